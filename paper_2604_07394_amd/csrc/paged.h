// Launchers of the paged 8-bit KV cache (each validates nothing: flux_api.hip has done it).
#pragma once

#include "flux_internal.h"

namespace flux {

constexpr int kPageTokens = FLUX_PAGE_TOKENS;
constexpr int kPlanRows = 1024;               // slots that a workgroup of flux_page_plan writes
constexpr float kPagedGuard = 1073741824.0f;  // 2^30: a page whose weights sum past this moves the softmax reference
constexpr long long kAppendPagedWaves = 4096; // an append takes as many as that where blocks may be many (see kv_append_paged_kernel)
constexpr int kPagedFewWgs = 256;            // workgroups of eight waves that a decode call takes at most
constexpr int kMinScaleExp = -100;            // of the scale of a block; its codes reach down to 2^-109

hipError_t launch_page_plan(const Ctx& c, const flux_page_table& pt, const int32_t* cu_new, int total_new, int32_t* slots, hipStream_t s);
hipError_t launch_page_release(const Ctx& c, const flux_page_table& pt, const int32_t* keep_len, hipStream_t s);
hipError_t launch_kv_append_paged(const Ctx& c, const flux_paged_kv& kv, int hkv, int d, const void* k_new, const void* v_new,
                                  const int32_t* slots, int total_new, hipStream_t s);

inline int pages_of(int tokens) { return tokens / kPageTokens + (tokens % kPageTokens != 0 ? 1 : 0); }
// A page of 8-bit codes has the bytes of 32 rows of a bf16 cache, the block that the plan of a decode call counts in.
// `one_each`: calls of few pages take workgroups of eight waves with a page each (see DecodePlan), of which a CU holds one at a time: up
// to kPagedFewWgs of them.  us of the kernel with at most 0 / 128 / 256 / 512, 32/8 heads of 128: 3 lists of 144 keys 7.4 / 7.3 / 6.9 /
// 7.2, 1 x 2000 9.0 / 8.9 / 8.7 / 8.8, 1 x 8000 11.6 / 11.8 / 10.2 / 10.5, 2 x 5000 12.0 / 12.0 / 10.9 / 11.1, 16 x 250 at 16/8 heads 7.5 /
// 7.6 / 6.9 / 7.6.
inline DecodePlan plan_decode_paged(const flux_attn_cfg& cfg, int batch, int max_kv_len, bool one_each = true) {
  DecodePlan p = plan_decode(cfg, batch, 32 * pages_of(max_kv_len));
  if (p.waves == 8 && !(one_each && p.wgs <= kPagedFewWgs)) {
    const long long by_four = (long long)batch * p.pps * (pages_of(max_kv_len) / 4 + (pages_of(max_kv_len) % 4 != 0 || max_kv_len == 0 ? 1 : 0));   // (one at least)
    p.waves = 4;
    // (the rows of parts go to the small region, which holds those of 512 workgroups up to 15 per part)
    if (2ll * (by_four < (1 << p.aligned_shift) ? by_four : (1 << p.aligned_shift)) * p.rpu * (cfg.head_dim + 2) * (long long)sizeof(float) > (long long)kSmallBytes) --p.aligned_shift;
    p.wgs = (int)(by_four < (1 << p.aligned_shift) ? by_four : (1 << p.aligned_shift));
  }
  return p;
}
hipError_t launch_decode_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, int max_kv_len, const flux_paged_kv& kv,
                               const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s);

// ---- prefill over pages: what its launch is bounded by (the plan itself is taken on the device, see paged_plan)
// Workgroups that the chip holds at once, per CU two at head dimension 128, three and (tiles of 64 rows) four at 64.  (With one
// register more than three of them have, 8192 tokens of 32/8 heads of 64 took 332 us, now 287.)
constexpr int paged_per_cu(int head_dim, int bm) { return head_dim == 128 ? 2 : (bm == 64 ? 4 : 3); }
constexpr int paged_resident(int head_dim, int bm) { return 256 * paged_per_cu(head_dim, bm); }
constexpr int kPagedMinPages = 8;             // a unit that shares a tile with others has at least so many pages
// Units of one (KV head, part) have ids of one residue mod 8, or of 8 / groups residues: units that `groups` of them take, some of
// them padding.
constexpr int share_shift(int groups) { return groups == 1 ? 3 : (groups == 2 ? 2 : (groups == 4 ? 1 : 0)); }
constexpr int unit_count(int groups, int tiles) {
  return share_shift(groups) > 0 ? ((tiles + (1 << share_shift(groups)) - 1) >> share_shift(groups)) * 8 : groups * tiles;
}
// n / d = (mulhi(n, mul) + n) >> shift for n < 2^31: the round-up method of Granlund and Montgomery (Division by invariant integers
// using multiplication, 1994), mul = floor(2^32 (2^shift - d) / d) + 1 with 2^shift >= d.
struct Reciprocal {
  uint32_t mul, shift;
};
inline Reciprocal reciprocal(uint32_t d) {
  uint32_t shift = 0;
  while (shift < 31 && (1ull << shift) < d) ++shift;
  return {(uint32_t)(((((uint64_t)1 << shift) - d) << 32) / d + 1), shift};
}
#ifdef __HIP__
__device__ __forceinline__ int quotient(int n, Reciprocal d) { return (int)(((uint32_t)(((uint64_t)(uint32_t)n * d.mul) >> 32) + (uint32_t)n) >> d.shift); }
#endif
struct PagedPrefillPlan {
  int bm;               // rows of a tile
  int tiles;            // of a sequence and KV head, at most
  long long wgs;        // workgroups launched
  int part_units;       // units whose rows the workspace has room for; 0: tiles are not shared out
  size_t info_bytes;    // of the table in front of these rows
};
inline PagedPrefillPlan plan_prefill_paged(const flux_attn_cfg& cfg, int batch, int max_q_len, int max_kv_len, size_t partials_bytes) {
  PagedPrefillPlan p;
  const long long rows = (long long)max_q_len * (cfg.n_q_heads / cfg.n_kv_heads);
  // Tiles of 64 rows where they run side by side and walk little more than their own queries: a page takes a wave half the MFMAs, and
  // nothing waits for a second round.  Behind a long context a tile of 128 rows converts and stages half as much.  us with 64 / 128
  // rows, 32/8 heads of 128 (512 workgroups of 64 rows side by side) unless said: 40 tokens 6.6 / 8.2, 100 7.6 / 9.6, 1000 25.4 / 29.0 and
  // a launch for shared tiles, 4 x 100 8.1 / 10.0, 16 x 60 to 140 (1024 tiles of 64) 17.2 / 14.4, at 8/2 heads of 64 (1024 side by side)
  // 512 tokens 10.5 / 12.8, 16 x 60 to 140 7.3 / 8.6; with the merge 64 tokens behind 8000 30.1 / 29.6, 128 behind 16000 61.2 / 51.8,
  // 512 behind 32000 382 / 274.  (What the bounds say counts: 4 x 300 to 700 tokens at 32/8 heads of 64 take 128 rows and 18.0 where 64
  // would be 16.8, as 1408 tiles of 64 are possible.)
  const long long tiles64 = (long long)batch * cfg.n_kv_heads * ((rows + 63) / 64);
  p.bm = rows <= 64 || (tiles64 <= paged_resident(cfg.head_dim, 64) && max_kv_len <= 2ll * max_q_len) ? 64 : 128;
  p.tiles = (int)((rows + p.bm - 1) / p.bm);
  p.wgs = (long long)batch * unit_count(cfg.n_kv_heads, p.tiles);
  p.part_units = 0;
  p.info_bytes = (((size_t)batch * cfg.n_kv_heads * p.tiles + 1) * 16 + 255) / 256 * 256;
  // worth a second launch (4 us where it finds nothing to do) where lists may be long and tiles few, or lists long and tiles no more than
  // two rounds: the tiles of the longest run of queries, and the device knows the others.  (From 64 pages on 3000 tokens behind 3000 took
  // 221 us, now 217 as without it; 5000 tokens at 8/2 heads of 64 64.)
  const long long longest = (long long)cfg.n_kv_heads * p.tiles, side_by_side = paged_resident(cfg.head_dim, p.bm);
  const bool few = 3 * longest < 2 * side_by_side;
  if (batch <= 64 && pages_of(max_kv_len) >= (few ? 2 : 16) * kPagedMinPages && longest <= 2 * side_by_side && p.info_bytes <= partials_bytes / 4) {
    const size_t fit = (partials_bytes - p.info_bytes) / ((size_t)p.bm * (cfg.head_dim + 2) * sizeof(float));
    const size_t want = (size_t)((few ? 2 : 3) * side_by_side + 8 * batch);
    p.part_units = (int)(fit < want ? fit : want);
    if (p.wgs < p.part_units) p.wgs = p.part_units;
  }
  return p;
}
// Short runs of queries behind a cached context (drafted tokens), whose rows take at most two blocks of 16 columns, are worked on like
// decode calls, by the kernel of those: a wave has a page to itself instead of a quarter of the rows.
constexpr int kRunRows = 32;
constexpr int runs_per_cu(int head_dim, int blocks) { return head_dim == 128 && blocks == 2 ? 1 : 2; }   // workgroups
inline DecodePlan plan_runs_paged(const flux_attn_cfg& cfg, int batch, int max_q_len, int max_kv_len) {
  flux_attn_cfg one = cfg;
  one.n_q_heads = cfg.n_kv_heads;                            // one pair per KV head
  DecodePlan p = plan_decode_paged(one, batch, max_kv_len, false);
  const long long by_four = (long long)batch * p.pps * ((pages_of(max_kv_len) + 3) / 4);
  p.rpu = max_q_len * (cfg.n_q_heads / cfg.n_kv_heads);
  p.aligned_shift = runs_per_cu(cfg.head_dim, (p.rpu + 15) / 16) == 1 ? kDecodeWgsShift : kDecodeAlignedShift;
  p.wgs = (int)(by_four < (1 << p.aligned_shift) ? by_four : (1 << p.aligned_shift));
  return p;
}
inline bool runs_paged(const Ctx& c, const flux_attn_cfg& cfg, int batch, int max_q_len, int max_kv_len) {
  const int group = cfg.n_q_heads / cfg.n_kv_heads;
  if (batch > 64 || max_q_len > kRunRows / group || pages_of(max_kv_len) < kPagedMinPages) return false;
  if ((long long)batch * cfg.n_kv_heads > 0x7FFFFFFFll / (pages_of(max_kv_len) + 16)) return false;   // pages are counted in 32 bits
  const DecodePlan p = plan_runs_paged(cfg, batch, max_q_len, max_kv_len);
  return c.decode_counters && (size_t)2 * p.wgs * p.rpu * (cfg.head_dim + 2) * sizeof(float) <= c.partials_bytes;
}
hipError_t launch_runs_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                             const flux_paged_kv& kv, const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s);
hipError_t launch_prefill_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                                const flux_paged_kv& kv, const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s);

}  // namespace flux
