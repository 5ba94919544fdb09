// flux_attn_prefill_paged: attention of the newest tokens of every sequence over a cache of 8-bit pages (Eq. 1 / Eq. 2, chosen per
// sequence by the mode byte).  The mathematics is that of decode_paged.hip, the shape that of prefill.hip: a workgroup of four
// waves owns a tile of query rows and walks the pages that a row of it sees, 64 keys at a time,
//   S^T[key][q]  = ck[key][:] . Q[q][:]            MFMA 16x16x32 bf16, A = keys from LDS, B = Q in registers
//   weights against a reference that moves only when a weight leaves the guarded range, rounded to bf16 (by 2^-8 of a weight at most,
//   2^-9 or so on average; the denominator sums the rounded ones).  One term, for fp32 outputs too, as in prefill.hip: a second one
//   is as many MFMAs again for this product.  2-norm of the error of bf16 outputs 1.9e-3 to 2.2e-3, of which their own rounding is 1.65e-3
//   O^T[d][q]   += (sv cv)^T[d][key] . p^T[key][q] V from LDS through the transposing read
//
// A tile is BM = 64 QB rows: the query rows of all heads of the group, token by token (row R is head R % group of token R /
// group), so that short runs of queries fill their tiles and K and V are read once per group.
//
// Codes become bf16 on their way into LDS: once per workgroup and page.  (In the waves' registers, behind the LDS reads, each of
// the four waves would convert every code.)  A page's codes are asked for one or two iterations ahead of that.  The
// scale of K goes into the exponent's factor, the power of two of V's into the conversion and what is left of it into the weights:
// nothing of K and V is rounded.
//
// What bounds it: the matrix pipe and the vector instructions beside it, at the clock that both leave (4096 tokens behind 28672 at 32/8
// heads of 128: pipe 57 % busy, no LDS bank conflicts, 1625 to 1705 us, 1.21 to 1.27 PFLOP/s; a bf16 cache takes 1540 to 1670, a large
// library product runs at 1.30 to 1.44).  512 behind 32000 take 237 (216), five prompts of 129 to 3001 tokens at 28/4 heads 93 (85 to 96: 1440
// tiles of 20 pages or so, each with a start and an end).
//
// Where the tiles do not fill the chip their pages are shared out over several workgroups, whose unnormalised rows a second
// launch merges (see paged_plan).
#include <type_traits>

#include "paged.h"

namespace flux {

typedef __attribute__((__vector_size__(4 * sizeof(int32_t)))) int32_t i32x4;

struct PagedPrefillArgs {
  const __bf16* q;        // [T, Hq, D]
  const int32_t* cu_q;
  const char *k, *v;
  const float *k_scale, *v_scale;
  int64_t stride_p, stride_h, stride_t;
  const int32_t* table;
  int table_pages, n_pages;
  const int32_t* kv_len;
  const uint8_t* mode;
  int max_q_len, max_kv_len;
  int hq, hkv, group, batch;
  Reciprocal by_group;
  int sink_lim, win_blocks, blk_shift;   // SA geometry (see sa_geom)
  int n_qtiles;           // tiles that a sequence has at most, by the host's bound
  int n_wg;
  float scale_log2;
  int out_fp32;
  void* out;
  uint32_t* status;
  int part_units;         // units whose rows the workspace holds; 0: tiles are never shared out
  float* part_o;          // unnormalised rows of a unit [unit][BM][D]
  float* part_ml;         // their reference (log2 units) and weight sum [unit][BM][2]
  i32x4* tile_info;       // whether tiles are shared out; behind it, [batch][hkv][n_qtiles]: first unit, unit stride, units of the tile
};

constexpr int kPagedNoSplit = 0x3FFFFFFF;

struct PagedSeq {
  int q_begin, n_q, len, rows, tiles, pages;   // rows: those within the bound on the queries; pages: of its longest tile (an upper bound for SA)
  bool sa, bad;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedPrefillArgs& a, int b, int bm) {
  PagedSeq s = {0, 0, 0, 0, 0, 0, false, false};
  if (b >= a.batch) return s;
  s.q_begin = a.cu_q[b];
  s.n_q = a.cu_q[b + 1] - s.q_begin;
  s.len = a.kv_len[b];
  s.sa = a.mode[b] == 0;
  const int cap = a.table_pages * kPageTokens;
  s.bad = s.n_q < 0 || s.len < 0 || s.len > cap || s.n_q > s.len || s.q_begin < 0 || s.len > a.max_kv_len;
  s.len = s.len < 0 ? 0 : min(s.len, cap);
  s.n_q = s.n_q < 0 || s.q_begin < 0 ? 0 : min(s.n_q, s.len);
  s.rows = min(s.n_q, a.max_q_len) * a.group;                // (max_q_len * group <= 2^30)
  s.tiles = (s.rows + bm - 1) / bm;
  s.pages = (s.len + 63) >> 6;
  if (s.sa) {
    const int64_t win = min((int64_t)a.win_blocks << a.blk_shift, (int64_t)s.len);
    s.pages = min(s.pages, ((min(a.sink_lim, s.len) + 63) >> 6) + (int)((win + bm) >> 6) + 2);
  }
  return s;
}

// ---- the plan of a launch, taken on the device by every wave: which unit of work a workgroup is.  A unit is (sequence, KV head,
// part, tile): part i of a tile has its pages [i * chunk, (i + 1) * chunk).  Where the tiles by themselves fill the chip
// more than twice, there is one part; otherwise see paged_chunk.
// Units of one (KV head, part) walk the same pages; workgroups go to the 8 XCDs by id mod 8, each with an L2 of its own, so these
// units get ids of one residue (or of 8 / groups residues).
struct PagedUnit {
  PagedSeq s;
  int b, kvh, tile, part, chunk, unit, stride;
  bool shared;            // some tile of the launch is shared out
  // b < 0: past the last unit; the tile's units are unit - part * stride + i * stride
};
// Over the 64 lanes, by moves between them as in wave_inclusive_sum; lane 63 has the result.  (Through LDS, a step takes a hundred
// cycles.)
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int old, int x) { return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus_moved(float x) { return x + __builtin_bit_cast(float, moved<CTRL, ROWS>(0, __builtin_bit_cast(int, x))); }
__device__ __forceinline__ float wave_sum(float x) {
  x = plus_moved<0x118, 0xf>(plus_moved<0x114, 0xf>(plus_moved<0x112, 0xf>(plus_moved<0x111, 0xf>(x))));
  x = plus_moved<0x143, 0xc>(plus_moved<0x142, 0xa>(x));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ __forceinline__ int wave_min(int x) {
  x = min(x, moved<0x111, 0xf>(x, x));
  x = min(x, moved<0x112, 0xf>(x, x));
  x = min(x, moved<0x114, 0xf>(x, x));
  x = min(x, moved<0x118, 0xf>(x, x));
  x = min(x, moved<0x142, 0xa>(x, x));
  x = min(x, moved<0x143, 0xc>(x, x));
  return __builtin_amdgcn_readlane(x, 63);
}
// Pages that a part has at most: every lane works out one candidate, from a fifth of the share that one of the resident workgroups has
// of all pages to three of them, by a model in units of one page, in which a part takes five pages more than it has, for its start
// and its end.  One round takes the longest part; more of them as many times the mean part, or what is shared out evenly and half of the
// longest part, whichever is less; and 0.03 for writing and merging the rows of a part.
// Calls of up to two rounds of tiles may be shared out.  us with none of more than two thirds of a round / so, 32/8 heads of 128 unless
// said: 3000 tokens behind 32000 (752 tiles where 512 run side by side) 1650 / 1380, six lists of 40 to 900 behind 500 to 20000 437 /
// 330, two of 600 to 2400 behind 6000 to 30000 660 / 549, three of 1000 to 3000 behind 100 to 60000 at 16/8 heads 1018 / 860, 4096
// behind 28672 at 32/8 heads of 64 1127 / 1070; but four of 500 to 1200 behind 1000 to 9000 230 / 241.
__device__ __forceinline__ int paged_chunk(const PagedPrefillArgs& a, int l, const PagedSeq& mine, int resident) {
  if (a.part_units == 0) return kPagedNoSplit;               // (the batch has at most 64 sequences otherwise)
  float tiles = (float)mine.tiles, pages = tiles * 0.5f * (float)(mine.pages + min(((mine.len - mine.n_q) >> 6) + 1, mine.pages));
  tiles = wave_sum(tiles) * (float)a.hkv;
  pages = wave_sum(pages) * (float)a.hkv;
  if (tiles > 2.f * (float)resident) return kPagedNoSplit;
  const float share = pages / (float)resident;
  const int cand = l == 63 ? kPagedNoSplit : max(kPagedMinPages, (int)(share * fast_exp2((float)l * (4.f / 62.f) - 2.3f)) + 1);
  const float inv = 1.0f / (float)cand;
  int units = 0, rows = 0;
  float longest = 0.f;
  for (int j = 0; j < a.batch; ++j) {
    const int t = __builtin_amdgcn_readlane(mine.tiles, j), p = __builtin_amdgcn_readlane(mine.pages, j);
    if (t == 0) continue;
    int n = (int)((float)(p - 1) * inv);                     // parts: (p - 1) / cand, put right by one, and one
    n += (n + 1) * cand <= p - 1 ? 1 : (n * cand > p - 1 ? -1 : 0);
    ++n;
    units += unit_count(a.hkv * n, t);
    rows += n > 1 ? a.hkv * n * t : 0;
    longest = fmaxf(longest, (float)p / (float)n);
  }
  const int rounds = (units + resident - 1) / resident;
  const float all = pages + 5.f * (float)units;
  longest += 5.f;
  float cost = (rounds <= 1 ? longest : fmaxf(longest, fminf((float)rounds * (all / (float)max(units, 1)), all / (float)resident + 0.5f * longest))) + 0.03f * (float)rows;
  if (units > a.n_wg || units > a.part_units) cost = 1e30f;
  if (l == 63) cost = fminf(cost, 1e29f);                    // (splits nothing, and always fits)
  const int best = wave_min((__builtin_bit_cast(int, cost) & ~63) | l) & 63;   // (positive floats order like their bits)
  return __builtin_amdgcn_readlane(rows, best) == 0 ? kPagedNoSplit : __builtin_amdgcn_readlane(cand, best);
}
__device__ __forceinline__ PagedSeq seq_from_lane(const PagedSeq& s, int i) {
  PagedSeq r;
  r.q_begin = __builtin_amdgcn_readlane(s.q_begin, i);
  r.n_q = __builtin_amdgcn_readlane(s.n_q, i);
  r.len = __builtin_amdgcn_readlane(s.len, i);
  r.rows = __builtin_amdgcn_readlane(s.rows, i);
  r.tiles = __builtin_amdgcn_readlane(s.tiles, i);
  r.pages = __builtin_amdgcn_readlane(s.pages, i);
  r.sa = __builtin_amdgcn_readlane((int)s.sa, i) != 0;
  r.bad = false;
  return r;
}
__device__ __forceinline__ PagedUnit paged_plan(const PagedPrefillArgs& a, int wg, int l, int bm, int resident) {
  const PagedSeq first = paged_seq(a, l, bm);
  PagedUnit u;
  u.b = -1;
  u.chunk = kPagedNoSplit;
  const int chunk = paged_chunk(a, l, first, resident);
  u.shared = chunk < kPagedNoSplit;
  int base = 0;
  bool bad = false;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const PagedSeq s = b0 == 0 ? first : paged_seq(a, b0 + l, bm);
    bad |= s.bad;
    const int parts = (s.pages + chunk - 1) / chunk, units = s.tiles > 0 ? unit_count(a.hkv * parts, s.tiles) : 0;
    // longest first, 64 sequences at a time
    int rank = l, units_s = units;
    if (a.batch > 1) {
      const int key = (s.pages << 6) | (63 - l);             // no two alike (pages <= 2^24)
      const int count = min(64, a.batch - b0);
      rank = 0;
      for (int j = 0; j < count; ++j) rank += __builtin_amdgcn_readlane(key, j) > key ? 1 : 0;
      rank = l < count ? rank : l;
      units_s = __builtin_amdgcn_ds_permute(4 * rank, units);
    }
    const int incl = base + wave_inclusive_sum(units_s);
    const int end = __builtin_amdgcn_readlane(incl, 63);
    if (u.b < 0 && wg < end) {                               // (uniform)
      const int place = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= wg));
      const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == place));
      u.s = seq_from_lane(s, at);
      u.b = b0 + at;
      const int n_parts = __builtin_amdgcn_readlane(parts, at), groups = a.hkv * n_parts, n_t = u.s.tiles;
      const int before = __builtin_amdgcn_readlane(incl, place) - unit_count(groups, n_t), local = wg - before;
      const int sh = share_shift(groups);
      int grp, t;
      if (sh > 0) {
        grp = (local & 7) & (groups - 1);
        t = ((local >> 3) << sh) + ((local & 7) >> (3 - sh));
      } else if ((groups & 7) == 0) {
        grp = ((local >> 3) / n_t) * 8 + (local & 7);
        t = (local >> 3) % n_t;
      } else {
        grp = local / n_t;
        t = local % n_t;
      }
      grp = __builtin_amdgcn_readfirstlane(grp);
      t = __builtin_amdgcn_readfirstlane(t);
      if (t >= n_t) {                                        // padding of the last round
        u.b = -1;
        return u;
      }
      u.part = __builtin_amdgcn_readfirstlane(grp / a.hkv);
      u.chunk = n_parts > 1 ? __builtin_amdgcn_readfirstlane((u.s.pages + n_parts - 1) / n_parts) : kPagedNoSplit;   // even parts
      u.kvh = grp - u.part * a.hkv;
      u.tile = n_t - 1 - t;                                  // heaviest first
      // rows of unit (kvh, part, tile) in the workspace: any numbering without gaps or clashes
      u.unit = before + (u.part * a.hkv + u.kvh) * n_t + u.tile;
      u.stride = a.hkv * n_t;
    }
    base = end;
    if (u.b >= 0 && wg != 0) break;
  }
  if (wg == 0 && threadIdx.x < 64 && bad) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_LENGTH);
  return u;
}

__device__ __forceinline__ u32x4 unpack8_scaled(uint32_t lo, uint32_t hi, float scale /*power of two*/) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}
template <int D, int QB>
__global__ __launch_bounds__(256, paged_per_cu(D, 64 * QB)) void paged_prompt_kernel(PagedPrefillArgs a) {
  constexpr int WR = 16 * QB;             // query rows per wave
  constexpr int BM = 4 * WR;              // query rows per workgroup
  constexpr int KC = D / 32;              // MFMA k-steps over the head dimension (QK^T)
  constexpr int DB = D / 16;              // 16-wide output blocks over the head dimension (PV)
  constexpr int KB = 4;                   // 16-key blocks of S^T per page
  constexpr int KS = 2;                   // 32-key steps of the PV product per page
  constexpr int AHEAD = QB == 1 ? 2 : 1;  // pages on their way, in registers: calls of few rows are bound by the memory
  constexpr int CPR = D / 16;             // 16-code chunks per row
  constexpr int NS = 64 * CPR / 256;      // chunks of K, and of V, that a thread stages
  constexpr int RPS = 256 / CPR;          // rows from one of them to the next
  constexpr int ROWB = 2 * D;             // bytes per row in LDS
  constexpr int TILE = 64 * ROWB;
  constexpr int STAGE = 2 * TILE;         // K, V
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = tid & 63;
  const int g = l >> 4, n = l & 15;
  const PagedUnit u = paged_plan(a, blockIdx.x, l, BM, paged_resident(D, BM));
  if (a.part_units > 0 && blockIdx.x == 0 && tid == 0) a.tile_info[0] = i32x4{u.shared, 0, 0, 0};
  if (u.b < 0) return;                                       // uniform for the workgroup

  // ---- rows and pages of the tile
  const int r0 = u.tile * BM, rows = min(u.s.rows - r0, BM);
  const int pos0 = u.s.len - u.s.n_q;                        // position of the sequence's first query
  auto token_of = [&](int r) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(quotient(r, a.by_group)); };   // (r: uniform)
  const int i_min = pos0 + token_of(r0), i_max = pos0 + token_of(r0 + rows - 1);
  const int last = i_max >> 6;                               // the page of the last query
  int seam = 0x7FFFFFFF, skip = 0;                           // list index x >= seam is page x + skip
  if (u.s.sa) {
    seam = min((int)(((int64_t)a.sink_lim + 63) >> 6), last + 1);
    skip = max((window_start(i_min, a.blk_shift, a.win_blocks) >> 6) - seam, 0);
  }
  const int list = last + 1 - skip;
  const int x0 = u.part * u.chunk;                           // (chunk < 2^30 / parts)
  const int parts = __builtin_amdgcn_readfirstlane((list + u.chunk - 1) / u.chunk);
  const bool split = parts > 1;
  if (u.shared && u.part == 0 && tid == 0)
    a.tile_info[1 + ((int64_t)u.b * a.hkv + u.kvh) * a.n_qtiles + u.tile] = i32x4{u.unit, u.stride, parts, 0};
  if (u.part >= parts) return;                               // (the bound on the pages was above this tile's)
  const int n_x = min(u.chunk, list - x0);                   // pages of this unit
  const int32_t* const pages = a.table + (int64_t)u.b * a.table_pages;
  auto page_at = [&](int x) __attribute__((always_inline)) { return x + (x >= seam ? skip : 0); };   // list index -> page of the sequence

  // ---- pages: lane i holds number and scales of the i-th page of 64: ids of the 64 that are being asked for, ids_next of the ones
  // behind them, ks and vs of the ones that are being staged, ks_next and vs_next of those in ids
  float ks, vs, ks_next, vs_next;
  auto load_ids = [&](int x) __attribute__((always_inline)) { return pages[page_at(x0 + min(x + l, n_x - 1))]; };
  int ids = load_ids(0), ids_next = load_ids(64);
  __builtin_amdgcn_sched_barrier(0);

  // ---- what a lane knows of its rows: position and start of the window; rows past the last one repeat it
  const int r_w0 = w * WR;
  int i_mine[QB], w_lo_mine[QB];
  bf16x8 qf[QB][KC];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int r = r0 + min(r_w0 + 16 * qb + n, rows - 1), tok = quotient(r, a.by_group), head = r - tok * a.group;
    i_mine[qb] = pos0 + tok;
    w_lo_mine[qb] = u.s.sa ? window_start(i_mine[qb], a.blk_shift, a.win_blocks) : 0;
    const __bf16* qrow = a.q + ((int64_t)(u.s.q_begin + tok) * a.hq + (int64_t)u.kvh * a.group + head) * D;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[qb][kc] = *(const bf16x8*)(qrow + 32 * kc + 8 * g);
  }
  const bool wave_active = r_w0 < rows;
  const int i_w_min = pos0 + token_of(r0 + min(r_w0, rows - 1)), i_w_max = pos0 + token_of(r0 + min(r_w0 + WR, rows) - 1);
  const int w_lo_first = u.s.sa ? window_start(i_w_min, a.blk_shift, a.win_blocks) : 0;
  const int w_lo_last = u.s.sa ? window_start(i_w_max, a.blk_shift, a.win_blocks) : 0;

  auto load_scales = [&]() __attribute__((always_inline)) {
    const int64_t page = (uint32_t)ids < (uint32_t)a.n_pages ? ids : 0;
    ks_next = a.k_scale[page * a.hkv + u.kvh];
    vs_next = a.v_scale[page * a.hkv + u.kvh];
  };
  const char* const kbase = a.k + (int64_t)u.kvh * a.stride_h;
  const char* const vbase = a.v + (int64_t)u.kvh * a.stride_h;
  u32x4 kcode[AHEAD][NS], vcode[AHEAD][NS];
  // The chunk that a thread stages: of 8 neighbouring lanes, which store at a time, half have a row whose swizzle takes their
  // chunks to the banks that the others leave out.
  const int st_c = D == 128 ? (tid & 3) | ((tid & 8) >> 1) : tid & 3;
  const int st_row = D == 128 ? ((tid >> 4) << 1) | ((tid >> 2) & 1) : ((tid >> 4) << 2) | ((tid >> 1) & 2) | ((tid >> 3) & 1);
  const int st_at = st_row * (int)a.stride_t + 16 * st_c;
  bool there_loaded[AHEAD], there = false;                   // whether a page in registers / the one in LDS is in the pool
  auto load_page = [&](int x, auto set_c) __attribute__((always_inline)) {   // x: page of this unit
    constexpr int SET = decltype(set_c)::value % AHEAD;
    if ((x & 63) == 0 && x > 0) {
      ids = ids_next;
      load_scales();
      ids_next = load_ids(x + 64);
    }
    const int id = __builtin_amdgcn_readlane(ids, x & 63);
    there_loaded[SET] = (uint32_t)id < (uint32_t)a.n_pages;
    const int64_t off = (int64_t)(there_loaded[SET] ? id : 0) * a.stride_p;
    // rows behind the length are not read: the last one stands in for them, with weight zero
    const int row_max = u.s.len - 1 - (page_at(x0 + x) << 6);
    const char *const kp = kbase + off, *const vp = vbase + off;
    if (row_max >= 63) {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        kcode[SET][i] = *(const u32x4*)(kp + i * RPS * a.stride_t + st_at);
        vcode[SET][i] = *(const u32x4*)(vp + i * RPS * a.stride_t + st_at);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int at = min(i * RPS + st_row, row_max) * (int)a.stride_t + 16 * st_c;
        kcode[SET][i] = *(const u32x4*)(kp + at);
        vcode[SET][i] = *(const u32x4*)(vp + at);
      }
    }
  };
  // K tile: 16-byte chunks XOR-swizzled by the row.  V tile: 32-byte units likewise (both as in prefill.hip), and of a unit the
  // two halves change places in every other row of a bank's.
  auto k_swz = [](int row) __attribute__((always_inline)) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto v_swz = [](int row) __attribute__((always_inline)) { return D == 128 ? row & 7 : (row >> 1) & 3; };
  auto v_half = [](int row) __attribute__((always_inline)) { return D == 128 ? row & 1 : (row >> 1) & 1; };
  // (the rows that a thread stages are 32 or 64 apart: the same swizzle)
  const int k_wr = st_row * ROWB + ((2 * st_c) ^ k_swz(st_row)) * 16, v_wr = TILE + st_row * ROWB + (st_c ^ v_swz(st_row)) * 32 + 16 * v_half(st_row);
  // The page in registers becomes bf16 in LDS, in 4 NS steps of 8 codes.  The scale of V: its power of two goes into
  // the conversion, which is exact; the rest, 1 <= r < 2, into the weights.
  float k_staged = 0.f, v_rest_staged = 1.f, v_power;        // of the page staged last
  auto begin_stage = [&](int x, bool is_there) __attribute__((always_inline)) {
    if ((x & 63) == 0) {
      ks = ks_next;
      vs = vs_next;
    }
    k_staged = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), x & 63));
    const uint32_t bits = max((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, vs), x & 63), 0x00800000u);
    v_power = __builtin_bit_cast(float, bits & 0x7F800000u);
    v_rest_staged = __builtin_bit_cast(float, (bits & 0x007FFFFFu) | 0x3F800000u);
    if (!is_there && tid == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_PAGE);
  };
  auto stage_step = [&](int j, auto set_c, FLUX_LDS char* st) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value % AHEAD;
    const int i = (j >> 1) % NS, h = j & 1;                  // chunk of the thread, half of the chunk
    if (j < 2 * NS) *(FLUX_LDS u32x4*)(st + (k_wr ^ (16 * h)) + i * RPS * ROWB) = unpack8_scaled(kcode[SET][i][2 * h], kcode[SET][i][2 * h + 1], 1.0f);
    else *(FLUX_LDS u32x4*)(st + (v_wr ^ (16 * h)) + i * RPS * ROWB) = unpack8_scaled(vcode[SET][i][2 * h], vcode[SET][i][2 * h + 1], v_power);
  };
  static_assert(4 * NS == DB, "a step of the staging for every output block");

  int k_rd[KC], v_rd[DB];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) k_rd[kc] = n * ROWB + ((4 * kc + g) ^ k_swz(n)) * 16;
  const int v_row = 4 * g + (n >> 2);
#pragma unroll
  for (int db = 0; db < DB; ++db) v_rd[db] = TILE + v_row * ROWB + (db ^ v_swz(v_row)) * 32 + ((8 * (n & 3)) ^ (16 * v_half(v_row)));

  // ---- accumulators.  A row's reference is -1e30 until it sees a key.
  float m_ref[QB], l_run[QB];
  f32x4 o[DB][QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m_ref[qb] = -1e30f;
    l_run[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  load_page(0, Even());
  load_scales();
  if (AHEAD == 2 && n_x > 1) load_page(1, Odd());
  begin_stage(0, there_loaded[0]);
#pragma unroll
  for (int j = 0; j < DB; ++j) stage_step(j, Even(), (FLUX_LDS char*)smem);
  float k_now = k_staged, v_rest = v_rest_staged;
  there = there_loaded[0];
  if (AHEAD == 2) {
    if (n_x > 2) load_page(2, Even());
  } else if (n_x > 1) {
    load_page(1, Odd());
  }
  __syncthreads();

  auto iteration = [&](int x, auto stg_c) __attribute__((always_inline)) {
    constexpr int STG = decltype(stg_c)::value;
    typedef std::integral_constant<int, STG ^ 1> Other;      // registers of the next page, and its stage
    FLUX_LDS char* const st = (FLUX_LDS char*)smem + STG * STAGE;
    const float c = fmaxf(a.scale_log2 * k_now, 0x1p-126f);  // (not 0: a masked score is -inf times this)
    const bool here = there;
    const bool more = x + 1 < n_x;                           // the next page goes into the other stage, the one behind it is asked for
    FLUX_LDS char* const st_next = (FLUX_LDS char*)smem + (STG ^ 1) * STAGE;
    float log_rest = 0.f, inv_rest = 1.f;
    if (__builtin_expect(v_rest != 1.f, 0)) {                // (uniform; the scales that the append writes are powers of two)
      log_rest = __builtin_amdgcn_logf(v_rest);
      inv_rest = 1.0f / v_rest;
    }
    const int j0 = page_at(x0 + x) << 6;
    bool hidden = !here || !wave_active || j0 > i_w_max;
    const bool all_sink = j0 + 64 <= a.sink_lim;
    hidden |= u.s.sa && j0 >= a.sink_lim && j0 + 63 < w_lo_first;
    if (more) begin_stage(x + 1, there_loaded[Other::value % AHEAD]);
    if (!hidden) {
      const bool causal = j0 + 63 > i_w_min, edge = u.s.sa && !all_sink && j0 < w_lo_last;
      f32x4 s[KB][QB];
      bf16x8 pf[QB][KS], kf[KB][KC], vf[KS][DB];
      auto read_k = [&](int kb, int kc) __attribute__((always_inline)) { kf[kb][kc] = *(FLUX_LDS bf16x8*)(st + k_rd[kc] + 16 * kb * ROWB); };
      auto read_v = [&](int h, int db) __attribute__((always_inline)) {
        FLUX_LDS char* const vp = st + v_rd[db] + 32 * h * ROWB;
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)vp);
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)(vp + 16 * ROWB));
        vf[h][db] = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
      };
      // wave priorities as in prefill.hip: the second product above the scores, those above the softmax and the staging
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) read_k(kb, kc);
      __builtin_amdgcn_sched_barrier(0);
      auto scores = [&]() __attribute__((always_inline)) {
        // S^T of keys 0..31 with the K fragments of keys 32..63 read between the MFMAs, then S^T of keys 32..63 with the V
        // fragments of keys 0..31 read between them
#pragma unroll
        for (int t = 0; t < 2 * KC; ++t) {
          const int kc = t >> 1, kb = t & 1;
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) s[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][kc], qf[qb][kc], s[kb][qb], 0, 0, 0);
          read_k(2 + kb, kc);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < 2 * KC; ++t) {
          const int kc = t >> 1, kb = 2 + (t & 1);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) s[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][kc], qf[qb][kc], s[kb][qb], 0, 0, 0);
#pragma unroll
          for (int db = t * DB / (2 * KC); db < (t + 1) * DB / (2 * KC); ++db) read_v(0, db);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if (causal || edge) {
        // element masks are put into the accumulators that the scores start from: key j0 + 4 g + c, c a constant
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const int hi = i_mine[qb] - j0 - 4 * g, lo = w_lo_mine[qb] - j0 - 4 * g, sl = a.sink_lim - j0 - 4 * g;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int k = 16 * kb + i;
              s[kb][qb][i] = (k <= hi) & ((k < sl) | (k >= lo)) ? 0.f : -INFINITY;
            }
        }
        scores();
      } else {                                               // (a path of its own: merged with the other one, the zeros would be moved into 32 registers)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) s[kb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
        scores();
      }
      __builtin_amdgcn_s_setprio(0);
      float l_page[QB];
      auto weights = [&]() __attribute__((always_inline)) {
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          l_page[qb] = 0.f;
          const float shift = log_rest - m_ref[qb];
#pragma unroll
          for (int h = 0; h < KS; ++h) {
            uint32_t pk[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const f32x4& sv = s[2 * h + (t >> 1)][qb];
              pk[t] = pack_bf16(fast_exp2(__builtin_fmaf(sv[2 * (t & 1)], c, shift)), fast_exp2(__builtin_fmaf(sv[2 * (t & 1) + 1], c, shift)));
              l_page[qb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[t]), ones, l_page[qb], false);
            }
            pf[qb][h] = __builtin_bit_cast(bf16x8, u32x4{pk[0], pk[1], pk[2], pk[3]});
          }
        }
      };
      weights();
      if (__builtin_amdgcn_ballot_w64(!(l_page[0] < kPagedGuard) | !(l_page[QB - 1] < kPagedGuard)) != 0) {
        // a row without a reference, or a weight that has left the guarded range: the rows that have one of 2^31 and more (which
        // trips the guard by itself, so that a row does not depend on those that share its wave) move the reference there
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          float m = s[0][qb][0];
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, s[kb][qb][i]);
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m, __shfl_xor(m, 32)) * c;
          const bool moves = m - m_ref[qb] >= 31.f;
          const float m_new = moves ? m : m_ref[qb];
          const float al = fast_exp2(m_ref[qb] - m_new);
          m_ref[qb] = m_new;
          l_run[qb] *= al;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db][qb] *= al;
        }
        weights();
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) l_run[qb] = __builtin_fmaf(l_page[qb], inv_rest, l_run[qb]);
      __builtin_amdgcn_s_setprio(2);
      __builtin_amdgcn_sched_barrier(0);
      // O^T += keys 0..31 with the V fragments of keys 32..63 read between the MFMAs
#pragma unroll
      for (int db = 0; db < DB; ++db) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[0][db], pf[qb][0], o[db][qb], 0, 0, 0);
        read_v(1, db);
        __builtin_amdgcn_sched_barrier(0);
      }
      // and those of keys 32..63 with the staging of the next page between them
      auto second = [&](auto stages) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[1][db], pf[qb][1], o[db][qb], 0, 0, 0);
          if constexpr (decltype(stages)::value) {
            stage_step(db, Other(), st_next);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      if (more) second(std::true_type());
      else second(std::false_type());
      __builtin_amdgcn_s_setprio(0);
    } else if (more) {
#pragma unroll
      for (int j = 0; j < DB; ++j) stage_step(j, Other(), st_next);
    }
    if (more) {
      k_now = k_staged;
      v_rest = v_rest_staged;
      there = there_loaded[Other::value % AHEAD];
      if (x + 1 + AHEAD < n_x) load_page(x + 1 + AHEAD, Other());
    }
    __syncthreads();                                         // this stage is free, and the other one written
  };
  for (int x = 0; x < n_x; x += 2) {
    iteration(x, Even());
    if (x + 1 < n_x) iteration(x + 1, Odd());
  }

  // ---- lane (n, g) holds d = 16 * db + 4 * g .. +3 of its rows
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    float l_tot = l_run[qb];
    l_tot += __shfl_xor(l_tot, 16);
    l_tot += __shfl_xor(l_tot, 32);
    const float inv = l_tot > 0.f || l_tot != l_tot ? 1.0f / l_tot : 0.f;   // (no key there: a row of zeros)
    // bf16 rows: of two output blocks side by side, the lanes of odd g hand their part of the first to the lane of g - 1 and
    // get its part of the second, so that a lane stores eight columns in a row (all lanes take part, whatever they store)
    u32x4 pk[DB / 2];
#pragma unroll
    for (int db = 0; db < DB; db += 2) {
      const f32x4 lo = o[db][qb] * inv, hi = o[db + 1][qb] * inv;
      const auto y0 = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[0], lo[1]), pack_bf16(hi[0], hi[1]), false, false);
      const auto y1 = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[2], lo[3]), pack_bf16(hi[2], hi[3]), false, false);
      pk[db / 2] = u32x4{y0[0], y1[0], y0[1], y1[1]};
    }
    const int x = r_w0 + 16 * qb + n;
    if (x >= rows) continue;
    if (split) {
      const int64_t row = (int64_t)u.unit * BM + x;
      if (g == 0) *(f32x2*)(a.part_ml + 2 * row) = f32x2{m_ref[qb], l_tot};
#pragma unroll
      for (int db = 0; db < DB; ++db) *(f32x4*)(a.part_o + row * D + 16 * db + 4 * g) = o[db][qb];
      continue;
    }
    const int r = r0 + x, tok = quotient(r, a.by_group), head = r - tok * a.group;
    const int64_t off = ((int64_t)(u.s.q_begin + tok) * a.hq + (int64_t)u.kvh * a.group + head) * D;
    if (a.out_fp32) {
#pragma unroll
      for (int db = 0; db < DB; ++db) *(f32x4*)((float*)a.out + off + 16 * db + 4 * g) = o[db][qb] * inv;
    } else {
      __bf16* const dst = (__bf16*)a.out + off + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
      for (int db = 0; db < DB; db += 2) *(u32x4*)(dst + 16 * db) = pk[db / 2];
    }
  }
}

// The merge of the units of a tile: out = sum_i w_i O_i / sum_i w_i l_i, w_i = 2^(m_i - max m).  D / 4 lanes per row, four columns
// each; a workgroup takes rows of one tile, and as many tiles as there are for it.
struct PagedMergeArgs {
  const int32_t *cu_q, *kv_len;
  const float *part_o, *part_ml;
  const i32x4* tile_info;
  int batch, hq, hkv, group, n_qtiles, bm, max_q_len, capacity, out_fp32;
  Reciprocal by_group;
  void* out;
};
template <int D>
__global__ __launch_bounds__(256) void paged_prompt_merge(PagedMergeArgs a) {
  constexpr int TPR = D / 4, RPW = 256 / TPR;                // rows that a workgroup has in work
  if (a.tile_info[0][0] == 0) return;
  const int groups = a.bm / RPW;
  const int items = a.batch * a.hkv * a.n_qtiles * groups;   // (64 sequences and twice paged_resident tiles of one at most)
  for (int it = blockIdx.x; it < items; it += gridDim.x) {
    const int t = it / groups, rg = it - t * groups;
    const int pair = t / a.n_qtiles, tile = t - pair * a.n_qtiles, b = pair / a.hkv, kvh = pair - b * a.hkv;
    const int q_begin = a.cu_q[b];
    int n_q = a.cu_q[b + 1] - q_begin, len = a.kv_len[b];
    len = len < 0 ? 0 : min(len, a.capacity);
    n_q = n_q < 0 || q_begin < 0 ? 0 : min(n_q, len);
    const int rows = min(min(n_q, a.max_q_len) * a.group - tile * a.bm, a.bm);   // (max_q_len * group <= 2^30)
    const int x = rg * RPW + threadIdx.x / TPR, d = 4 * (threadIdx.x % TPR);
    if (rg * RPW >= rows) continue;                          // (no such tile: what its entry holds is not read)
    const i32x4 info = a.tile_info[1 + t];
    if (info[2] < 2 || x >= rows) continue;
    float m = -INFINITY, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < info[2]; i0 += 8) {
      f32x2 ml[8];
      f32x4 o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t row = (int64_t)(info[0] + min(i0 + i, info[2] - 1) * info[1]) * a.bm + x;
        ml[i] = *(const f32x2*)(a.part_ml + 2 * row);
        o[i] = *(const f32x4*)(a.part_o + row * D + d);
      }
      float m_new = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) m_new = fmaxf(m_new, ml[i][0]);
      const float al = fast_exp2(m - m_new);                 // 0 for the first ones (every reference is -1e30 at least)
      num *= al;
      den *= al;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float wgt = i0 + i < info[2] ? fast_exp2(ml[i][0] - m_new) : 0.f;
        num += wgt * o[i];
        den += wgt * ml[i][1];
      }
      m = m_new;
    }
    const float inv = den > 0.f || den != den ? 1.0f / den : 0.f;
    const int r = tile * a.bm + x, tok = quotient(r, a.by_group), head = r - tok * a.group;
    const int64_t off = ((int64_t)(q_begin + tok) * a.hq + (int64_t)kvh * a.group + head) * D + d;
    const f32x4 y = num * inv;
    if (a.out_fp32) *(f32x4*)((float*)a.out + off) = y;
    else *(u32x2*)((__bf16*)a.out + off) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
  }
}

hipError_t launch_prefill_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                                const flux_paged_kv& kv, const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s) {
  if (max_q_len == 0) return hipSuccess;
  if (runs_paged(c, cfg, pt.batch, max_q_len, max_kv_len)) return launch_runs_paged(c, cfg, q, cu_q, max_q_len, max_kv_len, kv, pt, mode, out, s);
  const PagedPrefillPlan plan = plan_prefill_paged(cfg, pt.batch, max_q_len, max_kv_len, c.partials_bytes);
  PagedPrefillArgs a;
  a.q = (const __bf16*)q;
  a.cu_q = cu_q;
  a.k = (const char*)kv.k;
  a.v = (const char*)kv.v;
  a.k_scale = kv.k_scale;
  a.v_scale = kv.v_scale;
  a.stride_p = kv.stride_p;
  a.stride_h = kv.stride_h;
  a.stride_t = kv.stride_t;
  a.table = pt.table;
  a.table_pages = pt.table_pages;
  a.n_pages = kv.n_pages;
  a.kv_len = pt.kv_len;
  a.mode = mode;
  a.max_q_len = max_q_len;
  a.max_kv_len = max_kv_len;
  a.hq = cfg.n_q_heads;
  a.hkv = cfg.n_kv_heads;
  a.group = cfg.n_q_heads / cfg.n_kv_heads;
  a.by_group = reciprocal((uint32_t)a.group);
  a.batch = pt.batch;
  const SaGeom geom = sa_geom(cfg);
  a.sink_lim = geom.sink_lim;
  a.win_blocks = geom.win_blocks;
  a.blk_shift = geom.shift;
  a.n_qtiles = plan.tiles;
  a.n_wg = (int)plan.wgs;
  a.scale_log2 = (cfg.softmax_scale != 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)cfg.head_dim)) * kLog2e;
  a.out_fp32 = cfg.out_dtype;
  a.out = out;
  a.status = c.status;
  a.part_units = plan.part_units;
  a.tile_info = (i32x4*)c.partials;
  a.part_o = (float*)((char*)c.partials + plan.info_bytes);
  a.part_ml = a.part_o + (size_t)plan.part_units * plan.bm * cfg.head_dim;
  const dim3 grid((unsigned)plan.wgs), block(256);
  if (cfg.head_dim == 128) {
    if (plan.bm == 128) hipLaunchKernelGGL((paged_prompt_kernel<128, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_prompt_kernel<128, 1>), grid, block, 0, s, a);
  } else {
    if (plan.bm == 128) hipLaunchKernelGGL((paged_prompt_kernel<64, 2>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_prompt_kernel<64, 1>), grid, block, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.part_units == 0) return e;
  PagedMergeArgs m;
  m.cu_q = cu_q;
  m.kv_len = pt.kv_len;
  m.part_o = a.part_o;
  m.part_ml = a.part_ml;
  m.tile_info = a.tile_info;
  m.batch = pt.batch;
  m.hq = a.hq;
  m.hkv = a.hkv;
  m.group = a.group;
  m.by_group = a.by_group;
  m.n_qtiles = plan.tiles;
  m.bm = plan.bm;
  m.max_q_len = max_q_len;
  m.capacity = pt.table_pages * kPageTokens;
  m.out_fp32 = a.out_fp32;
  m.out = out;
  const long long items = (long long)pt.batch * a.hkv * plan.tiles * (plan.bm / (1024 / cfg.head_dim));
  const dim3 mgrid((unsigned)(items < 2048 ? items : 2048));
  if (cfg.head_dim == 128) hipLaunchKernelGGL(paged_prompt_merge<128>, mgrid, block, 0, s, m);
  else hipLaunchKernelGGL(paged_prompt_merge<64>, mgrid, block, 0, s, m);
  return hipGetLastError();
}

}  // namespace flux
