// flux_attn_cross: out = softmax(scale q K^T) V of packed query rows against all kv_len[b] keys of their sequence, with no order
// between queries and keys: the states of an encoder, of a length of their own.
//
// A workgroup has a tile of 64 or 128 rows of one KV head: the query rows of all heads of the group, token by token, so that K and V are
// read once for the group.  Four waves have 16 or 32 rows each and walk 64 keys at a time:
//     S^T[key][row] = K . Q      MFMA 16x16x32 bf16, K rows from LDS, Q in registers
//     p = 2^(scale (S - m))      m: the row's reference; it moves only when a block's weights sum past 2^30, so no block looks
//                                for its maximum first
//     O^T[d][row]  += V^T . p    the accumulators of two blocks of 16 keys are this product's operand as they are; V^T comes
//                                from row-major LDS through the transposing read
// K and V go to LDS without passing through registers, one block ahead.  The tiles' weights are rounded to bf16 (by 2^-8 of one at most), and the
// denominator sums the rounded ones, as in prefill.hip: a second term each would be half as many MFMAs again, in a kernel that the matrix pipe bounds.
// Where the tiles are few, the keys of a tile are shared out over several workgroups, and
// their unnormalised rows joined by a second launch.  Every workgroup finds out from the lengths which unit it is.
#include "cross.h"

namespace flux {

typedef __attribute__((__vector_size__(4 * sizeof(int32_t)))) int32_t i32x4;

struct CrossArgs {
  const __bf16* q;                // [T, Hq, D]
  const int32_t* cu;              // [batch + 1], null: q_len rows each
  const __bf16 *k, *v;
  int64_t stride_b, stride_h, stride_t;
  const int32_t* kv_len;
  int q_len, first;               // most rows of a sequence (null cu: of every one); first sequence of the launch
  int capacity, hq, hkv, group, batch;
  int n_tiles, max_blocks;        // by the host's bounds
  int n_wgs, part_units;
  float scale_log2;
  int out_fp32;
  void* out;
  float *part_o, *part_ml;        // unnormalised rows of a unit [unit][BM][D]; reference and sum of weights [unit][BM][2]
  i32x4* info;                    // of a tile [batch][hkv][n_tiles]: first unit, step between its units, how many; before them, whether any has more than one
  uint32_t* status;
};

constexpr float kGuard = 1073741824.0f;     // 2^30

struct CrossUnit {
  int b, kvh, tile, ci, parts;    // b < 0: none; part ci of `parts`
  int slot, slot_step;
  int q_begin, n_q, len;
};

__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_inclusive_sum(x), 63); }
// Largest of the lanes' numbers, none below 0: the moves of wave_inclusive_sum.
__device__ __forceinline__ int wave_most(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

// Keys of the tiles of a sequence in parts of at most so many blocks of 64.  A few sizes are tried on a model in units of a
// block (of tiles 1.6 us; of short runs 0.6 at head dimension 64 and 1.2 at 128, in which a CU takes its bytes in): the longest part where all run
// side by side, else their mean and half of the longest for unevenness; starting and ending a workgroup and the second launch are worth
// some blocks.
template <int D, int BM>
__device__ __forceinline__ CrossUnit cross_plan(const CrossArgs& a, int wg, int l) {
  constexpr int resident = BM <= 32 ? kCrossRunWgs : cross_resident(D);
  constexpr float kEnds = BM <= 32 ? (D == 64 ? 5.0f : 2.5f) : 2.5f, kJoin = BM <= 32 ? (D == 64 ? 6.0f : 3.0f) : 3.0f;
  CrossUnit u = {};
  int q_begin = 0, n_q = 0, len = 0, tiles = 0, nb = 0;
  bool bad = false;
  if (l < a.batch) {
    q_begin = a.cu ? a.cu[l] : (a.first + l) * a.q_len;
    n_q = a.cu ? a.cu[l + 1] - q_begin : a.q_len;
    len = a.kv_len[l];
    bad = n_q < 0 || n_q > a.q_len || len < 0 || len > a.capacity;
    n_q = min(max(n_q, 0), a.q_len);
    len = len < 0 ? 0 : min(len, a.capacity);
    tiles = (int)min(((int64_t)n_q * a.group + BM - 1) / BM, (int64_t)a.n_tiles);
    nb = max(1, (len + 63) >> 6);                            // (rows without keys are written too)
  }
  if (wg == 0 && threadIdx.x < 64 && bad) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_LENGTH);
  int nc = tiles > 0 ? 1 : 0;
  if (a.part_units > 0) {
    const int t_all = wave_total(tiles) * a.hkv;
    if (t_all < resident) {
      // (blocks of all tiles pass 32 bits in caches of 10^8 rows: their low 12 bits and the rest apart)
      const float work = ((float)wave_total(tiles * (nb & 4095)) + 4096.0f * (float)wave_total(tiles * (nb >> 12))) * (float)a.hkv, share = work / (float)resident;
      float best = 1e30f;
#pragma unroll
      for (int i = 0; i < 9; ++i) {
        const float factor[9] = {0.0f, 0.55f, 0.7f, 0.85f, 1.02f, 1.25f, 1.6f, 2.1f, 3.0f};      // (0: nothing is shared out)
        const int cand = i == 0 ? 0x3FFFFFFF : max(2, (int)(share * factor[i]) + 1);
        int n = i == 0 ? 0 : (int)((float)(nb - 1) / (float)cand);
        n += (int64_t)(n + 1) * cand <= nb - 1 ? 1 : (n * cand > nb - 1 && n > 0 ? -1 : 0);
        ++n;                                                 // ceil(nb / cand)
        const int units = wave_total(tiles * n) * a.hkv;
        const float longest = (float)wave_most(tiles > 0 ? (int)((float)nb / (float)n + 0.999f) : 0);
        float cost = units <= resident ? longest + kEnds : (work + kEnds * (float)units) / (float)resident + 0.5f * longest;
        if (i > 0) cost += kJoin + 0.004f * (float)units;
        if (i > 0 && (units + 8 * a.batch > a.n_wgs || units + 8 * a.batch > a.part_units)) cost = 1e30f;
        if (cost < best) {                                   // (uniform)
          best = cost;
          nc = tiles > 0 ? n : 0;
        }
      }
    }
  }
  const bool shared_out = __builtin_amdgcn_ballot_w64(nc > 1) != 0;
  if (a.part_units > 0 && wg == 0 && threadIdx.x == 0) a.info[-1] = i32x4{shared_out ? 1 : 0, 0, 0, 0};
  // Units of a sequence: one per (KV head, part, tile).  Workgroups go to the 8 XCDs by id mod 8, and the units of one (KV head,
  // part) walk the same rows of K and V: they get ids of one residue, or of 8 / groups residues.
  const int groups = a.hkv * nc;
  const int sh = groups == 1 ? 3 : (groups == 2 ? 2 : (groups == 4 ? 1 : 0));
  const int units = sh > 0 ? ((tiles + (1 << sh) - 1) >> sh) * 8 : groups * tiles;
  int units_s = units, idx_s = l, incl = wave_inclusive_sum(units);
  u.b = -1;
  if (wg >= __builtin_amdgcn_readlane(incl, 63)) return u;
  const int size = nc > 0 ? (int)((float)nb / (float)nc) : 0;
  if (__builtin_amdgcn_ballot_w64(l < a.batch && size != __builtin_amdgcn_readlane(size, 0)) != 0) {   // not all alike: longest first
    const int key = (size << 6) | (63 - l);
    int rank = 0;
    for (int j = 0; j < a.batch; ++j) rank += __builtin_amdgcn_readlane(key, j) > key ? 1 : 0;
    rank = l < a.batch ? rank : l;
    units_s = __builtin_amdgcn_ds_permute(4 * rank, units);
    idx_s = __builtin_amdgcn_ds_permute(4 * rank, l);
    incl = wave_inclusive_sum(units_s);
  }
  const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= wg));
  const int b = __builtin_amdgcn_readlane(idx_s, at);
  const int before = __builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(units_s, at), local = wg - before;
  const int n_t = __builtin_amdgcn_readlane(tiles, b), n_g = __builtin_amdgcn_readlane(groups, b), s = __builtin_amdgcn_readlane(sh, b);
  int grp, tt;
  if (s > 0) {
    grp = local & (n_g - 1);
    tt = ((local >> 3) << s) + ((local & 7) >> (3 - s));
  } else if ((n_g & 7) == 0) {
    const int j = local >> 3;
    tt = j % n_t;
    grp = j / n_t * 8 + (local & 7);
  } else {
    tt = local % n_t;
    grp = local / n_t;
  }
  tt = __builtin_amdgcn_readfirstlane(tt);
  grp = __builtin_amdgcn_readfirstlane(grp);
  if (tt >= n_t) return u;                                   // padding of the last round
  u.b = b;
  u.tile = tt;
  u.ci = grp / a.hkv;
  u.kvh = grp - u.ci * a.hkv;
  u.parts = __builtin_amdgcn_readlane(nc, b);
  u.slot = before + u.kvh * n_t + tt;
  u.slot_step = a.hkv * n_t;
  u.q_begin = __builtin_amdgcn_readlane(q_begin, b);
  u.n_q = __builtin_amdgcn_readlane(n_q, b);
  u.len = __builtin_amdgcn_readlane(len, b);
  return u;
}

// The first wave makes the plan for its workgroup: made by all four it takes the SIMDs four times as long (16 sequences, 600
// workgroups, us of the launch and the plan: 7.4 for 4.7).
template <int D, int BM>
__device__ __forceinline__ CrossUnit cross_unit(const CrossArgs& a, int w, int l, CrossUnit* shared) {
  if (w == 0) {
    const CrossUnit u = cross_plan<D, BM>(a, blockIdx.x, l);
    if (l == 0) *shared = u;
  }
  __syncthreads();
  CrossUnit u = *shared;
  int* words = (int*)&u;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(CrossUnit) / 4); ++i) words[i] = __builtin_amdgcn_readfirstlane(words[i]);
  return u;
}

#define FLUX_DMA_ONE(v, p, o) "s_add_u32 m0, %[lds], %[" o "]\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %[" v "], %[" p "]\n\t"
// The transfers of one wave for a tile of 64 keys, N of K and N of V, 1 KB each, every fourth KB of the stage at byte OFF.
template <int OFF, int KT, int N>
__device__ __forceinline__ void fetch_tile(const char* kt, const char* vt, const int (&ko)[N], const int (&vo)[N], uint32_t lds) {
  if constexpr (N == 4) {
    asm volatile(FLUX_DMA_ONE("k0", "kt", "o0") FLUX_DMA_ONE("k1", "kt", "o1") FLUX_DMA_ONE("k2", "kt", "o2") FLUX_DMA_ONE("k3", "kt", "o3")
                 FLUX_DMA_ONE("v0", "vt", "o4") FLUX_DMA_ONE("v1", "vt", "o5") FLUX_DMA_ONE("v2", "vt", "o6") FLUX_DMA_ONE("v3", "vt", "o7")
                 : : [k0] "v"(ko[0]), [k1] "v"(ko[1]), [k2] "v"(ko[2]), [k3] "v"(ko[3]), [v0] "v"(vo[0]), [v1] "v"(vo[1]), [v2] "v"(vo[2]), [v3] "v"(vo[3]),
                     [kt] "s"(kt), [vt] "s"(vt), [lds] "s"(lds), [o0] "i"(OFF), [o1] "i"(OFF + 4096), [o2] "i"(OFF + 8192), [o3] "i"(OFF + 12288),
                     [o4] "i"(OFF + KT), [o5] "i"(OFF + KT + 4096), [o6] "i"(OFF + KT + 8192), [o7] "i"(OFF + KT + 12288)
                 : "memory", "m0", "scc");
  } else {
    asm volatile(FLUX_DMA_ONE("k0", "kt", "o0") FLUX_DMA_ONE("k1", "kt", "o1") FLUX_DMA_ONE("v0", "vt", "o4") FLUX_DMA_ONE("v1", "vt", "o5")
                 : : [k0] "v"(ko[0]), [k1] "v"(ko[1]), [v0] "v"(vo[0]), [v1] "v"(vo[1]), [kt] "s"(kt), [vt] "s"(vt), [lds] "s"(lds),
                     [o0] "i"(OFF), [o1] "i"(OFF + 4096), [o4] "i"(OFF + KT), [o5] "i"(OFF + KT + 4096)
                 : "memory", "m0", "scc");
  }
}

// Bound by the matrix pipe (two thirds of the cycles of the CUs' SIMDs) and the vector instructions beside it: four sequences of 1000 to 5000 rows on 4001 to
// 9000 keys, 32 and 8 heads of 128 (986 GFLOP), 767 to 858 us from box to box, 1.15 to 1.29 PFLOP/s.
template <int D, int QB>
__global__ __launch_bounds__(256, 2) void cross_tile_kernel(CrossArgs a) {
  constexpr int WR = 16 * QB, BM = 4 * WR, BN = 64;
  constexpr int KC = D / 32, DB = D / 16, KB = BN / 16, KS = BN / 32;
  constexpr int CPR = D / 8, ROWB = 2 * D;
  constexpr int TILE = BN * ROWB, STAGE = 2 * TILE;          // K, then V
  constexpr int NT = BN * CPR / 64 / 4;                      // transfers of a wave for K, and for V
  constexpr int RPI = 64 / CPR;                              // rows of a transfer
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];

  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, g = l >> 4, n = l & 15;
  __shared__ CrossUnit s_unit;
  const CrossUnit u = cross_unit<D, BM>(a, w, l, &s_unit);
  if (u.b < 0) return;                                       // (uniform)
  const int64_t n_rows = (int64_t)u.n_q * a.group, row0 = (int64_t)u.tile * BM;
  const int rows = (int)min((int64_t)BM, n_rows - row0);
  const int tok0 = (int)(row0 / a.group), rem0 = (int)(row0 - (int64_t)tok0 * a.group);
  const int h0 = u.kvh * a.group;
  // element of q and out where row x of the tile begins (x and a group are small: the quotient is taken through floats)
  const float inv_grp = __builtin_amdgcn_rcpf((float)a.group);
  const int64_t tile_off = ((int64_t)(u.q_begin + tok0) * a.hq + h0) * D;
  auto row_off = [&](int x) {
    const int t = (int)(((float)(rem0 + x) + 0.5f) * inv_grp);
    return tile_off + ((int64_t)t * a.hq + (rem0 + x - t * a.group)) * D;
  };
  const int len = u.len, blocks = (len + BN - 1) / BN;
  if (a.part_units > 0 && tid == 0 && u.ci == 0) a.info[((int64_t)u.b * a.hkv + u.kvh) * a.n_tiles + u.tile] = i32x4{u.slot, u.slot_step, u.parts, 0};
  const int r_w0 = WR * w;                                   // first row of this wave
  const bool active = r_w0 < rows;
  int it0 = 0, n_iter = blocks;                              // this unit's blocks: it0 .. n_iter - 1
  if (u.parts > 1) {
    it0 = (int)((int64_t)u.ci * blocks / u.parts);
    n_iter = (int)((int64_t)(u.ci + 1) * blocks / u.parts);
  }
  it0 = __builtin_amdgcn_readfirstlane(it0);
  n_iter = __builtin_amdgcn_readfirstlane(n_iter);

  const char* kbase = (const char*)(a.k + (int64_t)u.b * a.stride_b + (int64_t)u.kvh * a.stride_h);
  const char* vbase = (const char*)(a.v + (int64_t)u.b * a.stride_b + (int64_t)u.kvh * a.stride_h);
  const int pitch = (int)a.stride_t * 2;
  const int64_t step_b = (int64_t)BN * pitch;
  // Transfer t of wave w covers rows (w + 4 t) * RPI .. of a tile; lane l lands at row l / CPR of them, piece l % CPR of 16 bytes,
  // and fetches the piece that the swizzle keeps there.  K: pieces XOR-swizzled by the row (head dimension 128: row & 15; 64, two rows per 64 banks: (row >> 1)
  // & 7); V: units of 32 bytes (row & 7; (row >> 1) & 3).  Both make the reads below free of bank conflicts.
  const int lrow = l / CPR;
  const int k_piece = (l % CPR) ^ ((4 * w + (l >> 4)) & (CPR - 1));
  const int v_piece = (l % CPR) ^ (D == 128 ? ((4 * (w & 1) + lrow) << 1) : (((lrow >> 1) & 3) << 1));
  auto k_slot = [&](int t, int rmax) __attribute__((always_inline)) { return min((w + 4 * t) * RPI + lrow, rmax) * pitch + k_piece * 16; };
  auto v_slot = [&](int t, int rmax) __attribute__((always_inline)) { return min((w + 4 * t) * RPI + lrow, rmax) * pitch + v_piece * 16; };
  int k_off[NT], v_off[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    k_off[t] = k_slot(t, BN);
    v_off[t] = v_slot(t, BN);
  }
  const uint32_t lds_w = (uint32_t)(uintptr_t)(FLUX_LDS char*)smem + 1024 * w;
  // a tile whose rows past the length are clamped to the last one
  auto fetch_clamped = [&](int tile, int stage) __attribute__((always_inline)) {
    const int rmax = len - 1 - tile * BN;
    const char *kt = kbase + tile * step_b, *vt = vbase + tile * step_b;
    const uint32_t at = lds_w + stage * STAGE;
#pragma unroll
    for (int t = 0; t < NT; ++t) lds_copy16(kt, k_slot(t, rmax), at + 4096 * t);
#pragma unroll
    for (int t = 0; t < NT; ++t) lds_copy16(vt, v_slot(t, rmax), at + TILE + 4096 * t);
  };
  if (n_iter > it0) fetch_clamped(it0, 0);

  bf16x8 qf[QB][KC];                                         // lane (n, g): d = 32 kc + 8 g .. + 7 of its rows (past the last one: that again)
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const __bf16* qrow = a.q + row_off(min(r_w0 + 16 * qb + n, rows - 1));
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[qb][kc] = *(const bf16x8*)(qrow + 32 * kc + 8 * g);
  }
  const int k_xr = D == 128 ? n : (n >> 1);
  int k_rd[KC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) k_rd[kc] = n * ROWB + (((4 * kc + g) ^ k_xr) * 16);
  const int v_row = 4 * g + (n >> 2), v_xr = D == 128 ? (v_row & 7) : ((v_row >> 1) & 3);
  int v_rd[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) v_rd[db] = TILE + v_row * ROWB + ((db ^ v_xr) * 32) + (n & 3) * 8;

  float m_ref[QB], mneg[QB], l_run[QB];                      // reference of a row (score units), -m * scale, this lane's part of the sum
  f32x4 o[DB][QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m_ref[qb] = -INFINITY;
    mneg[qb] = l_run[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool all_ref = false;
  const int whole = len / BN;                                // blocks that are wholly below the length
  const char* kt_n = kbase + (it0 + 1) * step_b;
  const char* vt_n = vbase + (it0 + 1) * step_b;

  auto iteration = [&](int it, auto stg_c) __attribute__((always_inline)) {
    constexpr int STG = decltype(stg_c)::value;
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // vmcnt(0): this wave's transfers have landed
    __syncthreads();                                         // ... and everyone's; the other stage is free
    if (__builtin_expect(it + 1 < n_iter, 1)) {              // the next tile, on its way during what follows
      if (__builtin_expect(it + 1 < whole, 1)) {
        fetch_tile<(STG ^ 1) * STAGE, TILE, NT>(kt_n, vt_n, k_off, v_off, lds_w);
        kt_n += step_b;
        vt_n += step_b;
      } else {
        fetch_clamped(it + 1, STG ^ 1);
      }
    }
    if (!active) return;
    FLUX_LDS char* st = (FLUX_LDS char*)smem + STG * STAGE;
    f32x4 s[KB][QB];             // s[kb][qb][i]: key 16 kb + 4 g + i of the block against row n of column block qb
    bf16x8 pf[QB][KS], kf[KB][KC], vf[KS][DB];
    auto read_k = [&](int kb, int kc) __attribute__((always_inline)) { kf[kb][kc] = *(FLUX_LDS bf16x8*)(st + k_rd[kc] + 16 * kb * ROWB); };
    auto read_v = [&](int ks, int db) __attribute__((always_inline)) {
      FLUX_LDS char* vp = st + v_rd[db] + 32 * ks * ROWB;
      const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)vp);
      const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)(vp + 16 * ROWB));
      vf[ks][db] = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    float l_blk[QB];
    auto weights = [&]() __attribute__((always_inline)) {
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        l_blk[qb] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint32_t pk[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const f32x4& sv = s[2 * ks + (t >> 1)][qb];
            const float p0 = fast_exp2(__builtin_fmaf(sv[2 * (t & 1)], a.scale_log2, mneg[qb]));
            const float p1 = fast_exp2(__builtin_fmaf(sv[2 * (t & 1) + 1], a.scale_log2, mneg[qb]));
            pk[t] = pack_bf16(p0, p1);
            l_blk[qb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[t]), ones, l_blk[qb], false);
          }
          pf[qb][ks] = __builtin_bit_cast(bf16x8, u32x4{pk[0], pk[1], pk[2], pk[3]});
        }
      }
    };
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) read_k(kb, kc);
    __builtin_amdgcn_sched_barrier(0);
    // reads of one half stand between the MFMAs of the other
    auto scores = [&]() __attribute__((always_inline)) {
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
    // the mask stands in the accumulators that the scores start from: -inf for a key past the length
    if (__builtin_expect(it >= whole, 0)) {
      const int hi = len - 1 - it * BN - 4 * g;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][qb][i] = 16 * kb + i <= hi ? 0.f : -INFINITY;
      scores();
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[kb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
      scores();
    }
    __builtin_amdgcn_s_setprio(0);
    weights();
    if (__builtin_expect(!all_ref || (__builtin_amdgcn_ballot_w64(!(l_blk[0] < kGuard)) | __builtin_amdgcn_ballot_w64(!(l_blk[QB - 1] < kGuard))) != 0, 0)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float top = s[0][qb][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kb][qb][i]);
        top = fmaxf(top, __shfl_xor(top, 16));               // over the 4 lanes of the row
        top = fmaxf(top, __shfl_xor(top, 32));
        // a row moves for its own reason alone: no reference yet, or a weight of 2^31 and more
        const bool moves = (m_ref[qb] == -INFINITY || __builtin_fmaf(top, a.scale_log2, mneg[qb]) >= 31.f) && top > m_ref[qb];
        const float al = moves ? fast_exp2((m_ref[qb] - top) * a.scale_log2) : 1.f;   // 0 for a row's first reference
        l_run[qb] *= al;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db][qb] *= al;
        m_ref[qb] = moves ? top : m_ref[qb];
        mneg[qb] = moves ? -top * a.scale_log2 : mneg[qb];
      }
      weights();
      all_ref = __builtin_amdgcn_ballot_w64((m_ref[0] == -INFINITY) | (m_ref[QB - 1] == -INFINITY)) == 0;
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l_run[qb] += l_blk[qb];
    __builtin_amdgcn_s_setprio(2);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[0][db], pf[qb][0], o[db][qb], 0, 0, 0);
      read_v(1, db);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[1][db], pf[qb][1], o[db][qb], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
  };
  for (int it = it0; it < n_iter; it += 2) {
    iteration(it, std::integral_constant<int, 0>());
    if (__builtin_expect(it + 1 < n_iter, 1)) iteration(it + 1, std::integral_constant<int, 1>());
  }

  // lane (n, g) holds d = 16 db + 4 g .. + 3 of its rows
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    float sum = l_run[qb];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const float inv = len > 0 ? 1.0f / sum : 0.f;            // (rows without keys are zero)
    // bf16: of two output blocks side by side, lanes of odd g hand their part of the first to the lane of g - 1 and get its part of the
    // second, so that a lane stores eight columns in a row
    u32x4 pk[DB / 2];
#pragma unroll
    for (int db = 0; db < DB; db += 2) {
      const f32x4 lo = o[db][qb] * inv, hi = o[db + 1][qb] * inv;
      const auto x0 = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[0], lo[1]), pack_bf16(hi[0], hi[1]), false, false);
      const auto x1 = __builtin_amdgcn_permlane16_swap(pack_bf16(lo[2], lo[3]), pack_bf16(hi[2], hi[3]), false, false);
      pk[db / 2] = u32x4{x0[0], x1[0], x0[1], x1[1]};
    }
    const int x = r_w0 + 16 * qb + n;
    if (x >= rows) continue;
    if (u.parts > 1) {
      const int64_t row = (int64_t)(u.slot + u.ci * u.slot_step) * BM + x;
      if (g == 0) {
        a.part_ml[2 * row] = m_ref[qb];
        a.part_ml[2 * row + 1] = sum;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) *(f32x4*)(a.part_o + row * D + 16 * db + 4 * g) = o[db][qb];
    } else if (a.out_fp32) {
#pragma unroll
      for (int db = 0; db < DB; ++db) *(f32x4*)((float*)a.out + row_off(x) + 16 * db + 4 * g) = o[db][qb] * inv;
    } else {
      __bf16* dst = (__bf16*)a.out + row_off(x) + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
      for (int db = 0; db < DB; db += 2) *(u32x4*)(dst + 16 * db) = pk[db / 2];
    }
  }
}

// Short runs: the rows of a KV head fit one or two blocks of 16 columns (a decode step of several beams, say), and a call is bound by the
// bytes of K and V.  The four waves of a workgroup take blocks of 32 keys in turn, K from memory into the MFMA's operand, V through
// LDS of their own, each block asked for while the one before is worked on, and join their rows in the end.  16 sequences of five rows on 1500 keys, 8
// heads of 64 (49 MB): 13.2 us of which the streaming is about 9, and 2.3 for the joining launch.
template <int D, int QB>
__global__ __launch_bounds__(256, 2) void cross_run_kernel(CrossArgs a) {
  constexpr int BM = 16 * QB, KC = D / 32, DB = D / 16, CPR = D / 8, ROWB = 2 * D, VL = 32 * CPR / 64;
  __shared__ __attribute__((aligned(1024))) char smem[4 * 32 * ROWB];              // a block of V per wave; the rows of O in the end
  __shared__ float s_m[4][BM], s_l[4][BM];
  static_assert(4 * 32 * ROWB >= 4 * 16 * D * 4, "one block of columns at a time is joined");
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, g = l >> 4, n = l & 15;
  __shared__ CrossUnit s_unit;
  const CrossUnit u = cross_unit<D, BM>(a, w, l, &s_unit);
  if (u.b < 0) return;                                       // (uniform)
  const int rows = u.n_q * a.group, len = u.len;             // (at most BM)
  if (a.part_units > 0 && tid == 0 && u.ci == 0) a.info[(int64_t)u.b * a.hkv + u.kvh] = i32x4{u.slot, u.slot_step, u.parts, 0};
  const int64_t tile_off = ((int64_t)u.q_begin * a.hq + u.kvh * a.group) * D;
  auto row_off = [&](int x) {
    const int t = (int)((uint32_t)x / (uint32_t)a.group);
    return tile_off + ((int64_t)t * a.hq + (x - t * a.group)) * D;
  };
  const int blocks = (len + 63) / 64;
  int k0 = 0, k1 = len;                                      // this unit's keys
  if (u.parts > 1) {
    k0 = 64 * (int)((int64_t)u.ci * blocks / u.parts);
    k1 = min(len, 64 * (int)((int64_t)(u.ci + 1) * blocks / u.parts));
  }
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k1 = __builtin_amdgcn_readfirstlane(k1);
  const char* kbase = (const char*)(a.k + (int64_t)u.b * a.stride_b + (int64_t)u.kvh * a.stride_h);
  const char* vbase = (const char*)(a.v + (int64_t)u.b * a.stride_b + (int64_t)u.kvh * a.stride_h);
  const int pitch = (int)a.stride_t * 2;
  u32x4 kreg[2][KC], vreg[VL];
  auto load_block = [&](int j0) __attribute__((always_inline)) {                   // (rows past the last key: that one again)
    const char *kt = kbase + (int64_t)j0 * pitch, *vt = vbase + (int64_t)j0 * pitch;
    const int last = k1 - 1 - j0;
#pragma unroll
    for (int sb = 0; sb < 2; ++sb)
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) kreg[sb][kc] = *(const u32x4*)(kt + min(16 * sb + n, last) * pitch + 64 * kc + 16 * g);
#pragma unroll
    for (int i = 0; i < VL; ++i) vreg[i] = *(const u32x4*)(vt + min((i * 64 + l) / CPR, last) * pitch + (l % CPR) * 16);
  };
  int j0 = k0 + 32 * w;
  if (j0 < k1) load_block(j0);
  bf16x8 qf[QB][KC];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const __bf16* qrow = a.q + row_off(min(16 * qb + n, rows - 1));
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[qb][kc] = *(const bf16x8*)(qrow + 32 * kc + 8 * g);
  }
  FLUX_LDS char* const vs = (FLUX_LDS char*)smem + w * 32 * ROWB;
  // V: units of 32 bytes XOR-swizzled by the row, as in the tiles
  int v_wr[VL];
#pragma unroll
  for (int i = 0; i < VL; ++i) {
    const int r = (i * 64 + l) / CPR;
    v_wr[i] = r * ROWB + (((l % CPR) ^ (D == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1)) * 16);
  }
  const int v_row = 4 * g + (n >> 2), v_xr = D == 128 ? (v_row & 7) : ((v_row >> 1) & 3);
  int v_rd[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) v_rd[db] = v_row * ROWB + ((db ^ v_xr) * 32) + (n & 3) * 8;
  float m[QB], sum[QB];
  f32x4 o[DB][QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = -INFINITY;
    sum[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  while (j0 < k1) {
#pragma unroll
    for (int i = 0; i < VL; ++i) *(FLUX_LDS u32x4*)(vs + v_wr[i]) = vreg[i];
    f32x4 s[2][QB];
#pragma unroll
    for (int sb = 0; sb < 2; ++sb)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        s[sb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) s[sb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kreg[sb][kc]), qf[qb][kc], s[sb][qb], 0, 0, 0);
      }
    const int left = k1 - j0;
    j0 += 128;
    __builtin_amdgcn_sched_barrier(0);
    if (j0 < k1) load_block(j0);                             // (its registers have been read by now)
    __builtin_amdgcn_sched_barrier(0);
    // A weight is the sum of two bf16 values, its upper bits and what they leave of it, to 2^-16 of it as in decode.hip: rows of several beams are scored as a
    // decode step scores one, and the matrix pipe is idle while a block arrives.  (2-norm of the error with fp32 outputs 1.2e-3 with one bf16 value, below 1.2e-5
    // with two; the call of the 49 MB above 16.0 us with either.)
    bf16x8 pf[QB], pr[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (left < 32) {
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[sb][qb][i] = 16 * sb + 4 * g + i < left ? s[sb][qb][i] : -INFINITY;
      }
      float top = m[qb];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[sb][qb][i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      // (a row whose scores are all -inf so far refers to 0)
      const float ref = top == -INFINITY ? 0.f : top, al = fast_exp2((m[qb] - ref) * a.scale_log2), mneg = -ref * a.scale_log2;
      m[qb] = top;
      uint32_t pk[4], rest[4];
      float add = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float p0 = fast_exp2(__builtin_fmaf(s[t >> 1][qb][2 * (t & 1)], a.scale_log2, mneg)), p1 = fast_exp2(__builtin_fmaf(s[t >> 1][qb][2 * (t & 1) + 1], a.scale_log2, mneg));
        pk[t] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p0), 0x07060302u);
        rest[t] = pack_bf16(p0 - bf16_lo(pk[t]), p1 - bf16_hi(pk[t]));
        add += p0 + p1;
      }
      sum[qb] = __builtin_fmaf(sum[qb], al, add);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][qb] *= al;
      pf[qb] = __builtin_bit_cast(bf16x8, u32x4{pk[0], pk[1], pk[2], pk[3]});
      pr[qb] = __builtin_bit_cast(bf16x8, u32x4{rest[0], rest[1], rest[2], rest[3]});
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)(vs + v_rd[db]));
      const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FLUX_LDS bf16x4*)(vs + v_rd[db] + 16 * ROWB));
      const bf16x8 vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qb], o[db][qb], 0, 0, 0);
        o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pr[qb], o[db][qb], 0, 0, 0);
      }
    }
  }
  // the waves' rows: references and sums first
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    sum[qb] += __shfl_xor(sum[qb], 16);
    sum[qb] += __shfl_xor(sum[qb], 32);
    if (g == 0) {
      s_m[w][16 * qb + n] = m[qb];
      s_l[w][16 * qb + n] = sum[qb];
    }
  }
  FLUX_LDS float* const so = (FLUX_LDS float*)(FLUX_LDS char*)smem;                // [wave][d / 4][column][4]
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    __syncthreads();                                         // (V, or the columns before, have been read)
    const float top = fmaxf(fmaxf(s_m[0][16 * qb + n], s_m[1][16 * qb + n]), fmaxf(s_m[2][16 * qb + n], s_m[3][16 * qb + n]));
    const float mine = m[qb] == -INFINITY ? 0.f : fast_exp2((m[qb] - top) * a.scale_log2);
#pragma unroll
    for (int db = 0; db < DB; ++db) *(FLUX_LDS f32x4*)(so + ((w * D / 4 + 4 * db + g) * 16 + n) * 4) = o[db][qb] * mine;
    __syncthreads();
    for (int e = tid; e < 16 * (D / 4); e += 256) {
      const int c = e / (D / 4), d4 = e - c * (D / 4), x = 16 * qb + c;
      if (x >= rows) continue;
      f32x4 num = {0.f, 0.f, 0.f, 0.f};
      float den = 0.f;
      const float ref = fmaxf(fmaxf(s_m[0][x], s_m[1][x]), fmaxf(s_m[2][x], s_m[3][x]));
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        num += *(FLUX_LDS f32x4*)(so + ((v * D / 4 + d4) * 16 + c) * 4);
        den += s_m[v][x] == -INFINITY ? 0.f : s_l[v][x] * fast_exp2((s_m[v][x] - ref) * a.scale_log2);
      }
      if (u.parts > 1) {
        const int64_t row = (int64_t)(u.slot + u.ci * u.slot_step) * BM + x;
        if (d4 == 0) {
          a.part_ml[2 * row] = ref;
          a.part_ml[2 * row + 1] = den;
        }
        *(f32x4*)(a.part_o + row * D + 4 * d4) = num;
      } else {
        const float inv = len > 0 ? 1.0f / den : 0.f;        // (rows without keys are zero)
        if (a.out_fp32) *(f32x4*)((float*)a.out + row_off(x) + 4 * d4) = num * inv;
        else *(u32x2*)((__bf16*)a.out + row_off(x) + 4 * d4) = u32x2{pack_bf16(num[0] * inv, num[1] * inv), pack_bf16(num[2] * inv, num[3] * inv)};
      }
    }
  }
}

// Tiles whose keys were shared out: out = sum_c w_c O_c / sum_c w_c l_c with w_c = 2^(scale (m_c - max m)), parts in order.  D / 4 threads
// per row, eight or sixteen rows of a tile per workgroup.
template <int D, int BM>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a) {
  constexpr int RPW = 1024 / D;
  constexpr int CHUNKS = BM < RPW ? 1 : BM / RPW;            // of a tile
  const int d = 4 * (threadIdx.x % (D / 4)), tiles = a.hkv * a.n_tiles, any = a.info[-1][0];
  for (int unit = blockIdx.x; unit < CHUNKS * tiles * a.batch; unit += gridDim.x) {
    const int at = unit / CHUNKS, b = at / tiles, kvh = (at - b * tiles) / a.n_tiles, tile = at - b * tiles - kvh * a.n_tiles;
    const int x0 = (unit - at * CHUNKS) * RPW, x = x0 + threadIdx.x / (D / 4);
    // (asked for together; what stands in a tile's entry counts only if it has rows)
    const i32x4 info = a.info[at];
    const int q_begin = a.cu ? a.cu[b] : (a.first + b) * a.q_len, n_q = a.cu ? min(a.cu[b + 1] - q_begin, a.q_len) : a.q_len;
    const int64_t n_rows = (int64_t)n_q * a.group;
    asm volatile("" : : "v"(any), "v"(info));
    if (any == 0) return;                                    // no tile was
    if ((int64_t)tile * BM + x0 >= n_rows) continue;
    const int parts = info[2];
    const int64_t row = (int64_t)tile * BM + x;
    if (parts < 2 || row >= n_rows) continue;
    const int64_t r0 = (int64_t)info[0] * BM + x, step = (int64_t)info[1] * BM;
    float m = -INFINITY, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < parts; c0 += 4) {                  // four at a time, their loads together (the last one again where there are fewer)
      float mc[4], lc[4];
      f32x4 oc[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int64_t r = r0 + min(c0 + v, parts - 1) * step;
        mc[v] = c0 + v < parts ? a.part_ml[2 * r] : -INFINITY;
        lc[v] = a.part_ml[2 * r + 1];
        oc[v] = *(const f32x4*)(a.part_o + r * D + d);
      }
      const float top = fmaxf(fmaxf(fmaxf(mc[0], mc[1]), fmaxf(mc[2], mc[3])), m);
      if (top == -INFINITY) continue;
      const float al = fast_exp2((m - top) * a.scale_log2);
      den *= al;
      num *= al;
      m = top;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float p = fast_exp2((mc[v] - m) * a.scale_log2);
        den += p * lc[v];
        num += p * oc[v];
      }
    }
    const float inv = 1.0f / den;
    const int64_t off = ((int64_t)(q_begin + row / a.group) * a.hq + (int64_t)kvh * a.group + row % a.group) * D + d;
    if (a.out_fp32) *(f32x4*)((float*)a.out + off) = num * inv;
    else *(u32x2*)((__bf16*)a.out + off) = u32x2{pack_bf16(num[0] * inv, num[1] * inv), pack_bf16(num[2] * inv, num[3] * inv)};
  }
}

namespace {
template <int D, int BM>
hipError_t launch_one(const CrossArgs& a, hipStream_t s) {
  if constexpr (BM <= 32) hipLaunchKernelGGL((cross_run_kernel<D, BM / 16>), dim3(a.n_wgs), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cross_tile_kernel<D, BM / 64>), dim3(a.n_wgs), dim3(256), 0, s, a);
  if (a.part_units == 0) return hipGetLastError();
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int RPW = 1024 / D, chunks = BM < RPW ? 1 : BM / RPW;
  const int units = chunks * a.hkv * a.n_tiles * a.batch;    // (below 2^31: see kCrossMostWgs)
  hipLaunchKernelGGL((cross_join_kernel<D, BM>), dim3(units < kCrossJoinWgs ? units : kCrossJoinWgs), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int D>
hipError_t launch_rows(const CrossArgs& a, int bm, hipStream_t s) {
  switch (bm) {
    case 16: return launch_one<D, 16>(a, s);
    case 32: return launch_one<D, 32>(a, s);
    case 64: return launch_one<D, 64>(a, s);
    default: return launch_one<D, 128>(a, s);
  }
}
}  // namespace

hipError_t launch_cross(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                        const flux_kv_cache& cache, void* out, hipStream_t s) {
  if (max_q_len == 0) return hipSuccess;
  const CrossPlan p = plan_cross(cfg, cache.batch, max_q_len, max_kv_len, c.partials_bytes);
  CrossArgs a = {};
  a.q = (const __bf16*)q;
  a.stride_b = cache.stride_b;
  a.stride_h = cache.stride_h;
  a.stride_t = cache.stride_t;
  a.q_len = max_q_len;
  a.capacity = max_kv_len < cache.capacity ? max_kv_len : cache.capacity;
  a.hq = cfg.n_q_heads;
  a.hkv = cfg.n_kv_heads;
  a.group = cfg.n_q_heads / cfg.n_kv_heads;
  a.n_tiles = p.tiles;
  a.n_wgs = (int)p.wgs;
  a.part_units = p.part_units;
  a.scale_log2 = (cfg.softmax_scale != 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)cfg.head_dim)) * kLog2e;
  a.out_fp32 = cfg.out_dtype;
  a.out = out;
  a.status = c.status;
  a.info = (i32x4*)c.partials + 1;
  a.part_o = (float*)((char*)c.partials + p.info_bytes);
  a.part_ml = a.part_o + (long long)p.part_units * p.bm * cfg.head_dim;
  for (a.first = 0; a.first < cache.batch; a.first += kCrossBatch) {
    a.batch = cache.batch - a.first < kCrossBatch ? cache.batch - a.first : kCrossBatch;
    a.cu = cu_q ? cu_q + a.first : nullptr;
    a.k = (const __bf16*)cache.k + a.first * cache.stride_b;
    a.v = (const __bf16*)cache.v + a.first * cache.stride_b;
    a.kv_len = cache.kv_len + a.first;
    const hipError_t e = cfg.head_dim == 128 ? launch_rows<128>(a, p.bm, s) : launch_rows<64>(a, p.bm, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace flux
