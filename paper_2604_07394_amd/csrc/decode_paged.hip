// flux_attn_decode_paged: decode attention (Eq. 1 / Eq. 2 with one query per sequence) over a cache of 8-bit pages.
//
//   o = sum_j p_j sv(j) cv_j / sum_j p_j,   p_j = exp(scale sk(j) (q . ck_j) - m)
// with the codes ck, cv of key j and the scales sk, sv of its page, so the scales cost a multiplication per score, not per
// code.  It is bound by reading the codes once from HBM: half the bytes of a bf16 cache.  The work of a (sequence, KV head)
// pair is the list of pages that hold a visible key, and the lists are shared out, cut and merged as those of the contiguous
// cache are (decode_cut.h): a page of 64 keys has the bytes of the 32-key blocks there.
//
// Measured, 32/8 heads of 128 unless said: 8 x 131072 keys 318 to 332 us, 6.5 to 6.75 TB/s of codes (a bf16 cache 605 to 626); 8 sparse lists
// of 4224 20.0 (28 to 30), of which 3.0 are the launch and the cut, 1 page numbers, 10.3 the streaming, 1.5 the last page, 1 the merge of the
// waves and 2.4 that of the parts; 32 ragged lists of 513 to 8400 at 28/4 heads 25.2 (38); one of 2001 at 8/2 heads of 64 7.3 (6.8:
// page numbers are a latency more).  16 runs of 5 queries behind 300 to 16000 keys
// 54.6 us, 240 MB: the loop over the pages takes more than half, the cut, two-block merges of waves and of parts the rest (the kernel for
// prompts took 63, a bf16 cache 95).
//
// Per wave, a page at a time:
//   S^T[key][q]  = ck[key][:] . Q[q][:]      MFMA 16x16x32 bf16.  A code is a bf16 value as it stands, so K is converted on its
//                                            way into the matrix cores (two codes an instruction) and the products are exact.
//                                            The order of d inside the contraction is free: lane (n, g) takes 16 codes of key
//                                            n, d = 64 kk + 16 g .., as two operands, so a load is 16 bytes
//   online softmax in the accumulator layout (one query per lane column, 16 keys per lane), in units of log2
//   O^T[d][q]   += cv^T[d][key] . (p sv)^T[key][q]   the codes of V go through wave-private LDS and come back with the
//                                            transposing 8-bit LDS read, 8 keys of one d per lane, in the order in which the
//                                            accumulators hold them; the weights as two bf16 terms (three for fp32 outputs)
#include <type_traits>

#include "decode_cut.h"
#include "paged.h"

namespace flux {

// What the cut is taken from.
struct PagedSplit {
  const int32_t* kv_len;
  const uint8_t* mode;
  int batch, capacity;    // capacity: positions that a table row can hold
  int sink_lim, win_blocks, blk_shift;   // SA geometry (see sa_geom)
  int max_pages;          // the host's bound on the pages of a list
  int pps, most_by_four, aligned_shift;  // see SplitArgs
  // us with 4 / 6 / 8 blocks of head dimension 128: 128 lists of 2 to 32 pages 64.4 / 60.2 / 60.5, 16 of 8 to 125 32.1 / 31.7 / 31.6, 32 ragged
  // ones of 28/4 heads 25.7 / 25.1 / 25.2
  static constexpr int seam_blocks(int head_dim) { return 768 / head_dim; }
};

// The pages of a list: all up to the query's, or, where `skip` > 0, the first `seam` (the sinks) and those from seam + skip on.
// Hidden in them: what lies behind the length, and of a sparse list the positions [s_end, tail_start).
struct PageList {
  int pages, seam, skip, s_end, tail_start;
};
__device__ __forceinline__ PageList page_list(const PagedSplit& s, int len, int md, int first) {   // first: position of the first query
  PageList r;
  r.s_end = min(len, s.sink_lim);
  const int lo = len > 0 ? window_start(first, s.blk_shift, s.win_blocks) : 0;
  r.tail_start = max(lo, r.s_end);
  if ((md & 1) != 0) r.tail_start = r.s_end;                 // FA: nothing is hidden
  r.seam = (r.s_end + 63) >> 6;
  r.skip = max((r.tail_start >> 6) - r.seam, 0);
  r.pages = ((len + 63) >> 6) - r.skip;
  return r;
}
__device__ __forceinline__ Seq load_counted(const PagedSplit& s, int b, bool& bad) {
  const int got = s.kv_len[b];
  Seq q;
  q.len = got < 0 ? 0 : min(got, s.capacity);
  q.md = s.mode[b] != 0 ? 1 : 0;
  q.nb = page_list(s, q.len, q.md, q.len - 1).pages;
  bad |= got != q.len || q.nb > s.max_pages;
  q.nb = min(q.nb, s.max_pages);
  return q;
}

// Runs of a few queries per sequence (batches of up to 64): every lane holds the number of its sequence's.
struct RunSplit : PagedSplit {
  int n_q;
  int max_kv_len;         // a longer sequence is reported, also where the bound holds all pages of its list
};
__device__ __forceinline__ Seq load_counted(const RunSplit& s, int b, bool& bad) {
  const int got = s.kv_len[b];
  Seq q;
  q.len = got < 0 ? 0 : min(got, s.capacity);
  q.md = s.mode[b] != 0 ? 1 : 0;
  const int n = s.n_q < 0 ? 0 : min(s.n_q, q.len);
  q.nb = n > 0 ? page_list(s, q.len, q.md, q.len - n).pages : 0;
  bad |= got != q.len || n != s.n_q || q.len > s.max_kv_len;   // (or the list may have more pages than the bound)
  q.nb = min(q.nb, s.max_pages);
  return q;
}

struct PagedDecodeArgs {
  const __bf16* q;        // [B, Hq, D]
  const char *k, *v;
  const float *k_scale, *v_scale;
  int64_t stride_p, stride_h, stride_t;
  const int32_t* table;
  int table_pages, n_pages;
  PagedSplit sp;
  int hq, hkv, group, qblocks, rpu;      // see DecodeArgs in decode.hip; runs: one pair per KV head, rpu = max_q * group
  const int32_t* cu_q;    // runs only
  int max_q, max_kv_len;  // ... queries of a run that are computed, and the host's bound on the lengths
  Reciprocal by_group;
  float scale_log2;
  float* part_o;
  float* part_ml;         // reference (log2 units) and weight sum
  uint32_t* status;
  uint32_t* arrived;
  void* out;
};

typedef __attribute__((__vector_size__(2 * sizeof(int)))) int i32x2;

// 8 codes times a power of two as bf16 values
__device__ __forceinline__ bf16x8 unpack8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)});
}

// FP32: the outputs are fp32, and a weight takes three bf16 terms (bf16 outputs: two).
// QB: 0, one query per sequence.  Otherwise the last n_q(b) positions of every sequence are queries (a step of speculative decoding),
// whose rows, token by token the heads of a group, take QB blocks of 16 columns: K and V are read once for all of them.
// (Two blocks at head dimension 128 take more registers than two workgroups per CU leave.)
template <int D, bool NT, int W, bool FP32, int QB>
__global__ __launch_bounds__(64 * W, runs_per_cu(D, QB)) void paged_decode_kernel(PagedDecodeArgs a) {
  constexpr bool RUN = QB > 0;
  constexpr int NB = RUN ? QB : 1;    // blocks of 16 columns
  constexpr int KK = D / 64;          // 16-byte K loads per lane and 16 keys
  constexpr int DB = D / 16;          // 16-wide output blocks over the head dimension
  constexpr int CPR = D / 16;         // 16-byte chunks per row
  constexpr int RPL = 64 / CPR;       // V rows per wave-wide load
  constexpr int VL = 64 / RPL;        // V loads per lane and page
  // LDS row of V and block of 16 of them (bytes): the 8 rows of each of two blocks that a pass of the transposing read takes lie in
  // different banks
  constexpr int VROW = D + 16, VBLOCK = 16 * VROW + 128;
  constexpr int RED = D + 4;          // floats from one row of the merge buffer to the next
  constexpr int VWAVE = 4 * VBLOCK - 128, STAGING = W * VWAVE, RED_BYTES = W * 16 * (RED + 2) * 4;
  __shared__ __attribute__((aligned(16))) char smem[STAGING > RED_BYTES ? STAGING : RED_BYTES];
  __shared__ int last_of_pair;

  const int tid = threadIdx.x;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int g = l >> 4, n = l & 15;
  const int wg = blockIdx.x;

  // ---- the range of this workgroup
  __shared__ u32x2 s_seq[W == 8 ? kDecodeFewWgs : kDecodeTable];   // (a call of eight waves has no more sequences than workgroups)
  SeqTable* const seqs = (SeqTable*)s_seq;
  Lanes lanes;
  typedef typename std::conditional<RUN, RunSplit, PagedSplit>::type Split;
  Split split;
  static_cast<PagedSplit&>(split) = a.sp;
  int q_begin_mine = 0;
  if constexpr (RUN) {
    split.max_kv_len = a.max_kv_len;
    split.n_q = 0;
    if (l < a.sp.batch) {
      q_begin_mine = a.cu_q[l];
      split.n_q = q_begin_mine < 0 ? -1 : a.cu_q[l + 1] - q_begin_mine;
    }
  }
  const Cut cut = find_cut<D, W>(split, l, w, seqs, lanes);
  if constexpr (W == 8) __builtin_assume(cut.align > 0);
  if (wg == 0 && lanes.bad) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_LENGTH);
  // rows of sequences without keys are zero: shared out over the workgroups
  auto zero_rows = [&]() __attribute__((always_inline)) {
    if constexpr (RUN) return;                               // (a run is not longer than what is cached)
    if (__builtin_amdgcn_ballot_w64(lanes.run > 1 || (l < a.sp.batch && lanes.q.nb == 0)) == 0) return;
    for (int b = wg; b < a.sp.batch; b += (int)gridDim.x) {
      const int i = b / lanes.run, j = b - i * lanes.run;
      if ((lanes.run == 1 ? __builtin_amdgcn_readlane(lanes.q.nb, i) : seq_at(split, seqs, lanes.run, i, j).nb) != 0) continue;
      const int64_t off = (int64_t)b * a.hq * D;
      for (int x = 8 * tid; x < a.hq * D; x += 8 * 64 * W) {
        const u32x4 zero = {0, 0, 0, 0};
        if constexpr (FP32) {
          *(u32x4*)((float*)a.out + off + x) = zero;
          *(u32x4*)((float*)a.out + off + x + 4) = zero;
        } else {
          *(u32x4*)((__bf16*)a.out + off + x) = zero;
        }
      }
    }
  };
  if (wg >= cut_wgs(cut) || cut.total == 0) {                // nothing to do: uniform for the whole workgroup
    zero_rows();
    return;
  }
  int at = range_begin(cut, wg);
  const int range_end = range_begin(cut, wg + 1);
  Place place = find_place(split, cut, lanes, l, seqs, at);
  const int rows_at = at - place.begin;
  int pair = __builtin_amdgcn_readfirstlane((int)((float)rows_at / (float)place.nb));   // (put right below: the quotient may be off by one)
  pair -= pair * place.nb > rows_at ? 1 : 0;
  pair += (pair + 1) * place.nb <= rows_at ? 1 : 0;

  // ---- the part in work: pages [x0, x1) of the list of (sequence place.b, pair), page x0 + w, x0 + w + W, ... by this wave
  int x0, x1, p;
  PageList list;
  const char *kbase, *vbase;
  const float *kscale, *vscale;
  const int32_t* pages;
  int first_pos, run_rows;                                   // position of the first query, rows of the run that are computed
  auto set_part = [&]() __attribute__((always_inline)) {
    const int kvh = a.qblocks == 1 ? pair : pair / a.qblocks;
    const int begin = place.begin + pair * place.nb;
    x0 = at - begin;
    x1 = min(place.real, range_end - begin);
    first_pos = place.len - 1;
    if constexpr (RUN) {
      const int n_q = min(__builtin_amdgcn_readlane(split.n_q, place.b), place.len);
      first_pos = place.len - n_q;
      run_rows = min(n_q, a.max_q) * a.group;
    }
    list = page_list(a.sp, place.len, place.md, first_pos);
    kbase = a.k + (int64_t)kvh * a.stride_h;
    vbase = a.v + (int64_t)kvh * a.stride_h;
    kscale = a.k_scale + kvh;
    vscale = a.v_scale + kvh;
    pages = a.table + (int64_t)place.b * a.table_pages;
  };
  set_part();

  // Lane i holds what is known of the wave's i-th page of 64: asked for 64 at a time, so that the loop waits for no table.
  // ids: those in work; ids_next: the ones behind them.
  int ids, ids_next;
  float ks, vs;
  auto load_ids = [&](int from) __attribute__((always_inline)) -> int {
    const int at_page = min(from + W * l, x1 - 1);
    return pages[at_page + (at_page >= list.seam ? list.skip : 0)];
  };
  auto load_scales = [&]() __attribute__((always_inline)) {
    const int64_t page = (uint32_t)ids < (uint32_t)a.n_pages ? ids : 0;
    ks = kscale[page * a.hkv];
    vs = vscale[page * a.hkv];
  };

  auto ld = [](const u32x4* x) -> u32x4 { return NT ? __builtin_nontemporal_load(x) : *x; };
  u32x4 kreg[4][KK], vreg[VL];
  const uint32_t k_lane = n * (uint32_t)a.stride_t + 16 * g;
  const uint32_t v_lane = (l / CPR) * (uint32_t)a.stride_t + 16 * (l % CPR);
  // the page's first position, and whether all of its positions are visible
  auto first_of = [&](int x) __attribute__((always_inline)) { return (x + (x >= list.seam ? list.skip : 0)) << 6; };
  auto is_full = [&](int pos) __attribute__((always_inline)) {   // (for loads: rows that some query sees are all of them)
    return pos + 64 <= place.len && (list.tail_start == list.s_end || pos + 64 <= list.s_end || pos >= list.tail_start);
  };
  auto load_page = [&](int x, int id) __attribute__((always_inline)) {   // both wave-uniform
    const int64_t page = (uint32_t)id < (uint32_t)a.n_pages ? id : 0;    // (one that is not there is left out below)
    const char* const kp = kbase + page * a.stride_p;
    const char* const vp = vbase + page * a.stride_p;
    const int pos = first_of(x);
    if (is_full(pos)) {
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kreg[sb][kk] = ld((const u32x4*)(kp + 16 * sb * a.stride_t + 64 * kk + k_lane));
#pragma unroll
      for (int i = 0; i < VL; ++i) vreg[i] = ld((const u32x4*)(vp + i * RPL * a.stride_t + v_lane));
    } else {
      // rows that are hidden are not read: the page's first visible one stands in for them, with weight zero
      const int stand_in = pos < list.s_end || pos >= list.tail_start ? 0 : list.tail_start - pos;
      auto row_of = [&](int r) __attribute__((always_inline)) {
        const int key = pos + r;
        return key < place.len && (list.tail_start == list.s_end || key < list.s_end || key >= list.tail_start) ? r : stand_in;
      };
      uint32_t krow[4], vrow[VL];
#pragma unroll
      for (int sb = 0; sb < 4; ++sb) krow[sb] = row_of(16 * sb + n) * (uint32_t)a.stride_t + 16 * g;
#pragma unroll
      for (int i = 0; i < VL; ++i) vrow[i] = row_of(i * RPL + l / CPR) * (uint32_t)a.stride_t + 16 * (l % CPR);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kreg[sb][kk] = ld((const u32x4*)(kp + 64 * kk + krow[sb]));
#pragma unroll
      for (int i = 0; i < VL; ++i) vreg[i] = ld((const u32x4*)(vp + vrow[i]));
    }
  };

  FLUX_LDS char* const vs_lds = (FLUX_LDS char*)smem + w * VWAVE;
  bf16x8 qf[NB][2 * KK];
  int i_mine[NB], w_lo_mine[NB], w_lo_last = 0;              // runs: position of a column's query, start of its window, of the last one's
  int id_now;                                                // number of the page in flight
  auto begin_part = [&]() __attribute__((always_inline)) {
    p = x0 + w;
    ids = ids_next = 0;
    ks = vs = 0.f;
    if (p < x1) {
      ids = load_ids(p);
      ids_next = load_ids(p + 64 * W);
      id_now = __builtin_amdgcn_readfirstlane(ids);
      load_page(p, id_now);
      load_scales();
    }
    __builtin_amdgcn_sched_barrier(0);
    // Q operand: lane (n, g) holds d = 64 kk + 16 g + 8 h .. +7 of its query row in qf[2 kk + h]: of query head kvh * group + 16 *
    // qb + n, or of the run's row 16 * qb + n (columns past the last one repeat a row; what they give is left out at the end)
    const int kvh = a.qblocks == 1 ? pair : pair / a.qblocks, qb = a.qblocks == 1 ? 0 : pair % a.qblocks;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const __bf16* qrow;
      if constexpr (RUN) {
        const int r = min(16 * b + n, run_rows - 1), tok = quotient(r, a.by_group);
        i_mine[b] = first_pos + tok;
        w_lo_mine[b] = place.md & 1 ? 0 : window_start(i_mine[b], a.sp.blk_shift, a.sp.win_blocks);
        qrow = a.q + ((int64_t)(__builtin_amdgcn_readlane(q_begin_mine, place.b) + tok) * a.hq + (int64_t)kvh * a.group + (r - tok * a.group)) * D;
      } else {
        const int qh = 16 * qb + n;
        qrow = a.q + ((int64_t)place.b * a.hq + (int64_t)kvh * a.group + (qh < a.group ? qh : 0)) * D;
      }
#pragma unroll
      for (int i = 0; i < 2 * KK; ++i) qf[b][i] = *(const bf16x8*)(qrow + 64 * (i >> 1) + 16 * g + 8 * (i & 1));
    }
    if constexpr (RUN) w_lo_last = place.md & 1 ? 0 : window_start(first_pos + quotient(run_rows - 1, a.by_group), a.sp.blk_shift, a.sp.win_blocks);
    __builtin_amdgcn_sched_barrier(0);
  };
  begin_part();

  for (;;) {
    // (a part of pages that are not there leaves this reference and a weight sum of almost nothing: zero rows)
    float m_run[NB], l_run[NB];
    f32x4 o[DB][NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      m_run[b] = -1e30f;
      l_run[b] = 0.f;
#pragma unroll
      for (int i = 0; i < DB; ++i) o[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int i = 0; p < x1; ++i) {
      const int pos = first_of(p), id = id_now;
      const float c = fmaxf(a.scale_log2 * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), i)), 0x1p-126f);   // (not 0: a masked score is -inf times this)
      // the scale of V: its power of two goes into the conversion, the rest, 1 <= r < 2, into the weights
      const uint32_t v_bits = max((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, vs), i), 0x00800000u);
      const float v_power = __builtin_bit_cast(float, v_bits & 0x7F800000u);
      float log_rest = 0.f, inv_rest = 1.f;
      if (__builtin_expect((v_bits & 0x007FFFFFu) != 0, 0)) {   // (uniform; the scales that the append writes are powers of two)
        const float rest = __builtin_bit_cast(float, (v_bits & 0x007FFFFFu) | 0x3F800000u);
        log_rest = __builtin_amdgcn_logf(rest);
        inv_rest = 1.0f / rest;
      }
#pragma unroll
      for (int j = 0; j < VL; ++j) *(FLUX_LDS u32x4*)(vs_lds + (j * RPL / 16) * VBLOCK + (j * RPL % 16 + l / CPR) * VROW + 16 * (l % CPR)) = vreg[j];
      // ---- scores: s[sb][b][i] is key 16 * sb + 4 * g + i of the page against query column (b, n)
      f32x4 s[4][NB];
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int b = 0; b < NB; ++b) s[sb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < 2 * KK; ++kk)
#pragma unroll
        for (int sb = 0; sb < 4; ++sb) {
          const bf16x8 kf = unpack8(kreg[sb][kk >> 1][2 * (kk & 1)], kreg[sb][kk >> 1][2 * (kk & 1) + 1], 1.0f);
#pragma unroll
          for (int b = 0; b < NB; ++b) s[sb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[b][kk], s[sb][b], 0, 0, 0);
        }
      __builtin_amdgcn_sched_barrier(0);
      const int next = x1 - p > W ? p + W : x1;
      if (next < x1) {
        id_now = i < 63 ? __builtin_amdgcn_readlane(ids, i + 1) : __builtin_amdgcn_readfirstlane(ids_next);
        load_page(next, id_now);
        if (i == 63) {                                       // the next 64 pages
          ids = ids_next;
          load_scales();
          ids_next = load_ids(next + 64 * W);
          i = -1;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      p = next;
      if ((uint32_t)id >= (uint32_t)a.n_pages) {             // (uniform)
        if (l == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_PAGE);
        continue;
      }
      if constexpr (RUN) {
        const bool all = pos + 63 <= first_pos && ((place.md & 1) != 0 || pos + 64 <= a.sp.sink_lim || pos >= w_lo_last);
        if (!all) {                                          // some column does not see all of the page
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int hi = i_mine[b] - pos - 4 * g, lo = w_lo_mine[b] - pos - 4 * g, sl = a.sp.sink_lim - pos - 4 * g;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int k = 16 * (j >> 2) + (j & 3);
              if (!((k <= hi) & ((k < sl) | (k >= lo)))) s[j >> 2][b][j & 3] = -INFINITY;
            }
          }
        }
      } else if (!is_full(pos)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int key = pos + 16 * (j >> 2) + 4 * g + (j & 3);
          if (key >= place.len || (list.tail_start != list.s_end && key >= list.s_end && key < list.tail_start)) s[j >> 2][0][j & 3] = -INFINITY;
        }
      }
      // ---- weights against the reference that the accumulators refer to, without looking for the page's maximum first: any
      // reference gives the same quotient.  Only where a weight leaves the guarded range, or a query has no reference yet, the
      // maximum is taken (over the 4 lane groups of a query), the references move there and the weights are taken again.
      // TERMS bf16 values make a weight: two leave 2^-16 of it (see decode.hip), three 2^-24, which is what an fp32 output holds
      // (8/2 heads of 64, 2001 keys: 2-norm of the error 3.7e-6 of the result's with two).
      // Runs take as many, so that a drafted token is scored as the decode step that it stands for would score it.  (With a term less 16
      // runs of 5 behind 300 to 16000 keys took 53.1 us for 54.6, 64 of them 158 for 166; 2-norm of the error 2.02e-3 and
      // now 1.65e-3, which is the rounding of a bf16 output.)
      constexpr int TERMS = FP32 ? 3 : 2;
      uint32_t pk[NB][TERMS][8];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float e[16], psum;
        auto weights = [&]() __attribute__((always_inline)) {
          const float shift = log_rest - m_run[b];
          psum = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            e[j] = fast_exp2(__builtin_fmaf(s[j >> 2][b][j & 3], c, shift));
            psum += e[j];
          }
        };
        weights();
        if (__builtin_amdgcn_ballot_w64(!(psum < kPagedGuard)) != 0) {
          float m = s[0][b][0];
#pragma unroll
          for (int j = 1; j < 16; ++j) m = fmaxf(m, s[j >> 2][b][j & 3]);
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m_run[b], fmaxf(m, __shfl_xor(m, 32)) * c);
          const float alpha = fast_exp2(m_run[b] - m);
          m_run[b] = m;
          l_run[b] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db][b] *= alpha;
          weights();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float x = e[2 * j], y = e[2 * j + 1];
#pragma unroll
          for (int t = 0; t < TERMS - 1; ++t) {              // the upper bits of what is left
            pk[b][t][j] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);
            x -= bf16_lo(pk[b][t][j]);
            y -= bf16_hi(pk[b][t][j]);
          }
          pk[b][TERMS - 1][j] = pack_bf16(x, y);
        }
        l_run[b] = __builtin_fmaf(psum, inv_rest, l_run[b]);
      }
      // ---- O^T += V^T P^T, 32 keys at a time: lane (n, g) has the keys 32 kh + 4 g + (0..3) and 16 more of P, and takes the same of V
#pragma unroll
      for (int kh = 0; kh < 2; ++kh) {
        const int j = n >> 1;
        FLUX_LDS char* const src = vs_lds + (2 * kh + (j >> 2)) * VBLOCK + (4 * g + (j & 3)) * VROW + 8 * (n & 1);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const i32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((FLUX_LDS i32x2*)(src + 16 * db));
          const bf16x8 vf = unpack8((uint32_t)t[0], (uint32_t)t[1], v_power);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < TERMS; ++i)
              o[db][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, u32x4{pk[b][i][4 * kh], pk[b][i][4 * kh + 1], pk[b][i][4 * kh + 2], pk[b][i][4 * kh + 3]}), o[db][b], 0, 0, 0);
        }
      }
    }

    __builtin_amdgcn_s_waitcnt(0x0F70);                     // vmcnt(0): nothing is in flight any more
    // ---- what the end of this part needs, and on to the next one: its first page is in flight meanwhile
    const int nq = RUN ? run_rows : min(16, a.group - (a.qblocks == 1 ? 0 : 16 * (pair % a.qblocks)));
    const int64_t out0 = ((int64_t)(RUN ? __builtin_amdgcn_readlane(q_begin_mine, place.b) : place.b) * a.hq +
                          (int64_t)(a.qblocks == 1 ? pair : pair / a.qblocks) * a.group + (a.qblocks == 1 ? 0 : 16 * (pair % a.qblocks))) * D;
    const int list0 = place.begin + pair * place.nb;
    const bool empty = x0 >= x1;                            // (the range begins in what is only counted behind a list)
    const bool whole = empty || (x0 == 0 && x1 == place.real);   // the pair lies in this range
    const int first = whole ? wg : range_of(cut, list0);
    const int parts = whole ? 1 : range_of(cut, list0 + place.real - 1) - first + 1;
    at = x1 < place.real ? range_end : list0 + place.nb;
    const bool more = W == 4 && at < range_end;
    if (more) {
      if (++pair == a.sp.pps) {
        place = find_place(split, cut, lanes, l, seqs, place.begin + a.sp.pps * place.nb);   // (the next one that has keys)
        pair = 0;
      }
      set_part();
      begin_part();
    }

    // ---- merge the waves through LDS, a block of columns at a time: red[w][n][0..D-1] = O, ml[w][n] = (m, l); only the columns of
    // rows that exist
    FLUX_LDS float* red = (FLUX_LDS float*)smem;
    FLUX_LDS f32x2* ml = (FLUX_LDS f32x2*)(red + W * 16 * RED);
    auto store_out = [&](int qi, int d, f32x4 r) __attribute__((always_inline)) {
      int64_t off = out0 + d;
      if constexpr (RUN) {
        const int tok = quotient(qi, a.by_group);
        off += (int64_t)(tok * a.hq + qi - tok * a.group) * D;
      } else {
        off += qi * D;
      }
      if constexpr (FP32) *(f32x4*)((float*)a.out + off) = r;
      else *(u32x2*)((__bf16*)a.out + off) = u32x2{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
    };
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int in_block = min(16, nq - 16 * b), row0 = part_place(first, wg - first) * a.rpu + 16 * b;
      if (RUN && in_block <= 0) break;                      // (uniform)
      float l_tot = l_run[b];
      l_tot += __shfl_xor(l_tot, 16);
      l_tot += __shfl_xor(l_tot, 32);
      __syncthreads();                                      // every wave is done with its V staging, or with the block before
      if (n < in_block) {
        FLUX_LDS float* mine = red + (w * 16 + n) * RED + 4 * g;
#pragma unroll
        for (int db = 0; db < DB; ++db) *(FLUX_LDS f32x4*)(mine + 16 * db) = o[db][b];
        if (g == 0) ml[w * 16 + n] = f32x2{m_run[b], l_tot};
      }
      __syncthreads();
      for (int idx = tid; !empty && idx < in_block * (D / 4); idx += 64 * W) {
        const int qi = idx / (D / 4), d = 4 * (idx % (D / 4));
        f32x2 x[W];
        float m = -1e30f;
#pragma unroll
        for (int ww = 0; ww < W; ++ww) {
          x[ww] = ml[ww * 16 + qi];
          m = fmaxf(m, x[ww][0]);
        }
        f32x4 val = {0.f, 0.f, 0.f, 0.f};
        float den = 0x1p-126f;                              // (no page there: 0 / this)
#pragma unroll
        for (int ww = 0; ww < W; ++ww) {
          const float wgt = fast_exp2(x[ww][0] - m);        // 0 for idle waves beside others
          val += wgt * *(FLUX_LDS f32x4*)(red + (ww * 16 + qi) * RED + d);
          den += wgt * x[ww][1];
        }
        if (whole) {                                        // nothing to merge with
          store_out(16 * b + qi, d, f32x4{val[0] / den, val[1] / den, val[2] / den, val[3] / den});
        } else {
          store16_dev(a.part_o, ((row0 + qi) * D + d) * 4, val);
          if (d == 0) __hip_atomic_store((unsigned long long*)(a.part_ml + 2 * (row0 + qi)), __builtin_bit_cast(unsigned long long, f32x2{m, den}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
    if (!whole) {
      // ---- the part that arrives last merges the pair
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wave's rows have reached the point all XCDs see
      __syncthreads();
      if (tid == 0) {
        uint32_t* count = a.arrived + kCounterStride * (1 + kDecodeGather + first);   // (a range holds the beginning of one unfinished pair at most)
        const bool done = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
        if (done) *count = 0;                               // ready for the next call on this stream
        last_of_pair = done;
      }
      __syncthreads();
      if (last_of_pair) merge_pair<D, true, W>(a.part_o, a.part_ml, a.rpu, first, parts, nq, 1.0f, smem, w, l, store_out);
    }
    if (!more) break;
    __syncthreads();                                        // the merge buffer becomes V staging again
  }
  zero_rows();
}

namespace {
template <bool NT, int W, int QB>
void launch_kernel(const PagedDecodeArgs& a, const flux_attn_cfg& cfg, int wgs, hipStream_t s) {
  const dim3 grid(wgs), block(64 * W);
  if (cfg.head_dim == 128) {
    if (cfg.out_dtype != 0) hipLaunchKernelGGL((paged_decode_kernel<128, NT, W, true, QB>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_decode_kernel<128, NT, W, false, QB>), grid, block, 0, s, a);
  } else {
    if (cfg.out_dtype != 0) hipLaunchKernelGGL((paged_decode_kernel<64, NT, W, true, QB>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_decode_kernel<64, NT, W, false, QB>), grid, block, 0, s, a);
  }
}

// What a call of one query per sequence and one of runs have in common.  `rows` leave a part, which go to `part_rows`.
PagedDecodeArgs decode_args(const Ctx& c, const flux_attn_cfg& cfg, const void* q, int max_kv_len, const flux_paged_kv& kv,
                            const flux_page_table& pt, const uint8_t* mode, void* out, const DecodePlan& plan, float* part_rows) {
  PagedDecodeArgs a;
  a.q = (const __bf16*)q;
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
  const SaGeom geom = sa_geom(cfg);
  a.sp.kv_len = pt.kv_len;
  a.sp.mode = mode;
  a.sp.batch = pt.batch;
  a.sp.capacity = pt.table_pages * kPageTokens;
  a.sp.sink_lim = geom.sink_lim;
  a.sp.win_blocks = geom.win_blocks;
  a.sp.blk_shift = geom.shift;
  a.sp.max_pages = pages_of(max_kv_len);
  a.sp.pps = plan.pps;
  a.sp.most_by_four = plan.most_by_four;
  a.sp.aligned_shift = plan.aligned_shift;
  a.hq = cfg.n_q_heads;
  a.hkv = cfg.n_kv_heads;
  a.group = cfg.n_q_heads / cfg.n_kv_heads;
  a.by_group = reciprocal((uint32_t)a.group);
  a.qblocks = plan.pps / cfg.n_kv_heads;
  a.rpu = plan.rpu;
  a.cu_q = nullptr;
  a.max_q = 1;
  a.max_kv_len = max_kv_len;
  a.scale_log2 = (cfg.softmax_scale != 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)cfg.head_dim)) * kLog2e;
  a.part_o = part_rows;
  a.part_ml = a.part_o + (size_t)2 * plan.wgs * plan.rpu * cfg.head_dim;
  a.status = c.status;
  a.arrived = c.decode_counters;
  a.out = out;
  return a;
}

// rows that are evicted before the next step are fetched with nontemporal loads (see launch_decode)
bool nontemporal(const flux_attn_cfg& cfg, const flux_page_table& pt, int max_kv_len) {
  return 2.0 * pt.batch * cfg.n_kv_heads * cfg.head_dim * (double)max_kv_len > 64.0 * 1024 * 1024;
}
}  // namespace

hipError_t launch_decode_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, int max_kv_len, const flux_paged_kv& kv,
                               const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s) {
  const DecodePlan plan = plan_decode_paged(cfg, pt.batch, max_kv_len);
  const PagedDecodeArgs a = decode_args(c, cfg, q, max_kv_len, kv, pt, mode, out, plan, plan.in_partials ? c.partials + decode_rows_at(plan, false) : c.small);
  if (plan.waves == 8) launch_kernel<false, 8, 0>(a, cfg, plan.wgs, s);
  else if (nontemporal(cfg, pt, max_kv_len)) launch_kernel<true, 4, 0>(a, cfg, plan.wgs, s);
  else launch_kernel<false, 4, 0>(a, cfg, plan.wgs, s);
  return hipGetLastError();
}

hipError_t launch_runs_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                             const flux_paged_kv& kv, const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s) {
  const DecodePlan plan = plan_runs_paged(cfg, pt.batch, max_q_len, max_kv_len);
  PagedDecodeArgs a = decode_args(c, cfg, q, max_kv_len, kv, pt, mode, out, plan, c.partials);
  a.cu_q = cu_q;
  a.max_q = max_q_len;
  const bool nt = nontemporal(cfg, pt, max_kv_len);
  if (plan.rpu <= 16) {
    if (nt) launch_kernel<true, 4, 1>(a, cfg, plan.wgs, s);
    else launch_kernel<false, 4, 1>(a, cfg, plan.wgs, s);
  } else {
    if (nt) launch_kernel<true, 4, 2>(a, cfg, plan.wgs, s);
    else launch_kernel<false, 4, 2>(a, cfg, plan.wgs, s);
  }
  return hipGetLastError();
}

}  // namespace flux
