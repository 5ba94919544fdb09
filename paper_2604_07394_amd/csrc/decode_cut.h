// How a decode call is shared out over the chip, and how the parts of a list are merged: what the decode kernels of the
// contiguous and of the paged cache have in common.  A call is described by a struct `s` with the members batch, pps,
// most_by_four and aligned_shift (see SplitArgs in decode.hip), for which load_counted(s, b, bad) says how many blocks
// sequence b has (32 keys of a bf16 cache or a page of 64 keys of an 8-bit one, the same bytes either way), and
// S::seam_blocks(head_dim) how many of them going on to the next list counts.
#pragma once

#include <utility>

#include "flux_internal.h"

namespace flux {

// ---- the cut.  Blocks of all pairs, sequence by sequence and pair by pair, numbered from 0.  While they are few (one per
// wave of two workgroups per CU) every list is rounded up to a multiple of 4 and a workgroup takes 4, so that none
// crosses from one pair into the next; 8 where every list has no more than that (nothing to merge) or more than 64 (half
// the rows to merge).  (Calls of eight waves: see kDecodeFewWgs.)  Of 256 to 512 short lists it takes one each.  Otherwise the
// lists lie end to end, and workgroup u of 256 or 512 takes [range_begin(u), range_begin(u + 1)): equal shares not of the
// blocks but of what they take, for which a list is counted as a multiple of the waves and some blocks more (see find_cut).
struct Cut {
  int total;        // blocks
  int shift;        // equal shares: log2 of the workgroups
  int align;        // log2 of the blocks that a workgroup takes of a list; 0: an equal share of all lists
  int round, pad;   // a list of nb blocks is counted as nb rounded up to a multiple of round + 1, and pad more
};
__device__ __forceinline__ int cut_wgs(Cut c) { return c.align > 0 ? c.total >> c.align : 1 << c.shift; }
__device__ __forceinline__ int range_begin(Cut c, int u) {
  return c.align > 0 ? u << c.align : (int)(((unsigned long long)(unsigned)u * (unsigned)c.total) >> c.shift);
}
// the workgroup whose range holds block x
__device__ __forceinline__ int range_of(Cut c, int x) {
  if (c.align > 0) return x >> c.align;
  int u = min((int)((float)x * ((float)(1 << c.shift) / (float)c.total)), (1 << c.shift) - 1);
  while (range_begin(c, u) > x) --u;
  while (range_begin(c, u + 1) <= x) ++u;
  return u;
}
// Where the rows of part `i` of a pair go whose first part lies in the range of workgroup `first`: a range holds at most one
// part that its pair goes on behind and one that its pair began before.
__device__ __forceinline__ int part_place(int first, int i) { return i == 0 ? 2 * first + 1 : 2 * (first + i); }

// ---- the sequences of a call.  Lane i of every wave looks after `run` of them from i * run on: one each in a batch of up to
// 64, which stays in registers; larger batches of up to kDecodeTable are read once, by all waves together, into a table in LDS.
// (Read in groups of 64, each behind the one before it, for both passes of the cut and for every list that a range goes on to:
// us before / now, 1000 lists of 20 to 200 keys at 28/4 heads 119.1 / 107.2, 512 of 50 to 300 at 32/8 130.9 / 127.0.)
constexpr int kDecodeTable = 2048;
struct Seq {
  int len, md, nb;  // rows, mode bits (see load_seq), blocks
};
typedef FLUX_LDS u32x2 SeqTable;   // [run][64]: sequence i * run + j is entry j * 64 + i; its rows, and 4 * blocks + mode bits

template <class S>
__device__ __forceinline__ Seq seq_at(const S& s, const SeqTable* table, int run, int i, int j) {
  if (run * 64 <= kDecodeTable) {
    const u32x2 e = table[j * 64 + i];
    return Seq{(int)e[0], (int)(e[1] & 3), (int)(e[1] >> 2)};
  }
  bool bad;
  return load_counted(s, i * run + j, bad);
}

struct Lanes {
  Seq q;            // batches of up to 64: this lane's sequence
  int run;          // sequences of a lane
  int incl;         // blocks up to and including this lane's
  bool bad;         // this lane saw a clamp trip
  bool merged;      // calls of eight waves: some list takes more than one workgroup
};
__device__ __forceinline__ int counted(Cut c, int nb) { return nb > 0 ? ((nb + c.round) & ~c.round) + c.pad : 0; }

// (called by all waves of a workgroup, w: this one, of W)
template <int D, int W, class S>
__device__ __forceinline__ Cut find_cut(const S& s, int lane, int w, SeqTable* table, Lanes& r) {
  // Going on from one list to the next, a workgroup stands still for a memory latency and the merge of its waves, about as long
  // as four blocks of head dimension 128 take, and for up to three waves without a block.  Ranges of equally many blocks that
  // held whole lists, such as the eight sparse ones of a sequence among long ones, were the last ones of their call: us
  // before / now per layer, 32/8 heads of 128: 13 lists of 1223 to 15370 keys, half of them cut at 144, 42.5 / 32.0, 32 ragged ones at
  // 28/4 heads 40.1 / 36.9, 16 ring lists of 2112 at 28/4 25.0 / 23.7, 13 of 144 to 13696 37.1 / 33.7, 29 of 139 to 2305 26.8
  // / 26.3, 21 of 296 to 4373 at head dimension 64 23.4 / 18.7.  (3 to 6 blocks, and 5 to 12 at head dimension 64, differ by 2 %.)
  // With two workgroups per CU (see kLists) the other one streams meanwhile, and a block takes twice as long: a list of head
  // dimension 128 is a multiple of two and two blocks more then.  us with four and four / so: 104 lists of 1 to 4 keys among 24 of 2000
  // 53.0 / 48.7, 128 of 50 to 299 31.2 / 30.4, 1000 of 20 to 199 at 28/4 heads 73.4 / 72.1, 53 of 36 to 1044 at 16/8 36.3 / 35.5.
  // At head dimension 64 there is nothing in it: 136 of 6 to 200 18.9 / 20.4, 122 of 39 to 1278 45.9 / 44.9.
  // (Over pages the next list's page numbers are a memory latency more: S says how many blocks a seam counts.)
  constexpr int kSeam = S::seam_blocks(D);
  // Two workgroups per CU where there are as many lists as CUs, since at most seams the other one goes on (us with one / two,
  // 32/8 heads of 128: 128 lists of 300 keys 39.9 / 34.5, 128 of 100 to 3000 61.8 / 52.6, 1000 of 20 to 200 at 28/4 heads 107 /
  // 82; but 16 lists of 2112, 128 in all, 29.4 / 31.0, 8 x 131072 629 / 665).  At head dimension 64 from a quarter of that on:
  // one workgroup has half the bytes in flight there (21 sequences of 296 to 4373 keys 22.8 / 20.5).
  constexpr int kLists = D == 64 ? 64 : 256;
  r.run = (s.batch + 63) >> 6;
  r.bad = false;
  r.q = Seq{0, 1, 0};
  if (__builtin_expect(r.run == 1, 1)) {
    if (lane < s.batch) r.q = load_counted(s, lane, r.bad);
  } else if (r.run * 64 <= kDecodeTable) {
    for (int j = w; j < r.run; j += W) {
      Seq q = {0, 1, 0};
      bool bad = false;
      if (lane * r.run + j < s.batch) q = load_counted(s, lane * r.run + j, bad);
      table[j * 64 + lane] = u32x2{(uint32_t)q.len, (uint32_t)(4 * q.nb + q.md)};
      r.bad |= bad;
    }
    __syncthreads();
  }
  // each(f): f(blocks) for every sequence of this lane
  auto take = [&](auto each) __attribute__((always_inline)) {
    Cut c = {0, kDecodeWgsShift, 0, 0, 0};
    if constexpr (W == 8) {
      bool merged = false;                                  // some list takes more than one workgroup
      int mine = 0, by_four = 0;
      each([&](int nb) __attribute__((always_inline)) {
        merged |= nb > 8;
        mine += (nb + 7) & ~7;
        by_four += (nb + 3) & ~3;
      });
      int incl = wave_inclusive_sum(s.pps * by_four);
      r.merged = __builtin_amdgcn_ballot_w64(merged) != 0;
      c.align = r.merged && __builtin_amdgcn_readlane(incl, 63) <= 4 * s.most_by_four ? 2 : 3;
      if (c.align == 3) incl = wave_inclusive_sum(s.pps * mine);
      c.round = (1 << c.align) - 1;
      r.incl = incl;
      c.total = __builtin_amdgcn_readlane(incl, 63);
      return c;
    }
    if (s.aligned_shift >= 0) {
      bool between = false;
      each([&](int nb) __attribute__((always_inline)) { between |= nb > 8 && nb <= 64; });
      c.align = __builtin_amdgcn_ballot_w64(between) == 0 ? 3 : 2;
      c.round = (1 << c.align) - 1;
    }
    // too many workgroups for that: one for each list where that pays, or an equal share of all lists: over how many ranges, and
    // what a list counts (calls of very many lists do not round)
    auto share = [&]() __attribute__((always_inline)) {
      int lists = 0, blocks = 0;
      each([&](int nb) __attribute__((always_inline)) {
        lists += nb != 0 ? s.pps : 0;
        blocks += s.pps * nb;
      });
      lists = __builtin_amdgcn_readlane(wave_inclusive_sum(lists), 63);
      const bool two = gridDim.x >= 2 << kDecodeWgsShift && lists >= kLists;   // workgroups per CU
      // 256 to 512 lists of up to 16 blocks take a workgroup each, none of which has a seam or anything to merge; up to 24 blocks
      // where there are hardly fewer lists than workgroups, and 24 (32 at head dimension 64) where every CU has one.  us in equal
      // ranges / so, 32/8 heads of 128 unless said: 64 lists of 200 to 328 keys 24.3 / 19.1, 64 of 50 to 296 21.1 / 16.4, 48 of
      // 300 to 508 25.7 / 23.2, 33 of 300 to 508 21.1 / 19.8, 40 of 50 to 439 at head dimension 64 13.8 / 11.2; 64 of 500 to 760
      // 39.6 / 35.1, 120 of 50 to 630 at 28/4 heads 28.8 / 24.8; 32 of 500 to 760 24.6 / 21.3, 32 of 50 to 760 20.9 / 19.7, 32 of
      // 50 to 630 at head dimension 64 13.4 / 11.1, 32 of 700 to 1010 there 17.0 / 15.2.
      // With fewer or longer lists the CU with two of the longest is the last (70 of 50 to 630 at 28/4 21.4 / 26.4, 48 of 700
      // to 1010 39.7 / 41.2, 33 of 500 to 760 26.7 / 27.9, 32 of 50 to 1010 22.4 / 23.8).
      if (s.aligned_shift >= 0 && two && lists >= 1 << kDecodeWgsShift && lists <= 1 << s.aligned_shift) {
        const int most = lists == 1 << kDecodeWgsShift ? (D == 64 ? 32 : 24) : lists > (7 << s.aligned_shift) / 8 ? 24 : 16;
        bool longer = false;
        each([&](int nb) __attribute__((always_inline)) { longer |= nb > most; });
        if (__builtin_amdgcn_ballot_w64(longer) == 0) {
          c.align = 5;
          c.round = 31;
          return;
        }
      }
      c.align = 0;
      c.shift = kDecodeWgsShift + (two ? 1 : 0);
      if (s.aligned_shift < 0) return;
      // Lists of one length that take a whole number of ranges each: no range has a seam, so they are cut evenly, and one
      // workgroup per CU is enough (8 lists of 4224 keys 29.6 / 29.4, 32 of 2048 50.9 / 47.3, 64 of 1000 at 28/4 heads 30.6 / 27.1)
      if ((lists & (lists - 1)) == 0 && lists <= 1 << c.shift) {
        blocks = __builtin_amdgcn_readlane(wave_inclusive_sum(blocks), 63);
        bool other = false;
        each([&](int nb) __attribute__((always_inline)) { other |= nb != 0 && (unsigned)nb * (unsigned)lists != (unsigned)blocks; });
        if (__builtin_amdgcn_ballot_w64(other) == 0) {
          if (lists <= 1 << kDecodeWgsShift) c.shift = kDecodeWgsShift;
          c.round = c.pad = 0;
          return;
        }
      }
      const bool beside = D == 128 && two;
      c.round = beside ? 1 : W - 1;
      c.pad = beside ? kSeam / 2 : kSeam;
    };
    if (s.aligned_shift < 0) share();
    for (;;) {
      int mine = 0;
      each([&](int nb) __attribute__((always_inline)) { mine += counted(c, nb); });
      r.incl = wave_inclusive_sum(s.pps * mine);
      c.total = __builtin_amdgcn_readlane(r.incl, 63);
      if (c.align == 0 || c.total <= 1 << (s.aligned_shift + c.align)) break;
      share();
    }
    if (c.align > 0) return c;
    // (lists that are not rounded up may have fewer blocks than there are workgroups: no range is empty, or it would be
    // counted among the parts of a list)
    while (c.shift > 0 && c.total >> c.shift == 0) --c.shift;
    return c;
  };
  if (__builtin_expect(r.run == 1, 1)) return take([&](auto f) __attribute__((always_inline)) { f(r.q.nb); });
  return take([&](auto f) __attribute__((always_inline)) {
    if (r.run * 64 <= kDecodeTable) {
      for (int j = 0; j < r.run; ++j) f(seq_at(s, table, r.run, lane, j).nb);
    } else {
      for (int j = 0; j < r.run && lane * r.run + j < s.batch; ++j) {
        bool bad = false;
        f(load_counted(s, lane * r.run + j, bad).nb);
        r.bad |= bad;
      }
    }
  });
}

// The sequence whose lists hold block x (x < total).
struct Place {
  int b, len, md;
  int begin;        // first block of its first pair
  int nb;           // blocks of a pair, as counted
  int real;         // ... that there are
};
template <class S>
__device__ __forceinline__ Place find_place(const S& s, Cut c, const Lanes& r, int lane, const SeqTable* table, int x) {
  const int i = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(r.incl <= x)));   // whose lane
  if (__builtin_expect(r.run == 1, 1)) {
    const int real = __builtin_amdgcn_readlane(r.q.nb, i), nb = counted(c, real);
    return Place{i, __builtin_amdgcn_readlane(r.q.len, i), __builtin_amdgcn_readlane(r.q.md, i), __builtin_amdgcn_readlane(r.incl, i) - s.pps * nb, nb, real};
  }
  Place p = {0, 0, 1, 0, 1, 1};
  int base = i > 0 ? __builtin_amdgcn_readlane(r.incl, i - 1) : 0;
  for (int j0 = 0; j0 < r.run; j0 += 64) {
    Seq q = {0, 1, 0};
    if (j0 + lane < r.run && i * r.run + j0 + lane < s.batch) q = seq_at(s, table, r.run, i, j0 + lane);
    const int nb = counted(c, q.nb), incl = base + wave_inclusive_sum(s.pps * nb);
    const int end = __builtin_amdgcn_readlane(incl, 63);
    if (x < end) {                                          // wave-uniform
      const int j = __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= x)));
      p.nb = __builtin_amdgcn_readlane(nb, j);
      p = Place{i * r.run + j0 + j, __builtin_amdgcn_readlane(q.len, j), __builtin_amdgcn_readlane(q.md, j), __builtin_amdgcn_readlane(incl, j) - s.pps * p.nb, p.nb, __builtin_amdgcn_readlane(q.nb, j)};
      break;
    }
    base = end;
  }
  return p;
}

// ---- rows that pass between workgroups of one launch, which may sit on different XCDs: written and read at device
// scope (past the L2s, which are not coherent with each other).  `base` is wave-uniform, `at` a byte offset.
__device__ __forceinline__ void store16_dev(float* base, int at, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), __builtin_amdgcn_make_buffer_rsrc(base, 0, -1, 0x00027000), at, 0, 16 /*sc1*/);
}
__device__ __forceinline__ f32x4 load16_dev(const float* base, int at) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, -1, 0x00027000), at, 0, 16));
}
template <bool DEV>
__device__ __forceinline__ f32x2 load_ml(const float* p) {
  if (!DEV) return *(const f32x2*)p;
  return __builtin_bit_cast(f32x2, __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// ---- the merge of a pair's parts: out = sum_c w_c O_c / sum_c w_c l_c, w_c = exp(m_c - max m).  A wave takes 64 / (D / 4)
// heads at a time, D / 4 lanes each with four columns, and the parts in runs of 16: lane i of every 16 works out the weight
// of part i, which the sum over the parts then takes from it.  The rows of a run are all asked for at once.
template <int CTRL>
__device__ __forceinline__ float row16(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float x) {           // over the 16 lanes of a row, the same in all of them
  x += row16<0x128>(x);                                     // row_ror:8, 4, 2, 1
  x += row16<0x124>(x);
  x += row16<0x122>(x);
  return x + row16<0x121>(x);
}
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, row16<0x128>(x));
  x = fmaxf(x, row16<0x124>(x));
  x = fmaxf(x, row16<0x122>(x));
  return fmaxf(x, row16<0x121>(x));
}
template <int... I>
__device__ __forceinline__ void add_weighted(f32x4& num, float w, const f32x4 (&o)[16], std::integer_sequence<int, I...>) {
  ((num += row16<0x150 + I>(w) * o[I]), ...);               // row_newbcast:I, the weight of part I
}
struct Merged {
  float m, den;
  f32x4 num;
};
// Lane l's columns of head `head0` + l / (D / 4), over the runs first_run, first_run + step, ...
template <int D, bool DEV>
__device__ __forceinline__ Merged merge_runs(const float* part_o, const float* part_ml, int rpu, int first, int parts, int nq, float scale_log2, int head0, int first_run, int step, int l) {
  constexpr int TPR = D / 4;
  const int row = min(head0 + l / TPR, nq - 1), d = 4 * (l % TPR), j = l & 15;
  Merged r = {-INFINITY, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int c0 = 16 * first_run; c0 < parts; c0 += 16 * step) {
    const f32x2 ml = load_ml<DEV>(part_ml + 2 * (part_place(first, min(c0 + j, parts - 1)) * rpu + row));
    f32x4 o[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = (part_place(first, min(c0 + i, parts - 1)) * rpu + row) * D + d;   // (the last part again where there are fewer)
      if (DEV) o[i] = load16_dev(part_o, at * 4);
      else o[i] = *(const f32x4*)(part_o + at);
    }
    const float mj = c0 + j < parts ? ml[0] : -INFINITY;
    const float m_new = fmaxf(r.m, max16(mj));
    const float al = fast_exp2((r.m - m_new) * scale_log2); // 0 for the first run (every part holds a key)
    const float w = fast_exp2((mj - m_new) * scale_log2);
    r.num *= al;
    r.den = r.den * al + sum16(w * ml[1]);
    r.m = m_new;
    add_weighted(r.num, w, o, std::make_integer_sequence<int, 16>());
  }
  return r;
}
// All heads of one pair by a workgroup of four waves; `store` is given (head, column, four values).  Where the heads take one
// or two waves and there are several runs, the other waves take every other run and all meet in LDS (Merged[4][64]).
template <int D, bool DEV, int W, class Store>
__device__ __forceinline__ void merge_pair(const float* part_o, const float* part_ml, int rpu, int first, int parts, int nq, float scale_log2, char* lds, int w, int l, Store store) {
  constexpr int TPR = D / 4, HPW = 64 / TPR;
  auto finish = [&](int head0, const Merged& r) __attribute__((always_inline)) {
    const int qi = head0 + l / TPR;
    if (qi < nq) store(qi, 4 * (l % TPR), f32x4{r.num[0] / r.den, r.num[1] / r.den, r.num[2] / r.den, r.num[3] / r.den});
  };
  const int groups = (nq + HPW - 1) / HPW;                  // of heads that a wave takes at a time
  const int split = groups > 2 || parts <= 16 ? 1 : 4 / groups;
  for (int i = w; i < groups * split; i += W) {
    const int head0 = (split == 1 ? i : i % groups) * HPW;
    const Merged r = merge_runs<D, DEV>(part_o, part_ml, rpu, first, parts, nq, scale_log2, head0, split == 1 ? 0 : i / groups, split, l);
    if (split == 1) finish(head0, r);
    else ((Merged*)lds)[64 * i + l] = r;
  }
  if (split == 1) return;                                   // uniform for the workgroup
  __syncthreads();
  if (w >= groups) return;
  float m = -INFINITY;
  for (int i = 0; i < split; ++i) m = fmaxf(m, ((Merged*)lds)[64 * (w + i * groups) + l].m);
  Merged t = {m, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  for (int i = 0; i < split; ++i) {
    const Merged r = ((Merged*)lds)[64 * (w + i * groups) + l];
    const float wgt = fast_exp2((r.m - m) * scale_log2);    // exp2(-inf) = 0 for a wave without runs
    t.num += wgt * r.num;
    t.den += wgt * r.den;
  }
  finish(w * HPW, t);
}

}  // namespace flux
