// flux_kv_append_paged: new K/V rows are quantised into the pages that their slots name.
//
// The new rows of one page and KV head are a BLOCK.  Its scale is 2^e, e the smallest exponent >= kMinScaleExp with
// amax <= 448 * 2^e (448 = 1.75 * 2^8 is the largest e4m3 value), which is read off the bits of amax; a code is x * 2^-e rounded to
// nearest even, and as the product is exact there is one rounding.  A page that holds rows already keeps its scale or takes
// the larger one of the new rows, and then its old codes are rounded once more.
//
// One wave per block, K or V: up to 64 rows stay in its registers between the maximum and the rounding, so every row is read once,
// with up to 16 KB on their way per wave, and nothing passes between waves.
// What bounds it: the memory for long prompts, latencies (slots, scale, row) for a decode step, and where pages take a larger scale
// the latencies of their old codes, RPS rows at a time: 64 sequences with a row each, 8 heads of 128, traced with every page so 10.8 us for 4.8.
#include "paged.h"

namespace flux {

struct PagedAppendArgs {
  const char *k_new, *v_new;      // bf16 [total, hkv, D]
  char *k, *v;
  float *k_scale, *v_scale;
  int64_t stride_p, stride_h, stride_t;
  const int32_t* slots;
  int hkv, total, n_pages;
  uint32_t units;                 // (tile of 64 token rows, head, K or V, 2^share)
  int share;
  uint32_t* status;
};

typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;

// largest of the values' magnitudes, as bits
__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  const u16x2 x = __builtin_bit_cast(u16x2, a), y = __builtin_bit_cast(u16x2, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}
__device__ __forceinline__ uint32_t finite_bits(uint32_t pair) {   // magnitudes, those that are not finite as 0
  const uint32_t lo = pair & 0x7FFFu, hi = (pair >> 16) & 0x7FFFu;
  return (lo < 0x7F80u ? lo : 0u) | (hi < 0x7F80u ? hi << 16 : 0u);
}

// Four values times `inv` as codes, to nearest even.  (The conversion would make a large number of an infinite value: it is NaN
// by then.)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, r, true);
}
__device__ __forceinline__ float finite_or_nan(float x) { return x - x == 0.f ? x : __builtin_nanf(""); }

// A wave looks at 64 token rows, where blocks begin in them, and does one block in 2^share for one head, K or V: in a decode step
// every row begins a block, in a long prompt one or two of 64 do, and only the slots tell which it is.  So short calls have as many
// waves as there may be blocks, and long ones about kAppendPagedWaves at least, most of which leave at once: us with 1024 / 2048 / 4096
// / 8192 of them, 8 heads of 128, one row of 256 sequences 8.6 / 6.6 / 5.8 / 5.7, five of each 14.1 / 9.4 / 7.5 / 7.1, 512 rows of one
// 5.4 / 6.2 / 6.5 / 8.9, 2100 rows of three 5.8 / 6.4 / 7.0 / 10.1, 8000 of four 13.2 / 13.2 / 12.0 / 12.0.  (32768 rows take 41.5 with
// any: 4.9 TB/s read and written, where a plain copy of 1 GB reaches 5.2.  64 sequences with a row each: 4.0, a launch, the slots,
// the scale and the row one behind the other.)
// A lane has 16 values of a row, two loads and one store of 16 bytes: with 8 values each a store of codes is 8 bytes, and 32768 rows
// took 42.4.
template <int D>
__global__ __launch_bounds__(256) void kv_append_paged_kernel(PagedAppendArgs a) {
  constexpr int LPR = D / 16;                                // lanes per row, 16 values each
  constexpr int RPS = 64 / LPR;                              // rows per step
  constexpr int STEPS = 64 / RPS;
  const int l = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t per_tile = (2u * a.hkv) << a.share;
  for (uint32_t u = blockIdx.x * 4 + w; u < a.units; u += gridDim.x * 4) {   // (units < 2^31, a launch below 2^25)
    const int tile = (int)(u / per_tile), rest = (int)(u - tile * per_tile);
    const int turn = rest & ((1 << a.share) - 1), h = rest >> (a.share + 1);
    const bool is_v = (rest >> a.share) & 1;
    const int t0 = tile * 64;
    // where blocks begin: a row whose slot does not follow that of the row before in the same page
    const int t_mine = t0 + l;
    const int s = t_mine < a.total ? a.slots[t_mine] : -1, p = t_mine > 0 && t_mine < a.total ? a.slots[t_mine - 1] : -1;
    uint64_t begins = __builtin_amdgcn_ballot_w64(s >= 0 && !(p == s - 1 && (s & 63) != 0));
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(begins >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)begins, 0));
    begins &= __builtin_amdgcn_ballot_w64((before & ((1 << a.share) - 1)) == turn);
    while (begins != 0) {
      const int t = t0 + __builtin_ctzll(begins);
      begins &= begins - 1;
      const int mine = t + l < a.total ? a.slots[t + l] : -1;
      const int slot = __builtin_amdgcn_readfirstlane(mine);
      const int page = slot >> 6, first = slot & 63;
      if (page >= a.n_pages) {
        if (l == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_PAGE);
        continue;
      }
      const uint64_t others = ~__builtin_amdgcn_ballot_w64(first + l < 64 && mine == slot + l);
      const int rows = others == 0 ? 64 : __builtin_ctzll(others);
      const char* src = (is_v ? a.v_new : a.k_new) + (((int64_t)t * a.hkv + h) * D + (l % LPR) * 16) * 2;
      const int64_t src_step = (int64_t)a.hkv * D * 2;
      float* const scale_at = (is_v ? a.v_scale : a.k_scale) + (int64_t)page * a.hkv + h;
      char* const dst = (is_v ? a.v : a.k) + (int64_t)page * a.stride_p + (int64_t)h * a.stride_h + (l % LPR) * 16;
      u32x4 x[STEPS][2];
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        x[i][0] = x[i][1] = u32x4{0, 0, 0, 0};
        if (i * RPS < rows) {                                // (uniform)
          const int r = i * RPS + l / LPR;
          if (r < rows) {
            x[i][0] = *(const u32x4*)(src + r * src_step);
            x[i][1] = *(const u32x4*)(src + r * src_step + 16);
          }
        }
      }
      const float old = first != 0 ? *scale_at : 0.f;
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = pk_max(top, x[i][j >> 2][j & 3] & 0x7FFF7FFFu);
      bool odd = (top & 0xFFFFu) >= 0x7F80u || (top >> 16) >= 0x7F80u;
      odd = __builtin_amdgcn_ballot_w64(odd) != 0;           // some value is not finite
      if (odd) {
        top = 0;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) top = pk_max(top, finite_bits(x[i][j >> 2][j & 3]));
      }
      int amax = max((int)(top & 0xFFFFu), (int)(top >> 16));
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) amax = max(amax, __shfl_xor(amax, off));
      amax = __builtin_amdgcn_readfirstlane(amax);
      // amax = (1 + f / 128) 2^(E - 127): it fits under 1.75 * 2^(8 + e) from e = E - 135 on, or one more where f > 96
      const int e = max((amax >> 7) - 135 + ((amax & 127) > 96 ? 1 : 0), kMinScaleExp);
      float scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
      scale = old > scale ? old : scale;
      const float inv = 1.0f / scale;                        // exact: a power of two
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        if (i * RPS >= rows) continue;
        const int r = i * RPS + l / LPR;
        uint32_t codes[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = x[i][j >> 1][2 * (j & 1)], hi = x[i][j >> 1][2 * (j & 1) + 1];
          float f[4] = {bf16_lo(lo), bf16_hi(lo), bf16_lo(hi), bf16_hi(hi)};
          if (odd) {
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] = finite_or_nan(f[k]);
          }
          codes[j] = codes4(f[0], f[1], f[2], f[3], inv);
        }
        if (r < rows) *(u32x4*)(dst + (first + r) * a.stride_t) = u32x4{codes[0], codes[1], codes[2], codes[3]};
      }
      if (first != 0 && scale > old) {                       // the rows that the page holds take the new scale too
        const float down = old * inv;
        for (int r0 = 0; r0 < first; r0 += RPS) {
          const int r = r0 + l / LPR;
          if (r >= first) continue;
          u32x4* const at = (u32x4*)(dst + r * a.stride_t);
          u32x4 c = *at;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], true);
            c[j] = codes4(lo[0], lo[1], hi[0], hi[1], down);
          }
          *at = c;
        }
      }
      if (l == 0 && (first == 0 || scale > old)) *scale_at = scale;
    }
  }
}

hipError_t launch_kv_append_paged(const Ctx& c, const flux_paged_kv& kv, int hkv, int d, const void* k_new, const void* v_new,
                                  const int32_t* slots, int total_new, hipStream_t s) {
  PagedAppendArgs a;
  a.k_new = (const char*)k_new;
  a.v_new = (const char*)v_new;
  a.k = (char*)kv.k;
  a.v = (char*)kv.v;
  a.k_scale = kv.k_scale;
  a.v_scale = kv.v_scale;
  a.stride_p = kv.stride_p;
  a.stride_h = kv.stride_h;
  a.stride_t = kv.stride_t;
  a.slots = slots;
  a.hkv = hkv;
  a.total = total_new;
  a.n_pages = kv.n_pages;
  a.status = c.status;
  const long long tiles = ((long long)total_new + 63) / 64 * 2 * hkv;
  a.share = 6;
  while (a.share > 0 && (tiles << a.share) > kAppendPagedWaves) --a.share;
  a.units = (uint32_t)(tiles << a.share);
  const long long wgs = ((long long)a.units + 3) / 4;
  const dim3 grid((unsigned)(wgs < kAppendMost ? wgs : kAppendMost)), block(256);
  if (d == 128) hipLaunchKernelGGL((kv_append_paged_kernel<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((kv_append_paged_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace flux
