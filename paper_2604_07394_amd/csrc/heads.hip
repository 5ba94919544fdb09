// flux_qk_norm_rope, flux_qkv_append, flux_qkv_append_paged: query and key heads of new tokens are normed and turned by their
// positions on their way from the projection to the attention and the cache.
//
// A head row x of D values:  y = x / sqrt(mean(x^2) + eps) * w;  of the first R dimensions the pairs (i, i + R/2), or (2i, 2i + 1), are
// turned by position * inv_freq[i] radians.  D / 16 lanes have a row, 16 values each: both dimensions of every pair lie in one lane, so a
// row passes between lanes for nothing but its sum of squares, and the angles of a lane are the same for all heads of a token.
// Angles are taken in 64 bits up to the fraction of a turn (a far position times a frequency has no such bits left in 32), the sine
// and cosine of that fraction by the instructions for turns.
#include "heads.h"

namespace flux {

struct HeadArgs {
  const char *q, *k, *v;
  int64_t stride_q, stride_k, stride_v;   // bytes between the rows of two tokens
  char *q_out, *k_out;
  const char *q_norm, *k_norm;
  const float* freq;
  const int32_t* pos;
  float eps;
  int hq, hkv, total, rot;
  int passes, waves;              // passes of a wave over all rows of a token, waves that share them
  // contiguous cache
  const int32_t* cu;
  char *kc, *vc;
  int64_t stride_b, stride_h, stride_t;   // bytes
  int32_t* kv_len;
  int batch, capacity;
  uint32_t *counter, *gather, *status;
};

constexpr double kTurnsPerRadian = 0.15915494309189533577;

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double x) {
  const u32x2 u = __builtin_bit_cast(u32x2, x);
  return __builtin_bit_cast(double, u32x2{(uint32_t)__builtin_amdgcn_mov_dpp((int)u[0], CTRL, 0xf, 0xf, true), (uint32_t)__builtin_amdgcn_mov_dpp((int)u[1], CTRL, 0xf, 0xf, true)});
}
// Sum over the 4, 8 or 16 lanes of a row: quad_perm 1 0 3 2, quad_perm 2 3 0 1, row_half_mirror, row_mirror.
template <int LANES, typename T>
__device__ __forceinline__ T row_sum(T x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  if constexpr (LANES >= 8) x += dpp<0x141>(x);
  if constexpr (LANES == 16) x += dpp<0x140>(x);
  return x;
}

// Position times frequency as a fraction of a turn, from -1/2 to 1/2.
__device__ __forceinline__ double turn_of(int pos, float freq) {
  const double t = (double)pos * ((double)freq * kTurnsPerRadian);
  return t - __builtin_rint(t);
}
__device__ __forceinline__ void sincos_turn(double t, float& s, float& c) {
  s = __builtin_amdgcn_sinf((float)t);
  c = __builtin_amdgcn_cosf((float)t);
}
// In 64 bits: the nearest quarter turn, and Taylor's series of what is left (at most pi / 4) to 2^-37.
__device__ __forceinline__ void sincos_turn(double t, double& s, double& c) {
  const double quarter = __builtin_rint(4.0 * t);
  const double x = (t - 0.25 * quarter) * 6.28318530717958647693, z = x * x;
  double a = -1.0 / 39916800, b = -1.0 / 3628800;
  a = __builtin_fma(a, z, 1.0 / 362880);
  b = __builtin_fma(b, z, 1.0 / 40320);
  a = __builtin_fma(a, z, -1.0 / 5040);
  b = __builtin_fma(b, z, -1.0 / 720);
  a = __builtin_fma(a, z, 1.0 / 120);
  b = __builtin_fma(b, z, 1.0 / 24);
  a = __builtin_fma(a, z, -1.0 / 6);
  b = __builtin_fma(b, z, -1.0 / 2);
  a = __builtin_fma(a * z, x, x);
  b = __builtin_fma(b, z, 1.0);
  const int n = (int)quarter;
  const double p = n & 1 ? b : a, r = n & 1 ? a : b;
  s = n & 2 ? -p : p;
  c = (n + 1) & 2 ? -r : r;
}

// Where the 16 values of lane i of a row lie: two pieces of eight.  Lanes below rot / 16 have eight whole pairs, the others none.
template <bool NEAR>
__device__ __forceinline__ void lane_places(int i, int rot, int& c0, int& c1, bool& turns) {
  turns = 16 * i < rot;
  const bool apart = !NEAR && turns;
  c0 = apart ? 8 * i : 16 * i;
  c1 = apart ? 8 * i + rot / 2 : 16 * i + 8;
}

__device__ __forceinline__ void unpack8(u32x4 x, float* f) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = bf16_lo(x[j]);
    f[2 * j + 1] = bf16_hi(x[j]);
  }
}

// The pairs of a lane turned: s, c of pair j.
template <bool NEAR, typename T>
__device__ __forceinline__ void turn_pairs(T* x, const T* s, const T* c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    T& a = NEAR ? x[2 * j] : x[j];
    T& b = NEAR ? x[2 * j + 1] : x[8 + j];
    const T a0 = a, b0 = b;
    a = __builtin_fma(-b0, s[j], a0 * c[j]);
    b = __builtin_fma(a0, s[j], b0 * c[j]);
  }
}

// The angles of a token for this lane.
template <typename T>
__device__ __forceinline__ void lane_angles(const float* freq, int i, int pos, T* s, T* c) {
  const f32x4 lo = *(const f32x4*)(freq + 8 * i), hi = *(const f32x4*)(freq + 8 * i + 4);
#pragma unroll
  for (int j = 0; j < 8; ++j) sincos_turn(turn_of(pos, j < 4 ? lo[j] : hi[j & 3]), s[j], c[j]);
}

// Rows of a token that a wave asks for at once.
constexpr int kPassesInFlight = 4;

// All rows of one token that this wave has: passes p0, p0 + step, ...  A pass is 64 / (D / 16) rows: the query heads first, then the
// key heads, then (V) the value heads, which are copied.
// q_at(h), k_at(h), v_at(h): where a finished row goes, null: nowhere.
template <int D, bool NEAR, bool V, typename KP, typename VP>
__device__ __forceinline__ void token_rows(const HeadArgs& a, int64_t t, int pos, int p0, int l, KP k_at, VP v_at) {
  constexpr int LPH = D / 16, RPP = 64 / LPH;
  const int i = l % LPH;
  int c0, c1;
  bool turns;
  lane_places<NEAR>(i, a.rot, c0, c1, turns);
  const int rows = a.hq + (V ? 2 : 1) * a.hkv;
  u32x4 wq[2], wk[2];
  if (a.q_norm) {
    wq[0] = *(const u32x4*)(a.q_norm + 2 * c0);
    wq[1] = *(const u32x4*)(a.q_norm + 2 * c1);
  }
  if (a.k_norm) {
    wk[0] = *(const u32x4*)(a.k_norm + 2 * c0);
    wk[1] = *(const u32x4*)(a.k_norm + 2 * c1);
  }
  float s[8], c[8];
  bool angles = false;
  for (int p = p0; p < a.passes; p += kPassesInFlight * a.waves) {
    u32x4 x[kPassesInFlight][2];
#pragma unroll
    for (int u = 0; u < kPassesInFlight; ++u) {
      const int r = (p + u * a.waves) * RPP + l / LPH;
      x[u][0] = x[u][1] = u32x4{0, 0, 0, 0};
      if (r < rows) {
        const char* src = r < a.hq ? a.q + t * a.stride_q + (int64_t)r * D * 2
                        : !V || r < a.hq + a.hkv ? a.k + t * a.stride_k + (int64_t)(r - a.hq) * D * 2
                                                 : a.v + t * a.stride_v + (int64_t)(r - a.hq - a.hkv) * D * 2;
        x[u][0] = *(const u32x4*)(src + 2 * c0);
        x[u][1] = *(const u32x4*)(src + 2 * c1);
      }
    }
    if (!angles) {                                           // (behind the rows, which take longer to come)
      angles = true;
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = 0.f, c[j] = 1.f;
      if (turns) lane_angles(a.freq, i, pos, s, c);
    }
#pragma unroll
    for (int u = 0; u < kPassesInFlight; ++u) {
      const int pass = p + u * a.waves;
      if (pass >= a.passes) break;                           // (uniform)
      const int r = pass * RPP + l / LPH;
      const bool is_q = r < a.hq, is_v = V && r >= a.hq + a.hkv;
      float f[16];
      unpack8(x[u][0], f);
      unpack8(x[u][1], f + 8);
      const bool norm = is_q ? a.q_norm != nullptr : !is_v && a.k_norm != nullptr;
      if (__builtin_amdgcn_ballot_w64(norm) != 0) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) sum = __builtin_fmaf(f[j], f[j], sum);
        sum = row_sum<LPH>(sum);
        float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / D, a.eps));
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(norm && !(sum < 0x1p100f)) != 0, 0)) {
          // squares that pass 32 bits, or are not numbers: the row in 64
          double big = 0.0;
#pragma unroll
          for (int j = 0; j < 16; ++j) big = __builtin_fma((double)f[j], (double)f[j], big);
          const double wide = 1.0 / __builtin_sqrt(row_sum<LPH>(big) * (1.0 / D) + (double)a.eps);
          const bool apart = !(sum < 0x1p100f);
#pragma unroll
          for (int j = 0; j < 16; ++j) f[j] = norm && apart ? (float)((double)f[j] * wide) : f[j];
          inv = apart ? 1.0f : inv;
        }
        float w[16];
        unpack8(is_q ? wq[0] : wk[0], w);
        unpack8(is_q ? wq[1] : wk[1], w + 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] = norm ? f[j] * inv * w[j] : f[j];
      }
      float y[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = f[j];
      turn_pairs<NEAR>(y, s, c);
      u32x4 o[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (a dimension that is not turned is not touched by the others of its lane, whatever they are)
        o[0][j] = turns ? pack_bf16(y[2 * j], y[2 * j + 1]) : pack_bf16(f[2 * j], f[2 * j + 1]);
        o[1][j] = turns ? pack_bf16(y[8 + 2 * j], y[9 + 2 * j]) : pack_bf16(f[8 + 2 * j], f[9 + 2 * j]);
        if (is_v) o[0][j] = x[u][0][j], o[1][j] = x[u][1][j];
      }
      char* dst = nullptr;
      if (is_q) dst = a.q_out + (t * a.hq + r) * D * 2;
      else if (r < rows) dst = is_v ? v_at(r - a.hq - a.hkv) : k_at(r - a.hq);
      if (dst) {
        *(u32x4*)(dst + 2 * c0) = o[0];
        *(u32x4*)(dst + 2 * c1) = o[1];
      }
    }
  }
}

template <int D, bool NEAR>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadArgs a) {
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)a.total * a.waves;
  for (int64_t u = (int64_t)blockIdx.x * 4 + w; u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / a.waves;
    const int pos = a.rot ? a.pos[t] : 0;
    token_rows<D, NEAR, false>(a, t, pos, (int)(u - t * a.waves), l, [&](int h) { return a.k_out + (t * a.hkv + h) * D * 2; }, [&](int) { return (char*)nullptr; });
  }
}

// Largest b of [0, batch) with cu[b] <= t, where cu ascends: 64 sequences at a time, one per lane.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int t, int l) {
  int lo = 0, n = batch;                                     // it is one of lo .. lo + n - 1
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const int at = lo + l * step;
    const int before = __builtin_popcountll(__builtin_amdgcn_ballot_w64(l * step < n && cu[min(at, batch - 1)] <= t));
    const int skip = before > 0 ? (before - 1) * step : 0;
    lo += skip;
    n = min(step, n - skip);
  }
  const int before = __builtin_popcountll(__builtin_amdgcn_ballot_w64(l < n && cu[min(lo + l, batch - 1)] <= t));
  return lo + (before > 0 ? before - 1 : 0);
}

// The contiguous cache: row r of sequence b goes to position kv_len[b] + r.  All waves read the lengths; the last workgroup to have read
// them moves them on (see kv_append.hip).
template <int D, bool NEAR>
__global__ __launch_bounds__(256) void qkv_rows_kernel(HeadArgs a) {
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)a.total * a.waves;
  const int end = a.cu[a.batch], begin = a.cu[0];
  bool overflow = false;
  for (int64_t u = (int64_t)blockIdx.x * 4 + w; u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / a.waves;
    if (t < begin || t >= end) continue;                     // rows of no sequence
    const int b = sequence_of(a.cu, a.batch, (int)t, l);
    const int64_t at = (int64_t)a.kv_len[b] + (t - a.cu[b]);
    const bool kept = at >= 0 && at < a.capacity;
    overflow |= !kept;
    const int64_t row = (int64_t)b * a.stride_b + at * a.stride_t;
    const int pos = a.pos ? a.pos[t] : (int)at;
    token_rows<D, NEAR, true>(a, t, pos, (int)(u - t * a.waves), l, [&](int h) { return kept ? a.kc + row + h * a.stride_h : nullptr; },
                              [&](int h) { return kept ? a.vc + row + h * a.stride_h : nullptr; });
  }
  if (overflow && l == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_KV_OVERFLOW);
  // (a wave holds the length that it read before it passes the barrier, as its rows' places come from it; the stores are not waited for)
  __shared__ int is_last;
  asm volatile("" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t n = gridDim.x, x = blockIdx.x & (kAppendGather - 1);
    bool last = true;
    if (n > kAppendOneWord) {
      uint32_t* word = a.gather + x * kCounterStride;
      last = atomicAdd(word, 1u) == (n - x + kAppendGather - 1) / kAppendGather - 1;
      if (last) *word = 0;                                   // ready for the next launch on this stream
    }
    if (last) last = atomicAdd(a.counter, 1u) == (n > kAppendOneWord ? (uint32_t)kAppendGather : n) - 1;
    is_last = last;
  }
  __syncthreads();
  if (!is_last) return;
  for (int b = threadIdx.x; b < a.batch; b += 256) {
    const int n = a.cu[b + 1] - a.cu[b];
    int len = a.kv_len[b];
    if (n > 0) len = (int)min((int64_t)len + n, (int64_t)a.capacity);
    a.kv_len[b] = min(len, a.capacity);
  }
  if (threadIdx.x == 0) *a.counter = 0;
}

// ---- pages
// K and V of the new rows are quantised as kv_append_paged.hip does it, K from its values in 64 bits: a code is rounded once, from
// the value that the formula names.  (From values in 32 bits 7 of 4.3 M codes came out on the other side of a border.)  A value is
// kept between the search for the block's largest one and the rounding as the upper 32 bits of its 64, the last of them set if any below it was (rounding
// to odd): 21 significant bits, from which the four of a code come out as from all of them, and which order like the values.
struct QuantArgs {
  HeadArgs h;
  char *k, *v;
  float *k_scale, *v_scale;
  int64_t stride_p, stride_h, stride_t;
  const int32_t* slots;
  int n_pages;
  uint32_t units;                 // (tile of 64 token rows, K or V, 2^share), of one head or of all
  int share;
  unsigned kv_wgs;                // workgroups that look after K and V; the others have the queries
};

__device__ __forceinline__ uint32_t to_odd(double x) {
  const u32x2 u = __builtin_bit_cast(u32x2, x);
  return u[1] | (u[0] != 0 ? 1u : 0u);
}
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t hi) {
  const uint32_t mag = hi & 0x7FFFFFFFu;
  return mag < 0x7FF00000u ? mag : 0u;
}
// A value as to_odd leaves it, divided by a scale: exact, or far below the smallest code.  What is not finite is NaN.
__device__ __forceinline__ float scaled(uint32_t hi, double inv) {
  const float x = (float)(__builtin_bit_cast(double, u32x2{0, hi}) * inv);
  return (hi & 0x7FF00000u) != 0x7FF00000u ? x : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ u32x4 codes16(const uint32_t* hi, double inv) {
  u32x4 codes;
#pragma unroll
  for (int j = 0; j < 4; ++j) codes[j] = codes4(scaled(hi[4 * j], inv), scaled(hi[4 * j + 1], inv), scaled(hi[4 * j + 2], inv), scaled(hi[4 * j + 3], inv));
  return codes;
}
// The scale of a block whose largest magnitude is `top` = (1 + f / 2^20) 2^(E - 1023): it fits under 1.75 * 2^(8 + e) from e = E - 1031 on, or
// one more where f > 0.75 * 2^20.  `old`: the scale that its page has, or 0.
__device__ __forceinline__ float block_scale(uint32_t top, float old) {
  const int e = max((int)(top >> 20) - 1031 + ((top & 0xFFFFFu) > 0xC0000u ? 1 : 0), kMinScaleExp);
  const float scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
  return old > scale ? old : scale;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, off));
  return x;
}
// 16 codes of a page that takes a larger scale.
__device__ __forceinline__ void scale_down(char* at, float down) {
  u32x4 c = *(u32x4*)at;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[j], true);
    c[j] = codes4(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down);
  }
  *(u32x4*)at = c;
}
__device__ __forceinline__ double value_of(const u32x4* x, int j) {
  const uint32_t u = x[j >> 3][(j & 7) >> 1];
  return (double)(j & 1 ? bf16_hi(u) : bf16_lo(u));
}
__device__ __forceinline__ void given_values(const u32x4* x, uint32_t* hi) {
#pragma unroll
  for (int j = 0; j < 16; ++j) hi[j] = to_odd(value_of(x, j));
}
// The 16 values of a lane normed (w not null) and turned by s, c.
template <int LPR, bool NEAR>
__device__ __forceinline__ void key_values(const u32x4* x, const u32x4* w, float eps, bool norm, bool turns, const double* s, const double* c, uint32_t* hi) {
  double inv = 1.0;
  if (norm) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) sum = __builtin_fma(value_of(x, j), value_of(x, j), sum);
    inv = 1.0 / __builtin_sqrt(row_sum<LPR>(sum) * (1.0 / (16 * LPR)) + (double)eps);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int u = NEAR ? 2 * j : j, v = NEAR ? 2 * j + 1 : 8 + j;
    double p = value_of(x, u), q = value_of(x, v);
    if (norm) {
      p = p * inv * value_of(w, u);
      q = q * inv * value_of(w, v);
    }
    const double p1 = __builtin_fma(-q, s[j], p * c[j]), q1 = __builtin_fma(p, s[j], q * c[j]);
    // (a dimension that is not turned is not touched by the other, whatever that is)
    hi[u] = to_odd(turns ? p1 : p);
    hi[v] = to_odd(turns ? q1 : q);
  }
}
template <bool NEAR>
__device__ __forceinline__ void key_angles(const HeadArgs& a, int i, int pos, bool turns, double* s, double* c) {
  f32x4 freq[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (turns) {
    freq[0] = *(const f32x4*)(a.freq + 8 * i);
    freq[1] = *(const f32x4*)(a.freq + 8 * i + 4);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sincos_turn(turn_of(pos, freq[j >> 2][j & 3]), s[j], c[j]);
}
__device__ __forceinline__ void put_codes(char* at, int c0, int c1, u32x4 codes) {
  *(u32x2*)(at + c0) = u32x2{codes[0], codes[1]};
  *(u32x2*)(at + c1) = u32x2{codes[2], codes[3]};
}

// Where blocks begin among the 64 token rows from t0 on: a row whose slot does not follow that of the row before in the same page; of
// those one in 2^share.
__device__ __forceinline__ uint64_t block_begins(const QuantArgs& a, int t0, int turn, int l) {
  const int t = t0 + l;
  const int s = t < a.h.total ? a.slots[t] : -1, p = t > 0 && t < a.h.total ? a.slots[t - 1] : -1;
  const uint64_t begins = __builtin_amdgcn_ballot_w64(s >= 0 && !(p == s - 1 && (s & 63) != 0));
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(begins >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)begins, 0));
  return begins & __builtin_amdgcn_ballot_w64((before & ((1 << a.share) - 1)) == turn);
}
// Slot and rows of the block that begins at t; false: its page is not in the pool.
__device__ __forceinline__ bool block_at(const QuantArgs& a, int t, int l, int& slot, int& rows) {
  const int mine = t + l < a.h.total ? a.slots[t + l] : -1;
  slot = __builtin_amdgcn_readfirstlane(mine);
  const uint64_t others = ~__builtin_amdgcn_ballot_w64((slot & 63) + l < 64 && mine == slot + l);
  rows = others == 0 ? 64 : __builtin_ctzll(others);
  if ((slot >> 6) < a.n_pages) return true;
  if (l == 0) atomicOr(a.h.status, (uint32_t)FLUX_DEV_BAD_PAGE);
  return false;
}

// Short calls: a workgroup per block, head and K or V, 16 rows per wave (most blocks of a decode step have one), and the queries beside them.
constexpr int kWaveRows = 16;
template <int D, bool NEAR>
__global__ __launch_bounds__(256) void qkv_quant_kernel(QuantArgs a) {
  constexpr int LPR = D / 16, RPS = 64 / LPR, STEPS = kWaveRows / RPS;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x >= a.kv_wgs) {
    const int64_t units = (int64_t)a.h.total * a.h.waves, step = (int64_t)(gridDim.x - a.kv_wgs) * 4;
    for (int64_t u = (int64_t)(blockIdx.x - a.kv_wgs) * 4 + w; u < units; u += step) {
      const int64_t t = u / a.h.waves;
      const int pos = a.h.rot ? a.h.pos[t] : 0;
      HeadArgs q = a.h;
      q.hkv = 0;
      token_rows<D, NEAR, false>(q, t, pos, (int)(u - t * a.h.waves), l, [&](int) { return (char*)nullptr; }, [&](int) { return (char*)nullptr; });
    }
    return;
  }
  __shared__ uint32_t tops[2][4];
  int turns_of = 0;                                          // (blocks take turns with the words: a barrier each)
  const int i = l % LPR;
  const uint32_t per_tile = (2u * a.h.hkv) << a.share;
  for (uint32_t u = blockIdx.x; u < a.units; u += a.kv_wgs) {                      // (units < 2^31, a launch below 2^25)
    const int tile = (int)(u / per_tile), rest = (int)(u - tile * per_tile), h = rest >> (a.share + 1);
    const bool is_v = (rest >> a.share) & 1;
    const bool norm = !is_v && a.h.k_norm != nullptr;
    int c0 = 16 * i, c1 = 16 * i + 8;
    bool turns = false;
    if (!is_v) lane_places<NEAR>(i, a.h.rot, c0, c1, turns);
    const char* src = (is_v ? a.h.v : a.h.k) + (int64_t)h * D * 2;
    const int64_t src_step = is_v ? a.h.stride_v : a.h.stride_k;
    uint64_t begins = block_begins(a, tile * 64, rest & ((1 << a.share) - 1), l);
    while (begins != 0) {                                    // (the same for all waves of the workgroup)
      const int t0 = tile * 64 + __builtin_ctzll(begins);
      begins &= begins - 1;
      int slot, rows;
      if (!block_at(a, t0, l, slot, rows)) continue;
      const int page = slot >> 6, held = slot & 63;
      float* const scale_at = (is_v ? a.v_scale : a.k_scale) + (int64_t)page * a.h.hkv + h;
      char* const dst = (is_v ? a.v : a.k) + (int64_t)page * a.stride_p + (int64_t)h * a.stride_h;
      u32x4 x[STEPS][2], wp[2];
      int pos[STEPS];
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int r = kWaveRows * w + k * RPS + l / LPR;
        x[k][0] = x[k][1] = u32x4{0, 0, 0, 0};
        pos[k] = 0;
        if (r < rows) {
          const char* at = src + (int64_t)(t0 + r) * src_step;
          x[k][0] = *(const u32x4*)(at + 2 * c0);
          x[k][1] = *(const u32x4*)(at + 2 * c1);
          if (turns) pos[k] = a.h.pos[t0 + r];
        }
      }
      const float old = held != 0 ? *scale_at : 0.f;
      if (norm) {
        wp[0] = *(const u32x4*)(a.h.k_norm + 2 * c0);
        wp[1] = *(const u32x4*)(a.h.k_norm + 2 * c1);
      }
      uint32_t val[STEPS][16], top = 0;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        if (kWaveRows * w + k * RPS >= rows) continue;       // (uniform)
        if (is_v) {
          given_values(x[k], val[k]);
        } else {
          double s[8], c[8];
          key_angles<NEAR>(a.h, i, pos[k], turns, s, c);
          key_values<LPR, NEAR>(x[k], wp, a.h.eps, norm, turns, s, c, val[k]);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) top = max(top, finite_or_zero(val[k][j]));
      }
      // (rows that the block does not have count as zeros)
      top = wave_max(top);
      turns_of ^= 1;
      if (l == 0) tops[turns_of][w] = top;
      __syncthreads();
      top = max(max(tops[turns_of][0], tops[turns_of][1]), max(tops[turns_of][2], tops[turns_of][3]));
      top = __builtin_amdgcn_readfirstlane(top);
      const float scale = block_scale(top, old), inv = 1.0f / scale;      // (exact: a power of two)
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int r = kWaveRows * w + k * RPS + l / LPR;
        if (r < rows) put_codes(dst + (int64_t)(held + r) * a.stride_t, c0, c1, codes16(val[k], (double)inv));
      }
      if (held != 0 && scale > old)                          // the rows that the page holds take the new scale too
        for (int r = w * RPS + l / LPR; r < held; r += 4 * RPS) scale_down(dst + (int64_t)r * a.stride_t + 16 * i, old * inv);
      if (threadIdx.x == 0 && (held == 0 || scale > old)) *scale_at = scale;
    }
  }
}

// Long calls: a workgroup per block, head and K or V, 16 rows per wave.  Keys are worked out in 32 bits.  Where the bounds of a value's error round to two different codes (one step of 8 or 16 rows in ten has such a
// value) the step is worked out again in 64 bits, and so is the block's largest value where it lies next to the border of its scale.
//
// The error in 32 bits, in units of 2^-24: the mean of squares takes 4 + 2 + 3 sums and one product, 10 of it; its root's reciprocal
// half of that and 2 for the instruction, 7; two products, 9 for each of a pair (a, b).  Sine and cosine are off by 4 at most, so a turned
// value by (9 + 4 + 2) (|a| + |b|) and 1 for its own rounding: below 2^-20 (|a| + |b|), where |a| + |b| is at most sqrt(2) times the
// sum of the turned magnitudes.
constexpr float kTurnedError = 0x1.7p-20f;                   // of the sum of a turned pair's magnitudes
constexpr uint32_t kBorder = 0x600000u, kBorderError = 64;   // 0.75 as a fraction; the error of a largest value in steps of it (2^-20 * 1.5 * 2 * 2^24, and more)

// Sine and cosine of `quarters` quarter turns in 32 bits: the nearest whole number of them (adding 1.5 * 2^52 rounds to one, whose low bits
// are then the low bits of the sum), and Taylor's series of what is left, at most pi / 4, whose remainders are 2^-29 and 2^-25.3; with the roundings
// of the argument and of the sums below 2^-22.
__device__ __forceinline__ void sincos_close(double quarters, float& s, float& c) {
  constexpr double kRound = 6755399441055744.0;
  const double m = quarters + kRound;
  const uint32_t n = __builtin_bit_cast(u32x2, m)[0];
  const float x = (float)(quarters - (m - kRound)) * 1.57079632679489661923f, z = x * x;
  float a = 1.0f / 362880, b = 1.0f / 40320;
  a = __builtin_fmaf(a, z, -1.0f / 5040);
  b = __builtin_fmaf(b, z, -1.0f / 720);
  a = __builtin_fmaf(a, z, 1.0f / 120);
  b = __builtin_fmaf(b, z, 1.0f / 24);
  a = __builtin_fmaf(a, z, -1.0f / 6);
  b = __builtin_fmaf(b, z, -0.5f);
  a = __builtin_fmaf(a * z, x, x);
  b = __builtin_fmaf(b, z, 1.0f);
  const float p = n & 1 ? b : a, r = n & 1 ? a : b;
  s = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, p) ^ ((n & 2) << 30));
  c = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, r) ^ (((n + 1) & 2) << 30));
}

// The values of a lane in 64 bits, pair by pair.  (Nothing of it is to be worked out before it is needed, or kept from what 32 bits took:
// with what both share held in registers the kernel has 200 of them in memory.)
template <int LPR, bool NEAR>
__device__ __forceinline__ void key_values_one_by_one(const u32x4* x_in, const u32x4* w_in, const f32x4* freq_in, float eps, bool norm, bool turns, int pos, uint32_t* hi) {
  u32x4 x[2] = {x_in[0], x_in[1]}, w[2] = {w_in[0], w_in[1]};
  f32x4 freq[2] = {freq_in[0], freq_in[1]};
  asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(w[0]), "+v"(w[1]), "+v"(freq[0]), "+v"(freq[1]), "+v"(pos));
  double inv = 1.0;
  if (norm) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) sum = __builtin_fma(value_of(x, j), value_of(x, j), sum);
    inv = 1.0 / __builtin_sqrt(row_sum<LPR>(sum) * (1.0 / (16 * LPR)) + (double)eps);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int u = NEAR ? 2 * j : j, v = NEAR ? 2 * j + 1 : 8 + j;
    double p = value_of(x, u), q = value_of(x, v);
    if (norm) {
      p = p * inv * value_of(w, u);
      q = q * inv * value_of(w, v);
    }
    if (turns) {
      double s, c;
      sincos_turn(turn_of(pos, freq[j >> 2][j & 3]), s, c);
      const double p0 = p, q0 = q;
      p = __builtin_fma(-q0, s, p0 * c);
      q = __builtin_fma(p0, s, q0 * c);
    }
    hi[u] = to_odd(p);
    hi[v] = to_odd(q);
    asm volatile("" : "+v"(hi[u]), "+v"(hi[v]));
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Rows `all` from token row t on, of head h of K (KEY) or V, into the page of `slot`: 16 of them per wave.
template <int D, bool NEAR, bool KEY>
__device__ __forceinline__ void quantise_block(const QuantArgs& a, int t, int slot, int all, int h, int l, int w, uint32_t* tops) {
  constexpr int LPR = D / 16, RPS = 64 / LPR, STEPS = kWaveRows / RPS;
  const int page = slot >> 6, held = slot & 63, i = l % LPR, r0 = kWaveRows * w + l / LPR;
  int c0 = 16 * i, c1 = 16 * i + 8;
  bool turns = false;
  if (KEY) lane_places<NEAR>(i, a.h.rot, c0, c1, turns);
  const int64_t src_step = KEY ? a.h.stride_k : a.h.stride_v;
  const char* src = (KEY ? a.h.k : a.h.v) + t * src_step + (int64_t)h * D * 2;
  const bool norm = KEY && a.h.k_norm != nullptr;
  float* const scale_at = (KEY ? a.k_scale : a.v_scale) + (int64_t)page * a.h.hkv + h;
  char* const dst = (KEY ? a.k : a.v) + (int64_t)page * a.stride_p + (int64_t)h * a.stride_h;
  u32x4 x[STEPS][2], wp[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  int pos[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    x[k][0] = x[k][1] = u32x4{0, 0, 0, 0};
    pos[k] = 0;
    const int r = r0 + k * RPS;
    if (r < all) {
      x[k][0] = *(const u32x4*)(src + r * src_step + 2 * c0);
      x[k][1] = *(const u32x4*)(src + r * src_step + 2 * c1);
      if (KEY && turns) pos[k] = a.h.pos[t + r];
    }
  }
  const float old = held != 0 ? *scale_at : 0.f;
  f32x4 freq[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (norm) {
    wp[0] = *(const u32x4*)(a.h.k_norm + 2 * c0);
    wp[1] = *(const u32x4*)(a.h.k_norm + 2 * c1);
  }
  if (KEY && turns) {
    freq[0] = *(const f32x4*)(a.h.freq + 8 * i);
    freq[1] = *(const f32x4*)(a.h.freq + 8 * i + 4);
  }
  // step k in 64 bits; its rows are read again
  auto in_full = [&](int k, uint32_t* hi) __attribute__((always_inline)) {
    const int r = r0 + k * RPS;
    u32x4 y[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    int p = 0;
    if (r < all) {
      y[0] = *(const u32x4*)(src + r * src_step + 2 * c0);
      y[1] = *(const u32x4*)(src + r * src_step + 2 * c1);
      if (KEY && turns) p = a.h.pos[t + r];
    }
    if (KEY) key_values_one_by_one<LPR, NEAR>(y, wp, freq, a.h.eps, norm, turns, p, hi);
    else given_values(y, hi);
  };
  float val[STEPS][16];
  uint32_t top = 0, odd = 0;                                 // largest magnitude; whether squares pass 32 bits
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    float* y = val[k];
    unpack8(x[k][0], y);
    unpack8(x[k][1], y + 8);
    if (norm) {
      float part[4] = {0.f, 0.f, 0.f, 0.f}, f[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) part[j & 3] = __builtin_fmaf(y[j], y[j], part[j & 3]);
      const float sum = row_sum<LPR>((part[0] + part[1]) + (part[2] + part[3]));
      const float inv = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.0f / D, a.h.eps));
      odd |= sum < 0x1p100f ? 0u : 1u;
      unpack8(wp[0], f);
      unpack8(wp[1], f + 8);
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = y[j] * inv * f[j];
    }
    if (KEY && a.h.rot != 0) {                               // (lanes that turn nothing turn by nothing)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float s, c;
        sincos_close((double)pos[k] * ((double)freq[j >> 2][j & 3] * (4.0 * kTurnsPerRadian)), s, c);
        float& u = NEAR ? y[2 * j] : y[j];
        float& v = NEAR ? y[2 * j + 1] : y[8 + j];
        const float u0 = u, v0 = v;
        u = __builtin_fmaf(-v0, s, u0 * c);
        v = __builtin_fmaf(u0, s, v0 * c);
        if (j % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) top = max(top, __builtin_bit_cast(uint32_t, y[j]) & 0x7FFFFFFFu);
  }
  auto most_of_all = [&](uint32_t y, uint32_t* at) __attribute__((always_inline)) {
    y = wave_max(y);                                         // (rows that the block does not have count as zeros)
    if (l == 0) at[w] = y;
    __syncthreads();
    return (uint32_t)__builtin_amdgcn_readfirstlane(max(max(at[0], at[1]), max(at[2], at[3])));
  };
  if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) top = 0x7F800000u;
  top = most_of_all(top, tops);
  const bool some_odd = top >= 0x7F800000u;                  // some value of the block is not finite, or left to 64 bits
  float scale;
  if (__builtin_expect(some_odd || (KEY && (top & 0x7FFFFFu) + kBorderError - kBorder <= 2 * kBorderError), 0)) {   // (the same for all waves)
    uint32_t most = 0;
#pragma unroll 1
    for (int k = 0; k < STEPS; ++k) {
      uint32_t hi[16];
      in_full(k, hi);
#pragma unroll
      for (int j = 0; j < 16; ++j) most = max(most, finite_or_zero(hi[j]));
    }
    scale = block_scale(most_of_all(most, tops + 4), old);
  } else {
    const int e = max((int)(top >> 23) - 135 + ((top & 0x7FFFFFu) > kBorder ? 1 : 0), kMinScaleExp);
    scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    scale = old > scale ? old : scale;
  }
  const float inv = 1.0f / scale;                            // exact: a power of two
  uint32_t again = some_odd ? ~0u : 0u;                      // steps that 32 bits do not settle
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    u32x4 codes;
    if (KEY) {
      uint32_t apart = 0;
      float below[16], above[16];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int u = NEAR ? 2 * j : j, v = NEAR ? 2 * j + 1 : 8 + j;
        const float p = val[k][u] * inv, q = val[k][v] * inv, off = (__builtin_fabsf(p) + __builtin_fabsf(q)) * kTurnedError;
        below[u] = p - off, above[u] = p + off;
        below[v] = q - off, above[v] = q + off;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        codes[j] = codes4(below[4 * j], below[4 * j + 1], below[4 * j + 2], below[4 * j + 3]);
        apart |= codes[j] ^ codes4(above[4 * j], above[4 * j + 1], above[4 * j + 2], above[4 * j + 3]);
      }
      if (__builtin_amdgcn_ballot_w64(apart != 0) != 0) again |= 1u << k;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) codes[j] = codes4(val[k][4 * j] * inv, val[k][4 * j + 1] * inv, val[k][4 * j + 2] * inv, val[k][4 * j + 3] * inv);
    }
    if (r0 + k * RPS < all) put_codes(dst + (int64_t)(held + r0 + k * RPS) * a.stride_t, c0, c1, codes);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll 1
  for (int k = 0; k < STEPS; ++k) {
    if (!((again >> k) & 1)) continue;
    uint32_t hi[16];
    in_full(k, hi);
    if (r0 + k * RPS < all) put_codes(dst + (int64_t)(held + r0 + k * RPS) * a.stride_t, c0, c1, codes16(hi, (double)inv));
  }
  if (held != 0 && scale > old)                              // the rows that the page holds take the new scale too
    for (int r = w * RPS + l / LPR; r < held; r += 4 * RPS) scale_down(dst + (int64_t)r * a.stride_t + 16 * i, old * inv);
  if (threadIdx.x == 0 && (held == 0 || scale > old)) *scale_at = scale;
}

template <int D, bool NEAR>
__global__ __launch_bounds__(256, 3) void quant_pages_kernel(QuantArgs a) {
  __shared__ uint32_t tops[2][8];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int turn = 0;                                              // (blocks take turns with the words: a barrier each)
  const uint32_t per_tile = (2u * a.h.hkv) << a.share;
  for (uint32_t u = blockIdx.x; u < a.units; u += gridDim.x) {                     // (units < 2^31, a launch below 2^25)
    const int tile = (int)(u / per_tile), rest = (int)(u - tile * per_tile), h = rest >> (a.share + 1);
    uint64_t begins = block_begins(a, tile * 64, rest & ((1 << a.share) - 1), l);
    while (begins != 0) {                                    // (the same for all waves of the workgroup)
      const int t0 = tile * 64 + __builtin_ctzll(begins);
      begins &= begins - 1;
      int slot, rows;
      if (!block_at(a, t0, l, slot, rows)) continue;
      turn ^= 1;
      if ((rest >> a.share) & 1) quantise_block<D, NEAR, false>(a, t0, slot, rows, h, l, w, tops[turn]);
      else quantise_block<D, NEAR, true>(a, t0, slot, rows, h, l, w, tops[turn]);
    }
  }
}

namespace {
HeadArgs head_args(const HeadRows& r, bool with_k, bool with_v) {
  HeadArgs a = {};
  a.q = (const char*)r.in.q;
  a.k = (const char*)r.in.k;
  a.v = (const char*)r.in.v;
  a.stride_q = 2 * r.in.stride_q;
  a.stride_k = 2 * r.in.stride_k;
  a.stride_v = 2 * r.in.stride_v;
  a.q_out = (char*)r.q_out;
  a.q_norm = (const char*)r.cfg.q_norm;
  a.k_norm = (const char*)r.cfg.k_norm;
  a.freq = r.cfg.inv_freq;
  a.pos = r.positions;
  a.eps = r.cfg.eps;
  a.hq = r.q_out ? r.cfg.n_q_heads : 0;
  a.hkv = r.cfg.n_kv_heads;
  a.total = r.total;
  a.rot = r.cfg.rotary_dim;
  const int rows = a.hq + (with_k ? a.hkv : 0) + (with_v ? a.hkv : 0), per_pass = 64 / (r.cfg.head_dim / 16);
  a.passes = (rows + per_pass - 1) / per_pass;
  a.waves = head_waves(r.total, a.passes);
  return a;
}
unsigned wgs_for(const HeadArgs& a) {
  const long long n = ((long long)a.total * a.waves + 3) / 4;
  return (unsigned)(n < kAppendMost ? n : kAppendMost);
}
}  // namespace

#define FLUX_HEADS(kernel, cfg, grid, threads, stream, args)                                                                       \
  do {                                                                                                                             \
    if ((cfg).head_dim == 128 && (cfg).interleaved) hipLaunchKernelGGL((kernel<128, true>), dim3(grid), dim3(threads), 0, stream, args);   \
    else if ((cfg).head_dim == 128) hipLaunchKernelGGL((kernel<128, false>), dim3(grid), dim3(threads), 0, stream, args);          \
    else if ((cfg).interleaved) hipLaunchKernelGGL((kernel<64, true>), dim3(grid), dim3(threads), 0, stream, args);                \
    else hipLaunchKernelGGL((kernel<64, false>), dim3(grid), dim3(threads), 0, stream, args);                                      \
  } while (0)

hipError_t launch_head_rows(const HeadRows& r, void* k_out, hipStream_t s) {
  HeadArgs a = head_args(r, k_out != nullptr, false);
  a.k_out = (char*)k_out;
  if (!k_out) a.hkv = 0;
  FLUX_HEADS(head_rows_kernel, r.cfg, wgs_for(a), 256, s, a);
  return hipGetLastError();
}

hipError_t launch_qkv_append(const Ctx& c, const HeadRows& r, const flux_kv_cache& cache, const int32_t* cu_new, hipStream_t s) {
  HeadArgs a = head_args(r, true, true);
  a.cu = cu_new;
  a.kc = (char*)cache.k;
  a.vc = (char*)cache.v;
  a.stride_b = 2 * cache.stride_b;
  a.stride_h = 2 * cache.stride_h;
  a.stride_t = 2 * cache.stride_t;
  a.kv_len = cache.kv_len;
  a.batch = cache.batch;
  a.capacity = cache.capacity;
  a.counter = c.counters + 0;
  a.gather = c.append_counters;
  a.status = c.status;
  FLUX_HEADS(qkv_rows_kernel, r.cfg, wgs_for(a), 256, s, a);
  return hipGetLastError();
}

hipError_t launch_qkv_append_paged(const Ctx& c, const HeadRows& r, const flux_paged_kv& kv, const int32_t* slots, hipStream_t s) {
  QuantArgs a;
  a.h = head_args(r, false, false);
  a.h.status = c.status;
  a.k = (char*)kv.k;
  a.v = (char*)kv.v;
  a.k_scale = kv.k_scale;
  a.v_scale = kv.v_scale;
  a.stride_p = kv.stride_p;
  a.stride_h = kv.stride_h;
  a.stride_t = kv.stride_t;
  a.slots = slots;
  a.n_pages = kv.n_pages;
  const long long tiles = ((long long)r.total + 63) / 64;
  if (r.total >= kQuantLong) {
    a.share = 6;
    while (a.share > 0 && (tiles * 2 * r.cfg.n_kv_heads << a.share) > kAppendPagedWaves) --a.share;
    a.units = (uint32_t)(tiles * 2 * r.cfg.n_kv_heads << a.share);
    if (a.h.passes > 0) {
      HeadArgs q = a.h;
      q.hkv = 0;
      FLUX_HEADS(head_rows_kernel, r.cfg, wgs_for(q), 256, s, q);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    FLUX_HEADS(quant_pages_kernel, r.cfg, a.units < (uint32_t)kAppendMost ? a.units : (uint32_t)kAppendMost, 256, s, a);
    return hipGetLastError();
  }
  a.share = 6;
  while (a.share > 0 && (tiles * 2 * r.cfg.n_kv_heads << a.share) > kAppendPagedWaves) --a.share;
  a.units = (uint32_t)(tiles * 2 * r.cfg.n_kv_heads << a.share);
  a.kv_wgs = a.units < (uint32_t)kAppendMost ? a.units : (uint32_t)kAppendMost;
  const unsigned q_wgs = a.h.passes > 0 ? wgs_for(a.h) : 0;
  FLUX_HEADS(qkv_quant_kernel, r.cfg, a.kv_wgs + q_wgs, 256, s, a);
  return hipGetLastError();
}

}  // namespace flux
