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
// In 64 bits: the nearest quarter turn, and Taylor's series of what is left (at most pi / 4): the sine up to x^11, which leaves x^13 / 13! or 2^-37, the cosine up to
// x^12, which leaves x^14 / 14! or 2^-41.
__device__ __forceinline__ void sincos_turn(double t, double& s, double& c) {
  const double quarter = __builtin_rint(4.0 * t);
  const double x = (t - 0.25 * quarter) * 6.28318530717958647693, z = x * x;
  double a = -1.0 / 39916800, b = 1.0 / 479001600;
  b = __builtin_fma(b, z, -1.0 / 3628800);
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

// Passes that a wave asks for at once.  us of the kernels with 4 / 3 / 2, 32/8 heads of 128, 32768 tokens 135 / 132 / 131; appended, 28/4 heads, 129 to
// 3001 tokens of five sequences 29.4 / 26.2 / 25.0 (of fewer registers more waves are at work).
constexpr int kPassesInFlight = 2;

// All rows of one token that this wave has: passes p0, p0 + step, ...  A pass is 64 / (D / 16) rows: the query heads first, then the
// key heads, then (V) the value heads, which are copied.  position(): of the token, asked when its first rows are on their way; k_at(h), v_at(h):
// where a finished row goes, null: nowhere.
template <int D, bool NEAR, bool V, typename PP, typename KP, typename VP>
__device__ __forceinline__ void token_rows(const HeadArgs& a, int64_t t, PP position, int p0, int l, KP k_at, VP v_at) {
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
      __builtin_amdgcn_sched_barrier(0);
      const int pos = position();
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

// A wave per token, or several where tokens are few.  Bound by the memory: 32768 tokens of 32 and 8 heads of 128 (671 MB) 124 us, 5.4 TB/s; 16 of 8 and 2 of 64
// 2.8, which is a launch and its two waits.
template <int D, bool NEAR>
__global__ __launch_bounds__(256) void head_rows_kernel(HeadArgs a) {
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)a.total * a.waves;
  for (int64_t u = (int64_t)blockIdx.x * 4 + w; u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / a.waves;
    token_rows<D, NEAR, false>(a, t, [&]() { return a.rot ? a.pos[t] : 0; }, (int)(u - t * a.waves), l, [&](int h) { return a.k_out + (t * a.hkv + h) * D * 2; }, [&](int) { return (char*)nullptr; });
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
// them moves them on (see kv_append.hip).  Five chunks of 129 to 3001 tokens, 28 and 4 heads of 128 (120 MB): 25 us, 4.8 TB/s; a step of 16
// sequences 4.8, in which the sequence of a row, its length and the arrivals wait for each other.
template <int D, bool NEAR>
__global__ __launch_bounds__(256) void qkv_rows_kernel(HeadArgs a) {
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t units = (int64_t)a.total * a.waves;
  // what the last workgroup needs of up to 256 sequences, one per thread
  const int own = min((int)threadIdx.x, a.batch - 1);
  const int my_cu = a.cu[own], my_end = a.cu[own + 1], my_len = a.kv_len[own];
  const int end = a.cu[a.batch], begin = a.cu[0];
  bool overflow = false;
  for (int64_t u = (int64_t)blockIdx.x * 4 + w; u < units; u += (int64_t)gridDim.x * 4) {
    const int64_t t = u / a.waves;
    if (t < begin || t >= end) continue;                     // rows of no sequence
    bool kept = false;
    int64_t row = 0;
    auto place = [&]() {
      const int b = sequence_of(a.cu, a.batch, (int)t, l);
      const int64_t at = (int64_t)a.kv_len[b] + (t - a.cu[b]);
      kept = at >= 0 && at < a.capacity;
      overflow |= !kept;
      row = (int64_t)b * a.stride_b + at * a.stride_t;
      return a.pos ? a.pos[t] : (int)at;
    };
    token_rows<D, NEAR, true>(a, t, place, (int)(u - t * a.waves), l, [&](int h) { return kept ? a.kc + row + h * a.stride_h : nullptr; },
                              [&](int h) { return kept ? a.vc + row + h * a.stride_h : nullptr; });
  }
  if (overflow && l == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_KV_OVERFLOW);
  // (a wave holds the length that it read before it passes the barrier, as its rows' places come from it; the stores are not waited for)
  __shared__ int is_last;
  asm volatile("" : : "v"(my_len), "v"(my_cu), "v"(my_end) : "memory");
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
    const int n = b < 256 ? my_end - my_cu : a.cu[b + 1] - a.cu[b];
    int len = b < 256 ? my_len : a.kv_len[b];
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
  int share;                      // 2^share workgroups look after a tile of 64 token rows, of K or V
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
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;
// The larger of each half.
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Largest of a wave's: within rows of 16 lanes, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_moved(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false)); }
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max_moved<0x111, 0xf>(x);
  x = max_moved<0x112, 0xf>(x);
  x = max_moved<0x114, 0xf>(x);
  x = max_moved<0x118, 0xf>(x);
  x = max_moved<0x142, 0xa>(x);
  return (uint32_t)__builtin_amdgcn_readlane((int)max_moved<0x143, 0xc>(x), 63);
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
typedef __attribute__((__vector_size__(2 * sizeof(double)))) double f64x2;
__device__ __forceinline__ double value_of(const u32x4* x, int j) {
  const uint32_t u = x[j >> 3][(j & 7) >> 1];
  return (double)(j & 1 ? bf16_hi(u) : bf16_lo(u));
}
// The 16 values of a lane normed and turned, in 64 bits, pair by pair (which keeps registers free).  `angles`: this thread's eight sines and cosines in
// LDS, THREADS apart; they are worked out where `fresh`, else found there.
template <int LPR, bool NEAR, int THREADS>
__device__ __forceinline__ void key_values(const HeadArgs& a, const u32x4* x, const u32x4* w, int i, int pos, bool norm, bool turns, bool fresh, f64x2* angles, uint32_t* hi) {
  double inv = 1.0;
  if (norm) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) sum = __builtin_fma(value_of(x, j), value_of(x, j), sum);
    inv = 1.0 / __builtin_sqrt(row_sum<LPR>(sum) * (1.0 / (16 * LPR)) + (double)a.eps);
  }
  if (fresh && a.rot != 0) {
    f32x4 freq[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if (turns) {
      freq[0] = *(const f32x4*)(a.freq + 8 * i);
      freq[1] = *(const f32x4*)(a.freq + 8 * i + 4);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      double s, c;
      sincos_turn(turn_of(pos, freq[j >> 2][j & 3]), s, c);
      angles[j * THREADS] = f64x2{s, c};
      if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int u = NEAR ? 2 * j : j, v = NEAR ? 2 * j + 1 : 8 + j;
    double p = value_of(x, u), q = value_of(x, v);
    if (norm) {
      p = p * inv * value_of(w, u);
      q = q * inv * value_of(w, v);
    }
    if (a.rot != 0) {
      const f64x2 turn = angles[j * THREADS];
      const double s = turn[0], c = turn[1];
      const double p1 = __builtin_fma(-q, s, p * c), q1 = __builtin_fma(p, s, q * c);
      // (a dimension that is not turned is not touched by the other, whatever that is)
      p = turns ? p1 : p;
      q = turns ? q1 : q;
    }
    hi[u] = to_odd(p);
    hi[v] = to_odd(q);
    asm volatile("" : "+v"(hi[u]), "+v"(hi[v]));             // (worked out here, not where they are used)
    if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
  }
}
__device__ __forceinline__ void put_codes(char* at, int c0, int c1, u32x4 codes) {
  *(u32x2*)(at + c0) = u32x2{codes[0], codes[1]};
  *(u32x2*)(at + c1) = u32x2{codes[2], codes[3]};
}

// The blocks of a tile of 64 token rows.  A row goes on a block if its slot follows that of the row before in the same page, and begins one
// otherwise; a block that the tile's last row has goes on in the next tile.
struct Tile {
  int slot;                       // of this lane's row, -1: none
  uint64_t begins, on, on_next;   // rows that begin a block, that go on one, and those of the next tile
};
__device__ __forceinline__ Tile load_tile(const QuantArgs& a, int t0, int l) {
  Tile x;
  const int t = t0 + l;
  x.slot = t < a.h.total ? a.slots[t] : -1;
  const int next = t + 64 < a.h.total ? a.slots[t + 64] : -1, first = t0 > 0 ? a.slots[t0 - 1] : -1;
  const int last = __builtin_amdgcn_readlane(x.slot, 63);
  const int up = __shfl_up(x.slot, 1), up_next = __shfl_up(next, 1);              // (by all lanes)
  const int p = l > 0 ? up : first, p_next = l > 0 ? up_next : last;
  const bool follows = x.slot >= 0 && p == x.slot - 1 && (x.slot & 63) != 0;
  x.begins = __builtin_amdgcn_ballot_w64(x.slot >= 0 && !follows);
  x.on = __builtin_amdgcn_ballot_w64(follows);
  x.on_next = __builtin_amdgcn_ballot_w64(next >= 0 && p_next == next - 1 && (next & 63) != 0);
  return x;
}
// Rows of the block that begins at this lane's row.
__device__ __forceinline__ int block_rows(const Tile& x, int l) {
  const uint64_t stop = l < 63 ? ~x.on >> (l + 1) : 0;       // (shifted-in zeros: the next tile)
  if (stop != 0) return 1 + __builtin_ctzll(stop);
  return 64 - l + (~x.on_next == 0 ? 64 : __builtin_ctzll(~x.on_next));
}
// Place of the n-th set bit of x (which has so many).
__device__ __forceinline__ int nth_set(uint64_t x, int n) {
  int at = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) {
    const int below = __builtin_popcountll(x & ((1ull << step) - 1));
    if (n >= below) {
      n -= below;
      at += step;
      x >>= step;
    }
  }
  return at;
}

// What a workgroup of W waves has of its tile's (block, head) pairs, which 2^share workgroups look after: a wave holds 64 / W rows at a time, so blocks of
// one row go to a wave for as many heads at once (kSingle), other blocks of up to 64 / W rows to a wave per head (kAlone), the rest to a whole workgroup per
// head (kShared).  one(pair, rows, how): while it is worked on, what fetch(pair, how) asks for of the next pair is on its way.
enum { kSingle, kAlone, kShared };
struct Pair {
  int at, slot, rows, head;       // row of the tile where the block begins, its slot; rows of the block; head, or first of them
};
struct Rows {                     // of a lane
  u32x4 x[2];
  int pos;
  float old;                      // scale that the page has
};
template <int W, typename G, typename F>
__device__ __forceinline__ void for_blocks(const QuantArgs& a, int tile, int turn, int l, int w, G fetch, F one) {
  const Tile x = load_tile(a, tile * 64, l);
  const int mine = block_rows(x, l), hkv = a.h.hkv;
  const bool begins = (x.begins >> l) & 1, in_pool = (x.slot >> 6) < a.n_pages;
  if (turn == 0 && w == 0 && __builtin_amdgcn_ballot_w64(begins && !in_pool) != 0 && l == 0) atomicOr(a.h.status, (uint32_t)FLUX_DEV_BAD_PAGE);
  const uint64_t single_ones = __builtin_amdgcn_ballot_w64(begins && in_pool && mine == 1);
  const uint64_t short_ones = __builtin_amdgcn_ballot_w64(begins && in_pool && mine > 1 && mine <= 64 / W);
  const uint64_t long_ones = __builtin_amdgcn_ballot_w64(begins && in_pool && mine > 64 / W);
#pragma unroll 1
  for (int how = kSingle; how <= kShared; ++how) {
    const bool alone = how != kShared;
    const uint64_t set = how == kSingle ? single_ones : (alone ? short_ones : long_ones);
    const int sharers = (alone ? W : 1) << a.share, me = alone ? W * turn + w : turn;
    const int per = how == kSingle ? (hkv + 64 / W - 1) / (64 / W) : hkv;          // of a block
    const int64_t pairs = (int64_t)__builtin_popcountll(set) * per;
    auto nth = [&](int64_t pair) __attribute__((always_inline)) {
      const int block = (int)((uint32_t)pair / (uint32_t)per), at = __builtin_amdgcn_readfirstlane(nth_set(set, block)), head = (int)pair - block * per;
      return Pair{at, __builtin_amdgcn_readlane(x.slot, at), __builtin_amdgcn_readlane(mine, at), how == kSingle ? head * (64 / W) : head};
    };
    if (me >= pairs) continue;
    Pair now = nth(me);
    Rows rows = fetch(now, how);
#pragma unroll 1
    for (int64_t pair = me; pair < pairs; pair += sharers) {
      Pair next = now;
      Rows next_rows = rows;
      if (pair + sharers < pairs) {
        next = nth(pair + sharers);
        next_rows = fetch(next, how);
      }
      one(now, rows, how);
      now = next;
      rows = next_rows;
    }
  }
}
// Largest of what the lanes of a row (kSingle), of a wave (kAlone) or of the workgroup have.
template <int W, int LPR>
__device__ __forceinline__ uint32_t block_max(uint32_t y, int how, uint32_t* words, int l, int w) {
  if (how == kSingle) {
    y = max(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0xB1, 0xf, 0xf, true));  // as in row_sum
    y = max(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x4E, 0xf, 0xf, true));
    if constexpr (LPR == 8) y = max(y, (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x141, 0xf, 0xf, true));
    return y;
  }
  y = wave_max(y);
  if (how == kShared) {
    if (l == 0) words[w] = y;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) y = max(y, words[i]);
  }
  return y;
}

// One launch: K, V, then the queries.  What bounds it: a decode step its latencies (slots, rows, the arithmetic of 64 bits), a long prompt the
// memory and that arithmetic together.  A workgroup with several heads of a block works their angles out once and keeps them in LDS.  us, 32/8 heads of 128:
// 64 sequences with a row each 6.5, 256 6.7, 1024 8.6 (a wave per head of each row: 35), 1024 rows of one 12.3, 4096 24, 16384 80 (369 MB, 4.6 TB/s; 118 with
// angles for every head, 89 with rows that are asked for when they are needed and K and V in turn).  Keys from 32 bits,
// worked out again in 64 where 32 do not settle a code, took 108 for the 16384 rows in launches of their own for queries, keys and values.
constexpr int quant_waves(int head_dim) { return head_dim == 128 ? 8 : 4; }   // of a workgroup: a row per D / 16 lanes, 64 rows in all
template <int D, bool NEAR>
__global__ __launch_bounds__(64 * quant_waves(D), 4) void qkv_quant_kernel(QuantArgs a) {
  constexpr int LPR = D / 16, W = quant_waves(D), RPW = 64 / W;
  static_assert(RPW * LPR == 64, "a wave holds its rows at once");
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x >= a.kv_wgs) {
    const int64_t units = (int64_t)a.h.total * a.h.waves, step = (int64_t)(gridDim.x - a.kv_wgs) * W;
    for (int64_t u = (int64_t)(blockIdx.x - a.kv_wgs) * W + w; u < units; u += step) {
      const int64_t t = u / a.h.waves;
      HeadArgs q = a.h;
      q.hkv = 0;
      q.k_norm = nullptr;                                    // (its registers)
      token_rows<D, NEAR, false>(q, t, [&]() { return a.h.rot ? a.h.pos[t] : 0; }, (int)(u - t * a.h.waves), l, [&](int) { return (char*)nullptr; }, [&](int) { return (char*)nullptr; });
    }
    return;
  }
  __shared__ uint32_t tops[2][W];
  __shared__ f64x2 s_angles[8 * 64 * W];
  int turn_of = 0;                                           // (blocks take turns with the words: a barrier each)
  int angles_of = -1;                                        // the block whose angles this wave has in LDS
  const int i = l % LPR;
  // K first, which takes longer (K and V in turn give all of K to every other XCD: 16384 rows 85 us for 79)
  const unsigned half = a.kv_wgs >> 1;
  const bool is_v = blockIdx.x >= half;
  const unsigned wg = blockIdx.x - (is_v ? half : 0);
  const int tile = (int)(wg >> a.share);
  const bool norm = !is_v && a.h.k_norm != nullptr;
  int c0 = 16 * i, c1 = 16 * i + 8;
  bool turns = false;
  if (!is_v) lane_places<NEAR>(i, a.h.rot, c0, c1, turns);
  const int64_t src_step = is_v ? a.h.stride_v : a.h.stride_k;
  auto fetch = [&](const Pair b, int how) __attribute__((always_inline)) {
    const int r = how == kSingle ? 0 : RPW * (how == kShared ? w : 0) + l / LPR, h = b.head + (how == kSingle ? l / LPR : 0);
    const int t = tile * 64 + b.at;
    Rows y = {{{0, 0, 0, 0}, {0, 0, 0, 0}}, 0, 0.f};         // (rows that the block does not have count as zeros)
    if (r < b.rows && h < a.h.hkv) {
      const char* src = (is_v ? a.h.v : a.h.k) + (int64_t)(t + r) * src_step + (int64_t)h * D * 2;
      y.x[0] = *(const u32x4*)(src + 2 * c0);
      y.x[1] = *(const u32x4*)(src + 2 * c1);
      if (turns) y.pos = a.h.pos[t + r];
    }
    if ((b.slot & 63) != 0 && h < a.h.hkv) y.old = (is_v ? a.v_scale : a.k_scale)[(int64_t)(b.slot >> 6) * a.h.hkv + h];
    return y;
  };
  for_blocks<W>(a, tile, (int)(wg & ((1u << a.share) - 1)), l, w, fetch, [&](const Pair b, const Rows& y, int how) __attribute__((always_inline)) {
    const bool single = how == kSingle, alone = how != kShared;
    const int at = b.at, page = b.slot >> 6, held = b.slot & 63, h = b.head + (single ? l / LPR : 0), pos = y.pos;
    const int part = alone ? 0 : w, r = single ? 0 : RPW * part + l / LPR;
    const bool has = r < b.rows && h < a.h.hkv;              // a row of its own
    float* const scale_at = (is_v ? a.v_scale : a.k_scale) + (int64_t)page * a.h.hkv + h;
    char* const dst = (is_v ? a.v : a.k) + (int64_t)page * a.stride_p + (int64_t)h * a.stride_h;
    const u32x4 (&x)[2] = y.x;
    const float old = y.old;
    float scale, inv;                                        // (inv: exact, a power of two)
    turn_of ^= alone ? 0 : 1;
    if (is_v) {
      // values as they are: their bits say which is the largest, and 32 bits hold all that a code needs
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = pair_max(most, x[j >> 2][j & 3] & 0x7FFF7FFFu);
      const bool odd = __builtin_amdgcn_ballot_w64((most & 0xFFFFu) >= 0x7F80u || (most >> 16) >= 0x7F80u) != 0;   // some value is not finite
      if (odd) {
        most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t lo = x[j >> 2][j & 3] & 0x7FFFu, hi = (x[j >> 2][j & 3] >> 16) & 0x7FFFu;
          most = pair_max(most, (lo < 0x7F80u ? lo : 0u) | (hi < 0x7F80u ? hi << 16 : 0u));
        }
      }
      most = block_max<W, LPR>(max(most & 0xFFFFu, most >> 16), how, tops[turn_of], l, w);
      // most = (1 + f / 128) 2^(E - 127): see block_scale
      const int e = max((int)(most >> 7) - 135 + ((most & 127) > 96 ? 1 : 0), kMinScaleExp);
      scale = __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
      scale = old > scale ? old : scale;
      inv = 1.0f / scale;
      float f[16];
      unpack8(x[0], f);
      unpack8(x[1], f + 8);
      if (odd) {
#pragma unroll
        for (int j = 0; j < 16; ++j) f[j] = f[j] - f[j] == 0.f ? f[j] : __builtin_nanf("");
      }
      u32x4 codes;
#pragma unroll
      for (int j = 0; j < 4; ++j) codes[j] = codes4(f[4 * j] * inv, f[4 * j + 1] * inv, f[4 * j + 2] * inv, f[4 * j + 3] * inv);
      if (has) *(u32x4*)(dst + (int64_t)(held + r) * a.stride_t + c0) = codes;
    } else {
      uint32_t val[16], top = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) val[j] = 0;
      if (RPW * part < b.rows) {                             // (uniform)
        u32x4 wp[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
        if (norm) {
          wp[0] = *(const u32x4*)(a.h.k_norm + 2 * c0);
          wp[1] = *(const u32x4*)(a.h.k_norm + 2 * c1);
        }
        key_values<LPR, NEAR, 64 * W>(a.h, x, wp, i, pos, norm, turns, angles_of != at, s_angles + threadIdx.x, val);
        angles_of = at;
#pragma unroll
        for (int j = 0; j < 16; ++j) top = max(top, finite_or_zero(val[j]));
      }
      top = block_max<W, LPR>(top, how, tops[turn_of], l, w);
      scale = block_scale(top, old);
      inv = 1.0f / scale;
      if (has) put_codes(dst + (int64_t)(held + r) * a.stride_t, c0, c1, codes16(val, (double)inv));
    }
    if (held != 0 && scale > old && h < a.h.hkv) {           // the rows that the page holds take the new scale too
      const int step = single ? 1 : (alone ? RPW : RPW * W);
      for (int y = r; y < held; y += step) scale_down(dst + (int64_t)y * a.stride_t + 16 * i, old * inv);
    }
    if (i == 0 && r == 0 && has && (held == 0 || scale > old)) *scale_at = scale;
  });
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
  a.share = quant_share(tiles, r.cfg.n_kv_heads);
  a.kv_wgs = (unsigned)(tiles << (a.share + 1));
  const int waves = quant_waves(r.cfg.head_dim);
  const long long q_wgs = a.h.passes > 0 ? ((long long)r.total * a.h.waves + waves - 1) / waves : 0;
  const unsigned grid = a.kv_wgs + (unsigned)(q_wgs < kHeadMost ? q_wgs : kHeadMost);
  FLUX_HEADS(qkv_quant_kernel, r.cfg, grid, 64 * waves, s, a);
  return hipGetLastError();
}

}  // namespace flux
