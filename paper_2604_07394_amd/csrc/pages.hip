// flux_page_plan and flux_page_release: the block tables, slots and free pages of a paged KV cache, from the lengths that the
// device holds.  What bounds both: latencies (a step of some hundred sequences moves a few KB).
// Traced, us: 256 sequences with a token each and three of them replaced by prompts of up to 500, plan 6.0 and release 2.7; 64
// sequences of which 16 are replaced by prompts of 1000 to 16384, 7.6 and 5.4.  An empty launch is about 2.
//
// Plan.  Sequence b of length L with n new rows lacks need(b) = ceil((L + n) / 64) - ceil(L / 64) pages; with start(b) the sum of
// need over the sequences before it, its j-th new page is free_pages[n_free - 1 - start(b) - j].  So everything follows from
// one prefix sum over the batch, which every workgroup takes for itself (a launch that left it behind for a second one would
// cost more than the sum does); the workgroup that finishes last writes the lengths, which the others read.
#include "paged.h"

namespace flux {

struct PageArgs {
  int32_t *table, *kv_len, *free_pages, *n_free;
  const int32_t* cu;        // plan: prefix sums of the new rows; release: lengths to keep
  int batch, table_pages, n_pages, total;
  int32_t* slots;
  uint32_t *counter, *status;
};

constexpr int kMaxBatch = FLUX_MAX_PAGED_BATCH;

// Largest i of [0, n) with a[i] <= x (a[0] <= x, ascending).
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sum over the workgroup of what the threads before this one give; `sums` holds W words.
template <int W>
__device__ __forceinline__ int exclusive_sum(int x, int* sums, int& total) {
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int incl = wave_inclusive_sum(x);
  if (l == 63) sums[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < W; ++i) {
    before += i < w ? sums[i] : 0;
    total += sums[i];
  }
  return before + incl - x;
}

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// A workgroup of 256 threads writes kPlanRows slots, a few per thread that are looked up side by side, and its share of the table
// entries.  What a step of some hundred sequences takes is memory latencies one behind the other: the lengths; the page that a
// sequence goes on in; the free pages, asked for together.  A launch of one workgroup has nobody to wait for.
__global__ __launch_bounds__(256) void page_plan_kernel(PageArgs a) {
  __shared__ int s_begin[kMaxBatch + 1], s_len[kMaxBatch], s_start[kMaxBatch], s_limit[kMaxBatch], s_page[kMaxBatch], s_free[256], s_sums[4], s_last;
  const int tid = threadIdx.x;
  const int cap = a.table_pages << 6;                        // (table_pages <= 2^24)
  const int n_free = *a.n_free, avail = clamped(n_free, 0, a.n_pages);
  const int next_free = tid < avail ? a.free_pages[avail - 1 - tid] : -1;   // the pages given out first: asked for along with the lengths
  uint32_t bad = n_free != avail ? FLUX_DEV_BAD_LENGTH : 0;
  const int run = (a.batch + 255) >> 8, b0 = tid * run, b1 = min(b0 + run, a.batch);
  // lengths and rows of this thread's sequences, the page that they go on in, and the pages that they lack
  int needed = 0;
  for (int b = b0; b < b1; ++b) {
    const int got = a.kv_len[b], from = a.cu[b], to = a.cu[b + 1];
    const int len = clamped(got, 0, cap), begin = clamped(from, 0, a.total), end = clamped(to, 0, a.total);
    if (got != len || begin != from || end != to || end < begin) bad |= FLUX_DEV_BAD_LENGTH;
    const int n = end > begin ? end - begin : 0;
    int limit = (int)min((int64_t)len + n, (int64_t)cap);    // the length with all rows that the table has room for
    int page = 0;
    if (n > 0 && (len & 63) != 0) {
      page = a.table[(int64_t)b * a.table_pages + (len >> 6)];
      if ((uint32_t)page >= (uint32_t)a.n_pages) {
        bad |= FLUX_DEV_BAD_PAGE;
        limit = len;
      }
    }
    if (limit - len < n) bad |= FLUX_DEV_KV_OVERFLOW;
    s_begin[b] = begin;
    if (b == a.batch - 1) s_begin[a.batch] = end;
    s_len[b] = len;
    s_page[b] = page;
    s_limit[b] = limit;
    s_start[b] = needed;
    needed += ((limit + 63) >> 6) - ((len + 63) >> 6);
  }
  s_free[tid] = next_free;
  int total;
  const int before = exclusive_sum<4>(needed, s_sums, total);
  for (int b = b0; b < b1; ++b) {
    const int start = s_start[b] + before, used = (s_len[b] + 63) >> 6, need = ((s_limit[b] + 63) >> 6) - used;
    s_start[b] = start;
    const int given = clamped(avail - start, 0, need);
    if (given < need) {
      bad |= FLUX_DEV_KV_OVERFLOW;
      s_limit[b] = min(s_limit[b], (used + given) << 6);
    }
  }
  if (blockIdx.x != 0) bad = 0;                              // (once per launch)
  __syncthreads();

  auto free_page = [&](int i) { return i < 256 ? s_free[i] : a.free_pages[avail - 1 - i]; };
  // the sequences of this thread's rows and of its first new page, looked up side by side
  constexpr int U = kPlanRows / 256;
  const int taken = min(total, avail), stride = gridDim.x * 256;
  const int64_t t0 = (int64_t)blockIdx.x * kPlanRows + tid;
  int i = blockIdx.x * 256 + tid;
  int seq[U + 1];
#pragma unroll
  for (int j = 0; j <= U; ++j) seq[j] = 0;
  for (int step = a.batch > 1 ? 1 << (31 - __builtin_clz(a.batch - 1)) : 0; step > 0; step >>= 1) {
#pragma unroll
    for (int j = 0; j <= U; ++j) {
      const int mid = seq[j] + step;
      const int first = mid < a.batch ? (j < U ? s_begin[mid] : s_start[mid]) : 0x7FFFFFFF;
      if (first <= (j < U ? (int)(t0 + 256 * j) : i)) seq[j] = mid;
    }
  }
  int slot[U], row[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t t = t0 + 256 * j;
    const int b = seq[j], len = s_len[b];
    const int64_t at = (int64_t)len + ((int)t - s_begin[b]);
    slot[j] = -1;
    row[j] = 0;
    if (t < a.total && t >= s_begin[b] && t < s_begin[b + 1] && at < s_limit[b]) {
      const int pos = (int)at, used = (len + 63) >> 6, p = pos >> 6;
      slot[j] = p >= used ? free_page(s_start[b] + p - used) : s_page[b];
      row[j] = pos & 63;
    }
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int64_t t = t0 + 256 * j;
    if (t < a.total) a.slots[t] = (uint32_t)slot[j] < (uint32_t)a.n_pages ? (slot[j] << 6) + row[j] : -1;
  }
  for (int b = seq[U]; i < taken;) {
    int page = free_page(i);
    if ((uint32_t)page >= (uint32_t)a.n_pages) {
      bad |= FLUX_DEV_BAD_PAGE;
      page = -1;
    }
    a.table[(int64_t)b * a.table_pages + ((s_len[b] + 63) >> 6) + (i - s_start[b])] = page;
    i += stride;
    if (i < taken) b = last_not_above(s_start, a.batch, i);
  }
  if (bad) atomicOr(a.status, bad);

  // the last workgroup to arrive writes the lengths: the others only read them, and a thread's loads have returned before the
  // barrier lets thread 0 count the arrival
  if (gridDim.x > 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(a.counter, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    if (tid == 0) *a.counter = 0;                            // ready for the next launch on this stream
  }
  for (int b = tid; b < a.batch; b += 256) a.kv_len[b] = s_limit[b];
  if (tid == 0) *a.n_free = avail - taken;
}

// Release.  One workgroup: the pages that go back, counted by sequence and place, are listed last one first, so that a plan
// that follows takes them in their order; which of them are in the pool (the others are not listed) is counted 1024 at a time.
__global__ __launch_bounds__(1024) void page_release_kernel(PageArgs a) {
  __shared__ int s_start[kMaxBatch], s_keep[kMaxBatch], s_sums[2][16];
  const int tid = threadIdx.x;
  const int cap = a.table_pages << 6;
  const int n_free = *a.n_free;
  int listed = clamped(n_free, 0, a.n_pages);
  uint32_t bad = n_free != listed ? FLUX_DEV_BAD_LENGTH : 0;
  const int run = (a.batch + 1023) >> 10, b0 = tid * run, b1 = min(b0 + run, a.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int got = a.kv_len[b], len = clamped(got, 0, cap), keep = clamped(a.cu[b], 0, len);
    if (got != len) bad |= FLUX_DEV_BAD_LENGTH;
    s_keep[b] = (keep + 63) >> 6;
    s_start[b] = mine;
    mine += ((len + 63) >> 6) - ((keep + 63) >> 6);
    if (keep != got) a.kv_len[b] = keep;
  }
  int total;
  const int before = exclusive_sum<16>(mine, s_sums[0], total);
  for (int b = b0; b < b1; ++b) s_start[b] += before;
  __syncthreads();
  for (int r0 = total - 1, turn = 1; r0 >= 0; r0 -= 1024, turn ^= 1) {
    const int r = r0 - tid;
    int page = -1;
    if (r >= 0) {
      const int b = last_not_above(s_start, a.batch, r);
      int32_t* entry = a.table + (int64_t)b * a.table_pages + s_keep[b] + (r - s_start[b]);
      page = *entry;
      *entry = -1;
    }
    const bool in_pool = (uint32_t)page < (uint32_t)a.n_pages;
    int found;
    const int at = listed + exclusive_sum<16>(in_pool ? 1 : 0, s_sums[turn], found);   // (the two sets of sums take turns: one barrier each)
    if (in_pool && at < a.n_pages) a.free_pages[at] = page;
    if (r >= 0 && (!in_pool || at >= a.n_pages)) bad |= FLUX_DEV_BAD_PAGE;
    listed = min(listed + found, a.n_pages);
  }
  if (tid == 0) *a.n_free = listed;
  if (bad) atomicOr(a.status, bad);
}

namespace {
PageArgs page_args(const Ctx& c, const flux_page_table& pt) {
  PageArgs a;
  a.table = pt.table;
  a.kv_len = pt.kv_len;
  a.free_pages = pt.free_pages;
  a.n_free = pt.n_free;
  a.batch = pt.batch;
  a.table_pages = pt.table_pages;
  a.n_pages = pt.n_pages;
  a.cu = nullptr;
  a.slots = nullptr;
  a.total = 0;
  a.counter = c.counters + 1;
  a.status = c.status;
  return a;
}
}  // namespace

hipError_t launch_page_plan(const Ctx& c, const flux_page_table& pt, const int32_t* cu_new, int total_new, int32_t* slots, hipStream_t s) {
  PageArgs a = page_args(c, pt);
  a.cu = cu_new;
  a.total = total_new;
  a.slots = slots;
  const unsigned wgs = (unsigned)(((long long)total_new + kPlanRows - 1) / kPlanRows);
  hipLaunchKernelGGL(page_plan_kernel, dim3(wgs), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_release(const Ctx& c, const flux_page_table& pt, const int32_t* keep_len, hipStream_t s) {
  PageArgs a = page_args(c, pt);
  a.cu = keep_len;
  hipLaunchKernelGGL(page_release_kernel, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace flux
