// flux_page_fork, flux_page_compact, flux_page_copy: pages of a paged KV cache change hands, change places, and are copied.
//
// Fork.  With n = min(keep_len[b], kv_len[parent[b]]), row b of the table becomes the first ceil(n / 64) entries of what row parent[b]
// was.  shares[p] is the number of rows that hold page p, less one (a free page has 0).  What follows is counted in shares by atomic
// additions, one for each entry that a row loses or gets (whose order does not show in the sums): a page that ends at -1 goes back.
// The new rows come from the old ones in place, so a workgroup takes a few columns of the table for all sequences, reads them all
// and then writes.  A second launch finds the pages that ended at -1 and gives copies to last pages that may not be shared.
// Compact.  One workgroup holds a bit per page in LDS; bits counted from either end say which page moves where.
// What bounds them: latencies (fork: two launches, each a chain of lengths, entries and sums; compact: the list of free
// pages, which one CU reads and writes); the copies of a layer are bound by the memory.
#include "page_moves.h"

namespace flux {

struct MoveArgs {
  int32_t *table, *kv_len, *free_pages, *n_free, *shares;
  const int32_t *parent, *keep;
  int32_t *list, *n_list;         // pages to copy: [.][3] from, to, rows; how many
  int batch, table_pages, n_pages, most;
  int cols_shift;                 // log2 of the columns that a workgroup of a fork takes
  int slots_shift;                // 32 less log2 of the places of the table of last pages
  int32_t* scratch;               // fork: counts and pages that went back; compact: where a page went, and from which page on they went
  uint32_t *counter, *status;
};

constexpr int kMaxBatch = FLUX_MAX_PAGED_BATCH;
constexpr int kSlots = 2 * kMaxBatch;

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
template <typename T>
__device__ __forceinline__ void put(T* at, T x) { __hip_atomic_store(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ T get(const T* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Sum over the workgroup's W waves of what the threads before this one give.  `sums` holds a word per wave; a barrier has to stand
// between two uses of it.
template <int W>
__device__ __forceinline__ int sum_before(int x, int* sums, int& total) {
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int incl = wave_inclusive_sum(x);
  if (l == 63) sums[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    before += i < w ? sums[i] : 0;
    total += sums[i];
  }
  return before + incl - x;
}

// Whose pages sequence b goes on with (-1: nobody's), and how many of its tokens.
__device__ __forceinline__ int goes_on(const MoveArgs& a, int b, int& p, uint32_t& bad) {
  const int cap = a.table_pages << 6;                        // (table_pages <= 2^24)
  p = a.parent ? a.parent[b] : b;
  if (p < -1 || p >= a.batch) {
    bad |= FLUX_DEV_BAD_LENGTH;
    p = -1;
  }
  if (p < 0) return 0;
  const int got = a.kv_len[p], len = clampi(got, 0, cap);
  if (got != len) bad |= FLUX_DEV_BAD_LENGTH;
  return a.keep ? clampi(a.keep[b], 0, len) : len;
}

// What the last workgroup of a fork finds out about the last pages that are partly filled: a table in LDS by page (open addressing) of how
// many sequences have it so, and which is the first.
struct LastPages {
  int *page, *holders, *first;
  int shift;                      // 32 less log2 of the places
  __device__ __forceinline__ int places() const { return 1 << (32 - shift); }
  __device__ __forceinline__ void clear() const {
    for (int i = threadIdx.x; i < places(); i += 1024) {
      page[i] = -1;
      holders[i] = 0;
      first[i] = 0x7FFFFFFF;
    }
  }
  __device__ __forceinline__ int add(int p, int b) const {
    int at = (int)(((uint32_t)p * 2654435769u) >> shift);    // (2^32 over the golden ratio: neighbours lie far apart)
    for (;;) {
      const int was = atomicCAS(&page[at], -1, p);
      if (was == -1 || was == p) break;
      at = (at + 1) & (places() - 1);                        // (twice as many places as sequences)
    }
    atomicAdd(&holders[at], 1);
    atomicMin(&first[at], b);
    return at;
  }
};
constexpr int kMine = kMaxBatch / 1024;     // sequences that a thread looks after: tid, tid + 1024, ..

// The lengths, and copies of last pages that may not be shared, in the order of the sequences.  len(b), last page and its holders less
// one (shares) as the first part left them; nth_free(j): the j-th free page, of `listed` in all.
template <typename F>
__device__ __forceinline__ void fork_copies(const MoveArgs& a, const int* s_len, const LastPages& t, const int (&page)[kMine], const int (&shares)[kMine],
                                            const int (&place)[kMine], int listed, int* s_sums, F nth_free, uint32_t& bad) {
  const int tid = threadIdx.x;
  int copies = 0, nth[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    bool copy = false;
    if (page[i] >= 0) copy = shares[i] > 0 && !(shares[i] + 1 == t.holders[place[i]] && t.first[place[i]] == tid + 1024 * i);
    int total = 0;
    nth[i] = -1;
    if (1024 * i < a.batch) {                                // (uniform)
      __syncthreads();
      const int j = copies + sum_before<16>(copy ? 1 : 0, s_sums, total);
      if (copy) nth[i] = j;
    }
    copies += total;
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int b = tid + 1024 * i;
    if (b >= a.batch) continue;
    int len = s_len[b];
    if (nth[i] >= 0) {
      const bool given = nth[i] < listed;
      int to = given ? nth_free(nth[i]) : -1;
      if (given && (uint32_t)to >= (uint32_t)a.n_pages) {
        bad |= FLUX_DEV_BAD_PAGE;
        to = -1;
      }
      if (!given) bad |= FLUX_DEV_KV_OVERFLOW;
      a.table[(int64_t)b * a.table_pages + (len >> 6)] = to;
      atomicSub(a.shares + page[i], 1);
      if (given) {
        a.list[3 * nth[i]] = to >= 0 ? page[i] : -1;
        a.list[3 * nth[i] + 1] = to;
        a.list[3 * nth[i] + 2] = len & 63;
      } else {
        len &= ~63;
      }
    }
    a.kv_len[b] = len;
  }
  if (tid == 0) {
    *a.n_free = listed - min(copies, listed);
    *a.n_list = min(copies, listed);
  }
}

// The first part, in columns; where the pool is small (ALL) the last workgroup to arrive does the rest, else a second launch does, whose
// workgroups look through the pool side by side.  What workgroups hand on is written past the caches, and waited for before they arrive.  us of the
// launch with 64 sequences and 680 pages / 256 and 8200: 26 / 58 in two launches of 64 columns per workgroup; now 10 / 12.
template <bool ALL>
__global__ __launch_bounds__(1024) void page_fork_kernel(MoveArgs a) {
  __shared__ int s_old[kMaxBatch], s_len[kMaxBatch], s_parent[kMaxBatch], s_work[3 * kSlots], s_sums[16], s_most, s_last;
  static_assert(3 * kSlots >= kForkEntries, "the entries of the first part, then the table of last pages");
  const int tid = threadIdx.x;
  if (tid == 0) s_most = 0;
  __syncthreads();
  uint32_t bad = 0, bad_page = 0;
  int most = 0;
  for (int b = tid; b < a.batch; b += 1024) {
    int p;
    const int n = goes_on(a, b, p, bad), had = (clampi(a.kv_len[b], 0, a.table_pages << 6) + 63) >> 6;
    s_old[b] = had;
    s_len[b] = n;
    s_parent[b] = p;
    most = max(most, max(had, (n + 63) >> 6));
  }
  if (most > 0) atomicMax(&s_most, most);
  __syncthreads();
  most = s_most;
  const int shift = a.cols_shift, cols = 1 << shift, entries = a.batch << shift;   // (at most kForkEntries)
  for (int64_t c0 = (int64_t)blockIdx.x * cols; c0 < most; c0 += (int64_t)gridDim.x * cols) {
    // entries of these columns, -1 where a row has none
    for (int i0 = tid; i0 < entries; i0 += 4096) {
      int page[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + 1024 * u, b = i >> shift, c = (int)c0 + (i & (cols - 1));
        page[u] = i < entries && c < s_old[b] ? a.table[(int64_t)b * a.table_pages + c] : -1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + 1024 * u;
        if (i >= entries) continue;
        if ((uint32_t)page[u] >= (uint32_t)a.n_pages) {
          if ((int)c0 + (i & (cols - 1)) < s_old[i >> shift]) bad_page = FLUX_DEV_BAD_PAGE;
          page[u] = -1;
        }
        s_work[i] = page[u];
      }
    }
    __syncthreads();
    for (int i = tid; i < entries; i += 1024) {
      const int b = i >> shift, x = i & (cols - 1), c = (int)c0 + x, p = s_parent[b];
      const int has = (s_len[b] + 63) >> 6, before = s_work[i], now = c < has ? s_work[(p << shift) + x] : -1;
      if (now != before) {
        if (before >= 0) atomicSub(a.shares + before, 1);
        if (now >= 0) atomicAdd(a.shares + now, 1);
      }
      if (c < max(s_old[b], has) && (p != b || c >= has)) put(a.table + (int64_t)b * a.table_pages + c, now);
    }
    __syncthreads();
  }
  if (blockIdx.x != 0) bad = 0;                              // (once per launch)
  bad |= bad_page;
  if (!ALL) {
    if (bad) atomicOr(a.status, bad);
    return;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s_last = atomicAdd(a.counter, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!s_last) {
    if (bad) atomicOr(a.status, bad);
    return;
  }
  if (tid == 0) *a.counter = 0;                              // ready for the next launch on this stream

  // the whole pool, from the highest page down, four pages per thread and turn; last pages; all asked for together
  constexpr int TURNS = kForkAlone / 4096;
  int have[TURNS][4], page[kMine], shares[kMine], place[kMine];
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = a.n_pages - 1 - 4096 * t - 4 * tid - i;
      have[t][i] = p >= 0 ? get(a.shares + p) : 0;
    }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int b = tid + 1024 * i;
    page[i] = b < a.batch && (s_len[b] & 63) != 0 ? get(a.table + (int64_t)b * a.table_pages + (s_len[b] >> 6)) : -1;
  }
  const int n_free = *a.n_free, avail = clampi(n_free, 0, a.n_pages);
  if (n_free != avail) bad |= FLUX_DEV_BAD_LENGTH;
  const LastPages last = {s_work, s_work + kSlots, s_work + 2 * kSlots, a.slots_shift};
  last.clear();
#pragma unroll
  for (int i = 0; i < kMine; ++i) shares[i] = page[i] >= 0 ? get(a.shares + page[i]) : 0;
  int* const s_low = s_old;                                  // of the pages that go back the lowest, from the lowest up (as many as there may be copies)
  int listed = avail, back_all = 0, n = 0;
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) n += have[t][i] < 0 ? 1 : 0;
  // (how many in all, so that the lowest are known by their place)
  sum_before<16>(n, s_sums, back_all);
  int done = 0;
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    if (4096 * t >= a.n_pages) continue;                     // (uniform)
    int m = 0, total;
#pragma unroll
    for (int i = 0; i < 4; ++i) m += have[t][i] < 0 ? 1 : 0;
    __syncthreads();
    int at = done + sum_before<16>(m, s_sums, total);
    done += total;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (have[t][i] >= 0) continue;
      const int p = a.n_pages - 1 - 4096 * t - 4 * tid - i;
      if (listed + at < a.n_pages) a.free_pages[listed + at] = p;
      else bad |= FLUX_DEV_BAD_PAGE;
      const int nth = back_all - 1 - at;
      if (nth < kMaxBatch) s_low[nth] = p;
      a.shares[p] = 0;
      if (have[t][i] < -1) bad |= FLUX_DEV_BAD_PAGE;         // more rows lost it than held it
      ++at;
    }
  }
  const bool fits = listed + back_all <= a.n_pages;          // (else the list would grow past the pool)
  listed = min(listed + back_all, a.n_pages);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMine; ++i) place[i] = page[i] >= 0 ? last.add(page[i], tid + 1024 * i) : 0;
  __syncthreads();
  fork_copies(a, s_len, last, page, shares, place, listed, s_sums,
              [&](int j) { return fits && j < back_all ? s_low[j] : a.free_pages[listed - 1 - j]; }, bad);
  if (bad) atomicOr(a.status, bad);
}

__global__ __launch_bounds__(1024) void page_fork_end_kernel(MoveArgs a) {
  __shared__ int s_sums[16], s_begin[1024], s_count[1024], s_last, s_len[kMaxBatch], s_work[3 * kSlots];
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  const int groups = (a.n_pages + kForkPages - 1) / kForkPages;
  int32_t* const counts = a.scratch;                         // of every workgroup's pages that go back
  int32_t* const found = a.scratch + groups;
  uint32_t bad = 0;
  {
    // pages that nobody holds, from the highest of this workgroup's down
    constexpr int PER = kForkPages / 1024;
    const int low = (int)blockIdx.x * kForkPages, top = min(low + kForkPages, a.n_pages) - 1 - PER * tid;
    int have[PER], n = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) have[i] = top - i >= low ? a.shares[top - i] : 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += have[i] < 0 ? 1 : 0;
    int at = sum_before<16>(n, s_sums, total);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (have[i] >= 0) continue;
      put(found + (int64_t)blockIdx.x * kForkPages + at++, top - i);
      a.shares[top - i] = 0;
      if (have[i] < -1) bad |= FLUX_DEV_BAD_PAGE;            // more rows lost it than held it
    }
    if (tid == 0) put(counts + blockIdx.x, total);
  }
  // the last workgroup to arrive does the rest; what the others found is in memory by then
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) s_last = atomicAdd(a.counter, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!s_last) {
    if (bad) atomicOr(a.status, bad);
    return;
  }
  if (tid == 0) *a.counter = 0;                              // ready for the next launch on this stream
  const LastPages last = {s_work, s_work + kSlots, s_work + 2 * kSlots, a.slots_shift};
  last.clear();
  uint32_t known = 0;                                        // (what the first launch has reported)
  for (int b = tid; b < a.batch; b += 1024) {
    int p;
    s_len[b] = goes_on(a, b, p, known);
  }
  const int n_free = *a.n_free, avail = clampi(n_free, 0, a.n_pages);
  if (n_free != avail) bad |= FLUX_DEV_BAD_LENGTH;
  __syncthreads();
  int page[kMine], shares[kMine], place[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int b = tid + 1024 * i;
    page[i] = b < a.batch && (s_len[b] & 63) != 0 ? a.table[(int64_t)b * a.table_pages + (s_len[b] >> 6)] : -1;
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) shares[i] = page[i] >= 0 ? get(a.shares + page[i]) : 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) place[i] = page[i] >= 0 ? last.add(page[i], tid + 1024 * i) : 0;
  // the list of free pages takes what goes back, the highest first
  int listed = avail;
  for (int g0 = groups - 1; g0 >= 0; g0 -= 1024) {
    const int g = g0 - tid;
    const int n = g >= 0 ? get(counts + g) : 0;
    int total;
    __syncthreads();
    s_begin[tid] = listed + sum_before<16>(n, s_sums, total);
    s_count[tid] = n;
    __syncthreads();
    for (int j = w; j < min(1024, g0 + 1); j += 16) {
      const int m = s_count[j], to = s_begin[j];
      for (int i = l; i < m; i += 64) {
        if (to + i < a.n_pages) a.free_pages[to + i] = get(found + (int64_t)(g0 - j) * kForkPages + i);
        else bad |= FLUX_DEV_BAD_PAGE;
      }
    }
    listed = min(listed + total, a.n_pages);
  }
  __threadfence_block();
  __syncthreads();
  fork_copies(a, s_len, last, page, shares, place, listed, s_sums, [&](int j) { return a.free_pages[listed - 1 - j]; }, bad);
  if (bad) atomicOr(a.status, bad);
}

// Free pages counted from the lowest, pages in use from the highest: as long as the free one is the lower of the two they change
// places.  A wave has a range of chunks of 64 pages, a lane one page of a chunk.
__global__ __launch_bounds__(1024) void page_compact_kernel(MoveArgs a) {
  __shared__ uint64_t s_free[kCompactPages / 64];
  __shared__ int s_sums[3][16];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int chunks = (a.n_pages + 63) / 64, run = (chunks + 15) / 16, k0 = min(w * run, chunks), k1 = min(k0 + run, chunks);
  uint32_t bad = 0;
  for (int i = tid; i < chunks; i += 1024) s_free[i] = 0;
  const int n_free = *a.n_free, avail = clampi(n_free, 0, a.n_pages);
  if (n_free != avail) bad |= FLUX_DEV_BAD_LENGTH;
  __syncthreads();
  constexpr int U = 16;
  for (int i0 = tid; i0 < avail; i0 += 1024 * U) {
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) page[u] = i0 + 1024 * u < avail ? a.free_pages[i0 + 1024 * u] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 1024 * u >= avail) continue;
      const bool in_pool = (uint32_t)page[u] < (uint32_t)a.n_pages;
      const uint32_t bit = 1u << (page[u] & 31);
      if (!in_pool || (atomicOr((uint32_t*)s_free + (page[u] >> 5), bit) & bit)) bad |= FLUX_DEV_BAD_PAGE;   // no page, or listed twice
    }
  }
  __syncthreads();
  int mine = 0;
  for (int k = k0 + l; k < k1; k += 64) mine += __builtin_popcountll(s_free[k]);
  mine = __builtin_amdgcn_readlane(wave_inclusive_sum(mine), 63);
  if (l == 0) s_sums[0][w] = mine;
  __syncthreads();
  int before = 0, free_all = 0;
  for (int i = 0; i < 16; ++i) {
    before += i < w ? s_sums[0][i] : 0;
    free_all += s_sums[0][i];
  }
  const int used = a.n_pages - free_all;                     // in the end the pages below it are the ones in use
  int low = 0;
  for (int k = k0 + l; k < k1; k += 64) {
    const int n = clampi(used - 64 * k, 0, 64);
    low += n > 0 ? __builtin_popcountll(s_free[k] << (64 - n)) : 0;
  }
  low = __builtin_amdgcn_readlane(wave_inclusive_sum(low), 63);
  if (l == 0) s_sums[1][w] = low;
  __syncthreads();
  int moves = 0;
  for (int i = 0; i < 16; ++i) moves += s_sums[1][i];
  moves = min(moves, a.most);
  // which pages move, and which are free afterwards.  A lane has one of 64 chunks and their ranks, and hands them to the wave
  int rank = before;                                         // of the next chunk's first free page
  mine = 0;
  for (int k = k0; k < k1; k += 64) {
    const uint64_t own = k + l < k1 ? s_free[k + l] : 0;
    const int count = __builtin_popcountll(own), incl = wave_inclusive_sum(count), first = rank + incl - count;
    // (free pages of a chunk move while they are among the lowest, pages in use while they are among the highest)
    const bool any = k + l < k1 && (first < moves || used - 64 * (k + l + 1) + first + count < moves);
    uint64_t after = own;
    for (uint64_t todo = __builtin_amdgcn_ballot_w64(any); todo != 0; todo &= todo - 1) {
      const int j = __builtin_ctzll(todo);
      const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)own, j), hi = __builtin_amdgcn_readlane((int)(uint32_t)(own >> 32), j);
      const int page = 64 * (k + j) + l, r = __builtin_amdgcn_readlane(first, j) + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
      const bool is_free = ((l < 32 ? lo : hi) >> (l & 31)) & 1;
      const int nth = is_free ? r : used - 1 - (page - r);   // from the lowest; from the highest
      const bool moved = page < a.n_pages && nth < moves;
      if (moved) {
        a.list[3 * nth + (is_free ? 1 : 0)] = page;
        if (!is_free) a.list[3 * nth + 2] = kPageTokens;
      }
      const uint64_t change = __builtin_amdgcn_ballot_w64(moved);
      if (l == j) after = own ^ change;
    }
    if (k + l < k1) s_free[k + l] = after;
    rank += __builtin_amdgcn_readlane(incl, 63);
    mine += __builtin_popcountll(after);
  }
  mine = __builtin_amdgcn_readlane(wave_inclusive_sum(mine), 63);
  if (l == 0) s_sums[2][w] = mine;
  __threadfence_block();
  __syncthreads();
  before = 0;
  for (int i = 0; i < w; ++i) before += s_sums[2][i];
  rank = before;
  for (int k = k0; k < k1; k += 64) {
    const uint64_t own = k + l < k1 ? s_free[k + l] : 0;
    const int count = __builtin_popcountll(own), incl = wave_inclusive_sum(count), first = rank + incl - count;
    for (uint64_t todo = __builtin_amdgcn_ballot_w64(own != 0); todo != 0; todo &= todo - 1) {
      const int j = __builtin_ctzll(todo);
      const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)own, j), hi = __builtin_amdgcn_readlane((int)(uint32_t)(own >> 32), j);
      const int r = __builtin_amdgcn_readlane(first, j) + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
      if (((l < 32 ? lo : hi) >> (l & 31)) & 1) a.free_pages[free_all - 1 - r] = 64 * (k + j) + l;   // the lowest page last
    }
    rank += __builtin_amdgcn_readlane(incl, 63);
  }
  // holders go along; where a page went, for the tables
  for (int j = tid; j < moves; j += 1024) {
    const int from = a.list[3 * j], to = a.list[3 * j + 1];
    a.scratch[1 + from] = to;
    if (a.shares) {
      a.shares[to] = a.shares[from];
      a.shares[from] = 0;
    }
  }
  if (tid == 0) {
    a.scratch[0] = moves > 0 ? a.list[3 * (moves - 1)] : a.n_pages;
    *a.n_list = moves;
    *a.n_free = free_all;
  }
  if (bad) atomicOr(a.status, bad);
}

// All pages in use from scratch[0] on have moved.
__global__ __launch_bounds__(256) void page_renumber_kernel(MoveArgs a) {
  int from = a.scratch[0], len = a.kv_len[blockIdx.y];       // (asked for together; there are no more rows of workgroups than sequences)
  asm volatile("" : "+s"(from), "+s"(len));
  if (from >= a.n_pages) return;
  uint32_t bad = 0;
  for (int b = blockIdx.y; b < a.batch; b += gridDim.y) {
    if (b != (int)blockIdx.y) len = a.kv_len[b];
    const int pages = (clampi(len, 0, a.table_pages << 6) + 63) >> 6;
    int32_t* const row = a.table + (int64_t)b * a.table_pages;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < pages; i += gridDim.x * 256) {
      const int page = row[i];
      if (page < from || page >= a.n_pages) {
        if ((uint32_t)page >= (uint32_t)a.n_pages) bad = FLUX_DEV_BAD_PAGE;
        continue;
      }
      const int to = a.scratch[1 + page];
      if ((uint32_t)to < (uint32_t)a.n_pages) row[i] = to;
      else bad = FLUX_DEV_BAD_PAGE;                          // (a page that the list called free)
    }
  }
  if (bad) atomicOr(a.status, bad);
}

struct CopyArgs {
  char *k, *v;
  float *k_scale, *v_scale;
  int64_t stride_p, stride_h, stride_t;
  const int32_t *list, *n_list;
  int hkv, n_pages, most;
  uint32_t* status;
};

// A wave per (entry, head, K or V): up to 8 KB on their way at once, 16 bytes per lane.
template <int D>
__global__ __launch_bounds__(256) void page_copy_kernel(CopyArgs a) {
  constexpr int LPR = D / 16, RPS = 64 / LPR, STEPS = 64 / RPS;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = 2 * a.hkv;
  int n = a.n_list ? *a.n_list : a.most;
  for (int64_t u = (int64_t)blockIdx.x * 4 + w; u < (int64_t)min(n, a.most) * per; u += (int64_t)gridDim.x * 4) {
    const int64_t j = u / per;
    const int part = (int)(u - j * per), h = part >> 1;
    int from = a.list[3 * j], to = a.list[3 * j + 1], rows = clampi(a.list[3 * j + 2], 0, kPageTokens);
    if (from == to && from == -1) continue;                  // (an entry that is left out)
    if ((uint32_t)from >= (uint32_t)a.n_pages || (uint32_t)to >= (uint32_t)a.n_pages) {
      if (l == 0 && part == 0) atomicOr(a.status, (uint32_t)FLUX_DEV_BAD_PAGE);
      continue;
    }
    char* const base = (part & 1) ? a.v : a.k;
    float* const scale = (part & 1) ? a.v_scale : a.k_scale;
    const int64_t in_page = (int64_t)h * a.stride_h + (l / LPR) * a.stride_t + (l % LPR) * 16;
    const char* src = base + (int64_t)from * a.stride_p + in_page;
    char* dst = base + (int64_t)to * a.stride_p + in_page;
    u32x4 x[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      if (i * RPS + l / LPR < rows) x[i] = *(const u32x4*)(src + (int64_t)i * RPS * a.stride_t);
    if (l == 0) scale[(int64_t)to * a.hkv + h] = scale[(int64_t)from * a.hkv + h];
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      if (i * RPS + l / LPR < rows) *(u32x4*)(dst + (int64_t)i * RPS * a.stride_t) = x[i];
  }
}

namespace {
MoveArgs move_args(const Ctx& c, const flux_page_table& pt, int32_t* shares, int32_t* list, int32_t* n_list, int most) {
  MoveArgs a = {};
  a.table = pt.table;
  a.kv_len = pt.kv_len;
  a.free_pages = pt.free_pages;
  a.n_free = pt.n_free;
  a.shares = shares;
  a.list = list;
  a.n_list = n_list;
  a.batch = pt.batch;
  a.table_pages = pt.table_pages;
  a.n_pages = pt.n_pages;
  a.most = most;
  a.scratch = (int32_t*)c.partials;
  a.counter = c.counters + 1;
  a.status = c.status;
  return a;
}
}  // namespace

hipError_t launch_page_fork(const Ctx& c, const flux_page_table& pt, int32_t* shares, const int32_t* parent, const int32_t* keep, int32_t* copies,
                            int32_t* n_copies, hipStream_t s) {
  MoveArgs a = move_args(c, pt, shares, copies, n_copies, pt.batch);
  a.parent = parent;
  a.keep = keep;
  // (16 columns are a line of memory of each row)
  a.cols_shift = 4;
  while (a.cols_shift > 2 && (pt.batch << a.cols_shift) > 4096) --a.cols_shift;
  a.slots_shift = 26;                                        // 64 places
  while ((1 << (32 - a.slots_shift)) < 2 * pt.batch) --a.slots_shift;
  const int wgs = (pt.table_pages + (1 << a.cols_shift) - 1) >> a.cols_shift;
  const dim3 grid(wgs < 1024 ? wgs : 1024), block(1024);
  if (pt.n_pages <= kForkAlone) {
    hipLaunchKernelGGL((page_fork_kernel<true>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((page_fork_kernel<false>), grid, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(page_fork_end_kernel, dim3((pt.n_pages + kForkPages - 1) / kForkPages), block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_compact(const Ctx& c, const flux_page_table& pt, int32_t* shares, int32_t* moves, int max_moves, int32_t* n_moves, hipStream_t s) {
  const MoveArgs a = move_args(c, pt, shares, moves, n_moves, max_moves);
  hipLaunchKernelGGL(page_compact_kernel, dim3(1), dim3(1024), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // about 2000 workgroups at most: a row of the table each, or shares of one
  const int rows = pt.batch < 1024 ? pt.batch : 1024, wide = (pt.table_pages + 255) / 256, most = 2048 / rows;
  hipLaunchKernelGGL(page_renumber_kernel, dim3(wide < most ? wide : most, rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_page_copy(const Ctx& c, const flux_paged_kv& kv, int hkv, int d, const int32_t* copies, const int32_t* n_copies, int max_copies, hipStream_t s) {
  CopyArgs a;
  a.k = (char*)kv.k;
  a.v = (char*)kv.v;
  a.k_scale = kv.k_scale;
  a.v_scale = kv.v_scale;
  a.stride_p = kv.stride_p;
  a.stride_h = kv.stride_h;
  a.stride_t = kv.stride_t;
  a.list = copies;
  a.n_list = n_copies;
  a.hkv = hkv;
  a.n_pages = kv.n_pages;
  a.most = max_copies;
  a.status = c.status;
  const long long wgs = ((long long)max_copies * 2 * hkv + 3) / 4;
  const dim3 grid((unsigned)(wgs < kCopyWgs ? wgs : kCopyWgs)), block(256);
  if (d == 128) hipLaunchKernelGGL((page_copy_kernel<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((page_copy_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace flux
