// flux_page_fork, flux_page_compact, flux_page_copy: pages of a paged KV cache change hands, change places, and are copied.
//
// Fork.  With n = min(keep_len[b], kv_len[parent[b]]), row b of the table becomes the first ceil(n / 64) entries of what row parent[b]
// was.  shares[p] is the number of rows that hold page p, less one (a free page has 0).  What follows is counted in shares by atomic
// additions, one for each entry that a row loses or gets (whose order does not show in the sums): a page that ends at -1 goes back.
// The new rows come from the old ones in place, so a workgroup takes a few columns of the table for all sequences, reads them all
// and then writes.  Then the pages that ended at -1 are found and last pages that may not be shared get copies: by the last workgroup to
// arrive, or in pools of more than kForkAlone pages by a second launch.
// Compact.  A bit per page; bits counted from either end say which page moves where.  One workgroup sets them, many write what follows.
// What bounds them: latencies (fork: a chain of parents, lengths, entries, sums and the arrival, 9 us with 64 sequences and 680 pages, 14 with 256
// and 8200; compact: the list of free pages, which one CU reads, and a second launch, 3 + 5 us with 1046 pages, 7 + 7 with 63595).  The copies of a layer are
// bound by the memory: 4096 pages of 2 heads of 64 in 26 us, 5.1 TB/s; 260 of 8 heads of 128 in 13.
#include "page_moves.h"

namespace flux {

struct MoveArgs {
  int32_t *table, *kv_len, *free_pages, *n_free, *shares;
  const int32_t *parent, *keep;
  int32_t *list, *n_list;         // pages to copy: [.][3] from, to, rows; how many
  int batch, table_pages, n_pages, most;
  int cols_shift;                 // log2 of the columns that a workgroup of a fork takes
  int slots_shift;                // 32 less log2 of the places of the table of last pages
  int32_t* scratch;               // fork of a large pool: counts and pages that went back; compact: CompactBits
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
    const int n = goes_on(a, b, p, bad), got = a.kv_len[b], len = clampi(got, 0, a.table_pages << 6), had = (len + 63) >> 6;
    if (got != len) bad |= FLUX_DEV_BAD_LENGTH;              // (whoever goes on with it)
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
        const int in_pool = page_of_entry(page[u], a.n_pages);
        if (in_pool < 0 && (int)c0 + (i & (cols - 1)) < s_old[i >> shift]) bad_page = FLUX_DEV_BAD_PAGE;
        s_work[i] = in_pool;
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
      if (fork_writes(c, s_old[b], has, p == b, before)) put(a.table + (int64_t)b * a.table_pages + c, now);
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
    page[i] = b < a.batch && (s_len[b] & 63) != 0 ? page_of_entry(get(a.table + (int64_t)b * a.table_pages + (s_len[b] >> 6)), a.n_pages) : -1;
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
    page[i] = b < a.batch && (s_len[b] & 63) != 0 ? page_of_entry(a.table[(int64_t)b * a.table_pages + (s_len[b] >> 6)], a.n_pages) : -1;
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
// places.  The first launch is one workgroup, which sets a bit for every free page and counts them; its bits, the free pages before every
// four words of them and the two totals are all that the second needs, whose workgroups then write the moves, the new list and the tables side by
// side: where a page goes is a rank among the bits of one kind and a search for the same rank among the others.  (A single workgroup that
// wrote the moves and the list as well took 28 us for a pool of 63595 pages, 4096 of which move, and the tables 5; now 7 and 7.)
constexpr int kWords = kCompactPages / 64, kFours = kWords / 4;

struct CompactBits {              // of the workspace
  int32_t free_all, moves, unused[2];
  uint64_t bits[1];               // a bit per page, then (behind whole fours of words) a count per four words
};

__global__ __launch_bounds__(1024) void page_compact_kernel(MoveArgs a) {
  __shared__ uint64_t s_free[kWords];
  __shared__ int s_sums[2][16];
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int fours = (a.n_pages + 255) / 256, run = (fours + 15) / 16, f0 = min(w * run, fours), f1 = min(f0 + run, fours);
  uint32_t bad = 0;
  const int n_free = *a.n_free, avail = clampi(n_free, 0, a.n_pages);
  for (int i = tid; i < 4 * fours; i += 1024) s_free[i] = 0;
  if (n_free != avail) bad |= FLUX_DEV_BAD_LENGTH;
  __syncthreads();
  constexpr int U = 8;
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
  auto count_of = [&](int f) { return __builtin_popcountll(s_free[4 * f]) + __builtin_popcountll(s_free[4 * f + 1]) + __builtin_popcountll(s_free[4 * f + 2]) + __builtin_popcountll(s_free[4 * f + 3]); };
  int mine = 0;
  for (int f = f0 + l; f < f1; f += 64) mine += count_of(f);
  mine = __builtin_amdgcn_readlane(wave_inclusive_sum(mine), 63);
  if (l == 0) s_sums[0][w] = mine;
  __syncthreads();
  int rank = 0, free_all = 0;
  for (int i = 0; i < 16; ++i) {
    rank += i < w ? s_sums[0][i] : 0;
    free_all += s_sums[0][i];
  }
  CompactBits* const out = (CompactBits*)a.scratch;
  int* const ranks = (int*)(out->bits + 4 * fours);
  const int used = a.n_pages - free_all;                     // in the end the pages below it are the ones in use
  int low = 0;                                               // free pages below it: as many move if they may
  for (int f = f0; f < f1; f += 64) {
    const bool there = f + l < f1;
    const int count = there ? count_of(f + l) : 0, incl = wave_inclusive_sum(count);
    if (there) {
      ranks[f + l] = rank + incl - count;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int word = 4 * (f + l) + i, n = clampi(used - 64 * word, 0, 64);
        out->bits[word] = s_free[word];
        low += n > 0 ? __builtin_popcountll(s_free[word] << (64 - n)) : 0;
      }
    }
    rank += __builtin_amdgcn_readlane(incl, 63);
  }
  low = __builtin_amdgcn_readlane(wave_inclusive_sum(low), 63);
  if (l == 0) s_sums[1][w] = low;
  __syncthreads();
  if (tid == 0) {
    int moves = 0;
    for (int i = 0; i < 16; ++i) moves += s_sums[1][i];
    moves = min(moves, a.most);
    out->free_all = free_all;
    out->moves = moves;
    *a.n_list = moves;
    *a.n_free = free_all;
  }
  if (bad) atomicOr(a.status, bad);
}

// Place of the n-th set bit of x (which has so many).
__device__ __forceinline__ int nth_bit(uint64_t x, int n) {
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

__global__ __launch_bounds__(1024) void page_renumber_kernel(MoveArgs a) {
  __shared__ uint64_t s_free[kWords];
  __shared__ int s_rank[kFours];
  const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fours = (a.n_pages + 255) / 256;
  const CompactBits* const in = (const CompactBits*)a.scratch;
  const int* const ranks = (const int*)(in->bits + 4 * fours);
  const int free_all = in->free_all, moves = in->moves, used = a.n_pages - free_all;
  int len = a.kv_len[min((int)blockIdx.x, a.batch - 1)];     // (of the first row: asked for along with the rest)
  for (int i = tid; i < 4 * fours; i += 1024) s_free[i] = in->bits[i];
  for (int i = tid; i < fours; i += 1024) s_rank[i] = ranks[i];
  __syncthreads();
  // free pages below one
  auto free_below = [&](int page) {
    const int f = page >> 8;
    int r = s_rank[f];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = clampi(page - 256 * f - 64 * i, 0, 64);
      r += n > 0 ? __builtin_popcountll(s_free[4 * f + i] << (64 - n)) : 0;
    }
    return r;
  };
  // the n-th page, from the lowest, of those that are free (or in use)
  auto nth_page = [&](int n, bool is_free) {
    int lo = 0, hi = fours;                                  // the last four words that have no more than n before them
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((is_free ? s_rank[mid] : 256 * mid - s_rank[mid]) <= n) lo = mid;
      else hi = mid;
    }
    n -= is_free ? s_rank[lo] : 256 * lo - s_rank[lo];
    int word = 4 * lo;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const int count = __builtin_popcountll(is_free ? s_free[word] : ~s_free[word]);
      if (n >= count && word == 4 * lo + i) {
        n -= count;
        ++word;
      }
    }
    return 64 * word + nth_bit(is_free ? s_free[word] : ~s_free[word], n);
  };
  const int from = moves > 0 ? nth_page(used - moves, false) : a.n_pages;          // all pages in use from here on move
  // the moves; holders go along
  for (int j = (int)blockIdx.x * 1024 + tid; j < moves; j += (int)gridDim.x * 1024) {
    const int src = nth_page(used - 1 - j, false), dst = nth_page(j, true);
    a.list[3 * j] = src;
    a.list[3 * j + 1] = dst;
    a.list[3 * j + 2] = kPageTokens;
    if (a.shares) {
      a.shares[dst] = a.shares[src];
      a.shares[src] = 0;
    }
  }
  // the list: pages from `from` on, and the free ones below it that no page moved to; the lowest last
  const int left = moves > 0 ? free_below(from) - moves : free_all;                // of the latter
  for (int word = (int)blockIdx.x * 16 + w; word < 4 * fours; word += (int)gridDim.x * 16) {
    const int page = 64 * word + l;
    const uint64_t bits = s_free[word];
    if (64 * word + 63 < from && bits == 0) continue;
    if (page >= a.n_pages) continue;
    int nth = -1;                                            // from the lowest
    if (page >= from) nth = left + page - from;
    else if ((bits >> l) & 1) nth = free_below(page) - moves;
    if (nth >= 0) a.free_pages[free_all - 1 - nth] = page;
  }
  uint32_t bad = 0;                                          // (entries are looked at where no page moves, too: an error in them is reported either way)
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    if (b != (int)blockIdx.x) len = a.kv_len[b];
    const int pages = (clampi(len, 0, a.table_pages << 6) + 63) >> 6;
    int32_t* const row = a.table + (int64_t)b * a.table_pages;
    for (int i = tid; i < pages; i += 1024) {
      const int page = row[i];
      if ((uint32_t)page >= (uint32_t)a.n_pages || (page >= from && ((s_free[page >> 6] >> (page & 63)) & 1))) {
        bad = FLUX_DEV_BAD_PAGE;                             // (no page, or one that the list called free)
      } else if (page >= from) {
        row[i] = nth_page(used - 1 - (page - free_below(page)), true);
      }
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
  // (16 columns are a line of memory of each row; more workgroups for many sequences: 256 of them, 8200 pages, us of fork and copy with up to 4096 / 2048 /
  // 1024 entries each 18.2 / 17.7 / 17.9)
  a.cols_shift = 4;
  while (a.cols_shift > 2 && (pt.batch << a.cols_shift) > 2048) --a.cols_shift;
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
  // a workgroup per row of the table or 4096 pages of the pool, one per CU at most
  const int wide = (pt.n_pages + 4095) / 4096, most = wide > pt.batch ? wide : pt.batch;
  hipLaunchKernelGGL(page_renumber_kernel, dim3(most < 256 ? most : 256), dim3(1024), 0, s, a);
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
