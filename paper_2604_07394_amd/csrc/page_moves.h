// Launchers of the calls that hand pages around, move and copy them (each validates nothing: flux_api.hip has done it).
#pragma once

#include "paged.h"

namespace flux {

constexpr int kForkAlone = 16384;           // pages of a pool up to which one workgroup of a fork looks through all of them
constexpr int kForkPages = 4096;            // pages that each of several looks through in a second launch
constexpr int kForkEntries = 16384;         // entries of the table that a workgroup holds in LDS
constexpr int kCompactPages = 1 << 20;      // pages of a pool that one workgroup holds a bit of each of in LDS (128 KB)
constexpr int kCopyWgs = 8192;              // workgroups that copy at most
static_assert(kForkEntries >= 4 * FLUX_MAX_PAGED_BATCH, "four columns of the table fit");

// An entry of a table as a page of the pool; -1: none.
constexpr int page_of_entry(int entry, int n_pages) { return (uint32_t)entry < (uint32_t)n_pages ? entry : -1; }
// Whether a fork writes a place of a row that had `had` places and goes on with `has`, of its own (`own`) or another row's; `before`: the page there, -1:
// none.  A page that a row keeps of its own stays as it is; a number outside the pool there becomes -1 like any other.
constexpr bool fork_writes(int place, int had, int has, bool own, int before) { return place < (had > has ? had : has) && (!own || place >= has || before < 0); }

// Bytes of the partials that the calls take: what every workgroup found and how much, or a bit per page and a count per 256.
inline size_t fork_bytes(int n_pages) {
  if (n_pages <= kForkAlone) return 0;
  const size_t groups = ((size_t)n_pages + kForkPages - 1) / kForkPages;
  return groups * (kForkPages + 1) * sizeof(int32_t);
}
inline size_t compact_bytes(int n_pages) { return 16 + ((size_t)n_pages + 255) / 256 * (4 * sizeof(uint64_t) + sizeof(int32_t)); }

hipError_t launch_page_fork(const Ctx& c, const flux_page_table& pt, int32_t* shares, const int32_t* parent, const int32_t* keep, int32_t* copies,
                            int32_t* n_copies, hipStream_t s);
hipError_t launch_page_compact(const Ctx& c, const flux_page_table& pt, int32_t* shares, int32_t* moves, int max_moves, int32_t* n_moves, hipStream_t s);
hipError_t launch_page_copy(const Ctx& c, const flux_paged_kv& kv, int hkv, int d, const int32_t* copies, const int32_t* n_copies, int max_copies, hipStream_t s);

}  // namespace flux
