// Launchers of the calls that norm and turn the heads of new tokens (each validates nothing: flux_api.hip has done it).
#pragma once

#include "paged.h"

namespace flux {

// What a call takes from the projection and how its heads are worked on.
struct HeadRows {
  flux_head_cfg cfg;
  flux_qkv_rows in;
  const int32_t* positions;   // null: nothing is turned, or (contiguous cache) the places of the rows
  int total;
  void* q_out;                // null: no queries
};

hipError_t launch_head_rows(const HeadRows& r, void* k_out, hipStream_t s);
hipError_t launch_qkv_append(const Ctx& c, const HeadRows& r, const flux_kv_cache& cache, const int32_t* cu_new, hipStream_t s);
hipError_t launch_qkv_append_paged(const Ctx& c, const HeadRows& r, const flux_paged_kv& kv, const int32_t* slots, hipStream_t s);

constexpr int kHeadWaves = 8192;            // waves that a launch takes where a token's heads can be shared out over so many
constexpr int kHeadMost = 1 << 20;          // workgroups for queries that such a launch takes at most
// Workgroups for K, and for V, up to which a tile of 64 rows has several of them: one per head at most, and up to kQuantFewWgs also more.  us with 256 and 128
// / 512 and 256, 8 heads of 128: 512 rows of one sequence 7.4 / 9.1, 1024 12.0 / 11.6, 1500 12.5 / 15.8, 4096 22 / 24, 16384 79 / 82.
constexpr int kQuantWgs = 256, kQuantFewWgs = 128;
inline int quant_share(long long tiles, int hkv) {
  int share = 0;
  while (share < 7 && tiles << share < ((1 << share) < hkv ? kQuantWgs : kQuantFewWgs)) ++share;
  return share;
}
// Waves that the heads of a token are shared out over, `passes` of 64 lanes in all.
inline int head_waves(int total, int passes) {
  const int most = total > 0 ? kHeadWaves / total : 1;
  return most < 1 ? 1 : (most < passes ? most : passes);
}

}  // namespace flux
