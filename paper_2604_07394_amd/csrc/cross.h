// Launch rules of flux_attn_cross (the launcher validates nothing: flux_api.hip has done it).
#pragma once

#include "flux_internal.h"

namespace flux {

constexpr int kCrossBatch = 64;             // sequences of a launch: a lane looks after each; longer batches take several launches
constexpr int kCrossMaxUnits = 1024;        // units of a launch whose tiles may be shared out (or one per tile, where those are more)
constexpr int kCrossMostWgs = 1 << 23;      // workgroups of a launch: fewer than 2^32 threads
constexpr int kCrossMostGroup = 1 << 20;    // query heads per KV head: (x + 1/2) / group in floats tells row x < 2 group of two tokens (from 2^22.5 on it does not)
constexpr int kCrossRunWgs = 512;           // workgroups of short runs that the chip holds at once
constexpr int kCrossJoinWgs = 4096;         // workgroups that join at most (24576 that find nothing to do take 11 us, 4096 take 3)
constexpr int cross_resident(int head_dim) { return 256 * (head_dim == 128 ? 2 : 3); }   // workgroups that the chip holds at once

struct CrossPlan {
  int bm;                 // rows of a tile; 16 or 32: short runs, of a tile each
  int tiles;              // of a sequence and KV head, at most
  long long wgs;          // workgroups of a launch
  int part_units;         // units whose rows the workspace holds; 0: tiles are not shared out
  size_t info_bytes;      // of the table in front of these rows
};
inline CrossPlan plan_cross(const flux_attn_cfg& cfg, int batch, int max_q_len, int max_kv_len, size_t partials_bytes) {
  CrossPlan p;
  const int n = batch < kCrossBatch ? batch : kCrossBatch;
  const long long rows = (long long)max_q_len * (cfg.n_q_heads / cfg.n_kv_heads);
  p.bm = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  p.tiles = (int)((rows + p.bm - 1) / p.bm);
  const long long tiles = (long long)n * cfg.n_kv_heads * p.tiles;
  p.wgs = tiles + 8 * n;                                     // (the units of a sequence are padded to whole rounds of the XCDs)
  p.part_units = 0;
  p.info_bytes = (((size_t)tiles + 1) * 16 + 255) / 256 * 256;
  // (tiles are shared out where all of them run side by side; the longest sequence alone says whether they may)
  if (max_kv_len > 128 && (long long)cfg.n_kv_heads * p.tiles < cross_resident(cfg.head_dim) && p.info_bytes <= partials_bytes / 4) {
    const size_t fit = (partials_bytes - p.info_bytes) / ((size_t)p.bm * (cfg.head_dim + 2) * sizeof(float));
    p.part_units = (int)(fit < (size_t)kCrossMaxUnits ? fit : (size_t)kCrossMaxUnits);
    if (p.wgs < p.part_units) p.wgs = p.part_units;
  }
  return p;
}

hipError_t launch_cross(const Ctx& c, const flux_attn_cfg& cfg, const void* q, const int32_t* cu_q, int max_q_len, int max_kv_len,
                        const flux_kv_cache& cache, void* out, hipStream_t s);

}  // namespace flux
