// Launchers of the paged 8-bit KV cache (each validates nothing: flux_api.hip has done it).
#pragma once

#include "flux_internal.h"

namespace flux {

constexpr int kPageTokens = FLUX_PAGE_TOKENS;
constexpr int kPlanRows = 2048;               // slots that a workgroup of flux_page_plan writes
constexpr long long kAppendPagedFew = 16384;  // (rows, heads) of an append up to which a wave looks after one row
constexpr int kMinScaleExp = -100;            // of the scale of a block; its codes reach down to 2^-109

hipError_t launch_page_plan(const Ctx& c, const flux_page_table& pt, const int32_t* cu_new, int total_new, int32_t* slots, hipStream_t s);
hipError_t launch_page_release(const Ctx& c, const flux_page_table& pt, const int32_t* keep_len, hipStream_t s);
hipError_t launch_kv_append_paged(const Ctx& c, const flux_paged_kv& kv, int hkv, int d, const void* k_new, const void* v_new,
                                  const int32_t* slots, int total_new, hipStream_t s);

inline int pages_of(int tokens) { return tokens / kPageTokens + (tokens % kPageTokens != 0 ? 1 : 0); }
// A page of 8-bit codes has the bytes of 32 rows of a bf16 cache, the block that the plan of a decode call counts in.
inline DecodePlan plan_decode_paged(const flux_attn_cfg& cfg, int batch, int max_kv_len) {
  return plan_decode(cfg, batch, 32 * pages_of(max_kv_len));
}
hipError_t launch_decode_paged(const Ctx& c, const flux_attn_cfg& cfg, const void* q, int max_kv_len, const flux_paged_kv& kv,
                               const flux_page_table& pt, const uint8_t* mode, void* out, hipStream_t s);

}  // namespace flux
