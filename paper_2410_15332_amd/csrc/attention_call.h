// What the attention entry points share (defined in api.cpp): checks, the kernels' arguments, profiling events.
#pragma once

#include "kernels.h"

namespace epic {

// What they ask of their config and plan.
epic_status check_attention(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes, const epic_plan* plan_dev);
AttnArgs attention_args(const epic_attn_cfg* cfg, const epic_plan_sizes* s, const epic_plan* p, const uint16_t* q_s,
                        const uint16_t* k_cache, const uint16_t* v_cache, uint16_t* out, float* lse, void* workspace);
// The calling thread's profiling event i, if it has one, on `stream`.
void record_profile_event(int i, hipStream_t stream);

}  // namespace epic
