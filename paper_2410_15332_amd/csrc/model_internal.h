// What the bf16 and the 8-bit model drivers share (defined in model.cpp).
#pragma once

#include <stddef.h>

#include "epic_link.h"

namespace epic {

epic_status validate_model(const epic_model_cfg* c);
// Configuration, plan and residual stream of a layer or model call.
epic_status check_model_call(const epic_model_cfg* c, const epic_plan_sizes* s, const epic_plan* p, const float* h);
epic_status check_workspace(const void* ws, size_t ws_bytes, size_t need);
// A call without rows: the re-rotated copies of every layer, if the plan has any.
epic_status link_write_only(const epic_model_cfg* c, const epic_plan_sizes* s, const epic_plan* p, uint16_t* const* kc,
                            uint16_t* const* vc, int n_layers, void* stream);
// The status of the launches so far.
epic_status hip_ok(const char* what);

}  // namespace epic
