// Status and message of the calling thread's last error, for every entry point.
#pragma once
#include <hip/hip_runtime.h>
#include <string>
#include "../../include/atspeed.h"

namespace atspeed {
// Records msg for atspeed_last_error and returns s.
atspeed_status fail(atspeed_status s, const std::string& msg);
// The arguments of atspeed_logit_rules that are not a call's logits and rows.
atspeed_status check_rules(const atspeed_logit_rules_args& a);
// atspeed_logit_rules where allowed columns come out at `lowest` at least.
atspeed_status logit_rules(const atspeed_logit_rules_args& a, float lowest, hipStream_t st);
}  // namespace atspeed

#define HIP_TRY(expr)                                                                      \
  do {                                                                                     \
    hipError_t _e = (expr);                                                                \
    if (_e != hipSuccess) return fail(ATSPEED_E_DEVICE, std::string(#expr) + ": " + hipGetErrorString(_e)); \
  } while (0)

#define ST_TRY(expr)                        \
  do {                                      \
    atspeed_status _s = (expr);             \
    if (_s != ATSPEED_OK) return _s;        \
  } while (0)
