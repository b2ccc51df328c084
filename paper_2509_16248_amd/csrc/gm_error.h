// gm_error.h -- return codes with the message that gm_last_error reports.
#pragma once
#include <hip/hip_runtime.h>

namespace gm {

// GM_E_INVAL / GM_E_HIP, after recording the message for the calling thread.
int inval(const char* what);
int hip_fail(hipError_t e, const char* what);

}  // namespace gm

#define HIP_TRY(call)                                       \
  do {                                                      \
    hipError_t e_ = (call);                                 \
    if (e_ != hipSuccess) return gm::hip_fail(e_, #call);   \
  } while (0)
