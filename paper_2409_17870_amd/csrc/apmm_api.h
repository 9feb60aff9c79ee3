// How the entry points of include/apmm.h report an error: its text is kept for apmm_last_error() on the calling thread.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/apmm.h"

namespace apmm {

apmm_status fail(apmm_status st, const char *msg);
apmm_status fail_hip(hipError_t e, const char *where);

}  // namespace apmm
