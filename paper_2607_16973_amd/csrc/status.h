// Status codes from HIP results, shared by the entry points' files.
#pragma once

#include <hip/hip_runtime.h>

#include "tq.h"

namespace tq {

tq_status device_ready();                              // TQ_EDEVICE without a usable GPU
tq_status hip_fail(hipError_t e, const char *what);

}  // namespace tq
