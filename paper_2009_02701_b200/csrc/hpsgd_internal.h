// What the translation units of libhpsgd share: the text of the last error, the launch count and
// the multiplicative mix of the counter hash.  Nothing here is exported.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/hpsgd.h"

#define HPSGD_HIDDEN __attribute__((visibility("hidden")))

namespace hpsgd {

// Record `code` with a printf-style text as the last error; returns `code`.
HPSGD_HIDDEN int report(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Count kernels launched by the operators (hpsgd_launch_count).
HPSGD_HIDDEN void count_launches(int n);

}  // namespace hpsgd
