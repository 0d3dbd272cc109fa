// The library's error record, shared by its translation units (defined in def_api.cu).
#pragma once

#include <cuda_runtime.h>

namespace defk {

// Stores a message for def_last_error() (thread-local) and returns `code`.
__attribute__((visibility("hidden"))) int fail(int code, const char *fmt, ...);
__attribute__((visibility("hidden"))) int cuda_fail(cudaError_t err, const char *what);

}  // namespace defk
