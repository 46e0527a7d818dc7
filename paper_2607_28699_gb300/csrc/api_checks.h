// What the extern "C" files share: the message of a refused call and small checks.  Host code.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/witcert.h"

namespace wc {

// Leaves the message for wc_last_error() (thread-local) and returns st.
wc_status fail(wc_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
wc_status cuda_fail(cudaError_t e, const char* what);
int current_sm_count(int* out);   // 0: ok
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace wc
