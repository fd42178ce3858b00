// Status and last-error helpers shared by the C entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

#include "cosa.h"

namespace cosa {

// Records the failure for cosa_last_error() of this thread and returns st.
cosa_status fail(cosa_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
cosa_status ok();
cosa_status hip_fail(hipError_t e, const char* what);

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace cosa
