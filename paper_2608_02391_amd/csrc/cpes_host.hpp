// cpes_host.hpp -- what the entry points share on the host: error reporting and
// small checks.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cpes {

// Clears, and sets, the calling thread's error message; fail returns `code`.
void clear_error();
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_status(hipError_t e, const char* what);

inline bool aligned16(const void* p)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
}

}  // namespace cpes
