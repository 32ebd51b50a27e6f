// What the library's host files share.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/sdtw.h"

namespace sdtw {

// Optional per-kernel timing (test/benchmark hook): when switched on, every kernel launch of the
// library is bracketed by two HIP events on the caller's stream.
bool profile_begin(const char *name, hipStream_t st);
void profile_end(hipStream_t st);

struct ProfScope {
    hipStream_t st;
    bool on;
    ProfScope(const char *name, hipStream_t s) : st(s), on(profile_begin(name, s)) {}
    ~ProfScope() { if (on) profile_end(st); }
};

inline int check_ws(const void *ws, size_t bytes, size_t need)
{
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || bytes < need) return SDTW_ERR_WORKSPACE;
    return SDTW_OK;
}

inline int hip_ok() { return hipGetLastError() == hipSuccess ? SDTW_OK : SDTW_ERR_HIP; }

}  // namespace sdtw
