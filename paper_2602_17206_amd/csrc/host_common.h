// What the library's host files share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

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

// The rule of a bias descriptor's buckets (train_ops.hip); false if the descriptor is invalid.
struct BucketRule;
bool position_bias_rule(const sdtw_bias_desc *d, BucketRule *rule);

// The position bias (train_ops.hip) as the Soft-DTW calls use it: with `penalty` negative table entries count as 0.
int position_bias_add(const sdtw_bias_desc *d, const void *table, bool penalty, const void *in, const int32_t *offsets,
                      const int32_t *row_len, const int32_t *col_len, void *out, hipStream_t st);
// ... and its table's gradient; penalty_table: 0 for the entries that are negative there, or nullptr;
// scale: [B], or [B, H] with scale_heads.
int position_bias_table_grad(const sdtw_bias_desc *d, const void *penalty_table, const void *grad, const float *scale, bool scale_heads,
                             const int32_t *offsets, const int32_t *row_len, const int32_t *col_len, float *dtable,
                             void *workspace, size_t workspace_bytes, hipStream_t st);

}  // namespace sdtw
