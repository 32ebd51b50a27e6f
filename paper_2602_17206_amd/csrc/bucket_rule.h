// The buckets of relative positions and what the kernels that use them share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace sdtw {

constexpr int kMaxBuckets = 256;

// The buckets of a side: distances below e one by one, bucket e + k from start[k] on (start[m]: beyond every distance).
struct BucketRule {
    int32_t n, e, m, two_sided;
    float per_octave, shift;  // bucket e + k is about per_octave * log2(d) + shift
    int32_t start[kMaxBuckets / 2 + 1];
    // first distance of bucket u of a side; of bucket n: beyond every distance
    __device__ __forceinline__ int first(int u) const { return u < e ? u : start[u - e]; }
    // The bucket of j - i - offset = r; `starts`: start[] in LDS.  The logarithm is a guess that the whole numbers correct:
    // it is off by less than a distance's rounding, so by one bucket at most where buckets are wider than that, and the
    // loops end at the right one in any case.
    __device__ __forceinline__ int bucket(int r, const int32_t *starts) const
    {
        const int d = two_sided ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
        int u = d;
        if (d >= e) {
            int k = min(max((int)(__builtin_amdgcn_logf((float)d) * per_octave + shift), 0), m - 1);
            while (d < starts[k]) --k;
            while (d >= starts[k + 1]) ++k;
            u = e + k;
        }
        return two_sided && r > 0 ? u + n : u;
    }
};

// A wavefront's accesses to LDS are carried out in the order of their issue.  Where one lane's place is another lane's before or
// after, this keeps the compiler from changing that order.
__device__ __forceinline__ void wavefront_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

__device__ __forceinline__ int clamp_len(const int32_t *len, int b, int full) { return len ? min(max(len[b], 0), full) : full; }

// The workgroup's number, renumbered so that neighbouring tiles are on one XCD (workgroups go round the eight of them).  Reading
// 32 planes of 8192 x 8192 float32 in tiles of 64 x 1024 runs at 6.7 TB/s so, and at 6.3 with the tiles dealt out in turn.
__device__ __forceinline__ int neighbours_together()
{
    const int id = blockIdx.x, n = gridDim.x / 8;
    return id < 8 * n ? id % 8 * n + id / 8 : id;
}

// a position difference as 32 bits: beyond 2^30 every distance is in the last bucket
__device__ __forceinline__ int clamp_rel(int64_t r) { return (int)min(max(r, (int64_t) - (1 << 30)), (int64_t)1 << 30); }

}  // namespace sdtw
