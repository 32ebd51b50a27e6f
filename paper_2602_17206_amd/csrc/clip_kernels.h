// The norm of many tensors together, and the tensors scaled by what it asks for.
//
// Few and small tensors: one workgroup does both, a wavefront for each chunk in turn.
// Else two launches (for up to 128 tensors, whose places come as kernel arguments: nothing is copied to the device): the squares, summed
// up in 64 bits by workgroups; then every workgroup adds those sums up itself, in one order, and scales its share.
// Both read all of the gradients.  The second walks from the end to the beginning: what was read last is still in
// the memory-side cache.
// What bounds it: reading twice and writing once, 386 us for 400 tensors of 430 MB bfloat16 that leave in float32 (1.7 GB, 4.5 TB/s); one
// read cannot be saved, as no element may be written before the norm is known and they do not fit on the chip.  Small lists wait
// for the launch: 13 tensors of 10000 elements, 8.3 us in one kernel.
#pragma once
#include "vector_io.h"

namespace sdtw {

constexpr int kClipTensors = 128;
constexpr int kClipChunk = 8192;  // elements
constexpr int kClipParts = 2048;

struct ClipList {
    const void *data[kClipTensors];
    void *out[kClipTensors];
    uint64_t count_types[kClipTensors];  // count, type << 56, out_type << 60
    int32_t first[kClipTensors + 1];     // chunks before each tensor
    int32_t tensors;
};

struct ClipParams {
    double *parts;    // [all_parts]
    int32_t part, all_parts;  // the first of this launch's
    float max_norm;
    float *norm;      // nullptr but for the launch that writes it
};

// The sum over the 256 threads of a workgroup, in every one of them.
__device__ __forceinline__ double workgroup_sum_f64(double v, double *lds)
{
    v = wave_sum_f64(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Calls f(tensor, first element, elements) for the workgroup's chunks, the last ones first if BACKWARD.
template <bool BACKWARD, typename F> __device__ __forceinline__ void clip_chunks(const ClipList &list, F f)
{
    const int64_t chunks = list.first[list.tensors];
    const int begin = (int)(chunks * blockIdx.x / gridDim.x), end = (int)(chunks * (blockIdx.x + 1) / gridDim.x);
    if (begin >= end) return;
    const int start = BACKWARD ? end - 1 : begin;
    int lo = 0, hi = list.tensors - 1;  // the tensor that holds chunk `start`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (list.first[mid] <= start) lo = mid;
        else hi = mid - 1;
    }
    int tensor = lo;
    for (int n = 0; n < end - begin; ++n) {
        const int chunk = BACKWARD ? start - n : start + n;
        while (chunk < list.first[tensor]) --tensor;
        while (chunk >= list.first[tensor + 1]) ++tensor;
        const int64_t count = (int64_t)(list.count_types[tensor] & 0xffffffffffffull);
        const int64_t at = (int64_t)(chunk - list.first[tensor]) * kClipChunk;
        f(tensor, at, (int)min(count - at, (int64_t)kClipChunk));
    }
}

template <typename T> __device__ __forceinline__ double clip_squares(const T *x, int n, int who, int threads)
{
    constexpr int W = Elem<T>::kWidth, kSteps = kClipChunk / 256 / W;
    double sum = 0.0, more = 0.0;
    if (n == kClipChunk && threads == 256) {
        Bits4 v[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) v[s] = load_vec<false>(x + (s * 256 + who) * W);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < W; e += 2) {
                const double a = Elem<T>::at(v[s], e), b = Elem<T>::at(v[s], e + 1);
                sum = fma(a, a, sum);
                more = fma(b, b, more);
            }
        return sum + more;
    }
    int i = who * W;
    for (; i + W <= n; i += threads * W) {
        const Bits4 v = load_vec<false>(x + i);
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const double a = Elem<T>::at(v, e);
            sum = fma(a, a, sum);
        }
    }
    for (; i < n; ++i) {  // (one thread's at most, fewer than a vector)
        const double a = Elem<T>::up(x[i]);
        sum = fma(a, a, sum);
    }
    return sum;
}

// What a thread takes at once: as many elements as make 16 bytes of the wider of the two types, so that neighbouring threads read and write
// neighbouring memory.  (16 bytes of bfloat16 each, written as twice 16 bytes of float32: 424 us where this takes 300, 400 tensors of 430 MB.)
template <int BYTES> struct Piece;
template <> struct Piece<16> { typedef Bits4Any Any; typedef Bits4 Bits; };
template <> struct Piece<8> {
    typedef uint32_t Bits __attribute__((ext_vector_type(2)));
    typedef Bits Any __attribute__((aligned(2)));
};

// The norm as it is returned: not finite only where an element is not, so that it says whether the gradients were left as they are.
__device__ __forceinline__ float clip_norm(double norm) { return norm < INFINITY ? (float)fmin(norm, 0x1.fffffep127) : (float)norm; }

// What the gradients are multiplied by, as `by` 2^octaves: octaves is 0, but for factors below the normal numbers, which would have
// few digits or none.
struct ClipFactor {
    float by;
    int octaves;
    bool scaled;
    __device__ __forceinline__ ClipFactor(double norm, float max_norm) : octaves(0), scaled(norm > (double)max_norm && norm < INFINITY)
    {
        double factor = scaled ? (double)max_norm / norm : 1.0;  // (a NaN is not scaled)
        if (factor < 0x1p-126) {
            octaves = __builtin_amdgcn_frexp_exp(factor);
            factor = __builtin_amdgcn_frexp_mant(factor);
        }
        by = (float)factor;
    }
    __device__ __forceinline__ float times(float x) const { return __builtin_amdgcn_ldexpf(x * by, octaves); }
};

template <typename T, typename U> __device__ __forceinline__ void clip_scale(const T *in, U *out, int n, const ClipFactor &factor, int who, int threads)
{
    // (a workgroup's whole chunk at once: 8 steps, or 4 between 16-bit types)
    constexpr int W = 16 / (sizeof(T) > sizeof(U) ? (int)sizeof(T) : (int)sizeof(U)), kSteps = kClipChunk / 256 / W;
    static_assert(kSteps * 256 * W == kClipChunk, "a chunk is dealt out evenly");
    typedef Piece<W * (int)sizeof(T)> In;
    typedef Piece<W * (int)sizeof(U)> Out;
    auto load = [&](int i) { return *reinterpret_cast<const typename In::Any *>(in + i); };
    auto store = [&](int i, typename In::Bits v) {
        Bits4 b{};
        for (int e = 0; e < (int)sizeof(v) / 4; ++e) b[e] = v[e];
        float x[Elem<U>::kWidth] = {};
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = factor.times(Elem<T>::at(b, e));
        const Bits4 y = Elem<U>::pack(x);
        typename Out::Bits z;
        for (int e = 0; e < (int)sizeof(z) / 4; ++e) z[e] = y[e];
        __builtin_nontemporal_store(z, reinterpret_cast<typename Out::Any *>(out + i));
    };
    int i = who * W;
    for (; i + (kSteps - 1) * threads * W + W <= n; i += kSteps * threads * W) {
        typename In::Bits v[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) v[s] = load(i + s * threads * W);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) store(i + s * threads * W, v[s]);
    }
    for (; i + W <= n; i += threads * W) store(i, load(i));
    for (; i < n; ++i) out[i] = Elem<U>::down(factor.times(Elem<T>::up(in[i])));  // (one thread's at most, fewer than a piece)
}

// Calls f with the element that SDTW_TYPE_* `type` stands for.
template <typename F> __device__ __forceinline__ void clip_typed(int type, F f)
{
    if (type == SDTW_TYPE_F32) f(float{});
    else if (type == SDTW_TYPE_F16) f(_Float16{});
    else f(Bf16{});
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipList list, ClipParams p)
{
    __shared__ double lds[4];
    double sum = 0.0;
    clip_chunks<false>(list, [&](int tensor, int64_t at, int n) {
        clip_typed((int)(list.count_types[tensor] >> 56 & 15), [&](auto t) {
            sum += clip_squares(static_cast<const decltype(t) *>(list.data[tensor]) + at, n, threadIdx.x, 256);
        });
    });
    sum = workgroup_sum_f64(sum, lds);
    if (threadIdx.x == 0) p.parts[p.part + blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void clip_scale_kernel(ClipList list, ClipParams p)
{
    __shared__ double lds[4];
    double sum = 0.0;
    for (int k = threadIdx.x; k < p.all_parts; k += 256) sum += p.parts[k];
    const double norm = sqrt(workgroup_sum_f64(sum, lds));
    if (p.norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = clip_norm(norm);
    const ClipFactor factor(norm, p.max_norm);
    clip_chunks<true>(list, [&](int tensor, int64_t at, int n) {
        if (!factor.scaled && list.out[tensor] == list.data[tensor]) return;
        const uint64_t types = list.count_types[tensor];
        clip_typed((int)(types >> 56 & 15), [&](auto t) {
            clip_typed((int)(types >> 60), [&](auto u) {
                clip_scale(static_cast<const decltype(t) *>(list.data[tensor]) + at, static_cast<decltype(u) *>(list.out[tensor]) + at, n,
                           factor, threadIdx.x, 256);
            });
        });
    });
}

__global__ __launch_bounds__(1024) void clip_small_kernel(ClipList list, ClipParams p)
{
    __shared__ double sums[16];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, chunks = list.first[list.tensors];
    auto each = [&](auto f) {  // (the tensors' chunks are dealt out to the wavefronts)
        int tensor = 0;
        for (int chunk = wave; chunk < chunks; chunk += 16) {
            while (chunk >= list.first[tensor + 1]) ++tensor;
            const int64_t count = (int64_t)(list.count_types[tensor] & 0xffffffffffffull);
            const int64_t at = (int64_t)(chunk - list.first[tensor]) * kClipChunk;
            f(tensor, at, (int)min(count - at, (int64_t)kClipChunk));
        }
    };
    double sum = 0.0;
    each([&](int tensor, int64_t at, int n) {
        clip_typed((int)(list.count_types[tensor] >> 56 & 15), [&](auto t) {
            sum += clip_squares(static_cast<const decltype(t) *>(list.data[tensor]) + at, n, lane, 64);
        });
    });
    sum = wave_sum_f64(sum);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < 16; ++w) sum += sums[w];
    const double norm = sqrt(sum);
    if (threadIdx.x == 0) *p.norm = clip_norm(norm);
    const ClipFactor factor(norm, p.max_norm);
    each([&](int tensor, int64_t at, int n) {
        if (!factor.scaled && list.out[tensor] == list.data[tensor]) return;
        const uint64_t types = list.count_types[tensor];
        clip_typed((int)(types >> 56 & 15), [&](auto t) {
            clip_typed((int)(types >> 60), [&](auto u) {
                clip_scale(static_cast<const decltype(t) *>(list.data[tensor]) + at, static_cast<decltype(u) *>(list.out[tensor]) + at, n,
                           factor, lane, 64);
            });
        });
    });
}

}  // namespace sdtw
