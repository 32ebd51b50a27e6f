// What the attention kernels are made of: tiles of rows in LDS, and products of such a tile with vectors that lanes hold.
//
// A wavefront works on 32 "columns" (queries, or keys in the kernel for the keys' gradients), column lane % 32 in the two lanes
// c and c + 32, and on tiles of 32 rows X [32][D] of what passes by.  With v_mfma_f32_32x32x* there are two products:
//   along_features   S [row][column] = sum_f X[row][f] R[column][f], R in registers
//   along_rows       O [f][column] += sum_row X[row][f] P[row][column], P in registers as S came out
// S leaves lane (c, half) with rows 8 (r / 4) + 4 half + r % 4 of its column in register r.  The order of a product's inner index
// is free as long as both operands have the same: along_rows takes the rows in that very order, so that P goes back into the
// matrix cores as it is, without a way through LDS, and statistics of a column stay in its two lanes.
#pragma once
#include <type_traits>

#include "bucket_rule.h"
#include "vector_io.h"

namespace sdtw {

typedef float Acc __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the row of register r within its tile
__device__ __forceinline__ constexpr int tile_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// The other half's value: of the two lanes of a column, each gets both.
struct Halves { float lower, upper; };
__device__ __forceinline__ Halves halves(float v)
{
    const uint32_t x = __float_as_uint(v);
    const auto w = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return {__uint_as_float(w[0]), __uint_as_float(w[1])};
}
__device__ __forceinline__ float both_sum(float v) { const Halves h = halves(v); return h.lower + h.upper; }
__device__ __forceinline__ float both_max(float v) { const Halves h = halves(v); return fmaxf(h.lower, h.upper); }

__device__ __forceinline__ int wave_min_i32(int v)
{
    for (int d = 1; d < 64; d *= 2) v = min(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max_i32(int v)
{
    for (int d = 1; d < 64; d *= 2) v = max(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}

// ------------------------------------------------------------------ tiles in LDS

// Rows of DP features (D and zeros behind it) without gaps, as memory is copied into LDS 64 chunks of 16 bytes at a time; a tile begins at
// a multiple of 256 bytes.  Within a row the chunks change places, chunk ch to ch ^ turn(row), so that what a read wants at once lies in
// different ones of the 16 chunks that the 64 banks hold: of 16 bytes a lane, rows 0-3, 12-15, 20-23 and 24-27 (and so on), which
// bits 2 and 3 of the row tell apart beside the lowest two; of the transposing read, four neighbouring chunks of four rows.
template <typename T, int DP> struct TileShape {
    static constexpr int W = Elem<T>::kWidth;
    static constexpr int kChunks = DP / W;  // 16-byte chunks of a row
    static constexpr int kStride = DP * (int)sizeof(T);
    static constexpr int kMask = kChunks % 16 == 0 ? 15 : kChunks % 8 == 0 ? 7 : 3;  // places change among so many chunks, plus one
    static constexpr int bytes(int rows) { return rows * kStride; }
    static __device__ __forceinline__ constexpr int turn(int row)
    {
        const int low = (row >> 2 & 1) | (row >> 3 & 1) << 1;
        return kMask == 15 ? (row & 3) << 2 | low : kMask == 7 ? (row >> 1 & 1) << 2 | low : low;
    }
};

// A matrix [rows][D] in memory whose features are contiguous and fill whole 16-byte chunks (others are packed beforehand).
template <typename T> struct Rows {
    const T *base;
    int64_t row;  // stride
};

// The memory from `base` on, `bytes` of it: what is read beyond them is 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void *base, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a), hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

typedef __attribute__((address_space(3))) char LdsByte;
__device__ __forceinline__ uint32_t lds_address(const char *p) { return (uint32_t)reinterpret_cast<uintptr_t>((LdsByte *)p); }

template <typename V> __device__ __forceinline__ V lds_read(uint32_t address, int offset)
{
    typedef __attribute__((address_space(3))) const char Byte;
    typedef __attribute__((address_space(3))) const V Value;
    return *(Value *)((Byte *)(uintptr_t)address + offset);
}

// 16 bytes a lane from the window straight into LDS, lane after lane from `lds` on.  Written out because the compiler, which cannot tell the
// tile that is being filled from the one that is being read, would wait for it before every read.  It does not look into what is written
// out, so the wait states that the hardware does not see to are here: one between m0's write and the copy that reads it, and five after a vector
// instruction that wrote a scalar register - the window comes from readfirstlane, or from lanes that scalar registers were spilled to -
// of which m0's write is one and s_nop 3 are four.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is reserved, so that naming it is warned of; it is not to be kept here)
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t from, uint32_t at, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(at), "s"(from),
                 "s"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// All that the wavefront asked for is there, and what it read from LDS has left it.  (The compiler does not reckon with this wait: what it
// loaded itself before a loop - a column's features - it waits for inside once more, before the first product.  Memory answers in order, so
// that the copies asked for in between are waited for as well: the next tile is on its way during what comes before that product only.)
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// All but the last N copies that the wavefront asked for are there.
template <int N> __device__ __forceinline__ void copies_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// What the wavefront read from LDS has left it.
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A tile of ROWS rows, copied by THREADS threads (`who`).  A tile's address is a scalar, each thread's places within it do not change,
// and rows and features behind the end come as zeros without a branch.
template <typename T, int DP, int ROWS, int THREADS> struct Stage {
    using Shape = TileShape<T, DP>;
    static constexpr int kEach = ROWS * Shape::kChunks / THREADS;
    static_assert(kEach * THREADS == ROWS * Shape::kChunks, "a tile is dealt out evenly");
    // Where the threads take whole groups of sixteen rows a thread's places are one, kStep rows further on each time.
    static constexpr int kStep = THREADS / Shape::kChunks;
    static constexpr bool kOne = THREADS % Shape::kChunks == 0 && kStep % 16 == 0;
    uint32_t at[kOne ? 1 : kEach];
    Rows<T> x;
    uint32_t row_bytes, last_bytes;
    __device__ __forceinline__ void begin(const Rows<T> &rows, int D, int who)
    {
        x = rows;
        row_bytes = (uint32_t)x.row * (uint32_t)sizeof(T);
        last_bytes = (uint32_t)D * (uint32_t)sizeof(T);
#pragma unroll
        for (int k = 0; k < (kOne ? 1 : kEach); ++k) {
            const int id = who + k * THREADS, row = id / Shape::kChunks;
            const uint32_t f = (uint32_t)((id % Shape::kChunks) ^ Shape::turn(row)) * 16;
            at[k] = f < last_bytes ? (uint32_t)row * row_bytes + f : 0x7fffffffu;
        }
    }
    // rows first .. first + ROWS; zeros from `limit` on (first < limit)
    __device__ __forceinline__ void copy(char *tile, int first, int limit, int who) const
    {
        const uint32_t to = lds_address(tile) + (uint32_t)(who / 64) * 1024u;
        const T *from = x.base + first * x.row;
        const int rows = min(limit - first, ROWS);
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int before = kOne ? k * kStep : 0;
            const uint32_t bytes = rows > before ? (uint32_t)(rows - before) * row_bytes - row_bytes + last_bytes : 0;
            copy_to_lds(window(from + before * x.row, bytes), at[kOne ? 0 : k], to + (uint32_t)k * (THREADS * 16u));
        }
    }
};

// Zeros for the rows of a tile whose document is negative: they may hold anything.  `documents`: of the ROWS rows, in LDS.
template <typename T, int DP, int ROWS, int THREADS> __device__ __forceinline__ void clear_rows(char *tile, const int32_t *documents, int who)
{
    using Shape = TileShape<T, DP>;
    for (int id = who; id < ROWS * Shape::kChunks; id += THREADS)
        if (documents[id / Shape::kChunks] < 0) *reinterpret_cast<Bits4 *>(tile + id * 16) = Bits4{};
}

// ------------------------------------------------------------------ products

// A column's features, as along_features takes them: chunks half, half + 2, ...
template <typename T, int DP> struct Column {
    static constexpr int kSteps = TileShape<T, DP>::kChunks / 2;
    Bits4 v[kSteps];
    __device__ __forceinline__ void load(const T *row, int D, bool valid, int half)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) v[s] = Bits4{};
        if (!valid) return;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            if ((2 * s + half) * Elem<T>::kWidth < D) v[s] = load_vec<false>(row + (2 * s + half) * Elem<T>::kWidth);
    }
};

template <typename T> __device__ __forceinline__ void mma(Acc &acc, const Bits4 &a, const Bits4 &b)
{
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = a[e], y = b[e];
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x), __uint_as_float(y), acc, 0, 0, 0);
        }
    } else if constexpr (std::is_same<T, Bf16>::value) {
        typedef __bf16 V __attribute__((ext_vector_type(8)));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
    } else {
        typedef _Float16 V __attribute__((ext_vector_type(8)));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), acc, 0, 0, 0);
    }
}

// S = X R for the 32 rows of `tile`, and what `acc` holds
template <typename T, int DP> __device__ __forceinline__ Acc along_features(const char *tile, const Column<T, DP> &col, int lane, Acc acc = Acc{})
{
    using Shape = TileShape<T, DP>;
    const int row = lane & 31;
    const uint32_t at = lds_address(tile) + (uint32_t)(row * Shape::kStride + ((lane >> 5) ^ Shape::turn(row)) * 16);  // chunk 2 s + half
#pragma unroll
    for (int s = 0; s < Column<T, DP>::kSteps; ++s)
        mma<T>(acc, lds_read<Bits4>(at ^ (uint32_t)(2 * s & Shape::kMask) * 16, (2 * s & ~Shape::kMask) * 16), col.v[s]);
    return acc;
}

// P [32 rows][column] as the matrix cores take it: rounded to T, except for float32.  Numbers of more digits would be two products for one, as
// in along_rows_twice; rounded once, they put out, dv and dk 1.1 to 1.45 times as far from 64 bits as the result's own rounding does.
template <typename T> struct Weights {
    Bits4 v[2];
    __device__ __forceinline__ explicit Weights(const Acc &p)
    {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float x[8] = {p[8 * s], p[8 * s + 1], p[8 * s + 2], p[8 * s + 3], p[8 * s + 4], p[8 * s + 5], p[8 * s + 6], p[8 * s + 7]};
            v[s] = Elem<T>::pack(x);
        }
    }
};
template <> struct Weights<float> {
    Acc v;
    __device__ __forceinline__ explicit Weights(const Acc &p) : v(p) {}
};

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) Short4 LdsShort4;

// O += X^T P: feature 32 ft + tile_row(r, half) of the column in register r of acc[ft]
// (`more`: other weights whose products are added as well)
template <typename T, int DP>
__device__ __forceinline__ void along_rows(Acc (&acc)[DP / 32], const char *tile, const Weights<T> &w, int lane, const Weights<T> *more = nullptr)
{
    using Shape = TileShape<T, DP>;
    constexpr int kStride = Shape::kStride, kMask = Shape::kMask;
    const int half = lane >> 5;
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 4 * half + (r & 3);  // (of the row, 8 (r / 4) is left out: it moves bit 1 of the place)
            const uint32_t at = lds_address(tile) + (uint32_t)(row * kStride + (((lane & 31) >> 2) ^ Shape::turn(row)) * 16 + (lane & 3) * 4);
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) {
                const float x = lds_read<float>(at ^ (uint32_t)((ft * 8 & kMask) ^ (r >> 2 & 1) << 1) * 16, 8 * (r >> 2) * kStride + (ft * 8 & ~kMask) * 16);
                acc[ft] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w.v[r], acc[ft], 0, 0, 0);
            }
        }
    } else {
        // ds_read_b64_tr_b16: sixteen lanes read 4 rows of 16 elements, four elements a lane, and each gets a column of them
        const int row = 4 * half + (lane >> 2 & 3), chunk = (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
        const uint32_t at = lds_address(tile) + (uint32_t)(row * kStride + (chunk ^ Shape::turn(row)) * 16 + (lane & 1) * 8);
        typedef __attribute__((address_space(3))) char Byte;
#pragma unroll
        for (int ft = 0; ft < DP / 32; ++ft)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Bits4 a;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const uint32_t place = at ^ (uint32_t)((ft * 4 & kMask) ^ q << 1) * 16;
                    const Short4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (LdsShort4 *)((Byte *)(uintptr_t)place + (16 * s + 8 * q) * kStride + (ft * 4 & ~kMask) * 16));
                    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
                    a[2 * q] = (uint32_t)bits;
                    a[2 * q + 1] = (uint32_t)(bits >> 32);
                }
                mma<T>(acc[ft], a, w.v[s]);
                if (more) mma<T>(acc[ft], a, more->v[s]);
            }
    }
}

// The same with P to twice the type's digits, as the sum of two numbers of the type: the tile's reads serve both.
template <typename T, int DP> __device__ __forceinline__ void along_rows_twice(Acc (&acc)[DP / 32], const char *tile, const Acc &p, int lane)
{
    if constexpr (std::is_same<T, float>::value) {
        along_rows<T, DP>(acc, tile, Weights<T>(p), lane);
    } else {
        const Weights<T> w(p);
        Acc rest;
#pragma unroll
        for (int r = 0; r < 16; ++r) rest[r] = p[r] - Elem<T>::at(w.v[r / 8], r % 8);
        const Weights<T> v(rest);
        along_rows<T, DP>(acc, tile, w, lane, &v);
    }
}

// A column's result, `factor` times acc, as row `out` of D features in memory.
template <typename T, int DP> __device__ __forceinline__ void store_column(T *out, int D, const Acc (&acc)[DP / 32], float factor, int half)
{
    typedef uint32_t Two __attribute__((ext_vector_type(2)));
    typedef Two TwoAny __attribute__((aligned(2)));
#pragma unroll
    for (int ft = 0; ft < DP / 32; ++ft)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int f = 32 * ft + 8 * g + 4 * half;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[ft][4 * g + e] * factor;
            if (f + 4 <= D) {
                if constexpr (sizeof(T) == 4)
                    store_vec<false>(out + f, Elem<T>::pack(x));
                else
                    *reinterpret_cast<TwoAny *>(out + f) = Two{Elem<T>::pack2(x[0], x[1]), Elem<T>::pack2(x[2], x[3])};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (f + e < D) out[f + e] = Elem<T>::down(x[e]);
            }
        }
}

// ------------------------------------------------------------------ scores

// What a kernel is compiled for; calls without any of it take one that has none of it, which has registers to spare.
enum { kBias = 1, kCap = 2, kDocuments = 4 };

struct AttentionParams {
    int32_t B, H, Hk, N, M, D;
    int32_t loaded;             // D rounded up to whole chunks, where D does not fill them
    int32_t buckets, table_type, causal;
    int32_t offset, prefix;
    float scale, scale2, unscale;  // of the products; times log2(e); 1 over it
    float cap, cap_in, cap_out; // 0: no cap; scale / cap; cap log2(e)
    const void *q, *k, *v, *table, *dout;
    void *out, *dq, *dk, *dv;
    float *lse;                 // [B, H, N]
    const int32_t *offsets, *prefixes, *row_len, *col_len, *row_document, *col_document;
    int64_t q_stride[4], k_stride[4], v_stride[4], out_stride[4], dout_stride[4], dq_stride[4], dk_stride[4], dv_stride[4];
    int64_t table_stride[2];
    // how the work is split
    int32_t row_tiles, key_tiles, splits, parts, table_columns;
    int32_t together;           // the rows' kernel sums delta up itself, in a walk over the keys before the one for gradients
    int32_t close;              // few keys: their gradients' weights to twice the type's digits
    int32_t near;               // diagonals of the neighbourhood that is laid out; 0: it is too wide
    float *part;                // [B, H, N, splits][D + 2]: unfinished sums, their reference and total
    float *delta;               // [B, H, N]
    float *key_part;            // [parts][2][B, Hk, M, D]: parts of dk and dv
    float *table_part;          // [H, buckets][B * row_tiles]
    float *dtable;              // [H, buckets]
};

template <typename T> __device__ __forceinline__ Rows<T> rows_of(const void *base, const int64_t (&stride)[4], int b, int h)
{
    return {static_cast<const T *>(base) + b * stride[0] + h * stride[1], stride[2]};
}
template <typename T> __device__ __forceinline__ T *row_of(void *base, const int64_t (&stride)[4], int b, int h, int64_t i)
{
    return static_cast<T *>(base) + b * stride[0] + h * stride[1] + i * stride[2];
}

// The workgroup's tile and unit (head of a sequence): all units' first tiles come first, so that those with the most work begin early, and
// where eight divides their number a unit's tiles are on one XCD (workgroups go round the eight of them), neighbouring units too.
struct Place {
    int tile, unit;
    __device__ __forceinline__ explicit Place(int units)
    {
        const int x = blockIdx.x;
        tile = x / units;
        unit = x - tile * units;
        if (units % 8 == 0) unit = unit % 8 * (units / 8) + unit / 8;
    }
};

// What a sequence's rows see: row i the keys below limit(i) (of its document).
struct Sight {
    int rows, keys, offset, prefix, causal;
    __device__ __forceinline__ Sight(const AttentionParams &p, int b)
    {
        rows = clamp_len(p.row_len, b, p.N);
        keys = clamp_len(p.col_len, b, p.M);
        // (|j - i| is below 2^28 and max_distance at most 2^24: beyond 2^29 nothing changes)
        offset = p.offsets ? min(max(p.offsets[b], -(1 << 29)), 1 << 29) : p.offset;
        prefix = p.prefixes ? p.prefixes[b] : p.prefix;
        causal = p.causal;
    }
    __device__ __forceinline__ int limit(int i) const { return causal ? min(keys, max(i + offset + 1, prefix)) : keys; }
    // the first row that sees key j, if any does
    __device__ __forceinline__ int first_row(int j) const { return causal && j >= prefix ? max(0, j - offset) : 0; }
};

// tanh from an exponential; for small arguments, where that cancels, Lambert's continued fraction to its fifth denominator (off by
// 3e-11 of the value at 0.5).  One division serves both.
__device__ __forceinline__ float tanh_fast(float x)
{
    const float y = fminf(fmaxf(x, -20.0f), 20.0f), z = y * y;  // (1 to the last bit from there on)
    const float e = exp2_fast(2.0f * kLog2e * y);
    const bool small = fabsf(y) < 0.5f;
    const float above = small ? y * fmaf(z + 105.0f, z, 945.0f) : e - 1.0f;
    const float below = small ? fmaf(fmaf(15.0f, z, 420.0f), z, 945.0f) : e + 1.0f;
    return x != x ? x : above * __builtin_amdgcn_rcpf(below);
}

// s = out tanh(in s).  Scores rarely come near their cap: where all of a wavefront's are below half of it, tanh(x) / x is a polynomial in x^2
// (interpolated at the Chebyshev nodes of [0, 1/4]; off by 1.4e-8, in float32 by 6e-8), which takes a third of the time.
__device__ __forceinline__ void cap_scores(Acc &s, float in, float out)
{
    float top = fabsf(s[0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, fabsf(s[r]));
    if (__all(top * in < 0.5f)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float x = s[r] * in, z = x * x;
            float y = fmaf(z, 0.017131344428621548f, -0.05298423882762508f);
            y = fmaf(y, z, 0.13324750504782334f);
            y = fmaf(y, z, -0.33333067944422656f);
            y = fmaf(y, z, 0.9999999867573899f);
            s[r] = out * x * y;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = out * tanh_fast(s[r] * in);
    }
}

// An entry times `unit`, which is at most 2^26; one below -1e30 forbids its cells, as -inf does, and one above 2^100 counts as that, so
// that the product stays finite.  NaN stays NaN.
__device__ __forceinline__ float entry_of(float v, float unit) { return v < -1e30f ? -INFINITY : (v > 0x1p100f ? 0x1p100f : v) * unit; }

// Diagonals kept on each side of those that are not all in one bucket: a tile of 64 x 32 cells that touches these reaches over by 94.
constexpr int kBiasMargin = 95;

// The bias of tiles of 32 x 32 cells.  Far from the diagonal it is one number.  Near it, cells take it from `at`, by their diagonal: of the
// whole neighbourhood, which is laid out once where that is small, else of the tile's 63 diagonals.  All of it by LDS addresses: a
// pointer that may be one of two would be read as memory, and wait for the tiles that are being copied.
struct WaveBias {
    uint32_t values;       // the head's entries
    const int32_t *starts;
    uint32_t near;         // the entry of j - i - offset = 0, and of its neighbours around it
    uint32_t near_bucket;
    bool have_near;
    float *diagonal;       // 64 of the wavefront's own
    uint8_t *bucket;       // 64 of the wavefront's own
    int last;              // first distance of a side's last bucket
    float one;             // the bias of all cells, where it is the same
    int one_bucket;
    bool same;
    uint32_t at;           // else: of the tile's lowest diagonal and those above it
    uint32_t at_bucket;
    // whether all cells with lowest <= j - i - offset <= highest are in the last bucket of their side (or in the one of all later keys)
    __device__ __forceinline__ bool far(const BucketRule &rule, int lowest, int highest)
    {
        const int before = highest <= -last ? rule.n - 1 : -1, behind = rule.two_sided ? (lowest >= last ? 2 * rule.n - 1 : -1) : lowest >= 0 ? 0 : -1;
        one_bucket = max(before, behind);
        same = one_bucket >= 0;
        if (same) one = lds_read<float>(values + 4 * (uint32_t)one_bucket, 0);
        return same;
    }
    // `lowest`: j - i - offset on the lowest of the diagonals
    __device__ __forceinline__ void look(const BucketRule &rule, int lowest, int lane)
    {
        if (far(rule, lowest, lowest + 62)) return;
        if (have_near) {
            at = near + 4 * (uint32_t)lowest;
            at_bucket = near_bucket + (uint32_t)lowest;
            return;
        }
        at = lds_address(reinterpret_cast<char *>(diagonal));
        at_bucket = lds_address(reinterpret_cast<char *>(bucket));
        const int u = rule.bucket(lowest + min(lane, 62), starts);
        wavefront_order();
        diagonal[lane] = lds_read<float>(values + 4 * (uint32_t)u, 0);
        bucket[lane] = (uint8_t)u;
        wavefront_order();
    }
    // The bias of 32 keys (registers) and 32 rows (columns).
    __device__ __forceinline__ Acc of_rows(int lane) const
    {
        if (same) return Acc{} + one;
        const uint32_t from = at + 4 * (uint32_t)(31 - (lane & 31) + 4 * (lane >> 5));
        Acc s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = lds_read<float>(from, 4 * tile_row(r, 0));
        return s;
    }
    // Adds it ...
    __device__ __forceinline__ void add_to_rows(Acc &s, int lane) const
    {
        if (same) {
            s += one;
            return;
        }
        const uint32_t from = at + 4 * (uint32_t)(31 - (lane & 31) + 4 * (lane >> 5));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] += lds_read<float>(from, 4 * tile_row(r, 0));
    }
    // ... or that of 32 rows (registers) and 32 keys (columns).
    __device__ __forceinline__ void add_to_keys(Acc &s, int lane) const
    {
        if (same) {
            s += one;
            return;
        }
        constexpr int kMost = tile_row(15, 0);
        const uint32_t from = at + 4 * (uint32_t)(31 + (lane & 31) - 4 * (lane >> 5) - kMost);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] += lds_read<float>(from, 4 * (kMost - tile_row(r, 0)));
    }
};

// LDS that the bias takes: 256 entries, the rule's starts, 64 diagonals (4 + 1 bytes) for each wavefront, and the neighbourhood.
constexpr int kBiasStarts = (kMaxBuckets / 2 + 1 + 3) / 4 * 4;
constexpr int bias_bytes(int waves, int near) { return kMaxBuckets * 4 + kBiasStarts * 4 + waves * 64 * 5 + (near + 3) / 4 * 4 * 5; }

// Lays the bias's part of LDS out and fills it with the entries times `unit`; a barrier has to follow.  The forward pass's
// products, unless they are capped, begin with the bias over the scale: in the matrix cores' accumulator it costs nothing more (68 to 62 us
// at 4 x 16 x 2048 x 2048 x 64 bfloat16 causal; the gradients' are slower so, 118 to 130).
__device__ __forceinline__ WaveBias begin_bias(const AttentionParams &p, const BucketRule &rule, float unit, char *lds, int h, int wave, int waves,
                                               int thread, int threads)
{
    float *values = reinterpret_cast<float *>(lds);
    int32_t *starts = reinterpret_cast<int32_t *>(values + kMaxBuckets);
    float *diagonal = reinterpret_cast<float *>(starts + kBiasStarts);
    float *near = diagonal + 64 * waves;
    uint8_t *near_bucket = reinterpret_cast<uint8_t *>(near + (p.near + 3) / 4 * 4);
    uint8_t *bucket = near_bucket + (p.near + 3) / 4 * 4;
    const int last = rule.first(rule.n - 1);
    if (p.buckets) {
        for (int u = thread; u < p.buckets; u += threads)
            values[u] = entry_of(load_typed(p.table, h * p.table_stride[0] + u * p.table_stride[1], p.table_type), unit);
        for (int k = thread; k <= rule.m; k += threads) starts[k] = rule.start[k];
        if (p.near) {
            __syncthreads();
            for (int d = thread; d < p.near; d += threads) {
                const int u = rule.bucket(d - last - kBiasMargin, starts);
                near[d] = values[u];
                near_bucket[d] = (uint8_t)u;
            }
        }
    }
    WaveBias b{};
    b.values = __builtin_amdgcn_readfirstlane(lds_address(reinterpret_cast<char *>(values)));
    b.starts = starts;
    b.have_near = p.near != 0;
    b.near = __builtin_amdgcn_readfirstlane(lds_address(reinterpret_cast<char *>(near + last + kBiasMargin)));
    b.near_bucket = __builtin_amdgcn_readfirstlane(lds_address(reinterpret_cast<char *>(near_bucket + last + kBiasMargin)));
    b.diagonal = diagonal + 64 * wave;
    b.bucket = bucket + 64 * wave;
    b.last = last;
    return b;
}

constexpr int kKeys = 64;  // keys of a tile in LDS

// A column's view of 32 positions that pass by: for the position of register r, whether it is below the column's limit and of its document.
// `documents`: those of the 32 positions, in LDS; `rest`: the column's limit less the first position less 4 half.
template <bool DOCUMENTS> struct Seen {
    bool at[16];
    __device__ __forceinline__ Seen(int rest, const int32_t *documents, int doc, int half)
    {
#pragma unroll
        for (int r = 0; r < 16; ++r) at[r] = tile_row(r, 0) < rest;
        if (DOCUMENTS) {
            typedef int32_t Four __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const Four d = *reinterpret_cast<const Four *>(documents + 8 * g + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) at[4 * g + e] = at[4 * g + e] && d[e] == doc;
            }
        }
    }
};

// The tiles of 64 keys (or rows) that a workgroup of 4 wavefronts walks through.  Where the sequence is packed from documents, those
// without one of the documents lowest .. highest are stepped over: found out for 256 tiles at a time.
template <bool DOCUMENTS> struct TileWalk {
    const int32_t *document;
    int keys, tiles, lowest, highest, batch;
    uint64_t *live;  // LDS, 4
    __device__ __forceinline__ int next(int t)  // the first tile from t on; `tiles` if there is none.  The same in all threads.
    {
        if (!DOCUMENTS || !document) return t;
        while (t < tiles) {
            if (t / 256 != batch) {
                batch = t / 256;
                const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, first = batch * 256 + wave * 64;
                uint64_t mine = 0;
#pragma unroll 8
                for (int k = 0; k < 64; ++k) {
                    const int j = (first + k) * 64 + lane;
                    const int d = j < keys ? document[j] : -1;
                    if (__any(d >= lowest && d <= highest)) mine |= (uint64_t)1 << k;
                }
                __syncthreads();
                if (lane == 0) live[wave] = mine;
                __syncthreads();
            }
            const uint64_t word = live[t % 256 / 64] >> (t % 64);
            if (word) return min(tiles, t + (int)__builtin_ctzll(word));
            t = (t / 64 + 1) * 64;
        }
        return tiles;
    }
};

struct PackParams {
    const void *in;
    void *out;
    int64_t stride[4], heads, rows, vectors;
    int32_t D, loaded;
};
// Rows of any strides into contiguous ones of whole chunks, zeros behind their D features.
template <typename U> __global__ __launch_bounds__(256) void attention_pack_kernel(PackParams p)
{
    constexpr int W = 16 / (int)sizeof(U);
    const int chunks = p.loaded / W;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < p.vectors; x += gridDim.x * (int64_t)256) {
        int64_t row = x / chunks;
        const int f = (int)(x - row * chunks) * W;
        const int64_t i = row % p.rows;
        row /= p.rows;
        const U *in = static_cast<const U *>(p.in) + row / p.heads * p.stride[0] + row % p.heads * p.stride[1] + i * p.stride[2];
        U v[W];
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = f + e < p.D ? in[(f + e) * p.stride[3]] : (U)0;
        Bits4 b;
        __builtin_memcpy(&b, v, 16);
        static_cast<Bits4 *>(p.out)[x] = b;
    }
}

}  // namespace sdtw
