// A learned relative position bias by buckets on planes [B, H, N, M], and the gradient of its table.
//
// The bias depends on the diagonal j - i alone.  Forward: a tile's diagonals are looked up once, into LDS, and
// every row of the tile reads the same values one place further left.  Backward: a wavefront walks down a strip of
// neighbouring diagonals - 8 rows and 8 columns further with every step - so that a diagonal's sum stays in one
// register the whole way and the memory is read in whole aligned-as-it-comes vectors; buckets come in at the end.
#pragma once
#include "vector_io.h"

namespace sdtw {

constexpr int kMaxBuckets = 256;

// The buckets of a side: distances below e one by one, bucket e + k from start[k] on.
struct BucketRule {
    int32_t n, e, m, two_sided;
    int32_t start[kMaxBuckets / 2];
    __device__ __forceinline__ int side(int d) const
    {
        if (d < e) return d;
        int b = e - 1;
        for (int k = 0; k < m; ++k) b += d >= start[k];
        return b;
    }
    __device__ __forceinline__ int bucket(int r) const
    {
        if (two_sided) return side(r < 0 ? -r : r) + (r > 0 ? n : 0);
        return side(r < 0 ? -r : 0);
    }
    // first distance of bucket u of a side; of bucket n: beyond every distance
    __device__ __forceinline__ int first(int u) const { return u < e ? u : (u < n ? start[u - e] : 0x7fffffff); }
};

struct BiasParams {
    int32_t B, H, N, M, buckets, table_type;
    int32_t penalty;  // negative table entries count as 0
    int64_t offset;
    int64_t in_stride[3], out_stride[3], table_stride[2];
    const void *table, *in;
    void *out;
    const int32_t *offsets, *row_len, *col_len;
    const float *scale;    // [B], or [B, H] with scale_heads
    int32_t scale_heads;
    float *dtable;
    // forward: tiles of (256 / ty * width) columns and ty * 8 rows
    int32_t tx, col_tiles, row_tiles;
    // backward: strips of diagonals, parts of the batch, parts of the way down
    int32_t strips, first_col, batch_parts, batch_per_part, step_parts, steps_per_part, parts;
    double *partial;  // [H][buckets][parts]
};

constexpr int kBiasRows = 8;

__device__ __forceinline__ int clamp_len(const int32_t *len, int b, int full) { return len ? min(max(len[b], 0), full) : full; }

// a position difference as 32 bits: beyond 2^30 every distance is in the last bucket
__device__ __forceinline__ int clamp_rel(int64_t r) { return (int)min(max(r, (int64_t) - (1 << 30)), (int64_t)1 << 30); }

__device__ __forceinline__ float load_bias(const BiasParams &p, int h, int u)
{
    const float v = load_typed(p.table, h * p.table_stride[0] + u * p.table_stride[1], p.table_type);
    return p.penalty && v < 0.0f ? 0.0f : v;
}

template <typename T>
__global__ __launch_bounds__(256) void position_bias_forward_kernel(BiasParams p, BucketRule rule)
{
    constexpr int W = Elem<T>::kWidth, R = kBiasRows;
    extern __shared__ __align__(16) unsigned char lds[];
    float *diag = reinterpret_cast<float *>(lds);  // [rows + cols - 1] of the tile
    int64_t id = blockIdx.x;
    const int ct = (int)(id % p.col_tiles);
    id /= p.col_tiles;
    const int rt = (int)(id % p.row_tiles);
    id /= p.row_tiles;
    const int h = (int)(id % p.H), b = (int)(id / p.H);
    const int ty = 256 / p.tx, cols = p.tx * W, rows = ty * R;
    const int j0 = ct * cols, i0 = rt * rows;
    const int64_t offset = p.offsets ? (int64_t)p.offsets[b] : p.offset;
    const int rlen = clamp_len(p.row_len, b, p.N), clen = clamp_len(p.col_len, b, p.M);
    // diag[q] is the bias at j - i = j0 - (i0 + rows - 1) + q
    const int nd = min(cols, p.M - j0) + rows - 1;
    for (int q = threadIdx.x; q < nd; q += 256) {
        const int u = rule.bucket(clamp_rel((int64_t)j0 - (i0 + rows - 1) + q - offset));
        diag[q] = load_bias(p, h, u);
    }
    __syncthreads();
    const int x = threadIdx.x % p.tx, y = threadIdx.x / p.tx;
    const int j = j0 + x * W, i = i0 + y * R;
    if (j >= p.M || i >= p.N) return;
    const T *in = p.in ? static_cast<const T *>(p.in) + b * p.in_stride[0] + h * p.in_stride[1] : nullptr;
    T *out = static_cast<T *>(p.out) + b * p.out_stride[0] + h * p.out_stride[1];
    const float *mine = diag + x * W + (rows - 1 - y * R);  // mine[w - k]: row i + k, column j + w
    const int nr = min(R, p.N - i);
    if (j + W <= p.M) {
        Bits4 v[R] = {};
        if (in)
#pragma unroll
            for (int k = 0; k < R; ++k) v[k] = load_vec<true>(in + (int64_t)(i + min(k, nr - 1)) * p.in_stride[2] + j);
        float d[W + R - 1];
#pragma unroll
        for (int q = 0; q < W + R - 1; ++q) d[q] = mine[q - (R - 1)];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k >= nr) break;
            float sum[W];
#pragma unroll
            for (int w = 0; w < W; ++w) sum[w] = Elem<T>::at(v[k], w) + d[w - k + R - 1];
            Bits4 o = Elem<T>::pack(sum);
            if (i + k >= rlen || j + W > clen) {
#pragma unroll
                for (int w = 0; w < W; ++w)
                    if (i + k >= rlen || j + w >= clen) Elem<T>::copy(o, w, v[k]);
            }
            store_vec<false>(out + (int64_t)(i + k) * p.out_stride[2] + j, o);
        }
    } else {
        for (int k = 0; k < nr; ++k)
            for (int w = 0; j + w < p.M; ++w) {
                T v = in ? in[(int64_t)(i + k) * p.in_stride[2] + j + w] : T{};
                if (i + k < rlen && j + w < clen) v = Elem<T>::down(Elem<T>::up(v) + mine[w - k]);
                out[(int64_t)(i + k) * p.out_stride[2] + j + w] = v;
            }
    }
}

// One strip of 64 * W + 7 diagonals, one part of the batch, one part of the way down, four wavefronts in turn.
// Step s covers rows 8 s .. 8 s + 7; lane l reads W columns from base + 8 s + W l on, so that element (a, w) of its
// patch lies on diagonal j - i = base + W l + w - a whatever s is: W + 7 sums per lane.  They are carried in float32 over
// at most 16 steps (128 terms) and in float64 beyond.
template <typename T>
__global__ __launch_bounds__(256) void position_bias_backward_kernel(BiasParams p, BucketRule rule)
{
    constexpr int W = Elem<T>::kWidth, R = kBiasRows, A = W + R - 1, Q = 64 * W + R - 1;
    __shared__ double diag[4][Q];
    __shared__ double bucket_sum[kMaxBuckets];
    int64_t id = blockIdx.x;
    const int strip = (int)(id % p.strips);
    id /= p.strips;
    const int sp = (int)(id % p.step_parts);
    id /= p.step_parts;
    const int bp = (int)(id % p.batch_parts), h = (int)(id / p.batch_parts);
    const int part = (bp * p.step_parts + sp) * p.strips + strip;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t base = p.first_col + (int64_t)strip * (64 * W);
    const int b0 = bp * p.batch_per_part, b1 = min(p.B, b0 + p.batch_per_part);
    for (int u = threadIdx.x; u < p.buckets; u += 256) bucket_sum[u] = 0.0;
    double acc[A];
#pragma unroll
    for (int k = 0; k < A; ++k) acc[k] = 0.0;
    auto to_buckets = [&](int64_t offset) {
        // the lanes' sums by diagonal: W of them at a time, which are W different places in every lane
        for (int q = lane; q < Q; q += 64) diag[wave][q] = 0.0;
        __syncthreads();
#pragma unroll
        for (int k0 = 0; k0 < A; k0 += W) {
#pragma unroll
            for (int k = k0; k < k0 + W && k < A; ++k) diag[wave][W * lane + k] += acc[k];
            __syncthreads();
        }
        // diagonal q is r = lowest + q; a bucket's are neighbours
        const int64_t lowest = base - (R - 1) - offset;
        for (int u = wave; u < p.buckets; u += 4) {
            const bool right = rule.two_sided && u >= rule.n;
            const int64_t d0 = rule.first(right ? u - rule.n : u), d1 = (int64_t)rule.first((right ? u - rule.n : u) + 1) - 1;
            int64_t lo, hi;
            if (right) {
                lo = max(d0, (int64_t)1);
                hi = d1 >= 0x7ffffffe ? (int64_t)1 << 62 : d1;
            } else {
                hi = !rule.two_sided && u == 0 ? (int64_t)1 << 62 : -d0;
                lo = d1 >= 0x7ffffffe ? -((int64_t)1 << 62) : -d1;
            }
            const int64_t qa = max(lo - lowest, (int64_t)0), qb = min(hi - lowest, (int64_t)Q - 1);
            if (qa > qb) continue;
            double s = 0.0;
            for (int q = (int)qa + lane; q <= (int)qb; q += 64) s += (diag[0][q] + diag[1][q]) + (diag[2][q] + diag[3][q]);
            s = wave_sum_f64(s);
            if (lane == 0) bucket_sum[u] += s;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < A; ++k) acc[k] = 0.0;
    };
    for (int b = b0; b < b1; ++b) {
        const int rlen = clamp_len(p.row_len, b, p.N), clen = clamp_len(p.col_len, b, p.M);
        const T *g = static_cast<const T *>(p.in) + b * p.in_stride[0] + h * p.in_stride[1];
        const double scale = p.scale ? (double)p.scale[p.scale_heads ? (int64_t)b * p.H + h : b] : 1.0;
        // the steps at which the strip touches the columns [0, clen) and the rows [0, rlen)
        const int64_t from = max((int64_t)sp * p.steps_per_part, base + 64 * W >= 0 ? (int64_t)0 : (-base - 64 * W) / 8);
        const int64_t past_cols = clen - base <= 0 ? 0 : (clen - base + 7) / 8;
        const int64_t to = min(min((int64_t)(sp + 1) * p.steps_per_part, (int64_t)((rlen + 7) / 8)), past_cols);
        float f[A];
#pragma unroll
        for (int k = 0; k < A; ++k) f[k] = 0.0f;
        int held = 0;
        for (int64_t s = from + wave; s < to; s += 4) {
            const int i = (int)(8 * s);
            const int64_t j = base + 8 * s + W * lane;
            if (j + W > 0 && j < clen) {
                if (j >= 0 && j + W <= clen && i + R <= rlen) {
                    Bits4 v[R];
#pragma unroll
                    for (int a = 0; a < R; ++a) v[a] = load_vec<true>(g + (int64_t)(i + a) * p.in_stride[2] + j);
#pragma unroll
                    for (int a = 0; a < R; ++a)
#pragma unroll
                        for (int w = 0; w < W; ++w) f[w - a + R - 1] += Elem<T>::at(v[a], w);
                } else {
#pragma unroll
                    for (int a = 0; a < R; ++a)
#pragma unroll
                        for (int w = 0; w < W; ++w)
                            if (i + a < rlen && j + w >= 0 && j + w < clen)
                                f[w - a + R - 1] += Elem<T>::up(g[(int64_t)(i + a) * p.in_stride[2] + j + w]);
                }
            }
            if (++held == 16) {
#pragma unroll
                for (int k = 0; k < A; ++k) {
                    acc[k] += scale * (double)f[k];
                    f[k] = 0.0f;
                }
                held = 0;
            }
        }
#pragma unroll
        for (int k = 0; k < A; ++k) acc[k] += scale * (double)f[k];
        if (p.offsets) to_buckets((int64_t)p.offsets[b]);  // (every sequence has its own diagonals' buckets)
    }
    __syncthreads();
    if (!p.offsets) to_buckets(p.offset);
    for (int u = threadIdx.x; u < p.buckets; u += 256) p.partial[((int64_t)h * p.buckets + u) * p.parts + part] = bucket_sum[u];
}

// dtable[h,u]: the parts in a fixed order.  With a table (a penalty) its negative entries, which count as 0, get 0.
__global__ __launch_bounds__(256) void position_bias_table_kernel(BiasParams p)
{
    __shared__ double sums[4];
    const double *src = p.partial + (int64_t)blockIdx.x * p.parts;
    double s = 0.0;
    for (int i = threadIdx.x; i < p.parts; i += 256) s += src[i];
    s = wave_sum_f64(s);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const int h = blockIdx.x / p.buckets, u = blockIdx.x % p.buckets;
        const bool off = p.table && load_typed(p.table, h * p.table_stride[0] + u * p.table_stride[1], p.table_type) < 0.0f;
        p.dtable[blockIdx.x] = off ? 0.0f : (float)((sums[0] + sums[1]) + (sums[2] + sums[3]));
    }
}

}  // namespace sdtw
