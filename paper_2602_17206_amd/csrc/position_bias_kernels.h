// A learned relative position bias by buckets on planes [B, H, N, M], and the gradient of its table.
//
// The bias depends on the diagonal j - i alone.  Forward: a tile's diagonals are looked up once, into LDS, and
// every row of the tile reads the same values one place further left.  Backward: the plane is read once in tiles of whole
// cache lines and summed up by diagonals; buckets, which are runs of neighbouring diagonals, come in at the end.
#pragma once
#include "vector_io.h"

#include <type_traits>

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

struct BiasParams {
    int32_t B, H, N, M, buckets, table_type;
    int32_t penalty;  // negative table entries count as 0, infinite ones as kForbidden
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
    // backward: tiles of `across` times 64 * width columns and 4 / across times wave_rows rows (col_tiles as above), parts of the batch
    int32_t wave_rows, tiles, across, batch_parts, batch_per_part, parts;
    double *partial;  // [H][buckets][parts]
};

constexpr int kBiasRows = 8;

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

// A penalty's entry of +inf forbids its cells: the sweeps take that as a cost of 3e38, as outside a band, and subtract costs.
constexpr float kForbidden = 3.0e38f;
__device__ __forceinline__ float load_bias(const BiasParams &p, int h, int u)
{
    const float v = load_typed(p.table, h * p.table_stride[0] + u * p.table_stride[1], p.table_type);
    if (!p.penalty) return v;
    return v < 0.0f ? 0.0f : v > kForbidden ? kForbidden : v;
}

// Bound by reading and writing the plane: 8 x 16 x 2048 x 2048 bfloat16 takes 357 us (6.0 TB/s both ways together), 8 x 16 x 1100 x
// 936 float16 82, with 937 columns, whose rows begin and end inside vectors, 103; a single row, 32 x 16 x 1 x 4097 bfloat16,
// 10 us, bound by the way from table to LDS to row.  STREAM_IN, STREAM_OUT: past the caches.
template <typename T, bool STREAM_IN, bool STREAM_OUT>
__global__ __launch_bounds__(256) void position_bias_forward_kernel(BiasParams p, BucketRule rule)
{
    constexpr int W = Elem<T>::kWidth, R = kBiasRows;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ int32_t starts[kMaxBuckets / 2 + 1];
    __shared__ float values[kMaxBuckets];
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
    for (int u = threadIdx.x; u < p.buckets; u += 256) values[u] = load_bias(p, h, u);
    for (int k = threadIdx.x; k <= rule.m; k += 256) starts[k] = rule.start[k];
    __syncthreads();
    // diag[q] is the bias at j - i = j0 - (i0 + rows - 1) + q
    const int nd = min(cols, p.M - j0) + rows - 1;
    for (int q = rows - min(rows, p.N - i0) + threadIdx.x; q < nd; q += 256)
        diag[q] = values[rule.bucket(clamp_rel((int64_t)j0 - (i0 + rows - 1) + q - offset), starts)];
    __syncthreads();
    const int x = threadIdx.x % p.tx, y = threadIdx.x / p.tx;
    const int j = j0 + x * W, i = i0 + y * R, nr = min(R, p.N - i);
    if (j >= p.M || i >= p.N) return;
    const T *in = p.in ? static_cast<const T *>(p.in) + b * p.in_stride[0] + h * p.in_stride[1] : nullptr;
    // (a vector that hangs over the row's end is read further in, and shifted: what it saw of its neighbours goes out)
    Bits4 v[R] = {};
    const int jc = min(j, p.M - W);
    if (in && jc >= 0)
#pragma unroll
        for (int k = 0; k < R; ++k) v[k] = load_vec<STREAM_IN>(in + (int64_t)(i + min(k, nr - 1)) * p.in_stride[2] + jc);
    T *out = static_cast<T *>(p.out) + b * p.out_stride[0] + h * p.out_stride[1];
    const float *mine = diag + x * W + (rows - 1 - y * R);  // mine[w - k]: row i + k, column j + w
    auto patch = [&](auto whole) {
        if (!whole) {
#pragma unroll
            for (int k = 0; k < R; ++k) v[k] = shift_vec(v[k], (j - jc) * 8 * (int)sizeof(T));
        }
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
            T *to = out + (int64_t)(i + k) * p.out_stride[2] + j;
            if (whole) {
                store_vec<STREAM_OUT>(to, o);
            } else {
#pragma unroll
                for (int w = 0; w < W - 1; ++w)
                    if (j + w < p.M) to[w] = element<T>(o, w);
            }
        }
    };
    if (j + W <= p.M) {
        patch(std::true_type{});
    } else if (p.M >= W) {
        patch(std::false_type{});
    } else {
        for (int k = 0; k < nr; ++k)
            for (int w = 0; j + w < p.M; ++w) {
                T v = in ? in[(int64_t)(i + k) * p.in_stride[2] + j + w] : T{};
                if (i + k < rlen && j + w < clen) v = Elem<T>::down(Elem<T>::up(v) + mine[w - k]);
                out[(int64_t)(i + k) * p.out_stride[2] + j + w] = v;
            }
    }
}

// One tile of the plane, for a part of the batch.  A wavefront takes wave_rows (at most 64) rows of 64 * W columns, 8 rows at a time: lane l reads W
// columns of each (whole cache lines from row to row), and element (a, w) of its patch lies on diagonal w - a of it: W + 7 sums
// in registers.  The next 8 rows move every diagonal 8 places on, so 8 of the sums are complete and go to the wavefront's diagonals
// in LDS (different places in all lanes, W of them at a time), and the others stay.  Float32 up to there: at most 64 terms; what
// a pass leaves there is added up in float64, scaled, and the buckets - neighbouring diagonals - are summed at the end.
// Bound by reading the plane: 32 x 1 x 8192 x 8192 float32 takes 1.28 ms (6.7 TB/s), 4 x 16 x 2048 x 2048 bfloat16 85 us
// (6.3 TB/s).  4 x 1 x 64 x 64 float32 takes 9 us: a wavefront's steps, then its buckets.  A walk along the diagonals, whose sums stay in
// registers the whole way, took 1.46 ms and 127 us: its rows' loads begin one place further on from row to row, so hardly any of
// them is whole cache lines.
template <typename T>
__global__ __launch_bounds__(256) void position_bias_backward_kernel(BiasParams p, BucketRule rule)
{
    constexpr int W = Elem<T>::kWidth, R = kBiasRows, A = W + R - 1, Z = 64 + R - W, Q = 64 * W + Z;
    typedef float Float4 __attribute__((ext_vector_type(4)));
    __shared__ __align__(16) float pass_sum[4][Q];  // each wavefront's own
    __shared__ double diag[4][Q];
    __shared__ double bucket_sum[kMaxBuckets], narrow_sum[4][64];
    int64_t id = neighbours_together();
    const int tile = (int)(id % p.tiles);
    id /= p.tiles;
    const int bp = (int)(id % p.batch_parts), h = (int)(id / p.batch_parts);
    const int part = bp * p.tiles + tile;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    // the tile's four wavefronts: `across` side by side, the others below
    const int across = p.across, down = 4 / across;
    const auto row_of = [&](int w) { return (tile / p.col_tiles * down + w / across) * p.wave_rows; };
    const auto col_of = [&](int w) { return (tile % p.col_tiles * across + w % across) * (64 * W); };
    const int i0 = row_of(wave), j0 = col_of(wave), j = j0 + W * lane;
    const int b0 = bp * p.batch_per_part, b1 = min(p.B, b0 + p.batch_per_part);
    for (int u = threadIdx.x; u < p.buckets; u += 256) bucket_sum[u] = 0.0;
    for (int q = lane; q < Q; q += 64) {
        diag[wave][q] = 0.0;
        pass_sum[wave][q] = 0.0f;
    }
    wavefront_order();
    // place q of a wavefront's diagonals is the difference j - i = col - row - Z + q
    auto to_buckets = [&](int64_t offset) {
        __syncthreads();
        int64_t lowest = (int64_t)1 << 62, highest = -lowest;
        for (int w = 0; w < 4; ++w) {
            lowest = min(lowest, (int64_t)col_of(w) - row_of(w) - Z - offset);
            highest = max(highest, (int64_t)col_of(w) - row_of(w) - Z - offset + Q - 1);
        }
        for (int u0 = 0; u0 < p.buckets; u0 += 64) {
            // a bucket's differences lo .. hi are neighbours; lane l looks at bucket u0 + l
            const int u = u0 + lane;
            const bool right = rule.two_sided && u >= rule.n;
            const int side = right ? u - rule.n : u;
            int64_t lo = 1, hi = 0;
            if (u < p.buckets) {
                const int64_t d0 = rule.first(side), d1 = (int64_t)rule.first(side + 1) - 1, end = (int64_t)1 << 62;
                const bool open = d1 >= 0x7ffffffe;
                lo = right ? max(d0, (int64_t)1) : open ? -end : -d1;
                hi = right ? (open ? end : d1) : !rule.two_sided && u == 0 ? end : -d0;
            }
            lo = max(lo, lowest);
            hi = min(hi, highest);
            const int from = (int)(lo - lowest), to = (int)(hi - lowest);
            // of up to 8 diagonals: all at once, a lane each, over this wavefront's own place among the diagonals
            const bool narrow = lo <= hi && to - from < 8;
            double own = 0.0;
            if (__any(narrow)) {
                const int shift = (int)((int64_t)col_of(wave) - row_of(wave) - Z - offset - lowest);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int q = from + k - shift;
                    const double x = diag[wave][max(0, min(q, Q - 1))];
                    own += narrow && from + k <= to && q >= 0 && q < Q ? x : 0.0;
                }
                narrow_sum[wave][lane] = own;
            }
            __syncthreads();
            if (wave == 0 && narrow) bucket_sum[u] += (own + narrow_sum[1][lane]) + (narrow_sum[2][lane] + narrow_sum[3][lane]);
            unsigned long long some = __ballot(lo <= hi && !narrow);
            for (int turn = 0; some != 0; ++turn, some &= some - 1) {
                if ((turn & 3) != wave) continue;
                const int l = __builtin_ctzll(some);
                const int qa = __builtin_amdgcn_readlane(from, l), qb = __builtin_amdgcn_readlane(to, l);
                double s = 0.0;
                for (int w = 0; w < 4; ++w) {
                    const int shift = (int)((int64_t)col_of(w) - row_of(w) - Z - offset - lowest);
                    for (int q = max(qa - shift, 0) + lane; q <= min(qb - shift, Q - 1); q += 64) s += diag[w][q];
                }
                s = wave_sum_f64(s);
                if (lane == 0) bucket_sum[u0 + l] += s;
            }
            __syncthreads();
        }
        __syncthreads();
    };
    for (int b = b0; b < b1; ++b) {
        const int rlen = clamp_len(p.row_len, b, p.N), clen = clamp_len(p.col_len, b, p.M);
        const T *g = static_cast<const T *>(p.in) + b * p.in_stride[0] + h * p.in_stride[1];
        const double scale = p.scale ? (double)p.scale[p.scale_heads ? (int64_t)b * p.H + h : b] : 1.0;
        const int steps = j0 < clen ? min((rlen - i0 + R - 1) / R, p.wave_rows / R) : 0;
        // A vector that hangs over the row's end is read further in and shifted, zeros coming in (rows shorter than one: by element).
        const int jc = min(j, clen - W);
        float f[A];
#pragma unroll
        for (int k = 0; k < A; ++k) f[k] = 0.0f;
        float *sums = pass_sum[wave] + W * lane + (Z - R + W);  // (the last step's are at W * lane: none lie before the first)
        for (int s = 0; s <= steps; ++s, sums -= R) {
            if (s < steps) {
                const int i = i0 + R * s;
                Bits4 v[R];
                if (clen >= W) {
#pragma unroll
                    for (int a = 0; a < R; ++a) v[a] = load_vec<true>(g + (int64_t)min(i + a, rlen - 1) * p.in_stride[2] + jc);
                    if (j0 + 64 * W > clen) {
                        const int shift = min(j - jc, W) * 8 * (int)sizeof(T);
#pragma unroll
                        for (int a = 0; a < R; ++a) v[a] = shift < 128 ? shift_vec(v[a], shift) : Bits4{};
                    }
                    if (i + R > rlen) {
#pragma unroll
                        for (int a = 0; a < R; ++a)
                            if (i + a >= rlen) v[a] = Bits4{};
                    }
#pragma unroll
                    for (int a = 0; a < R; ++a)
#pragma unroll
                        for (int w = 0; w < W; ++w) f[w - a + R - 1] += Elem<T>::at(v[a], w);
                } else {
#pragma unroll
                    for (int a = 0; a < R; ++a)
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            const float x = Elem<T>::up(g[(int64_t)min(i + a, rlen - 1) * p.in_stride[2] + min(j + w, clen - 1)]);
                            f[w - a + R - 1] += i + a < rlen && j + w < clen ? x : 0.0f;
                        }
                }
            }
            // sums W - 1 .. W + 6 are complete; those below are W - 1 .. of the next rows' patch
            // (float4 at a time; with W = 4 the second four are the next lane's first ones, after it has stored them)
#pragma unroll
            for (int k0 = 0; k0 < R; k0 += 4) {
                Float4 *at = reinterpret_cast<Float4 *>(sums + k0);
                Float4 x = *at;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] += f[W - 1 + k0 + k];
                *at = x;
                wavefront_order();
            }
#pragma unroll
            for (int k = A - 1; k >= R; --k) f[k] = f[k - R];
#pragma unroll
            for (int k = 0; k < R; ++k) f[k] = 0.0f;
        }
        // The diagonals that have a cell; the others hold zeros still, and no weight is looked at for them (1 / 0 where a sequence is empty).
        const int nr = min(rlen - i0, p.wave_rows), nc = min(clen - j0, 64 * W);
        if (nr > 0 && nc > 0)
            for (int q = Z - nr + 1 + lane; q < Z + nc; q += 64) {
                diag[wave][q] += scale * (double)pass_sum[wave][q];
                pass_sum[wave][q] = 0.0f;
            }
        wavefront_order();
        if (p.offsets) {  // (every sequence has its own diagonals' buckets)
            to_buckets((int64_t)p.offsets[b]);
            for (int q = lane; q < Q; q += 64) diag[wave][q] = 0.0;
        }
    }
    if (!p.offsets) to_buckets(p.offset);
    for (int u = threadIdx.x; u < p.buckets; u += 256) p.partial[((int64_t)h * p.buckets + u) * p.parts + part] = bucket_sum[u];
}

// dtable[h,u]: the parts in a fixed order; 2 to 5 us.  With a table (a penalty) its negative entries, which count as 0, get 0.
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
