// Softmax attention under a learned position bias, forward.
//
//   s[i,j] = cap tanh(scale <q_i, k_j> / cap) + table[h, bucket(j - i - offset)]  over the keys j that row i sees
//   out[i] = sum_j exp(s[i,j] - lse[i]) v_j,   lse[i] = log sum_j exp(s[i,j])
// in one pass over the keys: a running reference m, total l and unfinished sum o per row; with exponents in octaves
//   m' = max(m, max_j s),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j.
#pragma once
#include "attention_tiles.h"

namespace sdtw {

// A row's running softmax; its two lanes hold the same m and half of l each.
template <int DP> struct Running {
    float m, l;
    Acc o[DP / 32];
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int ft = 0; ft < DP / 32; ++ft) o[ft] = Acc{};
    }
    // takes scores in, and leaves 2^(s - m) in their place
    __device__ __forceinline__ void take(Acc &s)
    {
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = both_max(top);
        if (__any(top > m)) {
            const float to = fmaxf(m, top);
            const float factor = m == to ? 1.0f : exp2_fast(m - to);
            m = to;
            l *= factor;
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) o[ft] *= factor;
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = exp2_fast(s[r] - ref);
            sum += s[r];
        }
        l += sum;
    }
};

// 4 wavefronts of 32 * NT rows each, one head of one sequence.
template <typename T, int DP, int NT>
__global__ __launch_bounds__(256, 1) void attention_forward_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    extern __shared__ __align__(16) char lds[];
    __shared__ uint64_t live[4];
    __shared__ int shared[4][4];
    char *ktile = lds, *vtile = lds + Shape::bytes(kKeys);
    const int thread = threadIdx.x, wave = thread / 64, lane = thread % 64, c = lane % 32, half = lane / 32;
    int64_t id = neighbours_together();
    const int rt = p.row_tiles - 1 - (int)(id % p.row_tiles);  // (the last rows see the most keys of a causal sequence: they go first)
    id /= p.row_tiles;
    const int h = (int)(id % p.H), b = (int)(id / p.H), hk = h / (p.H / p.Hk);
    const Sight sight(p, b);
    const int32_t *col_document = p.col_document ? p.col_document + (int64_t)b * p.M : nullptr;
    WaveBias bias = begin_bias(p, rule, lds + 2 * Shape::bytes(kKeys), h, wave, 4, thread, 256);

    const int first_row = rt * 128 * NT + wave * 32 * NT;
    const Rows<T> q = rows_of<T>(p.q, p.q_stride, b, h);
    Column<T, DP> col[NT];
    int lim[NT], doc[NT];
    bool valid[NT];
    int from = 0x7fffffff, to = 0, low = 0x7fffffff, high = -1;  // limits and documents of the wavefront's rows
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int i = first_row + 32 * n + c;
        valid[n] = i < sight.rows;
        doc[n] = 0;
        if (p.row_document && valid[n]) {
            doc[n] = p.row_document[(int64_t)b * p.N + i];
            valid[n] = doc[n] >= 0;
        }
        lim[n] = valid[n] ? sight.limit(i) : 0;
        if (valid[n]) from = min(from, lim[n]), to = max(to, lim[n]), low = min(low, doc[n]), high = max(high, doc[n]);
        else lim[n] = 0x7fffffff;  // (what such a row computes is not looked at)
        col[n].load(q.base + i * q.row, q.feature, p.D, valid[n], half);
    }
    from = wave_min_i32(from), to = wave_max_i32(to), low = wave_min_i32(low), high = wave_max_i32(high);
    if (lane == 0) shared[wave][0] = to, shared[wave][1] = low, shared[wave][2] = high;
    __syncthreads();
    int end = 0, lowest = 0x7fffffff, highest = -1;
    for (int w = 0; w < 4; ++w) end = max(end, shared[w][0]), lowest = min(lowest, shared[w][1]), highest = max(highest, shared[w][2]);

    Running<DP> run[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) run[n].clear();
    const Rows<T> k = rows_of<T>(p.k, p.k_stride, b, hk), v = rows_of<T>(p.v, p.v_stride, b, hk);
    TileWalk walk{col_document, end, (end + kKeys - 1) / kKeys, lowest, highest, -1, live};
    Stage<T, DP, kKeys, 256> ks, vs;
    int t = walk.next(0);
    if (t < walk.tiles) {
        ks.load(k, p.D, t * kKeys, end, col_document, thread);
        vs.load(v, p.D, t * kKeys, end, col_document, thread);
    }
    while (t < walk.tiles) {
        __syncthreads();
        ks.store(ktile, thread);
        vs.store(vtile, thread);
        __syncthreads();
        const int now = t;
        t = walk.next(t + 1);
        if (t < walk.tiles) {
            ks.load(k, p.D, t * kKeys, end, col_document, thread);
            vs.load(v, p.D, t * kKeys, end, col_document, thread);
        }
#pragma unroll
        for (int sub = 0; sub < kKeys / 32; ++sub) {
            const int j0 = now * kKeys + sub * 32;
            if (j0 >= to) break;
            bool open = j0 + 32 <= from;  // every row sees all of these keys
            int key_doc = -1;
            if (col_document) {
                key_doc = j0 + c < end ? col_document[j0 + c] : -1;
                open = open && low == high && __all(key_doc == low);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Acc s = along_features<T, DP>(ktile + Shape::bytes(sub * 32), col[n], lane);
                scale_scores(s, p);
                if (p.buckets) {
                    const int i0 = first_row + 32 * n;
                    bias.look(rule, j0 - (i0 + 31) - sight.offset, lane);
                    if (bias.same) {
                        s += bias.one;
                    } else {
                        const float *at = bias.diagonal + 31 - c + 4 * half;
#pragma unroll
                        for (int r = 0; r < 16; ++r) s[r] += at[tile_row(r, 0)];
                    }
                }
                if (!open) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (j0 + tile_row(r, half) >= lim[n]) s[r] = -INFINITY;
                    if (col_document) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (__shfl(key_doc, tile_row(r, half)) != doc[n]) s[r] = -INFINITY;
                    }
                }
                run[n].take(s);
                along_rows<T, DP>(run[n].o, vtile + Shape::bytes(sub * 32), Weights<T>(s), lane);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int i = first_row + 32 * n + c;
        const float total = both_sum(run[n].l);
        const bool some = valid[n] && total != 0.0f;  // (a NaN is something)
        if (i >= p.N) continue;
        const float factor = some ? 1.0f / total : 0.0f;
        if (!some) {
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) run[n].o[ft] = Acc{};
        }
        store_column<T, DP>(row_of<T>(p.out, p.out_stride, b, h, i), p.D, run[n].o, factor, half);
        if (half == 0) p.lse[((int64_t)b * p.H + h) * p.N + i] = some ? (run[n].m + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
    }
}

// A few rows against many keys.  The rows of a group of heads that share their keys stand in one wavefront's columns together: row t is
// query t / G of head t % G of the group.  Each of 4 wavefronts takes every fourth 32 keys of the workgroup's share, on its own; then
// they are joined in LDS, and the workgroups of a row by attention_join_kernel.
template <typename T, int DP>
__global__ __launch_bounds__(256, 1) void attention_few_rows_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    extern __shared__ __align__(16) char lds[];
    __shared__ float ref[4][32], tot[4][32];
    const int thread = threadIdx.x, wave = thread / 64, lane = thread % 64, c = lane % 32, half = lane / 32;
    char *ktile = lds + wave * 2 * Shape::bytes(32), *vtile = ktile + Shape::bytes(32);
    int64_t id = neighbours_together();
    const int split = (int)(id % p.splits);
    id /= p.splits;
    const int rt = (int)(id % p.row_tiles);
    id /= p.row_tiles;
    const int hk = (int)(id % p.Hk), b = (int)(id / p.Hk), G = p.H / p.Hk;
    const Sight sight(p, b);
    const int32_t *col_document = p.col_document ? p.col_document + (int64_t)b * p.M : nullptr;
    const int row = rt * 32 + c, i = row / G, h = hk * G + row % G;
    bool valid = i < sight.rows;
    int doc = 0;
    if (p.row_document && valid) {
        doc = p.row_document[(int64_t)b * p.N + i];
        valid = doc >= 0;
    }
    int lim = valid ? sight.limit(i) : 0;
    const int to = wave_max_i32(lim);
    if (!valid) lim = 0x7fffffff;
    const int from = wave_min_i32(lim);
    Column<T, DP> col;
    {
        const Rows<T> q = rows_of<T>(p.q, p.q_stride, b, valid ? h : 0);
        col.load(q.base + (valid ? i : 0) * q.row, q.feature, p.D, valid, half);
    }
    // the entries of every head that is here, and the rule's starts
    float *values = reinterpret_cast<float *>(lds + 8 * Shape::bytes(32));
    int32_t *starts = reinterpret_cast<int32_t *>(values + min(G, 32) * p.buckets);
    const int first_head = G <= 32 ? 0 : rt * 32 % G;  // (the heads of 32 rows of a larger group follow each other, round its end)
    if (p.buckets) {
        for (int u = thread; u < min(G, 32) * p.buckets; u += 256) {
            const int head = hk * G + (first_head + u / p.buckets) % G;
            values[u] = octaves_of_entry(load_typed(p.table, head * p.table_stride[0] + u % p.buckets * p.table_stride[1], p.table_type));
        }
        for (int u = thread; u <= rule.m; u += 256) starts[u] = rule.start[u];
        __syncthreads();
    }
    const float *mine = values + ((row % G - first_head + G) % G) * p.buckets;

    // the workgroup's tiles of 128 keys
    const int tiles = (to + 127) / 128, each = (tiles + p.splits - 1) / p.splits;
    const int begin = min(tiles, split * each), end = min(tiles, begin + each);
    const Rows<T> k = rows_of<T>(p.k, p.k_stride, b, hk), v = rows_of<T>(p.v, p.v_stride, b, hk);
    Running<DP> run;
    run.clear();
    Stage<T, DP, 32, 64> ks, vs;
    if (begin < end) {
        ks.load(k, p.D, begin * 128 + wave * 32, to, col_document, lane);
        vs.load(v, p.D, begin * 128 + wave * 32, to, col_document, lane);
    }
    for (int t = begin; t < end; ++t) {
        const int j0 = t * 128 + wave * 32;
        wavefront_order();
        ks.store(ktile, lane);
        vs.store(vtile, lane);
        wavefront_order();
        if (t + 1 < end) {
            ks.load(k, p.D, j0 + 128, to, col_document, lane);
            vs.load(v, p.D, j0 + 128, to, col_document, lane);
        }
        if (j0 >= to) continue;
        Acc s = along_features<T, DP>(ktile, col, lane);
        scale_scores(s, p);
        if (p.buckets) {
            const int near = j0 - i - sight.offset;
            const int u0 = rule.bucket(near, starts), u1 = rule.bucket(near + 31, starts);
            if (__all(u0 == u1 && (near > 0 || near + 31 <= 0))) {
                s += mine[u0];
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] += mine[rule.bucket(near + tile_row(r, half), starts)];
            }
        }
        if (j0 + 32 > from) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (j0 + tile_row(r, half) >= lim) s[r] = -INFINITY;
        }
        if (col_document) {
            const int key_doc = j0 + c < to ? col_document[j0 + c] : -1;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (__shfl(key_doc, tile_row(r, half)) != doc) s[r] = -INFINITY;
        }
        run.take(s);
        along_rows<T, DP>(run.o, vtile, Weights<T>(s), lane);
    }
    const float total = both_sum(run.l);
    if (half == 0) ref[wave][c] = run.m, tot[wave][c] = total;
    __syncthreads();  // (the tiles are not read any more either)
    float m = ref[0][c];
    for (int w = 1; w < 4; ++w) m = fmaxf(m, ref[w][c]);
    const float factor = run.m == m ? 1.0f : exp2_fast(run.m - m);
    // [4][32][DP + 4]: rows of a wavefront's sums, a column each
    float *sums = reinterpret_cast<float *>(lds);
    constexpr int kRow = DP + 4;
#pragma unroll
    for (int ft = 0; ft < DP / 32; ++ft)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const Acc &o = run.o[ft];
            *reinterpret_cast<float4 *>(sums + (wave * 32 + c) * kRow + 32 * ft + 8 * g + 4 * half) =
                float4{o[4 * g] * factor, o[4 * g + 1] * factor, o[4 * g + 2] * factor, o[4 * g + 3] * factor};
        }
    __syncthreads();
    const int rows = min(32, p.N * G - rt * 32);
    for (int x = thread; x < 32 * DP; x += 256) {
        const int r = x / DP, f = x % DP;
        if (r >= rows || f >= p.D) continue;
        const int t = rt * 32 + r, ri = t / G, rh = hk * G + t % G;
        const int64_t place = ((int64_t)b * p.H + rh) * p.N + ri;
        float top = ref[0][r], all = 0.0f, sum = 0.0f;
        for (int w = 1; w < 4; ++w) top = fmaxf(top, ref[w][r]);
        for (int w = 0; w < 4; ++w) {
            all += tot[w][r] * (ref[w][r] == top ? 1.0f : exp2_fast(ref[w][r] - top));
            sum += sums[(w * 32 + r) * kRow + f];
        }
        if (p.splits == 1) {
            const bool seen = ri < sight.rows && !(p.row_document && p.row_document[(int64_t)b * p.N + ri] < 0) && all != 0.0f;
            row_of<T>(p.out, p.out_stride, b, rh, ri)[f] = Elem<T>::down(seen ? sum / all : 0.0f);
            if (f == 0) p.lse[place] = seen ? (top + __builtin_amdgcn_logf(all)) * kLn2 : -INFINITY;
        } else {
            float *part = p.part + (place * p.splits + split) * (p.D + 2);
            part[f] = sum;
            if (f == 0) part[p.D] = top, part[p.D + 1] = all;
        }
    }
}

// A row's parts joined, in their order: a workgroup of 128 threads for each row.
template <typename T> __global__ __launch_bounds__(128) void attention_join_kernel(AttentionParams p)
{
    __shared__ float factor[1024];
    const int64_t place = blockIdx.x;
    const int i = (int)(place % p.N), h = (int)(place / p.N % p.H), b = (int)(place / p.N / p.H);
    const float *part = p.part + place * p.splits * (p.D + 2);
    const Sight sight(p, b);
    const bool valid = i < sight.rows && !(p.row_document && p.row_document[(int64_t)b * p.N + i] < 0);
    float top = -INFINITY, all = 0.0f;
    for (int s = 0; s < p.splits; ++s) top = fmaxf(top, part[s * (p.D + 2) + p.D]);
    for (int s = threadIdx.x; s < p.splits; s += 128) {
        const float m = part[s * (p.D + 2) + p.D];
        factor[s] = m == top ? 1.0f : exp2_fast(m - top);
    }
    __syncthreads();
    for (int s = 0; s < p.splits; ++s) all += part[s * (p.D + 2) + p.D + 1] * factor[s];
    const bool seen = valid && all != 0.0f;
    for (int f = threadIdx.x; f < p.D; f += 128) {
        float sum = 0.0f;
        for (int s = 0; s < p.splits; ++s) sum += part[s * (p.D + 2) + f] * factor[s];
        row_of<T>(p.out, p.out_stride, b, h, i)[f] = Elem<T>::down(seen ? sum / all : 0.0f);
    }
    if (threadIdx.x == 0) p.lse[place] = seen ? (top + __builtin_amdgcn_logf(all)) * kLn2 : -INFINITY;
}

}  // namespace sdtw
