// Softmax attention under a learned position bias, forward.
//
//   s[i,j] = cap tanh(scale <q_i, k_j> / cap) + table[h, bucket(j - i - offset)]  over the keys j that row i sees
//   out[i] = sum_j exp(s[i,j] - lse[i]) v_j,   lse[i] = log sum_j exp(s[i,j])
// in one pass over the keys: a running reference m, total l and unfinished sum o per row; with exponents in octaves
//   m' = max(m, max_j s),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  o' = o 2^(m - m') + sum_j 2^(s_j - m') v_j.
// Scores and their exponentials never leave registers: 32 rows stand in a wavefront's columns, 64 keys at a time come through LDS, copied
// there directly; the next tile is asked for before this one is worked on, and waited for before its first product (see copies_done).
// What bounds it: at D = 64 the vector units, which take 32 exponents, maxima, sums and conversions a lane for each tile and are busy 77 % of the
// time (4 x 16 x 2048 x 2048 bfloat16 causal with bias 54 to 60 us, 573 to 638 TFLOP/s with the skipped half not counted; without mask and bias 89
// us, 775 TFLOP/s); at D = 128 they and the matrix cores in turn, and the wait for tiles (152 us, 902 TFLOP/s, where a large library product
// reaches 1250; capped, with documents, vector units 51 % and matrix cores 21 %).  float32: the matrix cores (332 us at D = 64, 104
// TFLOP/s of a library product's 153).
// Tried: no maximum taken within a tile (77 us for 62 then: scalar registers spilled); three wavefronts a SIMD instead of four (slower).
#pragma once
#include "attention_tiles.h"

namespace sdtw {

// A row's running softmax; its two lanes hold the same m and half of l each.  m follows the largest score only where that is ahead by
// more than 8 octaves: the sums' scale does not matter within float32's range, and rescaling them for every new maximum
// would cost as much as a tenth of the work.
template <int DP> struct Running {
    static constexpr float kAhead = 8.0f;
    float m, l;
    bool far;  // some reference of the wavefront's is so large that its rounding would show in an exponent
    Acc o[DP / 32];
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY;
        far = false;
        l = 0.0f;
#pragma unroll
        for (int ft = 0; ft < DP / 32; ++ft) o[ft] = Acc{};
    }
    // a new largest score
    __device__ __forceinline__ void raise(float top)
    {
        if (__any(top > m + kAhead)) {
            const float to = fmaxf(m, top);
            const float factor = m == to ? 1.0f : exp2_fast(m - to);
            m = to;
            far = far || __any(fabsf(m) > 65536.0f && fabsf(m) < INFINITY);
            l *= factor;
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) o[ft] *= factor;
        }
    }
    // Takes in scores of SUBS * 32 keys and leaves 2^(score - m) in their place.  The scores are s * factor + add.
    template <int SUBS> __device__ __forceinline__ void take(Acc (&s)[SUBS], float factor, float add)
    {
        float top[SUBS];
#pragma unroll
        for (int x = 0; x < SUBS; ++x) {
            top[x] = fmaxf(s[x][0], s[x][1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) top[x] = fmaxf(fmaxf(s[x][r], s[x][r + 1]), top[x]);
        }
        raise(fmaf(both_max(SUBS == 2 ? fmaxf(top[0], top[SUBS - 1]) : top[0]), factor, add));
        if (far) {  // then scores are rounded as their maximum was, before it is subtracted
#pragma unroll
            for (int x = 0; x < SUBS; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[x][r] = fmaf(s[x][r], factor, add);
            factor = 1.0f;
            add = 0.0f;
        }
        const float from = add - (m == -INFINITY ? 0.0f : m);
        float sum[2] = {};
#pragma unroll
        for (int x = 0; x < SUBS; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[x][r] = exp2_fast(fmaf(s[x][r], factor, from));
                sum[r & 1] += s[x][r];
            }
        l += sum[0] + sum[1];
    }
};

// Wavefronts on a SIMD that registers are kept for.
template <typename T, int DP, int F>
constexpr int kForwardWaves = (sizeof(T) == 4 ? (DP <= 32 ? 4 : DP <= 64 ? 3 : 1) : DP <= 64 ? 4 : DP <= 96 ? 3 : 2) - (F & kCap && DP <= 96 ? 1 : 0);

// 4 wavefronts of 32 rows each, one head of one sequence.
template <typename T, int DP, int F>
__global__ __launch_bounds__(256, (kForwardWaves<T, DP, F>)) void attention_forward_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    constexpr int SUBS = kKeys / 32;
    constexpr bool BIAS = F & kBias, CAP = F & kCap, DOCUMENTS = F & kDocuments;
    extern __shared__ __align__(256) char lds[];
    __shared__ uint64_t live[4];
    __shared__ int shared[4][4];
    __shared__ __align__(16) int32_t documents[2][kKeys];
    constexpr int kTile = Shape::bytes(kKeys);  // (two tiles of keys, then two of values: one is read while the other is filled)
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread / 64), lane = thread % 64, c = lane % 32, half = lane / 32;
    const Place place(p.B * p.H);
    const int rt = p.row_tiles - 1 - place.tile;  // (the last rows see the most keys of a causal sequence)
    const int h = place.unit % p.H, b = place.unit / p.H, hk = h / (p.H / p.Hk);
    const Sight sight(p, b);
    const int32_t *col_document = DOCUMENTS && p.col_document ? p.col_document + (int64_t)b * p.M : nullptr;

    const int first_row = rt * 128 + wave * 32, i = first_row + c;
    bool valid = i < sight.rows;
    int doc = 0;
    if (DOCUMENTS && p.row_document && valid) {
        doc = p.row_document[(int64_t)b * p.N + i];
        valid = doc >= 0;
    }
    int lim = valid ? sight.limit(i) : 0;
    const int to = wave_max_i32(lim);
    if (!valid) lim = 0x7fffffff;  // (what such a row computes is not looked at)
    const int from = wave_min_i32(lim);  // every row sees the keys below it
    const int low = wave_min_i32(valid ? doc : 0x7fffffff), high = wave_max_i32(valid ? doc : -1);
    Column<T, DP> col;
    {
        const Rows<T> q = rows_of<T>(p.q, p.q_stride, b, h);
        col.load(q.base + i * q.row, p.loaded, valid, half);
    }
    if (lane == 0) shared[wave][0] = to, shared[wave][1] = low, shared[wave][2] = high;
    __syncthreads();
    int end = 0, lowest = 0x7fffffff, highest = -1;
    for (int w = 0; w < 4; ++w) end = max(end, shared[w][0]), lowest = min(lowest, shared[w][1]), highest = max(highest, shared[w][2]);
    end = __builtin_amdgcn_readfirstlane(end);

    TileWalk<DOCUMENTS> walk{col_document, end, (end + kKeys - 1) / kKeys, lowest, highest, -1, live};
    Stage<T, DP, kKeys, 256> ks, vs;
    ks.begin(rows_of<T>(p.k, p.k_stride, b, hk), p.loaded, thread);
    vs.begin(rows_of<T>(p.v, p.v_stride, b, hk), p.loaded, thread);
    const float scale2 = p.scale2, cap_out = p.cap_out;
    const bool fold = !CAP || cap_out == 0.0f;  // the bias comes in with the products
    const int base = first_row + 31 + sight.offset;  // j less this: the lowest diagonal of the wavefront's rows
    auto fetch = [&](int t, int buffer) {
        ks.copy(lds + buffer * kTile, t * kKeys, end, thread);
        vs.copy(lds + (2 + buffer) * kTile, t * kKeys, end, thread);
        if (DOCUMENTS && thread < kKeys)
            documents[buffer][thread] = t * kKeys + thread >= end ? -1 : col_document ? col_document[t * kKeys + thread] : 0;
    };
    int t = walk.next(0), buffer = 0;
    if (t < walk.tiles) fetch(t, 0);
    WaveBias bias;  // (laid out while the first tile is on its way)
    if (BIAS) bias = begin_bias(p, rule, fold ? p.unscale : kLog2e, lds + 4 * kTile, h, wave, 4, thread, 256);
    Running<DP> run;
    run.clear();
    while (t < walk.tiles) {
        const int j0 = t * kKeys;
        char *const ktile = lds + buffer * kTile, *const vtile = lds + (2 + buffer) * kTile;
        const int32_t *const document = documents[buffer];
        copies_done();
        __syncthreads();
        if (DOCUMENTS && __any(document[lane] < 0)) {  // (the same in all wavefronts)
            clear_rows<T, DP, kKeys, 256>(ktile, document, thread);
            clear_rows<T, DP, kKeys, 256>(vtile, document, thread);
            __syncthreads();
        }
        t = walk.next(t + 1);
        buffer ^= 1;
        if (t < walk.tiles) fetch(t, buffer);
        if (j0 < to) {
            Acc s[SUBS];
            bool open = j0 + kKeys <= from;
            if (DOCUMENTS) open = open && low == high && __all(document[lane] == low);
            // The scores are the products times a number, plus a number; or made so, by 1 and 0.
            float factor = scale2, add = 0.0f;
            if (BIAS && fold && !bias.far(rule, j0 - base, j0 - base + 94)) {
#pragma unroll
                for (int x = 0; x < SUBS; ++x) {
                    bias.look(rule, j0 + 32 * x - base, lane);
                    s[x] = bias.of_rows(lane);
                }
            } else {
#pragma unroll
                for (int x = 0; x < SUBS; ++x) s[x] = Acc{};
                if (BIAS && fold) add = bias.one * scale2;
            }
#pragma unroll
            for (int x = 0; x < SUBS; ++x) s[x] = along_features<T, DP>(ktile + Shape::bytes(x * 32), col, lane, s[x]);
            if (CAP && !fold) {
                factor = 1.0f;
#pragma unroll
                for (int x = 0; x < SUBS; ++x) {
                    cap_scores(s[x], p.cap_in, cap_out);
                    if (BIAS) {
                        bias.look(rule, j0 + 32 * x - base, lane);
                        bias.add_to_rows(s[x], lane);
                    }
                }
            }
            if (!open) {
#pragma unroll
                for (int x = 0; x < SUBS; ++x) {
                    const Seen<DOCUMENTS> seen(lim - j0 - 32 * x - 4 * half, document + 32 * x, doc, half);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[x][r] = seen.at[r] ? s[x][r] : -INFINITY;
                }
            }
            run.take(s, factor, add);
#pragma unroll
            for (int x = 0; x < SUBS; ++x) along_rows<T, DP>(run.o, vtile + Shape::bytes(x * 32), Weights<T>(s[x]), lane);
        }
    }
    const float total = both_sum(run.l);
    const bool some = valid && total != 0.0f;  // (a NaN is something)
    if (i >= p.N) return;
    if (!some) {
#pragma unroll
        for (int ft = 0; ft < DP / 32; ++ft) run.o[ft] = Acc{};
    }
    store_column<T, DP>(row_of<T>(p.out, p.out_stride, b, h, i), p.D, run.o, some ? 1.0f / total : 0.0f, half);
    if (half == 0) p.lse[((int64_t)b * p.H + h) * p.N + i] = some ? (run.m + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
}

// LDS of the kernel below: its wavefronts' tiles, or their sums, [4][32][DP + 4].
template <typename T, int DP> constexpr int few_rows_bytes()
{
    const int tiles = 4 * 2 * TileShape<T, DP>::bytes(32), sums = 4 * 32 * (DP + 4) * 4;
    return tiles > sums ? tiles : sums;
}

// A few rows against many keys.  The rows of a group of heads that share their keys stand in one wavefront's columns together: row t is
// query t / G of head t % G of the group.  Each of 4 wavefronts takes every fourth 32 keys of the workgroup's share, on its own; then
// they are joined in LDS, and the workgroups of a row by attention_join_kernel.
// What bounds it: reading the keys and values.  32 x 16 heads in groups of 4, one row each, 4097 keys of 128 bfloat16: 165 MB in 33 us, 4.9 TB/s,
// where a copy of 1 GiB reaches 5.1 both ways; in float32 336 MB in 129, 2.6 TB/s, at one wavefront a SIMD.  131072 float16 keys, 4 rows: 268 MB
// in 54 us capped and 52 as they are.
template <typename T, int DP, int F>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attention_few_rows_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    constexpr bool BIAS = F & kBias, CAP = F & kCap, DOCUMENTS = F & kDocuments;
    extern __shared__ __align__(256) char lds[];
    __shared__ float ref[4][32], tot[4][32];
    __shared__ __align__(16) int32_t documents[4][32];
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread / 64), lane = thread % 64, c = lane % 32, half = lane / 32;
    constexpr int kTile = Shape::bytes(32);
    char *const ktile = lds + wave * 2 * kTile, *const vtile = ktile + kTile;
    int64_t id = neighbours_together();
    const int split = (int)(id % p.splits);
    id /= p.splits;
    const int rt = (int)(id % p.row_tiles);
    id /= p.row_tiles;
    const int hk = (int)(id % p.Hk), b = (int)(id / p.Hk), G = p.H / p.Hk;
    const Sight sight(p, b);
    const int32_t *col_document = DOCUMENTS && p.col_document ? p.col_document + (int64_t)b * p.M : nullptr;
    const int row = rt * 32 + c, i = row / G, h = hk * G + row % G;
    bool valid = i < sight.rows;
    int doc = 0;
    if (DOCUMENTS && p.row_document && valid) {
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
        col.load(q.base + (valid ? i : 0) * q.row, p.loaded, valid, half);
    }
    // the workgroup's tiles of 128 keys
    const int tiles = (to + 127) / 128, each = (tiles + p.splits - 1) / p.splits;
    const int begin = min(tiles, split * each), end = min(tiles, begin + each);
    Running<DP> run;
    run.clear();
    Stage<T, DP, 32, 64> ks, vs;
    ks.begin(rows_of<T>(p.k, p.k_stride, b, hk), p.loaded, lane);
    vs.begin(rows_of<T>(p.v, p.v_stride, b, hk), p.loaded, lane);
    // The next keys are asked for as soon as the products with these are done, the next values likewise.  (Before the first product with keys
    // all that was asked for is waited for, see copies_done: from there to the next request nothing is on its way.)
    auto fetch_keys = [&](int t) { if (t < end && t * 128 + wave * 32 < to) ks.copy(ktile, t * 128 + wave * 32, to, lane); };
    auto fetch_values = [&](int t) { if (t < end && t * 128 + wave * 32 < to) vs.copy(vtile, t * 128 + wave * 32, to, lane); };
    fetch_keys(begin);
    fetch_values(begin);
    // the entries of every head that is here, and the rule's starts
    float *values = reinterpret_cast<float *>(lds + few_rows_bytes<T, DP>());
    int32_t *starts = reinterpret_cast<int32_t *>(values + min(G, 32) * p.buckets);
    uint8_t *near = reinterpret_cast<uint8_t *>(starts + kBiasStarts);  // the buckets of the diagonals around 0
    const int last = rule.first(rule.n - 1);
    const int first_head = G <= 32 ? 0 : rt * 32 % G;  // (the heads of 32 rows of a larger group follow each other, round its end)
    if (BIAS) {
        for (int u = thread; u < min(G, 32) * p.buckets; u += 256) {
            const int head = hk * G + (first_head + u / p.buckets) % G;
            values[u] = entry_of(load_typed(p.table, head * p.table_stride[0] + u % p.buckets * p.table_stride[1], p.table_type), kLog2e);
        }
        for (int u = thread; u <= rule.m; u += 256) starts[u] = rule.start[u];
        __syncthreads();
        for (int d = thread; d < p.near; d += 256) near[d] = (uint8_t)rule.bucket(d - last - kBiasMargin, starts);
        if (p.near) __syncthreads();
    }
    const float *const mine = values + ((row % G - first_head + G) % G) * p.buckets;
    // (beyond the neighbourhood all is as on its edge)
    auto bucket = [&](int r) { return p.near ? (int)near[min(max(r + last + kBiasMargin, 0), p.near - 1)] : rule.bucket(r, starts); };

    for (int t = begin; t < end; ++t) {
        const int j0 = t * 128 + wave * 32;
        if (j0 >= to) break;
        int doc_here = 0;
        if (DOCUMENTS) {
            doc_here = j0 + c >= to ? -1 : col_document ? col_document[j0 + c] : 0;
            if (half == 0) documents[wave][c] = doc_here;
            copies_done();
            if (__any(doc_here < 0)) {
                clear_rows<T, DP, 32, 64>(ktile, documents[wave], lane);
                clear_rows<T, DP, 32, 64>(vtile, documents[wave], lane);
            }
            wavefront_order();
        } else {
            copies_left<decltype(vs)::kEach>();  // (the values may still be on their way)
        }
        Acc scores[1] = {along_features<T, DP>(ktile, col, lane)};
        Acc &s = scores[0];
        reads_done();
        fetch_keys(t + 1);
        if (CAP && p.cap_out != 0.0f) cap_scores(s, p.cap_in, p.cap_out);
        else s *= p.scale2;
        if (BIAS) {
            const int first = j0 - i - sight.offset, u0 = bucket(first), u1 = bucket(first + 31);
            if (__all(u0 == u1 && (first > 0 || first + 31 <= 0))) {
                s += mine[u0];
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] += mine[bucket(first + tile_row(r, half))];
            }
        }
        if (DOCUMENTS || j0 + 32 > from) {
            const Seen<DOCUMENTS> seen(lim - j0 - 4 * half, documents[wave], doc, half);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = seen.at[r] ? s[r] : -INFINITY;
        }
        run.take(scores, 1.0f, 0.0f);
        if (t + 1 < end && j0 + 128 < to) copies_left<decltype(ks)::kEach>();
        else copies_left<0>();
        along_rows<T, DP>(run.o, vtile, Weights<T>(s), lane);
        reads_done();
        fetch_values(t + 1);
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

// A row's parts joined, in one order: a workgroup of 256 threads for each row.  (512 rows of 4 parts 4.0 us, 128 rows of 128 parts 6.5: a
// launch and three dependent reads.)
template <typename T> __global__ __launch_bounds__(256) void attention_join_kernel(AttentionParams p)
{
    __shared__ float factor[1024], sums[256];
    __shared__ float best[4];
    const int64_t place = blockIdx.x;
    const int thread = threadIdx.x, i = (int)(place % p.N), h = (int)(place / p.N % p.H), b = (int)(place / p.N / p.H);
    const int pitch = p.D + 2;
    const float *part = p.part + place * p.splits * pitch;
    const Sight sight(p, b);
    const bool valid = i < sight.rows && !(p.row_document && p.row_document[(int64_t)b * p.N + i] < 0);
    float top = -INFINITY;
    for (int s = thread; s < p.splits; s += 256) {
        factor[s] = part[s * pitch + p.D];
        top = fmaxf(top, factor[s]);
    }
    top = wave_max_all_f32(top);
    if (thread % 64 == 0) best[thread / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
    float all = 0.0f;
    for (int s = thread; s < p.splits; s += 256) {
        const float m = factor[s];
        factor[s] = m == top ? 1.0f : exp2_fast(m - top);
        all = fmaf(part[s * pitch + p.D + 1], factor[s], all);
    }
    all = wave_sum_all_f32(all);
    __syncthreads();
    if (thread % 64 == 0) best[thread / 64] = all;
    __syncthreads();
    all = (best[0] + best[1]) + (best[2] + best[3]);
    const bool seen = valid && all != 0.0f;
    // `groups` threads for each feature
    const int wide = p.D <= 32 ? 32 : p.D <= 64 ? 64 : 128, groups = 256 / wide, f = thread % wide;
    float sum = 0.0f;
    if (f < p.D) {
#pragma unroll 8
        for (int s = thread / wide; s < p.splits; s += groups) sum = fmaf(part[s * pitch + f], factor[s], sum);
    }
    sums[thread] = sum;
    __syncthreads();
    if (thread < p.D) {
        sum = sums[thread];
        for (int g = 1; g < groups; ++g) sum += sums[thread + g * wide];
        row_of<T>(p.out, p.out_stride, b, h, i)[thread] = Elem<T>::down(seen ? sum / all : 0.0f);
    }
    if (thread == 0) p.lse[place] = seen ? (top + __builtin_amdgcn_logf(all)) * kLn2 : -INFINITY;
}

}  // namespace sdtw
