// Softmax attention under a learned position bias, backward.
//
// With p[i,j] = exp(s[i,j] - lse[i]), made again from the products, and dp[i,j] = <dout_i, v_j>:
//   delta[i] = sum_j p dp,   ds = p (dp - delta),   dtable[h,u] = sum of ds where bucket(j - i - offset) = u
//   dx = ds (1 - tanh^2) where scores are capped, else ds
//   dv_j = sum_i p dout_i,   dq_i = scale sum_j dx k_j,   dk_j = scale sum_i dx q_i   (the last two over a group's heads too)
// Two kernels, each the sole writer of what it sums: no atomics on memory, the same bits from the same inputs.
//   rows   wavefronts own queries and walk over the keys: delta, dq, dtable
//   keys   wavefronts own keys and walk over the queries of all heads of the group: dk, dv
// The products are made twice, which is 14 D operations a cell for the formula's 10 (18 D with delta's walk); one kernel that made them once
// would have to add dq up in memory, by atomics or by 32-bit parts of all keys.
// What bounds them: matrix cores and vector units in turn, at two wavefronts a SIMD, which is what registers leave, and in the keys' kernel
// the wait for tiles: the rows' lse and delta are read behind a tile's copies, and so waited for with them.  4 x 16 x 2048 x 2048 x 64
// bfloat16 causal with bias and its table: delta 58 us, rows 141 to 152, keys 120 to 128; 2 x 16 heads in groups of 4, 4096 x 4096 x 128
// causal with prefixes: rows 315 to 361 (matrix cores busy 55 % of the time), keys 348 to 421 (44 %), their parts added up 25.
// In float32 the kernels for rows and keys stand at one wavefront a SIMD: the first of these 352, 641 and 759 us, 49 of a library
// product's 153 TFLOP/s.
#pragma once
#include "attention_tiles.h"

namespace sdtw {

// Times 1 - tanh^2, where `capped` holds the capped scores and `inverse` is 1 over the cap; 0 without a cap.
__device__ __forceinline__ void through_cap(Acc &x, const Acc &capped, float inverse)
{
    const Acc t = capped * inverse;
    x = x - x * t * t;
}

// float16 has 30 octaves for numbers that may be of any size (gradients of a mean are small): a column's numbers go into the
// matrix cores times a power of two of the column's own, chosen from the first of them and made smaller whenever one would not fit.
template <typename T, int DP> struct ColumnScale {
    __device__ __forceinline__ void fit(Acc &, Acc (&)[DP / 32]) {}
    __device__ __forceinline__ float undo() const { return 1.0f; }
};
template <int DP> struct ColumnScale<_Float16, DP> {
    float by = 0.0f;  // 0: nothing but zeros so far
    __device__ __forceinline__ void fit(Acc &x, Acc (&sums)[DP / 32])
    {
        float top = fabsf(x[0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, fabsf(x[r]));
        top = both_max(top);
        const bool change = by == 0.0f ? top > 0.0f : top * by > 16384.0f;
        if (__any(change)) {
            if (change) {  // the largest to 8 .. 16: 10 octaves of room above, 17 below
                const int e = __builtin_amdgcn_frexp_expf(fminf(top, 1e38f));
                const float next = __builtin_amdgcn_ldexpf(1.0f, min(max(4 - e, -126), 126));
                const float factor = by == 0.0f ? 0.0f : next / by;
                by = next;
#pragma unroll
                for (int ft = 0; ft < DP / 32; ++ft) sums[ft] *= factor;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] *= by;
    }
    __device__ __forceinline__ float undo() const { return by == 0.0f ? 0.0f : 1.0f / by; }
};

// The table's gradient of a wavefront's 32 rows, in LDS: [buckets][columns].  Where all cells of a tile are in one bucket its sum stays in a
// register until the bucket changes.  Else the cells are added up by their diagonals first and then lane d adds diagonal d to its bucket,
// in a column that it shares with the lanes d' = d (modulo columns), taking turns: one order of additions, whatever happens.
// (LDS's own atomic additions are one instruction, but take 3 cycles a lane: 224 us against 99 without the table's gradient at
// 4 x 16 x 2048 x 2048 x 64 bfloat16 causal.)
struct TableSum {
    static constexpr int kPitch = 33, kTile = 32 * kPitch;
    float *sum;       // [buckets][columns]
    float *tile;      // [32 rows][kPitch]
    int columns, bucket;  // bucket: of `running`
    float running;
    __device__ __forceinline__ void turns(int lane, int u, float v)
    {
        for (int first = 0; first < 64; first += columns) {
            wavefront_order();
            if (lane >= first && lane < first + columns) sum[u * columns + lane - first] += v;
        }
        wavefront_order();
    }
    __device__ __forceinline__ void flush(int lane)
    {
        if (bucket >= 0) turns(lane, bucket, running);
        bucket = -1;
        running = 0.0f;
    }
    // ds of 32 keys and 32 rows; `buckets`: of the 63 diagonals key - row + 31, and one more, in LDS.  Lane l of a half walks over 16 keys t and
    // the rows (t + 31 - l) mod 32: diagonal l as far as t <= l, and diagonal l + 32 from there on.
    __device__ __forceinline__ void by_diagonals(const Acc &ds, int lane, uint32_t buckets)
    {
        const int l = lane & 31, half = lane >> 5;
        float *const to = tile + l * kPitch + 4 * half;
        wavefront_order();
#pragma unroll
        for (int r = 0; r < 16; ++r) to[tile_row(r, 0)] = ds[r];
        wavefront_order();
        const float *const low = tile + (31 - l) * kPitch + half * 16 * (kPitch + 1), *const high = low - kTile;
        const int turn = l - half * 16;  // the last key of diagonal l among this half's
        float first = 0.0f, all = 0.0f;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const float v = (t <= turn ? low : high)[t * (kPitch + 1)];
            all += v;
            first = t <= turn ? all : first;
        }
        const float mine = both_sum(first), next = both_sum(all - first);
        turns(lane, lds_read<uint8_t>(buckets + (uint32_t)lane, 0), half ? next : mine);
    }
};

// Both products of a tile before anything else, where there are registers for it: the matrix cores go on while the scores are worked on.
template <int DP> constexpr bool kEarly = DP < 128;

// Whether the rows' kernel can sum delta up itself (beyond that there are no registers for it).
template <int DP> constexpr bool kTogether = DP <= 96;

// Wavefronts on a SIMD that registers are kept for.
template <typename T, int DP> constexpr int kDeltaWaves = sizeof(T) == 4 ? (DP <= 32 ? 4 : DP <= 64 ? 2 : 1) : DP <= 64 ? 4 : 3;
template <typename T, int DP, bool MORE> constexpr int kBackwardWaves = sizeof(T) == 4 ? (DP <= 32 ? 2 : 1) : DP <= 32 ? 3 : DP <= 96 || !MORE ? 2 : 1;

// The weights of dq go into the matrix cores as two numbers, the second what the first was rounded off by: rows whose ds nearly cancel, as
// under long causal masks, would show one rounding to 8 bits (beyond 1.5 times the error of a chain in 32 bits).
//
// 4 wavefronts of 32 rows each, one head of one sequence.  delta comes from the rows' outputs - sum_j p dp = <dout, out> - unless the table's
// gradient is wanted: that is kept in 32 bits, and its sums over whole diagonals would show the rounding of a 16-bit `out`; then, and for
// 16-bit gradients over few keys, the keys are walked over once more beforehand, for delta alone.  (So is float32, whose `out` is not rounded:
// its table's gradient from <dout, out> has not been held against 64 bits.)
enum { kRowsPlain, kRowsDelta, kRowsTable, kRowsGiven };
template <typename T, int DP, int F, int WORK>
__global__ __launch_bounds__(256, (WORK == kRowsDelta ? kDeltaWaves<T, DP> : kBackwardWaves<T, DP, false>)) void attention_rows_gradient_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    constexpr bool TABLE = WORK == kRowsTable;
    constexpr bool BIAS = F & kBias, CAP = F & kCap, DOCUMENTS = F & kDocuments;
    extern __shared__ __align__(256) char lds[];
    __shared__ uint64_t live[4];
    __shared__ int shared[4][4];
    __shared__ __align__(16) int32_t documents[2][kKeys];
    constexpr int kTile = Shape::bytes(kKeys);
    constexpr int kBuffers = TABLE && kTile >= 16384 ? 1 : 2;  // (with one, two workgroups still fit into LDS beside the table's sums)
    // (16-bit results take exponents in octaves as they are; 32-bit ones want them rounded as late as can be)
    constexpr bool OCTAVES = sizeof(T) == 2 && (WORK == kRowsPlain || WORK == kRowsGiven);
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread / 64), lane = thread % 64, c = lane % 32, half = lane / 32;
    const Place at_work(p.B * p.H);
    const int rt = p.row_tiles - 1 - at_work.tile;  // (the last rows see the most keys of a causal sequence)
    const int h = at_work.unit % p.H, b = at_work.unit / p.H, hk = h / (p.H / p.Hk);
    const Sight sight(p, b);
    const int32_t *col_document = DOCUMENTS && p.col_document ? p.col_document + (int64_t)b * p.M : nullptr;
    const int table_columns = TABLE ? p.table_columns : 0;
    float *const table_sums = reinterpret_cast<float *>(lds + 2 * kBuffers * kTile + bias_bytes(4, p.near));
    TableSum table{table_sums + wave * p.buckets * table_columns, table_sums + 4 * p.buckets * table_columns + wave * TableSum::kTile, table_columns, -1, 0.0f};
    if (TABLE)
        for (int x = thread; x < 4 * p.buckets * table_columns; x += 256) table_sums[x] = 0.0f;

    const int first_row = rt * 128 + wave * 32, i = first_row + c;
    const int64_t place = ((int64_t)b * p.H + h) * p.N + i;
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
    const int low = wave_min_i32(valid ? doc : 0x7fffffff), high = wave_max_i32(valid ? doc : -1);
    // (a row that sees nothing has no p: 2^(score - inf))
    float lse = valid ? p.lse[place] : -INFINITY;
    lse = lse == -INFINITY ? INFINITY : OCTAVES ? lse * kLog2e : lse;
    Column<T, DP> q, dout;
    {
        const Rows<T> x = rows_of<T>(p.q, p.q_stride, b, h), y = rows_of<T>(p.dout, p.dout_stride, b, h);
        q.load(x.base + i * x.row, p.loaded, valid, half);
        dout.load(y.base + i * y.row, p.loaded, valid, half);
    }
    float delta = 0.0f;
    // With the delta that there is, a row's ds add up to what delta is off by: the kernel for the keys gets the better one.
    float rest = 0.0f;
    constexpr bool GIVEN = TABLE || WORK == kRowsGiven, BOTH = GIVEN && kTogether<DP>;
    bool summing = BOTH && p.together;  // this walk over the keys is for delta
    if (GIVEN && !summing && valid) delta = p.delta[place];
    if (WORK == kRowsPlain) {
        const Rows<T> x = rows_of<T>(p.out, p.out_stride, b, h);
        Column<T, DP> out;
        out.load(x.base + i * x.row, p.loaded, valid, half);
#pragma unroll
        for (int s = 0; s < Column<T, DP>::kSteps; ++s)
#pragma unroll
            for (int e = 0; e < Elem<T>::kWidth; ++e) delta = fmaf(Elem<T>::at(dout.v[s], e), Elem<T>::at(out.v[s], e), delta);
        delta = both_sum(delta);
    }
    if (lane == 0) shared[wave][0] = to, shared[wave][1] = low, shared[wave][2] = high;
    __syncthreads();
    int end = 0, lowest = 0x7fffffff, highest = -1;
    for (int w = 0; w < 4; ++w) end = max(end, shared[w][0]), lowest = min(lowest, shared[w][1]), highest = max(highest, shared[w][2]);

    Acc dq[DP / 32];
#pragma unroll
    for (int ft = 0; ft < DP / 32; ++ft) dq[ft] = Acc{};
    ColumnScale<T, DP> fit;
    const float cap = OCTAVES ? p.cap_out : p.cap, inverse_cap = CAP && cap != 0.0f ? 1.0f / cap : 0.0f, scale = OCTAVES ? p.scale2 : p.scale;
    TileWalk<DOCUMENTS> walk{col_document, end, (end + kKeys - 1) / kKeys, lowest, highest, -1, live};
    Stage<T, DP, kKeys, 256> ks, vs;
    const int base = first_row + 31 + sight.offset;  // j less this: the lowest diagonal of the wavefront's rows
    ks.begin(rows_of<T>(p.k, p.k_stride, b, hk), p.loaded, thread);
    vs.begin(rows_of<T>(p.v, p.v_stride, b, hk), p.loaded, thread);
    auto fetch = [&](int t, int buffer) {
        ks.copy(lds + buffer * kTile, t * kKeys, end, thread);
        vs.copy(lds + (kBuffers + buffer) * kTile, t * kKeys, end, thread);
        if (DOCUMENTS && thread < kKeys)
            documents[buffer][thread] = t * kKeys + thread >= end ? -1 : col_document ? col_document[t * kKeys + thread] : 0;
    };
    int t = walk.next(0), buffer = 0;
    if (kBuffers == 2 && t < walk.tiles) fetch(t, 0);
    WaveBias bias;
    if (BIAS) bias = begin_bias(p, rule, OCTAVES ? kLog2e : 1.0f, lds + 2 * kBuffers * kTile, h, wave, 4, thread, 256);
    while (t < walk.tiles) {
        const int first = t * kKeys;
        char *const ktile = lds + buffer * kTile, *const vtile = lds + (kBuffers + buffer) * kTile;
        const int32_t *const document = documents[buffer];
        if (kBuffers == 1) {
            __syncthreads();
            fetch(t, 0);
        }
        copies_done();
        __syncthreads();
        if (DOCUMENTS && __any(document[lane] < 0)) {
            clear_rows<T, DP, kKeys, 256>(ktile, document, thread);
            clear_rows<T, DP, kKeys, 256>(vtile, document, thread);
            __syncthreads();
        }
        t = walk.next(t + 1);
        const bool for_delta = summing;
        if (BOTH && summing && t >= walk.tiles) {
            summing = false;
            t = walk.next(0);
        }
        if (kBuffers == 2) {
            buffer ^= 1;
            if (t < walk.tiles) fetch(t, buffer);
        }
#pragma unroll 1
        for (int sub = 0; sub < kKeys / 32; ++sub) {
            const int j0 = first + sub * 32;
            const char *const kt = ktile + Shape::bytes(sub * 32), *const vt = vtile + Shape::bytes(sub * 32);
            if (j0 >= to) break;
            bool open = j0 + 32 <= from;
            if (DOCUMENTS) open = open && low == high && __all(document[sub * 32 + c] == low);
            Acc s = along_features<T, DP>(kt, q, lane), dp, capped;
            if (kEarly<DP>) dp = along_features<T, DP>(vt, dout, lane);
            if (CAP) {
                if (cap != 0.0f) cap_scores(s, p.cap_in, cap);
                else s *= scale;
                capped = s;
            }
            // (the difference first: what is left to round is small)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = CAP ? s[r] - lse : fmaf(s[r], scale, -lse);
            if (BIAS) {
                bias.look(rule, j0 - base, lane);
                bias.add_to_rows(s, lane);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = OCTAVES ? exp2_fast(s[r]) : exp2_fast(s[r] * kLog2e);
            if (!open) {
                const Seen<DOCUMENTS> seen(lim - j0 - 4 * half, document + sub * 32, doc, half);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = seen.at[r] ? s[r] : 0.0f;
            }
            if (!kEarly<DP>) dp = along_features<T, DP>(vt, dout, lane);
            if (WORK == kRowsDelta || (BOTH && for_delta)) {  // (a tile's sum first: hundreds of additions to one number would show)
                float sum = s[0] * dp[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) sum = fmaf(s[r], dp[r], sum);
                delta += sum;
                continue;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
            float sum = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) sum += s[r];
            if (WORK == kRowsPlain) rest += sum;
            if (TABLE) {
                if (bias.same) {
                    if (bias.one_bucket != table.bucket) {
                        table.flush(lane);
                        table.bucket = bias.one_bucket;
                    }
                    table.running += sum;
                } else {
                    table.by_diagonals(s, lane, bias.at_bucket);
                }
            }
            if (CAP) through_cap(s, capped, inverse_cap);
            fit.fit(s, dq);
            along_rows_twice<T, DP>(dq, kt, s, lane);
        }
        if (BOTH && for_delta && !summing) delta = both_sum(delta);
    }
    if (BOTH && p.together && half == 0 && i < p.N) p.delta[place] = delta;
    if (WORK == kRowsDelta) {
        delta = both_sum(delta);
        if (half == 0 && i < p.N) p.delta[place] = delta;
        return;
    }
    if (WORK == kRowsPlain) {
        rest = both_sum(rest);
        if (half == 0 && i < p.N) p.delta[place] = delta + rest;
    }
    if (i < p.N) {
        if (!valid) {
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) dq[ft] = Acc{};
        }
        store_column<T, DP>(row_of<T>(p.dq, p.dq_stride, b, h, i), p.D, dq, p.scale * fit.undo(), half);
    }
    if (TABLE) {
        table.flush(lane);
        __syncthreads();
        for (int u = thread; u < p.buckets; u += 256) {
            float sum = 0.0f;
            for (int w = 0; w < 4; ++w)
                for (int x = 0; x < table_columns; ++x) sum += table_sums[(w * p.buckets + u) * table_columns + (x + u) % table_columns];
            p.table_part[((int64_t)h * p.buckets + u) * ((int64_t)p.B * p.row_tiles) + (int64_t)b * p.row_tiles + rt] = sum;
        }
    }
}

// dtable [h][u] from its parts, in 64 bits and in a fixed order: a wavefront for each entry.
__global__ __launch_bounds__(64) void attention_table_kernel(AttentionParams p)
{
    const int64_t parts = (int64_t)p.B * p.row_tiles;
    const float *x = p.table_part + blockIdx.x * parts;
    double sum = 0.0;
    for (int64_t k = threadIdx.x; k < parts; k += 64) sum += x[k];
    sum = wave_sum_f64(sum);
    if (threadIdx.x == 0) p.dtable[blockIdx.x] = (float)sum;
}

// 4 wavefronts of 32 keys each, of one head of keys of one sequence; the queries of the group's heads go by in tiles of 64, or one part
// of them does: then attention_keys_join_kernel adds the parts up.
template <typename T, int DP, int F>
__global__ __launch_bounds__(256, (kBackwardWaves<T, DP, (F & kCap) != 0>)) void attention_keys_gradient_kernel(AttentionParams p, BucketRule rule)
{
    using Shape = TileShape<T, DP>;
    constexpr bool OCTAVES = sizeof(T) == 2;
    constexpr bool BIAS = F & kBias, CAP = F & kCap, DOCUMENTS = F & kDocuments;
    extern __shared__ __align__(256) char lds[];
    __shared__ uint64_t live[4];
    __shared__ int shared[4][4];
    __shared__ __align__(16) float row_lse[2][kKeys], row_delta[2][kKeys];
    __shared__ __align__(16) int32_t row_doc[2][kKeys];
    constexpr int kTile = Shape::bytes(kKeys);
    const int thread = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(thread / 64), lane = thread % 64, c = lane % 32, half = lane / 32;
    const Place at_work(p.B * p.Hk);
    const int kt = at_work.tile / p.parts, part = at_work.tile % p.parts;  // (the first keys are seen by the most rows of a causal sequence)
    const int hk = at_work.unit % p.Hk, b = at_work.unit / p.Hk, G = p.H / p.Hk;
    const Sight sight(p, b);
    const int32_t *row_document = DOCUMENTS && p.row_document ? p.row_document + (int64_t)b * p.N : nullptr;
    const int first_key = kt * 128 + wave * 32, j = first_key + c;
    bool valid = sight.rows > 0 && j < sight.limit(sight.rows - 1);  // (the last row sees the most; other keys may hold NaN)
    int doc = 0;
    if (DOCUMENTS && p.col_document && valid) {
        doc = p.col_document[(int64_t)b * p.M + j];
        valid = doc >= 0;
    }
    const int low = wave_min_i32(valid ? doc : 0x7fffffff), high = wave_max_i32(valid ? doc : -1);
    const bool any = __any(valid);
    Column<T, DP> k, v;
    {
        const Rows<T> x = rows_of<T>(p.k, p.k_stride, b, hk), y = rows_of<T>(p.v, p.v_stride, b, hk);
        k.load(x.base + j * x.row, p.loaded, valid, half);
        v.load(y.base + j * y.row, p.loaded, valid, half);
    }
    if (lane == 0) shared[wave][1] = low, shared[wave][2] = high, shared[wave][3] = any;
    __syncthreads();
    int lowest = 0x7fffffff, highest = -1, some = 0;
    for (int w = 0; w < 4; ++w) lowest = min(lowest, shared[w][1]), highest = max(highest, shared[w][2]), some |= shared[w][3];
    // rows that see one of the keys: from first_row(the first key) on, as limits rise with the rows
    const int begin = sight.first_row(kt * 128), mine = sight.first_row(first_key);
    const int end = some ? sight.rows : 0;
    Acc dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int ft = 0; ft < DP / 32; ++ft) dk[ft] = Acc{}, dv[ft] = Acc{};
    ColumnScale<T, DP> fit;
    const float cap = OCTAVES ? p.cap_out : p.cap, inverse_cap = CAP && cap != 0.0f ? 1.0f / cap : 0.0f, scale = OCTAVES ? p.scale2 : p.scale;
    constexpr float kWeight = std::is_same<T, _Float16>::value ? 16384.0f : 1.0f;  // p <= 1 (to rounding) into float16's upper octaves
    TileWalk<DOCUMENTS> walk{row_document, end, (end + kKeys - 1) / kKeys, lowest, highest, -1, live};
    Stage<T, DP, kKeys, 256> qs, ds;
    // tiles from_tile .. walk.tiles of each head, all heads' one after the other: this part's share of them
    const int from_tile = min(begin / kKeys, walk.tiles), each = walk.tiles - from_tile;
    const int64_t all = (int64_t)G * each;
    const int64_t share_begin = all * part / p.parts, share_end = all * (part + 1) / p.parts;
    const int first_head = each ? (int)(share_begin / each) : 0, last_head = each ? (int)((share_end + each - 1) / each) : 0;
#pragma unroll 1
    for (int g = first_head; g < last_head; ++g) {
        const int h = hk * G + g;
        const int first_tile = from_tile + (int)max(share_begin - (int64_t)g * each, (int64_t)0);
        walk.tiles = from_tile + (int)min(share_end - (int64_t)g * each, (int64_t)each);
        __syncthreads();
        const float *lse = p.lse + ((int64_t)b * p.H + h) * p.N, *delta = p.delta + ((int64_t)b * p.H + h) * p.N;
        qs.begin(rows_of<T>(p.q, p.q_stride, b, h), p.loaded, thread);
        ds.begin(rows_of<T>(p.dout, p.dout_stride, b, h), p.loaded, thread);
        auto fetch = [&](int t, int buffer) {
            qs.copy(lds + buffer * kTile, t * kKeys, end, thread);
            ds.copy(lds + (2 + buffer) * kTile, t * kKeys, end, thread);
            if (thread < kKeys) {
                const int i = t * kKeys + thread, d = i >= end ? -1 : row_document ? row_document[i] : 0;
                const float x = d >= 0 ? lse[i] : -INFINITY;
                row_doc[buffer][thread] = d;
                row_lse[buffer][thread] = x == -INFINITY ? INFINITY : OCTAVES ? x * kLog2e : x;
                row_delta[buffer][thread] = d >= 0 ? delta[i] : 0.0f;
            }
        };
        int t = walk.next(first_tile), buffer = 0;
        if (t < walk.tiles) fetch(t, 0);
        WaveBias bias;
        if (BIAS) bias = begin_bias(p, rule, OCTAVES ? kLog2e : 1.0f, lds + 4 * kTile, h, wave, 4, thread, 256);
        while (t < walk.tiles) {
            const int first = t * kKeys, now = buffer;
            char *const qtile = lds + buffer * kTile, *const dtile = lds + (2 + buffer) * kTile;
            copies_done();
            __syncthreads();
            if (DOCUMENTS && row_document && __any(row_doc[now][lane] < 0)) {
                clear_rows<T, DP, kKeys, 256>(qtile, row_doc[now], thread);
                clear_rows<T, DP, kKeys, 256>(dtile, row_doc[now], thread);
                __syncthreads();
            }
            t = walk.next(t + 1);
            buffer ^= 1;
            if (t < walk.tiles) fetch(t, buffer);
#pragma unroll 1
            for (int sub = 0; sub < kKeys / 32; ++sub) {
                const int i0 = first + sub * 32;
                const char *const qt = qtile + Shape::bytes(sub * 32), *const dt = dtile + Shape::bytes(sub * 32);
                if (i0 + 32 <= mine || i0 >= end || !any) continue;
                bool open = sight.limit(i0) >= min(first_key + 32, sight.keys);
                if (DOCUMENTS) open = open && low == high && __all(row_doc[now][sub * 32 + c] == low);
                const float *at_lse = row_lse[now] + sub * 32 + 4 * half, *at_delta = row_delta[now] + sub * 32 + 4 * half;
                Acc s = along_features<T, DP>(qt, k, lane), dp, capped;
                if (kEarly<DP>) dp = along_features<T, DP>(dt, v, lane);
                if (CAP) {
                    if (cap != 0.0f) cap_scores(s, p.cap_in, cap);
                    else s *= scale;
                    capped = s;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = CAP ? s[r] - at_lse[tile_row(r, 0)] : fmaf(s[r], scale, -at_lse[tile_row(r, 0)]);
                if (BIAS) {
                    bias.look(rule, first_key - (i0 + 31) - sight.offset, lane);
                    bias.add_to_keys(s, lane);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = exp2_fast(OCTAVES ? s[r] : s[r] * kLog2e);
                if (!kEarly<DP>) dp = along_features<T, DP>(dt, v, lane);
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = s[r] * (dp[r] - at_delta[tile_row(r, 0)]);
                if (CAP) through_cap(dp, capped, inverse_cap);
                if (!open) {  // (a key that only rows in no document would see may hold NaN: both are chosen, not multiplied away)
                    // rows from `before` on see the key; documents of rows behind the last are negative
                    const int before = j < sight.prefix || !sight.causal ? -0x40000000 : j - sight.offset;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        bool seen = tile_row(r, 0) >= before - i0 - 4 * half;
                        if (DOCUMENTS) seen = seen && row_doc[now][sub * 32 + 4 * half + tile_row(r, 0)] == doc;
                        s[r] = seen ? s[r] : 0.0f;
                        dp[r] = seen ? dp[r] : 0.0f;
                    }
                }
                if (kWeight != 1.0f) s *= kWeight;
                along_rows<T, DP>(dv, dt, Weights<T>(s), lane);
                fit.fit(dp, dk);
                if (DP <= 96 && p.close) along_rows_twice<T, DP>(dk, qt, dp, lane);
                else along_rows<T, DP>(dk, qt, Weights<T>(dp), lane);
            }
        }
    }
    if (j < p.M) {
        if (!valid) {
#pragma unroll
            for (int ft = 0; ft < DP / 32; ++ft) dk[ft] = Acc{}, dv[ft] = Acc{};
        }
        if (p.parts == 1) {
            store_column<T, DP>(row_of<T>(p.dk, p.dk_stride, b, hk, j), p.D, dk, p.scale * fit.undo(), half);
            store_column<T, DP>(row_of<T>(p.dv, p.dv_stride, b, hk, j), p.D, dv, 1.0f / kWeight, half);
        } else {
            float *const out = p.key_part + ((int64_t)part * 2 * p.B * p.Hk + b * p.Hk + hk) * p.M * p.D + (int64_t)j * p.D;
            store_column<float, DP>(out, p.D, dk, p.scale * fit.undo(), half);
            store_column<float, DP>(out + (int64_t)p.B * p.Hk * p.M * p.D, p.D, dv, 1.0f / kWeight, half);
        }
    }
}

// dk and dv from their parts, in their order.  key_part [parts][2][B, Hk, M, D]; four features a thread where four divide D.
template <typename T, int W> __global__ __launch_bounds__(256) void attention_keys_join_kernel(AttentionParams p)
{
    const int64_t all = (int64_t)p.B * p.Hk * p.M * p.D;
    const int64_t x = (blockIdx.x * (int64_t)256 + threadIdx.x) * W;
    if (x >= 2 * all) return;
    float sum[W] = {};
    for (int part = 0; part < p.parts; ++part) {
        const float *in = p.key_part + part * 2 * all + x;
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] += in[e];
    }
    const int64_t y = x < all ? x : x - all, row = y / p.D;
    const int64_t j = row % p.M, hk = row / p.M % p.Hk, b = row / p.M / p.Hk;
    T *out = x < all ? row_of<T>(p.dk, p.dk_stride, b, hk, j) : row_of<T>(p.dv, p.dv_stride, b, hk, j);
#pragma unroll
    for (int e = 0; e < W; ++e) out[y - row * p.D + e] = Elem<T>::down(sum[e]);
}

}  // namespace sdtw
