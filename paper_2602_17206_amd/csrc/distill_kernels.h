// Distillation from a teacher's top logits: loss per row and its gradient.
//
// With a = z / temperature, p = softmax(a) and the teacher's kept probabilities q_k (and the rest q_r):
//   loss = sum_k q_k (log q_k - a[id_k] + lse) + q_r (log q_r - lse_out + lse),
//   lse over all tokens, lse_out over those outside the kept ones.
//   dz   = (Q p_v - q_v) / temperature on a kept token, p_v (Q - q_r / p_r) / temperature on the others.
// The sum outside the kept tokens is gathered directly - a bit per token marks the kept ones - since the difference
// of two nearly equal sums would lose it where the student is as sure as the teacher.
#pragma once
#include "vector_io.h"

namespace sdtw {

constexpr int kMaxTop = 1024;
constexpr double kLn2 = 0.69314718055994530942;

// What the forward pass leaves of a row (SDTW_DISTILL_STATS floats).
struct RowStats {
    float m;        // maximum of the logits
    float top;      // Q / the sum of the exponentials relative to m: a kept token's gradient is top * exp_at(z, m) - q
    float off;      // the others' is out * exp_at(z, off)
    float out;
    float t_ref;    // a kept teacher logit t has the probability exp((t - t_ref) / temperature - lq)
    float lq_hi;    // lq in two parts
    float lq_lo;
    uint32_t flags;
};
static_assert(sizeof(RowStats) == SDTW_DISTILL_STATS * sizeof(float), "stats layout");
enum : uint32_t { kRowNoTarget = 1, kRowInvalid = 2, kRowRepeated = 4 };

struct DistillParams {
    int32_t rows, vocab, top, teacher_rows;
    int32_t teacher_type, id64, tail;
    int32_t slices, slice_vecs;     // a row is shared by `slices` workgroups, slice_vecs vectors each
    float inv_temperature, scale2;  // 1 / temperature and log2(e) / temperature
    double inv_temperature_d;
    double student_inv_temperature;  // scale2 log(2): see exp_at
    int64_t logit_stride, grad_stride, teacher_stride, id_stride;
    const void *logits, *teacher_logits, *teacher_ids;
    const float *teacher_lse;
    const int32_t *teacher_row;
    const float *grad_loss;
    float *loss;
    RowStats *stats;
    float4 *partial;                // [rows][slices]: maximum, sum, 1 if an id is there twice
    void *dlogits;
};

// The teacher's row of student row t; -1: none; teacher_rows or more: invalid.
__device__ __forceinline__ int teacher_row_of(const DistillParams &p, int t)
{
    return p.teacher_row ? p.teacher_row[t] : t;
}

// A slot as it lies in memory, in two halves each: loaded without a branch on its types, so that nothing waits for it before
// it is used.
struct RawSlot { uint32_t id_lo, id_hi, t_lo, t_hi; };
__device__ __forceinline__ RawSlot fetch_slot(const DistillParams &p, int r, int k)
{
    const char *id = static_cast<const char *>(p.teacher_ids) + (((int64_t)r * p.id_stride + k) << (p.id64 ? 3 : 2));
    const bool wide = p.teacher_type == SDTW_TYPE_F32;
    const char *t = static_cast<const char *>(p.teacher_logits) + (((int64_t)r * p.teacher_stride + k) << (wide ? 2 : 1));
    return {*reinterpret_cast<const uint32_t *>(id), *reinterpret_cast<const uint32_t *>(id + (p.id64 ? 4 : 0)),
            *reinterpret_cast<const uint16_t *>(t), *reinterpret_cast<const uint16_t *>(t + (wide ? 2 : 0))};
}
// Its token as 32 bits: -1 if unused, vocab if there is no such token.
__device__ __forceinline__ int slot_id(const DistillParams &p, const RawSlot &s)
{
    const int lo = (int)s.id_lo, hi = p.id64 ? (int)s.id_hi : lo >> 31;
    if (hi < 0) return -1;
    return hi > 0 || s.id_lo >= (uint32_t)p.vocab ? p.vocab : lo;
}
__device__ __forceinline__ float slot_logit(const DistillParams &p, const RawSlot &s)
{
    if (p.teacher_type == SDTW_TYPE_F32) return __uint_as_float(s.t_hi << 16 | s.t_lo);
    if (p.teacher_type == SDTW_TYPE_BF16) return __uint_as_float(s.t_lo << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)s.t_lo);
}

// Exponentials are powers of two: exp(x / temperature) = 2^(c x), c = log2(e) / temperature in float32 (`scale2`; what that rounds c
// by is a change of the temperature, the same for every term).  They are taken relative to a reference near the maximum m.  As long as
// |c m| is at most 2^22, where float32 still holds quarters, that is the whole power R(m) = 2^rint(c m), off by less than one octave:
// 2^fma(x, c, -R) rounds its exponent once, and moving a sum to another maximum is exact.  Beyond (masks of -1e9, -1e30, the type's
// lowest value) rounding c m would cost octaves, and the reference is m itself, subtracted from x before the scaling: what lies within
// a factor of 2 of m is subtracted exactly, and everything else is more than 2^21 octaves away.
constexpr float kWhole = 4194304.0f;
__device__ __forceinline__ bool huge_ref(float m, float c) { return !(fabsf(m * c) <= kWhole); }
__device__ __forceinline__ float whole_ref(float m, float c) { return huge_ref(m, c) ? 0.0f : rintf(m * c); }
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.0f : m; }
// what is subtracted from x before the scaling
__device__ __forceinline__ float sub_ref(float m, float c) { return huge_ref(m, c) ? finite_ref(m) : 0.0f; }
// 2^(c x) relative to the reference of m; what the hot loops spell out
__device__ __forceinline__ float exp_at(float x, float m, float c)
{
    return __builtin_amdgcn_exp2f(fmaf(x - sub_ref(m, c), c, -whole_ref(m, c)));
}
// from the reference of a to that of m >= a (a maximum of -inf: nothing was summed), whichever kinds they are
__device__ __forceinline__ float move_ref(float a, float m, float c)
{
    if (a == -INFINITY) return 0.0f;
    return __builtin_amdgcn_exp2f(fmaf(sub_ref(a, c) - sub_ref(m, c), c, whole_ref(a, c) - whole_ref(m, c)));
}

// Maximum m of some logits and sum s of their exponentials relative to its reference.
struct MaxSum { float m, s; };
__device__ __forceinline__ float moved(MaxSum v, float m, float c) { return v.m == -INFINITY ? v.s : v.s * move_ref(v.m, m, c); }
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c)
{
    const float m = fmaxf(a.m, b.m);
    return {m, moved(a, m, c) + moved(b, m, c)};
}
// over the lanes of a wavefront, the same in every lane
__device__ __forceinline__ MaxSum wave_join(MaxSum v, float c)
{
    const float m = wave_max_all_f32(v.m);
    return {m, wave_sum_all_f32(moved(v, m, c))};
}
// over a workgroup, the same in every thread; red: one MaxSum per wavefront
__device__ __forceinline__ MaxSum block_join(MaxSum v, float c, MaxSum *red)
{
    v = wave_join(v, c);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    const int lane = threadIdx.x & 63;
    return wave_join(lane < (int)(blockDim.x >> 6) ? red[lane] : MaxSum{-INFINITY, 0.0f}, c);
}

// A row as the aligned 16-byte vectors that hold it: column c is element `pre` + c of them.  The first and the last one may
// hold other memory too - its elements count as -inf, and are not written - so that whatever the row's length and start are,
// loads are whole cache lines and there is no remainder.  (An aligned vector with one element of the row in it lies in the
// row's allocation or in the same 16 bytes as its first or last element: it can be read.)
template <typename T> struct Row {
    static constexpr int W = Elem<T>::kWidth;
    const T *base;
    int pre, vocab, vecs;
    unsigned before, behind;  // bit e: element e of the first, the last vector is not of the row
    __device__ __forceinline__ Row(const T *row, int vocab_) : vocab(vocab_)
    {
        pre = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
        base = row - pre;
        vecs = (pre + vocab + W - 1) / W;
        before = (1u << pre) - 1u;
        behind = (~0u << (pre + vocab - (vecs - 1) * W)) & ((1u << W) - 1u);
    }
    // the same of vector i
    __device__ __forceinline__ unsigned outside(int i) const
    {
        return (i == 0 ? before : 0u) | (i == vecs - 1 ? behind : 0u) | (i >= vecs ? ~0u : 0u);
    }
};
template <typename T> __device__ __forceinline__ Row<T> logits_row(const DistillParams &p, int64_t row)
{
    return Row<T>(static_cast<const T *>(p.logits) + row * p.logit_stride, p.vocab);
}
template <typename T> __device__ __forceinline__ T *dlogits_row(const DistillParams &p, int64_t row)
{
    return static_cast<T *>(p.dlogits) + row * p.grad_stride;
}

// Vector i of a row's gradient; `out` as Row::outside.
template <typename T> __device__ __forceinline__ void store_gradient(T *dz, const Row<T> &r, int i, const float (&d)[Row<T>::W], unsigned out)
{
    T *at = dz - r.pre + (int64_t)i * Row<T>::W;
    if (out == 0) {
        store_vec<true>(at, Elem<T>::pack(d));
    } else {
#pragma unroll
        for (int w = 0; w < Row<T>::W; ++w)
            if (!(out >> w & 1)) at[w] = Elem<T>::down(d[w]);
    }
}

// The slots of a row in LDS.
struct Slots {
    int *id;
    float *t, *z;
    uint32_t *bits;  // a mark per element of the slice's vectors: kept tokens
};
__device__ __forceinline__ Slots carve_slots(unsigned char *lds, int top)
{
    Slots s;
    s.id = reinterpret_cast<int *>(lds);
    s.t = reinterpret_cast<float *>(s.id + top);
    s.z = s.t + top;
    s.bits = reinterpret_cast<uint32_t *>(s.z + top);
    return s;
}
// the marks of vector i
template <typename T> __device__ __forceinline__ unsigned vector_marks(const uint32_t *bits, int i)
{
    const unsigned char *marks = reinterpret_cast<const unsigned char *>(bits);
    return Elem<T>::kWidth == 8 ? marks[i] : (unsigned)(marks[i >> 1] >> (4 * (i & 1))) & 15u;
}

// A slot's id and teacher logit into LDS, and a mark if element `at` is one of the slice's `count`; *repeated is set where there
// was one already.
template <typename R>
__device__ __forceinline__ void put_slot(const Slots &sl, int k, int id, float t, int at, int count, R *repeated)
{
    sl.id[k] = id;
    sl.t[k] = t;
    if (at >= 0 && at < count) {
        const uint32_t bit = 1u << (at & 31);
        if (atomicOr(&sl.bits[at >> 5], bit) & bit) *repeated = 1;
    }
}
// where a token's mark is, in a slice that begins with element `first`: -1 for what is no token
__device__ __forceinline__ int mark_of(int id, int vocab, int pre, int first) { return id >= 0 && id < vocab ? id + pre - first : -1; }

// All slots, by one wavefront.
template <typename R>
__device__ __forceinline__ void load_slots(const DistillParams &p, int r, int pre, int first, int count, const Slots &sl, R *repeated)
{
    for (int k = threadIdx.x & 63; k < p.top; k += 64) {
        const RawSlot raw = fetch_slot(p, r, k);
        const int id = slot_id(p, raw);
        put_slot(sl, k, id, slot_logit(p, raw), mark_of(id, p.vocab, pre, first), count, repeated);
    }
}

// ... and, by the same one, the student's logits of these tokens.
template <typename T> __device__ __forceinline__ float kept_logit(const Row<T> &row, int id)
{
    return id >= 0 && id < row.vocab ? Elem<T>::up(row.base[row.pre + id]) : 0.0f;
}
// the same as it lies in memory, and any other's for what is no token (reduce_slots does not look at those)
template <typename T> __device__ __forceinline__ T kept_logit_ahead(const Row<T> &row, int id)
{
    return row.base[row.pre + max(0, min(id, row.vocab - 1))];
}
template <typename T> __device__ __forceinline__ void load_kept(const DistillParams &p, const Row<T> &row, const Slots &sl)
{
    for (int k = threadIdx.x & 63; k < p.top; k += 64) sl.z[k] = kept_logit(row, sl.id[k]);
}

// log(x) for x > 0 to about 1e-7, without 64-bit arithmetic in a chain: the exponent is whole and the rest, log2 of 0.5 .. 1, small.
__device__ __forceinline__ double log_of(float x)
{
    int k;
    const float f = frexpf(x, &k);
    return ((double)k + (double)__builtin_amdgcn_logf(f)) * kLn2;
}

// What one wavefront makes of a row's slots, in LDS: all that depends on the kept tokens alone.
struct Kept {
    double mass;    // sum of q_k (1 if renormalised)
    double rest;    // what the tail holds of the teacher's mass; 0 if there is no tail
    double inner;   // sum of q_k (log q_k - (z_k - m) / temperature)
    float m, s;     // maximum of the student's kept logits and sum of their exponentials, each token once
    float t_ref, lq_hi, lq_lo;  // as in RowStats
    float Q, tail;  // mass + rest, and rest, in float32
    float q_scale;  // reduce_slots leaves q_k / q_scale where the slots' teacher logits were
    int tokens;     // how many different ones
    float g;        // distill_rows_kernel: the row's upstream gradient / temperature
    uint32_t flags;
};

__device__ __forceinline__ bool has_tail(const DistillParams &p, const Kept &kept) { return p.tail && kept.tokens < p.vocab; }

// The rest of a wavefront's work on the slots.  Sums in 64 bits: they are few, and the tail is what they leave of 1.
__device__ __forceinline__ Kept reduce_slots(const DistillParams &p, int r, const Slots &sl, bool repeated)
{
    const int lane = threadIdx.x & 63;
    const double it = p.inv_temperature_d;
    Kept o{};
    bool used = false, invalid = false;
    float mt = -INFINITY, mk = -INFINITY;
    for (int k = lane; k < p.top; k += 64) {
        const int id = sl.id[k];
        const float t = sl.t[k];
        invalid = invalid || id >= p.vocab;
        if (id < 0) continue;
        used = used || p.tail || t != -INFINITY;  // (renormalised: nothing but -inf leaves no target)
        mt = fmaxf(mt, t);
        mk = fmaxf(mk, sl.z[k]);
    }
    if (__any(invalid) || !__any(used)) {
        o.flags = __any(invalid) ? kRowInvalid : kRowNoTarget;
        return o;
    }
    // (renormalised: the logarithm of the sum stays apart from the largest logit, beside which it could vanish)
    o.t_ref = p.tail ? 0.0f : finite_ref(wave_max_all_f32(mt));
    const double lse = p.tail ? (double)p.teacher_lse[r] : 0.0;
    mk = wave_max_all_f32(mk);
    const float z_ref = finite_ref(mk);
    double sum = 0.0, inner = 0.0, lq = lse;
    float sk = 0.0f;
    int tokens = 0;
    for (int k = lane; k < p.top; k += 64) {
        const int id = sl.id[k];
        if (id < 0) continue;
        const double lk = ((double)sl.t[k] - (double)o.t_ref) * it - lse, w = exp(lk);
        sum += w;
        sl.t[k] = (float)w;
        if (w != 0.0) inner += w * (lk - ((double)sl.z[k] - (double)z_ref) * p.student_inv_temperature);
        bool first = true;
        if (repeated)
            for (int j = 0; j < k; ++j) first = first && sl.id[j] != id;
        if (!first) continue;
        ++tokens;
        sk += exp_at(sl.z[k], mk, p.scale2);
    }
    sum = wave_sum_f64(sum);
    inner = wave_sum_f64(inner);
    if (p.tail) {
        o.q_scale = 1.0f;
        o.mass = sum;
        o.inner = inner;
    } else {
        const double log_sum = log_of((float)sum);
        lq = log_sum;
        o.q_scale = (float)(1.0 / sum);
        o.mass = sum == sum ? 1.0 : sum;  // (a NaN among the teacher's logits stays one)
        o.inner = inner / sum - log_sum;
    }
    o.lq_hi = (float)lq;
    o.lq_lo = (float)(lq - (double)o.lq_hi);
    o.m = mk;
    o.s = wave_sum_all_f32(sk);
    o.tokens = (int)wave_sum_all_f32((float)tokens);
    o.rest = has_tail(p, o) ? fmax(0.0, 1.0 - o.mass) : 0.0;
    o.Q = (float)(o.mass + o.rest);
    o.tail = (float)o.rest;
    o.flags = repeated ? kRowRepeated : 0;
    return o;
}

// The factors of a row's gradient (finish_row) and its loss from the kept tokens' part and the streamed columns' `sum` - of all of
// them, or those outside the kept tokens (tail).
__device__ __forceinline__ RowStats finish_row(const DistillParams &p, const Kept &kept, MaxSum sum)
{
    RowStats st{};
    st.flags = kept.flags;
    if (kept.flags & (kRowInvalid | kRowNoTarget)) return st;
    const MaxSum all = p.tail ? join(sum, MaxSum{kept.m, kept.s}, p.scale2) : sum;
    if (all.m == -INFINITY && all.s == 0.0f) {  // no token has any mass
        st.flags = kRowInvalid;
        return st;
    }
    const bool tail = has_tail(p, kept);
    st.m = all.m;
    st.top = kept.Q * __builtin_amdgcn_rcpf(all.s);
    st.off = tail ? sum.m : all.m;
    st.out = st.top;
    if (tail) {
        // with no mass outside the gradient there is 0 (NaN in a row that holds one)
        st.out = sum.s == 0.0f ? 0.0f * st.top : st.top * move_ref(sum.m, all.m, p.scale2) - kept.tail * __builtin_amdgcn_rcpf(sum.s);
    }
    st.t_ref = kept.t_ref;
    st.lq_hi = kept.lq_hi;
    st.lq_lo = kept.lq_lo;
    return st;
}

// The reference of m as a natural logarithm, less x / temperature.  (Two of 1e38, of masks, are subtracted before anything else.)
__device__ __forceinline__ double log_ref(const DistillParams &p, float m, float x)
{
    const double sub = (double)x * p.student_inv_temperature;
    return huge_ref(m, p.scale2) ? ((double)finite_ref(m) - (double)x) * p.student_inv_temperature
                                 : (double)whole_ref(m, p.scale2) * kLn2 - sub;
}
__device__ __forceinline__ float row_loss(const DistillParams &p, const Kept &kept, MaxSum sum, const RowStats &st)
{
    if (st.flags & (kRowInvalid | kRowNoTarget)) return st.flags & kRowInvalid ? NAN : 0.0f;
    const MaxSum all = p.tail ? join(sum, MaxSum{kept.m, kept.s}, p.scale2) : sum;
    const double rest = kept.rest, log_s = log_of(all.s);
    double v = kept.inner + kept.mass * (log_ref(p, all.m, finite_ref(kept.m)) + log_s);
    if (rest > 0.0) {
        const float out = finite_ref(sum.m);
        v += rest * ((log_ref(p, all.m, out) - log_ref(p, sum.m, out)) + log_of(kept.tail) + log_s - log_of(sum.s));
    }
    return (float)v;
}

// A thread's share of vectors [v0, v1) of a row: v0 + tid, + n, ..., U at a time, the next ones on their way while these are
// summed up.  STREAM: see load_vec.  MARKED: without the elements marked in `bits`, whose first vector is v0.
template <typename T, int U, bool STREAM> struct RowStream {
    static constexpr int W = Elem<T>::kWidth;
    Row<T> row;
    int v0, v1, tid, n;
    Bits4 v[U];

    // (past the end: the last vector once more, so that no load hides behind a branch)
    __device__ __forceinline__ void fetch(Bits4 (&d)[U], int i0) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) d[u] = load_vec<STREAM>(row.base + (int64_t)min(i0 + u * n, v1 - 1) * W);
    }
    __device__ __forceinline__ RowStream(const Row<T> &row_, int v0_, int v1_, int tid_, int n_) : row(row_), v0(v0_), v1(v1_), tid(tid_), n(n_)
    {
        fetch(v, v0 + tid);
    }
    template <bool MARKED> __device__ __forceinline__ MaxSum run(const uint32_t *bits, float scale2)
    {
        MaxSum acc{-INFINITY, 0.0f};
        float acc_ref = 0.0f, acc_sub = 0.0f;  // the reference of acc.m
        for (int i0 = v0 + tid; i0 < v1; i0 += U * n) {
            Bits4 next[U];
            fetch(next, i0 + U * n);
            float x[W * U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * n;
#pragma unroll
                for (int e = 0; e < W; ++e) x[u * W + e] = Elem<T>::at(v[u], e);
                unsigned out = i < v1 ? row.outside(i) : ~0u;
                if (MARKED && i < v1) out |= vector_marks<T>(bits, i - v0);
                if (out) {  // (few vectors hold a kept token)
#pragma unroll
                    for (int e = 0; e < W; ++e) x[u * W + e] = out >> e & 1 ? -INFINITY : x[u * W + e];
                }
            }
            float m = acc.m;
#pragma unroll
            for (int e = 0; e < W * U; ++e) m = fmaxf(m, x[e]);
            const float ref = whole_ref(m, scale2), sub = sub_ref(m, scale2);
            if (sub != 0.0f) {
#pragma unroll
                for (int e = 0; e < W * U; ++e) x[e] -= sub;
            }
            // (move_ref with the references at hand; two sums side by side)
            const float move = __builtin_amdgcn_exp2f(fmaf(acc_sub - sub, scale2, acc_ref - ref));
            float s2[2] = {acc.m == -INFINITY ? acc.s : acc.s * move, 0.0f};
#pragma unroll
            for (int e = 0; e < W * U; ++e) s2[e & 1] += __builtin_amdgcn_exp2f(fmaf(x[e], scale2, -ref));
            acc = {m, s2[0] + s2[1]};
            acc_ref = ref;
            acc_sub = sub;
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = next[u];
        }
        return acc;
    }
};

// One workgroup per row, or per slice of a row.  The first wavefront works on the slots while the others stream the columns.
// Bound by reading the logits once: 8192 x 131072 bfloat16 takes 314 us (6.8 TB/s), 4096 x 32768 47 us.  A single row of 32768 takes
// 5 us, the way from its slots' addresses over their logits and exponentials to the loss.
template <typename T, bool STREAM, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 320 ? 8 : 4) void distill_forward_kernel(DistillParams p)
{
    constexpr int W = Elem<T>::kWidth;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ MaxSum red[THREADS / 64];
    __shared__ Kept kept;
    __shared__ int repeated;
    const int row = blockIdx.x / p.slices, slice = blockIdx.x % p.slices;
    const int r = teacher_row_of(p, row);
    if (r < 0 || r >= p.teacher_rows) {
        if (p.slices == 1 && threadIdx.x == 0) {
            RowStats st{};
            st.flags = r < 0 ? kRowNoTarget : kRowInvalid;
            p.stats[row] = st;
            p.loss[row] = r < 0 ? 0.0f : NAN;
        }
        return;
    }
    const Row<T> z = logits_row<T>(p, row);
    const int v0 = slice * p.slice_vecs, v1 = min(z.vecs, v0 + p.slice_vecs);
    if (v0 >= v1) {  // (the last slice of a row that begins on a vector)
        if (threadIdx.x == 0) p.partial[(int64_t)row * p.slices + slice] = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
        return;
    }
    const Slots sl = carve_slots(lds, p.top);
    const bool slots_wave = threadIdx.x < 64;
    RowStream<T, 2, STREAM> stream(z, v0, v1, slots_wave ? 0 : threadIdx.x - 64, blockDim.x - 64);
    for (int w = threadIdx.x; w < ((v1 - v0) * W + 31) / 32; w += blockDim.x) sl.bits[w] = 0;
    if (threadIdx.x == 0) repeated = 0;
    __syncthreads();
    if (slots_wave) load_slots(p, r, z.pre, v0 * W, (v1 - v0) * W, sl, &repeated);
    __syncthreads();
    MaxSum v{-INFINITY, 0.0f};
    if (slots_wave) {
        if (p.slices == 1) {
            load_kept(p, z, sl);
            const Kept k = reduce_slots(p, r, sl, repeated != 0);
            if (threadIdx.x == 0) kept = k;
        }
    } else {
        v = p.tail ? stream.template run<true>(sl.bits, p.scale2) : stream.template run<false>(sl.bits, p.scale2);
    }
    v = block_join(v, p.scale2, red);
    if (threadIdx.x != 0) return;
    if (p.slices > 1) {
        p.partial[(int64_t)row * p.slices + slice] = make_float4(v.m, v.s, repeated ? 1.0f : 0.0f, 0.0f);
    } else {
        const RowStats st = finish_row(p, kept, v);
        p.stats[row] = st;
        p.loss[row] = row_loss(p, kept, v, st);
    }
}

// Joins the slices of a row: one wavefront.
template <typename T>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillParams p)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int row = blockIdx.x, r = teacher_row_of(p, row);
    Kept kept{};
    MaxSum v{-INFINITY, 0.0f};
    if (r < 0 || r >= p.teacher_rows) {
        kept.flags = r < 0 ? kRowNoTarget : kRowInvalid;
    } else {
        const Row<T> z = logits_row<T>(p, row);
        const Slots sl = carve_slots(lds, p.top);
        load_slots(p, r, 0, 0, 0, sl, (int *)nullptr);  // (no marks)
        load_kept(p, z, sl);
        bool repeated = false;
        for (int i = threadIdx.x; i < p.slices; i += 64) {
            const float4 q = p.partial[(int64_t)row * p.slices + i];
            v = join(v, MaxSum{q.x, q.y}, p.scale2);
            repeated = repeated || q.z != 0.0f;
        }
        __syncthreads();
        v = wave_join(v, p.scale2);
        kept = reduce_slots(p, r, sl, __any(repeated));
    }
    if (threadIdx.x == 0) {
        const RowStats st = finish_row(p, kept, v);
        p.stats[row] = st;
        p.loss[row] = row_loss(p, kept, v, st);
    }
}

// dlogits over a slice of a row: every element as one outside the kept ones, then the kept ones over it.  A workgroup a slice,
// or a wavefront (TEAM 64, with at most TOP slots), where rows are short.  Bound by reading and writing: 1024 x 100003 float32 takes
// 137 us (6.0 TB/s both ways together).
template <typename T, int TEAM, int TOP>
__global__ __launch_bounds__(256) void distill_backward_kernel(DistillParams p)
{
    constexpr int W = Elem<T>::kWidth, U = 4;
    __shared__ int team_ids[256 / TEAM][TOP];
    __shared__ float team_qs[256 / TEAM][TOP];
    const int team = TEAM == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0, thread = threadIdx.x % TEAM;
    int *ids = team_ids[team];
    float *qs = team_qs[team];
    const int64_t at_slice = (int64_t)blockIdx.x * (256 / TEAM) + team;
    if (TEAM == 64 && at_slice >= (int64_t)p.rows * p.slices) return;
    const int row = (int)(at_slice / p.slices), slice = (int)(at_slice % p.slices);
    // all of the slice's threads have come this far
    auto meet = [] {
        if (TEAM == 64)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        else
            __syncthreads();
    };
    const Row<T> z = logits_row<T>(p, row);
    const int v0 = slice * p.slice_vecs, v1 = min(z.vecs, v0 + p.slice_vecs);
    if (v0 >= v1) return;
    T *dz = dlogits_row<T>(p, row);
    const RowStats st = p.stats[row];
    if (st.flags & (kRowNoTarget | kRowInvalid)) {
        float fill[W];
#pragma unroll
        for (int e = 0; e < W; ++e) fill[e] = st.flags & kRowInvalid ? NAN : 0.0f;
        for (int i = v0 + thread; i < v1; i += TEAM) store_gradient(dz, z, i, fill, z.outside(i));
        return;
    }
    const int r = teacher_row_of(p, row);
    const float g = (p.grad_loss ? p.grad_loss[row] : 1.0f) * p.inv_temperature;
    constexpr int kMine = TOP / TEAM;
    int id[kMine];
    float val[kMine];
    const double lq = (double)st.lq_hi + (double)st.lq_lo;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int k = thread + i * TEAM;
        id[i] = -1;
        if (k >= p.top) continue;
        const RawSlot raw = fetch_slot(p, r, k);
        id[i] = slot_id(p, raw);
        val[i] = (float)exp(((double)slot_logit(p, raw) - (double)st.t_ref) * p.inv_temperature_d - lq);
        ids[k] = id[i];
        qs[k] = val[i];
    }
    meet();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = mark_of(id[i], p.vocab, z.pre, v0 * W);
        if (at < 0 || at >= (v1 - v0) * W) { id[i] = -1; continue; }
        float q = val[i];
        if (st.flags & kRowRepeated) {  // slots of one id add up: each of them stores the same sum
            q = 0.0f;
            for (int j = 0; j < p.top; ++j) q += ids[j] == id[i] ? qs[j] : 0.0f;
        }
        val[i] = g * (st.top * exp_at(kept_logit(z, id[i]), st.m, p.scale2) - q);
    }
    meet();  // dlogits may be the logits: the kept ones have been read
    const float out = g * st.out, sub = sub_ref(st.off, p.scale2), ref = whole_ref(st.off, p.scale2);
    for (int i0 = v0 + thread; i0 < v1; i0 += U * TEAM) {
        Bits4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_vec<true>(z.base + (int64_t)min(i0 + u * TEAM, v1 - 1) * W);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * TEAM;
            float d[W];
#pragma unroll
            for (int e = 0; e < W; ++e) d[e] = out * __builtin_amdgcn_exp2f(fmaf(Elem<T>::at(v[u], e) - sub, p.scale2, -ref));
            if (i < v1) store_gradient(dz, z, i, d, z.outside(i));
        }
    }
    meet();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (id[i] >= 0) dz[id[i]] = Elem<T>::down(val[i]);
}

// The gradient of a row's kept tokens.  Slots of one id add up: each of them stores the same sum.
template <typename T>
__device__ __forceinline__ void store_kept(const DistillParams &p, const Slots &sl, float q_scale, const RowStats &st, float g, T *dz,
                                           int first, int step)
{
    for (int k = first; k < p.top; k += step) {
        const int id = sl.id[k];
        if (id < 0) continue;
        float q = sl.t[k];
        if (st.flags & kRowRepeated) {
            q = 0.0f;
            for (int j = 0; j < p.top; ++j) q += sl.id[j] == id ? sl.t[j] : 0.0f;
        }
        dz[id] = Elem<T>::down(g * (st.top * exp_at(sl.z[k], st.m, p.scale2) - q * q_scale));
    }
}

// The lane's number, counted anew: what is computed from it is not kept in registers from one use to the next.
__device__ __forceinline__ int lane_again()
{
    int zero = 0;
    asm volatile("" : "+v"(zero));
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

// Loss and gradient of rows that stay in registers from their one read to their one write: NV vectors a thread, whose
// exponentials are kept as float32.  A workgroup takes row after row, `gridDim.x` apart.  The streaming wavefronts have a row's
// vectors on their way while they finish the one before it; the slots' wavefront runs two rows ahead, and stores a row's
// kept tokens when the others are known to have stored their vectors.  One barrier a row.  At most kRowsTop slots.
// Bound by reading and writing: 4096 x 32768 bfloat16 takes 113 us (4.8 TB/s both ways together), two passes 142; 2048 x 12000 float32 42 and 53,
// and 2048 x 40000, twelve vectors a thread, 127 (5.2 TB/s) and 155.
constexpr int kRowsTop = 128;
template <typename T, int NV, int WAVES_PER_SIMD>
__global__ __launch_bounds__(1024, WAVES_PER_SIMD) void distill_rows_kernel(DistillParams p, int ring_bytes)
{
    constexpr int W = Elem<T>::kWidth;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ MaxSum red[2][16];
    __shared__ Kept kept[3];
    __shared__ Bits4 edge[2][2];  // the gradient in a row's first and last vector, where they are not the row's alone
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int stride = gridDim.x, rows = (p.rows - blockIdx.x + stride - 1) / stride;  // of this workgroup
    auto row_of = [&](int i) { return (int64_t)blockIdx.x + (int64_t)i * stride; };
    // maximum and sum of row i, from the streaming wavefronts' own (behind the barrier)
    auto join_waves = [&](int i, int lane) {
        return wave_join(lane < waves - 1 ? red[i & 1][lane] : MaxSum{-INFINITY, 0.0f}, p.scale2);
    };
    if (wave == 0) {
        // Step t: row t - 3's kept tokens are stored, row t's slots go to LDS, row t - 2 is finished and row t's slots are
        // reduced; row t + 1's are on their way meanwhile, and the number of row t + 2's teacher.
        RowStats before{};
        float g_before = 0.0f;
        RawSlot ahead[2];
        // (loads that nothing branches on, so that nothing waits for them early: without a vector, any address that can be read)
        const int32_t *teacher_rows = p.teacher_row ? p.teacher_row : reinterpret_cast<const int32_t *>(p.loss);
        const float *weights = p.grad_loss ? p.grad_loss : p.loss;
        auto teacher_raw = [&](int i) { return teacher_rows[row_of(min(i, rows - 1))]; };
        auto teacher_of = [&](int i, int raw) { return i >= rows ? -1 : p.teacher_row ? raw : (int)row_of(i); };
        auto fetch_slots = [&](int r) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // (of a row without a target, or past the last slot: any other's, which nobody looks at)
                ahead[j] = fetch_slot(p, max(0, min(r, p.teacher_rows - 1)), min(lane + 64 * j, p.top - 1));
            }
        };
        int r = teacher_of(0, teacher_raw(0)), raw_next = teacher_raw(1);
        fetch_slots(r);
        for (int t = 0; t < rows + 3; ++t) {
            if (t >= 2) __syncthreads();
            if (t >= 3) {
                const int b = (t - 3) % 3;
                T *dz = dlogits_row<T>(p, row_of(t - 3));
                const Row<T> z = logits_row<T>(p, row_of(t - 3));
                // the row's share of its first and last vector, then the kept tokens
                const int last = z.vecs - 1, i = lane < W ? 0 : last, w = lane & (W - 1);
                const unsigned out = z.outside(i);
                if (lane < 2 * W && (lane < W || last > 0) && out != 0 && !(out >> w & 1))
                    dz[(int64_t)i * W + w - z.pre] = reinterpret_cast<const T *>(&edge[(t - 3) & 1][i ? 1 : 0])[w];
                if (!(before.flags & (kRowNoTarget | kRowInvalid)))
                    store_kept<T>(p, carve_slots(lds + b * ring_bytes, p.top), kept[b].q_scale, before, g_before, dz, lane, 64);
            }
            const bool target = t < rows && r >= 0 && r < p.teacher_rows;
            const Slots sl = carve_slots(lds + t % 3 * ring_bytes, p.top);
            bool repeated = false;
            T ahead_z[2];
            if (target) {
                const Row<T> z = logits_row<T>(p, row_of(t));
                for (int w = lane; w < (z.vecs * W + 31) / 32; w += 64) sl.bits[w] = 0;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int id = slot_id(p, ahead[j]);
                    ahead_z[j] = kept_logit_ahead(z, id);
                    if (lane + 64 * j < p.top)
                        put_slot(sl, lane + 64 * j, id, slot_logit(p, ahead[j]), mark_of(id, p.vocab, z.pre, 0), z.vecs * W, &repeated);
                }
            }
            const float weight = weights[row_of(min(t, rows - 1))];
            const int r_now = r;
            r = teacher_of(t + 1, raw_next);
            raw_next = teacher_raw(t + 2);
            fetch_slots(r);
            if (t >= 2 && t < rows + 2) {
                const MaxSum sum = join_waves(t - 2, lane);
                before = finish_row(p, kept[(t - 2) % 3], sum);
                g_before = kept[(t - 2) % 3].g;
                if (lane == 0) p.loss[row_of(t - 2)] = row_loss(p, kept[(t - 2) % 3], sum, before);
            }
            if (t < rows) {
                Kept k{};
                k.flags = r_now < 0 ? kRowNoTarget : kRowInvalid;
                if (target) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (lane + 64 * j < p.top) sl.z[lane + 64 * j] = Elem<T>::up(ahead_z[j]);
                    k = reduce_slots(p, r_now, sl, __any(repeated));
                }
                k.g = (p.grad_loss ? weight : 1.0f) * p.inv_temperature;
                if (lane == 0) kept[t % 3] = k;
            }
            if (t == 1) __syncthreads();
        }
        return;
    }
    const int wave_first = 64 * (wave - 1), n = blockDim.x - 64;
    Bits4 v[NV];
    auto fetch = [&](int i, int tid) {
        const Row<T> z = logits_row<T>(p, row_of(i));
        GlobalByte *base = shared_row(z.base);
#pragma unroll
        for (int u = 0; u < NV; ++u) v[u] = load_at<true>(base, 16u * min(tid + u * n, z.vecs - 1));
    };
    fetch(0, wave_first + lane);
    __syncthreads();
    for (int i = 0; i < rows; ++i) {
        const int tid = wave_first + lane_again();
        const Row<T> z = logits_row<T>(p, row_of(i));
        const Kept &k = kept[i % 3];
        const uint32_t *bits = carve_slots(lds + i % 3 * ring_bytes, p.top).bits;
        MaxSum own{-INFINITY, 0.0f};
        float e[NV * W];
        // (whole aligned rows that fill the workgroup hold nothing that is not of the row)
        const bool look = p.tail || z.vecs != n * NV || z.pre != 0 || p.vocab % W != 0;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
#pragma unroll
            for (int w = 0; w < W; ++w) e[u * W + w] = Elem<T>::at(v[u], w);
            if (look) {
                const int at = tid + u * n;
                unsigned out = z.outside(at);
                if (p.tail) out |= vector_marks<T>(bits, min(at, z.vecs - 1));
                if (out) {  // (few vectors hold a kept token)
#pragma unroll
                    for (int w = 0; w < W; ++w) e[u * W + w] = out >> w & 1 ? -INFINITY : e[u * W + w];
                }
            }
#pragma unroll
            for (int w = 0; w < W; ++w) own.m = fmaxf(own.m, e[u * W + w]);
        }
        if (huge_ref(own.m, p.scale2) && own.m != -INFINITY) {
#pragma unroll
            for (int q = 0; q < NV * W; ++q) e[q] -= own.m;
        }
        if (i + 1 < rows) fetch(i + 1, tid);
        const float ref = whole_ref(own.m, p.scale2);
        float s4[4] = {};  // (four sums side by side: additions do not wait for each other)
#pragma unroll
        for (int q = 0; q < NV * W; ++q) {
            e[q] = __builtin_amdgcn_exp2f(fmaf(e[q], p.scale2, -ref));
            s4[q & 3] += e[q];
        }
        own.s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
        const MaxSum wave_sum = wave_join(own, p.scale2);
        if (lane_again() == 0) red[i & 1][wave - 1] = wave_sum;
        __syncthreads();
        const RowStats st = finish_row(p, k, join_waves(i, lane_again()));
        const int tid_again = wave_first + lane_again();
        GlobalByte *dz = shared_row(dlogits_row<T>(p, row_of(i)) - z.pre);
        // what turns an exponential relative to the thread's maximum into a gradient
        const float factor = k.g * st.out * move_ref(own.m, st.off, p.scale2);
        const uint32_t flags = __builtin_amdgcn_readfirstlane(st.flags);
        if (flags & (kRowNoTarget | kRowInvalid)) {  // 0 or NaN whatever the row held
            float fill[W];
#pragma unroll
            for (int w = 0; w < W; ++w) fill[w] = flags & kRowInvalid ? NAN : 0.0f;
            for (int at = tid_again; at < z.vecs; at += n) {
                if (z.outside(at) == 0)
                    store_at<true>(dz, 16u * at, Elem<T>::pack(fill));
                else
                    edge[i & 1][at ? 1 : 0] = Elem<T>::pack(fill);
            }
            continue;
        }
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float d[W];
#pragma unroll
            for (int w = 0; w < W; ++w) d[w] = e[u * W + w] * factor;
            const int at = tid_again + u * n;
            const unsigned out = z.outside(at);
            if (out == 0)
                store_at<true>(dz, 16u * at, Elem<T>::pack(d));
            else if (at < z.vecs)
                edge[i & 1][at ? 1 : 0] = Elem<T>::pack(d);
        }
    }
    __syncthreads();
}

// Short rows: a wavefront each, four of them a workgroup that know nothing of each other.  The row stays in registers, NV vectors a
// lane, from its one read on; with GRAD its gradient is written, else its stats.  All loads of the row are on their way before
// the slots' chain of dependent ones begins - which is what bounds it: with ten slots 32 us at 16384 x 1000 float32 (4.1 TB/s) and 55 at
// 2000 (4.8), with 64 of them 46 and 87.
template <typename T, int NV, bool GRAD>
__global__ __launch_bounds__(256) void distill_short_kernel(DistillParams p, int team_bytes)
{
    constexpr int W = Elem<T>::kWidth;
    extern __shared__ __align__(16) unsigned char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= p.rows) return;
    // what lanes of this wavefront wrote is there for the others
    auto meet = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"); };
    const Row<T> z = logits_row<T>(p, row);
    T *dz = GRAD ? dlogits_row<T>(p, row) : nullptr;
    Bits4 v[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) v[u] = load_vec<GRAD>(z.base + (int64_t)min(lane + 64 * u, z.vecs - 1) * W);
    const int r = teacher_row_of(p, (int)row);
    const Slots sl = carve_slots(lds + wave * team_bytes, p.top);
    Kept kept{};
    bool repeated = false;
    const bool target = r >= 0 && r < p.teacher_rows;
    if (target) {
        for (int w = lane; w < (z.vecs * W + 31) / 32; w += 64) sl.bits[w] = 0;
        meet();
        load_slots(p, r, z.pre, 0, z.vecs * W, sl, &repeated);
        meet();
        load_kept(p, z, sl);
    }
    float e[NV * W];
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int at = lane + 64 * u;
        unsigned out = z.outside(at);
        if (p.tail && target) out |= vector_marks<T>(sl.bits, min(at, z.vecs - 1));
#pragma unroll
        for (int w = 0; w < W; ++w) {
            e[u * W + w] = out >> w & 1 ? -INFINITY : Elem<T>::at(v[u], w);
            m = fmaxf(m, e[u * W + w]);
        }
    }
    m = wave_max_all_f32(m);
    const float sub = sub_ref(m, p.scale2), ref = whole_ref(m, p.scale2);
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < NV * W; ++q) {
        e[q] = __builtin_amdgcn_exp2f(fmaf(e[q] - sub, p.scale2, -ref));
        s += e[q];
    }
    const MaxSum sum{m, wave_sum_all_f32(s)};
    if (target) {
        meet();
        kept = reduce_slots(p, r, sl, __any(repeated));
    } else {
        kept.flags = r < 0 ? kRowNoTarget : kRowInvalid;
    }
    const RowStats st = finish_row(p, kept, sum);
    if (lane == 0) {
        p.loss[row] = row_loss(p, kept, sum, st);
        if (!GRAD) p.stats[row] = st;
    }
    if constexpr (GRAD) {
        const float g = (p.grad_loss ? p.grad_loss[row] : 1.0f) * p.inv_temperature;
        const bool fill = st.flags & (kRowNoTarget | kRowInvalid);  // 0 or NaN whatever the row held
        const float filler = st.flags & kRowInvalid ? NAN : 0.0f, factor = g * st.out * move_ref(m, st.off, p.scale2);
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int at = lane + 64 * u;
            float d[W];
#pragma unroll
            for (int w = 0; w < W; ++w) d[w] = fill ? filler : e[u * W + w] * factor;
            if (at < z.vecs) store_gradient(dz, z, at, d, z.outside(at));
        }
        if (fill) return;
        meet();
        store_kept<T>(p, sl, kept.q_scale, st, g, dz, lane, 64);
    }
}

}  // namespace sdtw
