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
constexpr float kLog2e = 1.44269504088896340736f;

// What the forward pass leaves of a row (SDTW_DISTILL_STATS floats).
struct RowStats {
    float m;        // maximum of the logits
    float top;      // Q / sum exp((z - m) / temperature): a kept token's gradient is top * exp(..) - q
    float off;      // the others' is out * exp((z - off) / temperature)
    float out;
    float lq_hi;    // logarithm of the teacher's normaliser, in two parts
    float lq_lo;
    float spare;
    uint32_t flags;
};
static_assert(sizeof(RowStats) == SDTW_DISTILL_STATS * sizeof(float), "stats layout");
enum : uint32_t { kRowNoTarget = 1, kRowInvalid = 2, kRowRepeated = 4 };

struct DistillParams {
    int32_t rows, vocab, top, teacher_rows;
    int32_t teacher_type, id64, tail;
    int32_t slices, slice_cols;     // a row is shared by `slices` workgroups, slice_cols (a multiple of 8) columns each
    float inv_temperature, scale2;  // 1 / temperature and log2(e) / temperature
    double inv_temperature_d;
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

// A token id as 32 bits; whatever does not fit stays invalid (negative: unused).
__device__ __forceinline__ int load_id(const DistillParams &p, int r, int k)
{
    const int64_t i = (int64_t)r * p.id_stride + k;
    if (!p.id64) return static_cast<const int32_t *>(p.teacher_ids)[i];
    const int64_t v = static_cast<const int64_t *>(p.teacher_ids)[i];
    return v < 0 ? -1 : (v >= p.vocab ? p.vocab : (int)v);
}

// Running maximum m and sum s of exp((x - m) / temperature).  A maximum of -inf is never subtracted.
struct MaxSum { float m, s; };
__device__ __forceinline__ float exp_rel(float x, float m, float scale2) { return __builtin_amdgcn_exp2f((x - m) * scale2); }
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float scale2)
{
    const float m = fmaxf(a.m, b.m), ref = finite_ref(m);
    return {m, a.s * exp_rel(a.m, ref, scale2) + b.s * exp_rel(b.m, ref, scale2)};
}

// The same over a workgroup; red: one MaxSum per wavefront.  The result is the same in every thread.
__device__ __forceinline__ MaxSum block_join(MaxSum v, float scale2, MaxSum *red)
{
    const float m = wave_max_all_f32(v.m);
    v.s = wave_sum_all_f32(v.s * exp_rel(v.m, finite_ref(m), scale2));
    v.m = m;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    MaxSum r = red[0];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) r = join(r, red[w], scale2);
    return r;
}

// The slots of a row in LDS.
struct Slots {
    int *id;
    float *t, *z;
    uint32_t *bits;  // one per column of the slice
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

// Finishes a row, by one wavefront: `sum` is over the columns outside the kept ones (tail) or over all of them.
template <typename T>
__device__ void finish_row(const DistillParams &p, int row, int r, MaxSum sum, bool repeated, const Slots &sl, RowStats *out, float *loss)
{
    const int lane = threadIdx.x & 63;
    const double it = p.inv_temperature_d;
    int used = 0, invalid = 0;
    float mt = -INFINITY;  // the teacher's largest kept logit
    for (int k = lane; k < p.top; k += 64) {
        const int id = sl.id[k];
        used |= id >= 0 && (p.tail || sl.t[k] != -INFINITY);  // (renormalised: nothing but -inf leaves no target)
        invalid |= id >= p.vocab;
        if (id >= 0) mt = fmaxf(mt, sl.t[k]);
    }
    used = __any(used);
    invalid = __any(invalid);
    RowStats st{};
    if (!used || invalid) {
        st.flags = invalid ? kRowInvalid : kRowNoTarget;
        *out = st;
        *loss = invalid ? NAN : 0.0f;
        return;
    }
    double lq;
    if (p.tail) {
        lq = (double)p.teacher_lse[r];
    } else {
        mt = wave_max_all_f32(mt);
        double s = 0.0;
        for (int k = lane; k < p.top; k += 64)
            if (sl.id[k] >= 0) s += exp(((double)sl.t[k] - (double)finite_ref(mt)) * it);
        lq = (double)finite_ref(mt) * it + log(wave_sum_f64(s));
    }
    // maximum and sum over all columns, and how many different tokens are kept
    float m = sum.m;
    double s = (double)sum.s;
    int kept = 0;
    if (p.tail) {
        float mk = -INFINITY;
        for (int k = lane; k < p.top; k += 64)
            if (sl.id[k] >= 0) mk = fmaxf(mk, sl.z[k]);
        m = fmaxf(m, wave_max_all_f32(mk));
        double sk = 0.0;
        for (int k = lane; k < p.top; k += 64) {
            const int id = sl.id[k];
            bool first = id >= 0;
            if (repeated)
                for (int j = 0; j < k; ++j) first = first && sl.id[j] != id;
            if (!first) continue;
            ++kept;
            sk += (double)exp_rel(sl.z[k], finite_ref(m), p.scale2);
        }
        s = wave_sum_f64(sk) + (double)(sum.s * exp_rel(sum.m, finite_ref(m), p.scale2));
        kept = (int)wave_sum_all_f32((float)kept);
    }
    const double log_s = log(s);
    double part = 0.0, mass = 0.0;
    for (int k = lane; k < p.top; k += 64) {
        if (sl.id[k] < 0) continue;
        const double lk = (double)sl.t[k] * it - lq, q = exp(lk);
        mass += q;
        if (q > 0.0) part += q * (lk - ((double)sl.z[k] - (double)m) * it + log_s);
    }
    part = wave_sum_f64(part);
    mass = wave_sum_f64(mass);
    double Q = p.tail ? mass : 1.0;
    if (m == -INFINITY) {  // no token has any mass
        st.flags = kRowInvalid;
        *out = st;
        *loss = NAN;
        return;
    }
    st.m = m;
    st.off = m;
    if (!p.tail && !(mass == mass)) Q = mass;  // a NaN among the teacher's logits
    double outside = Q / s;
    if (p.tail && kept < p.vocab) {
        const double rest = fmax(0.0, 1.0 - mass);
        Q += rest;
        st.off = finite_ref(sum.m);
        // what the student has outside, relative to off; with no mass there the others' gradient is 0
        const double so = (double)sum.s, to_all = exp(((double)st.off - (double)m) * it) / s;
        if (rest > 0.0) part += rest * (log(rest) - (log(so) + ((double)st.off - (double)m) * it - log_s));
        outside = so > 0.0 ? Q * to_all - rest / so : (so == 0.0 ? 0.0 : so);
    }
    st.top = (float)(Q / s);
    st.out = (float)outside;
    st.lq_hi = (float)lq;
    st.lq_lo = (float)(lq - (double)st.lq_hi);
    st.flags = repeated ? kRowRepeated : 0;
    *out = st;
    *loss = (float)part;
}

// Columns [c0, c1) of a row: maximum and sum, without the columns marked in `bits` (bit 0 = column c0) if MARKED.
template <typename T, bool MARKED>
__device__ __forceinline__ MaxSum stream_max_sum(const T *row, int c0, int c1, const uint32_t *bits, float scale2)
{
    constexpr int W = Vec<T>::W, U = 4;
    const unsigned char *marks = reinterpret_cast<const unsigned char *>(bits);
    const int n = c1 - c0, whole = n / W;
    MaxSum acc{-INFINITY, 0.0f};
    auto take = [&](float (&x)[W * U]) {
        float m = x[0];
#pragma unroll
        for (int e = 1; e < W * U; ++e) m = fmaxf(m, x[e]);
        m = fmaxf(m, acc.m);
        const float ref = finite_ref(m);
        float s = acc.s * exp_rel(acc.m, ref, scale2);
#pragma unroll
        for (int e = 0; e < W * U; ++e) s += exp_rel(x[e], ref, scale2);
        acc = {m, s};
    };
    for (int v0 = threadIdx.x; v0 < whole; v0 += U * blockDim.x) {
        Vec<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = v0 + u * blockDim.x;
            v[u] = load_vec(row + c0 + (int64_t)(i < whole ? i : v0) * W);
        }
        float x[W * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = v0 + u * blockDim.x;
            const bool in = i < whole;
#pragma unroll
            for (int e = 0; e < W; ++e) x[u * W + e] = in ? Elem<T>::up(v[u].e[e]) : -INFINITY;
            if (MARKED && in) {
                const unsigned b = W == 8 ? marks[i] : (unsigned)(marks[i >> 1] >> (4 * (i & 1))) & 15u;
                if (b) {
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        if (b >> e & 1) x[u * W + e] = -INFINITY;
                }
            }
        }
        take(x);
    }
    const int rest = n - whole * W;
    if ((int)threadIdx.x < rest) {
        const int c = whole * W + threadIdx.x;
        float x = Elem<T>::up(row[c0 + c]);
        if (MARKED && (bits[c >> 5] >> (c & 31) & 1)) x = -INFINITY;
        acc = join(acc, MaxSum{x, x == -INFINITY ? 0.0f : exp_rel(x, x, scale2)}, scale2);
    }
    return acc;
}

// Loads the slots and marks those inside [c0, c1); *repeated is set where an id comes up twice.
template <typename T>
__device__ __forceinline__ void load_slots(const DistillParams &p, const T *row, int r, int c0, int c1, const Slots &sl, int *repeated)
{
    const int words = (c1 - c0 + 31) / 32;
    for (int w = threadIdx.x; w < words; w += blockDim.x) sl.bits[w] = 0;
    if (threadIdx.x == 0) *repeated = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < p.top; k += blockDim.x) {
        const int id = load_id(p, r, k);
        sl.id[k] = id;
        sl.t[k] = load_typed(p.teacher_logits, (int64_t)r * p.teacher_stride + k, p.teacher_type);
        const bool valid = id >= 0 && id < p.vocab;
        sl.z[k] = valid ? Elem<T>::up(row[id]) : 0.0f;
        if (valid && id >= c0 && id < c1) {
            const uint32_t bit = 1u << ((id - c0) & 31);
            if (atomicOr(&sl.bits[(id - c0) >> 5], bit) & bit) *repeated = 1;
        }
    }
    __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(512) void distill_forward_kernel(DistillParams p)
{
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ MaxSum red[8];
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
    const T *z = static_cast<const T *>(p.logits) + (int64_t)row * p.logit_stride;
    const int c0 = slice * p.slice_cols, c1 = min(p.vocab, c0 + p.slice_cols);
    const Slots sl = carve_slots(lds, p.top);
    load_slots(p, z, r, c0, c1, sl, &repeated);
    MaxSum v = p.tail ? stream_max_sum<T, true>(z, c0, c1, sl.bits, p.scale2) : stream_max_sum<T, false>(z, c0, c1, sl.bits, p.scale2);
    v = block_join(v, p.scale2, red);
    if (p.slices > 1) {
        if (threadIdx.x == 0) p.partial[(int64_t)row * p.slices + slice] = make_float4(v.m, v.s, repeated ? 1.0f : 0.0f, 0.0f);
        return;
    }
    if (threadIdx.x < 64) {
        RowStats st;
        float loss;
        finish_row<T>(p, row, r, v, repeated != 0, sl, &st, &loss);
        if (threadIdx.x == 0) {
            p.stats[row] = st;
            p.loss[row] = loss;
        }
    }
}

// Joins the slices of a row: one wavefront.
template <typename T>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillParams p)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int row = blockIdx.x, r = teacher_row_of(p, row);
    RowStats st{};
    float loss;
    if (r < 0 || r >= p.teacher_rows) {
        st.flags = r < 0 ? kRowNoTarget : kRowInvalid;
        loss = r < 0 ? 0.0f : NAN;
    } else {
        const T *z = static_cast<const T *>(p.logits) + (int64_t)row * p.logit_stride;
        const Slots sl = carve_slots(lds, p.top);
        for (int k = threadIdx.x; k < p.top; k += 64) {
            const int id = load_id(p, r, k);
            sl.id[k] = id;
            sl.t[k] = load_typed(p.teacher_logits, (int64_t)r * p.teacher_stride + k, p.teacher_type);
            sl.z[k] = id >= 0 && id < p.vocab ? Elem<T>::up(z[id]) : 0.0f;
        }
        MaxSum v{-INFINITY, 0.0f};
        bool repeated = false;
        for (int i = threadIdx.x; i < p.slices; i += 64) {
            const float4 q = p.partial[(int64_t)row * p.slices + i];
            v = join(v, MaxSum{q.x, q.y}, p.scale2);
            repeated = repeated || q.z != 0.0f;
        }
        __syncthreads();
        const float m = wave_max_all_f32(v.m);
        v = {m, wave_sum_all_f32(v.s * exp_rel(v.m, finite_ref(m), p.scale2))};
        finish_row<T>(p, row, r, v, __any(repeated), sl, &st, &loss);
    }
    if (threadIdx.x == 0) {
        p.stats[row] = st;
        p.loss[row] = loss;
    }
}

// dlogits over columns [c0, c1): every element as one outside the kept ones, then the kept ones over it.
template <typename T>
__global__ __launch_bounds__(256) void distill_backward_kernel(DistillParams p)
{
    constexpr int W = Vec<T>::W, U = 4;
    __shared__ int ids[kMaxTop];
    __shared__ float qs[kMaxTop];
    const int row = blockIdx.x / p.slices, slice = blockIdx.x % p.slices;
    const int c0 = slice * p.slice_cols, c1 = min(p.vocab, c0 + p.slice_cols);
    const T *z = static_cast<const T *>(p.logits) + (int64_t)row * p.logit_stride;
    T *dz = static_cast<T *>(p.dlogits) + (int64_t)row * p.grad_stride;
    const RowStats st = p.stats[row];
    if (st.flags & (kRowNoTarget | kRowInvalid)) {
        const T fill = Elem<T>::down(st.flags & kRowInvalid ? NAN : 0.0f);
        for (int c = c0 + threadIdx.x; c < c1; c += blockDim.x) dz[c] = fill;
        return;
    }
    const int r = teacher_row_of(p, row);
    const float g = (p.grad_loss ? p.grad_loss[row] : 1.0f) * p.inv_temperature;
    constexpr int kMine = kMaxTop / 256;
    int id[kMine];
    float val[kMine];
    const double lq = (double)st.lq_hi + (double)st.lq_lo;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int k = threadIdx.x + i * 256;
        id[i] = -1;
        if (k < p.top) {
            id[i] = load_id(p, r, k);
            const float t = load_typed(p.teacher_logits, (int64_t)r * p.teacher_stride + k, p.teacher_type);
            const float q = (float)exp((double)t * p.inv_temperature_d - lq);
            ids[k] = id[i];
            qs[k] = q;
            val[i] = q;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if (id[i] < c0 || id[i] >= c1) { id[i] = -1; continue; }
        float q = val[i];
        if (st.flags & kRowRepeated) {  // slots of one id add up: each of them stores the same sum
            q = 0.0f;
            for (int j = 0; j < p.top; ++j) q += ids[j] == id[i] ? qs[j] : 0.0f;
        }
        val[i] = g * (st.top * exp_rel(Elem<T>::up(z[id[i]]), st.m, p.scale2) - q);
    }
    __syncthreads();  // dlogits may be the logits: the kept ones have been read
    const float out = g * st.out;
    const int n = c1 - c0, whole = n / W;
    for (int v0 = threadIdx.x; v0 < whole; v0 += U * blockDim.x) {
        Vec<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = v0 + u * blockDim.x;
            if (i < whole) v[u] = load_vec(z + c0 + (int64_t)i * W);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = v0 + u * blockDim.x;
            if (i < whole) {
#pragma unroll
                for (int e = 0; e < W; ++e) v[u].e[e] = Elem<T>::down(out * exp_rel(Elem<T>::up(v[u].e[e]), st.off, p.scale2));
                store_vec(dz + c0 + (int64_t)i * W, v[u]);
            }
        }
    }
    const int rest = n - whole * W;
    if ((int)threadIdx.x < rest) {
        const int c = c0 + whole * W + threadIdx.x;
        dz[c] = Elem<T>::down(out * exp_rel(Elem<T>::up(z[c]), st.off, p.scale2));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (id[i] >= 0) dz[id[i]] = Elem<T>::down(val[i]);
}

}  // namespace sdtw
