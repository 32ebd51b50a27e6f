// C entry points of the operators beside Soft-DTW (declared in include/sdtw.h): distillation from a teacher's top
// logits and the learned relative position bias.  Argument checks, workspace carving and kernel launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "distill_kernels.h"
#include "host_common.h"
#include "layout.h"
#include "position_bias_kernels.h"

namespace {

using namespace sdtw;

bool type_ok(int t) { return t == SDTW_TYPE_F32 || t == SDTW_TYPE_F16 || t == SDTW_TYPE_BF16; }

// Calls f with a value of the element type.
template <typename F> void with_type(int type, F f)
{
    if (type == SDTW_TYPE_F32)
        f(float{});
    else if (type == SDTW_TYPE_F16)
        f(_Float16{});
    else
        f(Bf16{});
}

int width_of(int type) { return type == SDTW_TYPE_F32 ? 4 : 8; }

// A grid has fewer than 2^32 threads.
bool grid_ok(int64_t workgroups, int threads) { return workgroups <= 0xffffffffll / threads; }

// ---------------------------------------------------------------- distillation

struct DistillPlan {
    int32_t slices, slice_vecs, threads;  // forward
    int32_t back_slices, back_vecs;       // backward
    size_t off_stats, off_partial, total;
};

// log2(e) / temperature in float32, what the kernels scale a logit by
float octaves_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

bool distill_ok(const sdtw_distill_desc *d)
{
    if (!d) return false;
    if (d->rows < 0 || d->vocab < 1 || d->vocab >= 1 << 30 || d->top < 1 || d->top > kMaxTop) return false;
    if (d->teacher_rows < (d->rows > 0 ? 1 : 0)) return false;
    if (!(d->temperature > 0.0f) || !std::isfinite(d->temperature) || !std::isfinite(octaves_of(d->temperature))) return false;
    if (d->target != SDTW_DISTILL_RENORMALIZED && d->target != SDTW_DISTILL_TAIL) return false;
    if (!type_ok(d->logit_type) || !type_ok(d->teacher_type)) return false;
    if (d->id_type != SDTW_ID_I32 && d->id_type != SDTW_ID_I64) return false;
    if (d->flags != 0) return false;
    if (d->logit_stride < d->vocab || d->grad_stride < d->vocab || d->teacher_stride < d->top || d->id_stride < d->top) return false;
    const int64_t most = (int64_t)1 << 60;  // no address overflows 64 bits
    const int64_t rows = std::max<int64_t>(1, std::max(d->rows, d->teacher_rows));
    return d->logit_stride <= most / rows && d->grad_stride <= most / rows && d->teacher_stride <= most / rows && d->id_stride <= most / rows;
}

// Vectors of a slice when `rows` rows of `vecs` vectors are shared by about `want` workgroups, none with fewer than `least`.
int32_t slice_vectors(int64_t rows, int64_t vecs, int64_t want, int64_t least, int64_t most)
{
    const int64_t per_row = std::max<int64_t>(1, (want + rows - 1) / rows);
    const int64_t n = (vecs + per_row - 1) / per_row;
    return (int32_t)((std::min(std::max(n, least), most) + 7) / 8 * 8);
}

DistillPlan distill_plan(const sdtw_distill_desc *d)
{
    DistillPlan P{};
    const int W = width_of(d->logit_type);
    const int64_t rows = std::max(d->rows, 1), vecs = (d->vocab + W - 1) / W + 1;  // (a row may begin inside a vector)
    // Many rows: a workgroup each, of one streaming wavefront up to 2048 vectors, three up to 16384, then four, next to the
    // one for the slots.  (One / three / four of them: 33 / 34 / 42 us at 8192 x 8000 bfloat16, 47 each at 4096 x 32768,
    // 384 / 324 / 313 at 8192 x 131072; 40 / 23 / 23 at 1024 x 32000 float32.)
    // Fewer than 512: up to fifteen, so that a row is on its way at once: 12.3 us at 1 x 32768 and at 400 x 32768 bfloat16,
    // 15.3 at 200 x 100000 float32; slices of a row and a second kernel that joins them take 15.1, 17.7 and 43.5.
    // Slices are for the few long rows (16 x 200000 bfloat16 15.1 us against 16.7; for one of 131072, 15.1 against 12.3, the second
    // launch costs more than they give), and for those whose marks - one bit an element in LDS - would take more than 32 KB.
    const int64_t most = (1 << 18) / W;
    if (rows >= 512) {
        P.slice_vecs = slice_vectors(1, vecs, 1, 1, most);
        P.threads = 64 * (P.slice_vecs < 2048 ? 2 : P.slice_vecs < 16384 ? 4 : 5);
    } else if (rows >= 64 || vecs < 16384) {
        P.slice_vecs = slice_vectors(1, vecs, 1, 1, most);
        P.threads = 64 * (int)std::min<int64_t>(16, 1 + (P.slice_vecs + 127) / 128);
    } else {
        P.slice_vecs = slice_vectors(rows, vecs, 512, 512, most);
        P.threads = 64 * 2;
    }
    P.slices = (int32_t)((vecs + P.slice_vecs - 1) / P.slice_vecs);
    // The gradient alone: workgroups whose whole slice is on its way at once, four vectors a thread, where that makes 1024 of them
    // or more: 137 us at 1024 x 100003 float32 (6.0 TB/s), 90 at 4096 x 32768 and 346 at 8192 x 65536 bfloat16; slices of 2048
    // take 154, 92 and 367, whole rows 185, 101 and 418.  Fewer rows: two vectors a thread at least.
    P.back_vecs = slice_vectors(rows, vecs, 1024, 512, 1024);
    P.back_slices = (int32_t)((vecs + P.back_vecs - 1) / P.back_vecs);
    size_t o = 0;
    P.off_stats = o;
    o = align_up(o + (size_t)rows * sizeof(RowStats), 256);
    P.off_partial = o;
    if (P.slices > 1) o = align_up(o + (size_t)rows * P.slices * sizeof(float4), 256);
    P.total = o;
    return P;
}

bool distill_args_ok(const sdtw_distill_desc *d, const void *logits, const void *teacher_logits, const void *teacher_ids,
                     const float *teacher_lse, const int32_t *teacher_row)
{
    if (!logits || !teacher_logits || !teacher_ids) return false;
    if ((d->target == SDTW_DISTILL_TAIL) != (teacher_lse != nullptr)) return false;
    return teacher_row || d->teacher_rows >= d->rows;
}

DistillParams distill_params(const sdtw_distill_desc *d, const void *logits, const void *teacher_logits, const void *teacher_ids,
                             const float *teacher_lse, const int32_t *teacher_row)
{
    DistillParams p{};
    p.rows = d->rows; p.vocab = d->vocab; p.top = d->top; p.teacher_rows = d->teacher_rows;
    p.teacher_type = d->teacher_type; p.id64 = d->id_type == SDTW_ID_I64; p.tail = d->target == SDTW_DISTILL_TAIL;
    p.inv_temperature_d = 1.0 / (double)d->temperature;
    p.inv_temperature = (float)p.inv_temperature_d;
    p.scale2 = octaves_of(d->temperature);
    p.student_inv_temperature = (double)p.scale2 * kLn2;
    p.logit_stride = d->logit_stride; p.grad_stride = d->grad_stride;
    p.teacher_stride = d->teacher_stride; p.id_stride = d->id_stride;
    p.logits = logits; p.teacher_logits = teacher_logits; p.teacher_ids = teacher_ids;
    p.teacher_lse = teacher_lse; p.teacher_row = teacher_row;
    return p;
}

void launch_distill_forward(const DistillPlan &P, DistillParams p, int type, bool stream, hipStream_t st)
{
    p.slices = P.slices;
    p.slice_vecs = P.slice_vecs;
    const size_t slots = (size_t)p.top * 12;
    const int W = width_of(type);
    const size_t marks = ((size_t)std::min((p.vocab + W - 1) / W + 1, P.slice_vecs) * W + 31) / 32 * 4;
    const unsigned grid = (unsigned)(p.rows * (int64_t)P.slices);
    {
        ProfScope ps("distill_forward", st);
        with_type(type, [&](auto t) {
            using T = decltype(t);
            if (P.threads > 320)  // (few rows)
                distill_forward_kernel<T, true, 1024><<<grid, P.threads, slots + marks, st>>>(p);
            else if (stream)
                distill_forward_kernel<T, true, 320><<<grid, P.threads, slots + marks, st>>>(p);
            else
                distill_forward_kernel<T, false, 320><<<grid, P.threads, slots + marks, st>>>(p);
        });
    }
    if (P.slices > 1) {
        ProfScope ps("distill_join", st);
        with_type(type, [&](auto t) { distill_join_kernel<decltype(t)><<<(unsigned)p.rows, 64, slots, st>>>(p); });
    }
}

// The gradient alone of rows of at most 512 vectors is a wavefront's each: with ten slots 29 against 43 us at 16384 x 1000 float32, 20 against
// 37 in bfloat16, and 53 against 50 at 16384 x 2000 float32 (64 slots at 1000: 46 and 51); with twice as many vectors 54 against 46 at 8192 x 4000.
bool wavefront_slices(const DistillPlan &P, int top) { return P.back_slices == 1 && P.back_vecs <= 512 && top <= kRowsTop; }

// (256 threads each)
int64_t distill_backward_workgroups(const DistillPlan &P, int32_t rows, int top)
{
    const int64_t slices = rows * (int64_t)P.back_slices;
    return wavefront_slices(P, top) ? (slices + 3) / 4 : slices;
}

void launch_distill_backward(const DistillPlan &P, DistillParams p, int type, hipStream_t st)
{
    p.slices = P.back_slices;
    p.slice_vecs = P.back_vecs;
    ProfScope ps("distill_backward", st);
    const unsigned grid = (unsigned)distill_backward_workgroups(P, p.rows, p.top);
    with_type(type, [&](auto t) {
        if (wavefront_slices(P, p.top))
            distill_backward_kernel<decltype(t), 64, kRowsTop><<<grid, 256, 0, st>>>(p);
        else
            distill_backward_kernel<decltype(t), 256, kMaxTop><<<grid, 256, 0, st>>>(p);
    });
}

// 16-byte vectors of a row (rows that begin anywhere may take one more)
int64_t row_vectors(const sdtw_distill_desc *d, const void *logits)
{
    const int W = width_of(d->logit_type), size = 16 / W;
    const bool aligned = (reinterpret_cast<uintptr_t>(logits) % 16 == 0) && d->logit_stride * size % 16 == 0;
    return ((int64_t)d->vocab + (aligned ? W - 1 : 2 * W - 2)) / W;
}

// Rows of up to 512 vectors are a wavefront's: its vectors a lane, 0 for longer rows.  Loss and gradient of 16384 x 1000 float32 take 32 us
// with ten slots and 46 with 64, with a workgroup to a row (distill_rows_kernel) 45 and 52, of 16384 x 2000 55 and 87 against 60 and 79; with more
// vectors a lane there are too few wavefronts.  The loss alone only with many rows: 20 against 27 us at 16384 x 1000; 256 x 4000 bfloat16 waits for the
// host, 12.5 us either way.
int short_vectors(const sdtw_distill_desc *d, const void *logits, bool gradient)
{
    const int64_t vecs = row_vectors(d, logits);
    if (d->top > kRowsTop || (!gradient && d->rows < 1024)) return 0;
    return vecs <= 256 ? 4 : vecs <= 512 ? 8 : 0;
}

// The shape of the one-read kernel for longer rows: vectors a thread and wavefronts, or 0 for rows that are too long.  Eight vectors a
// thread, and twelve where only they hold a row of float32.  (Four take 62 us at 8192 x 8000 bfloat16 and 73 at 4096 x 24000, eight 66 and 83:
// they were slower, 77 and 92, in an earlier form of the kernel, and hold rows of half the length.)
struct RowsShape { int vectors, waves, per_simd; };
RowsShape rows_shape(const sdtw_distill_desc *d, const void *logits)
{
    const int W = width_of(d->logit_type);
    const int64_t vecs = row_vectors(d, logits);
    auto waves = [&](int nv) { return 1 + (int)std::min<int64_t>(99, (vecs + 64 * nv - 1) / (64 * nv)); };
    if (waves(8) <= 16) return {8, waves(8), W == 4 ? 5 : 4};
    if (W == 4 && waves(12) <= 16) return {12, waves(12), 4};
    return {0, 0, 0};
}

// (256 threads each)
int64_t short_workgroups(const sdtw_distill_desc *d) { return ((int64_t)d->rows + 3) / 4; }

template <bool GRAD> void launch_distill_short(const sdtw_distill_desc *d, int vectors, const DistillParams &p, hipStream_t st)
{
    const int team = (d->top * 12 + vectors * 8 * width_of(d->logit_type) + 15) / 16 * 16;
    const unsigned grid = (unsigned)short_workgroups(d);
    ProfScope ps(GRAD ? "distill_step" : "distill_forward", st);
    with_type(d->logit_type, [&](auto t) {
        using T = decltype(t);
        if (vectors == 4)
            distill_short_kernel<T, 4, GRAD><<<grid, 256, 4 * team, st>>>(p, team);
        else
            distill_short_kernel<T, 8, GRAD><<<grid, 256, 4 * team, st>>>(p, team);
    });
}

// LDS of the one-read kernel for a row's slots and marks (one for every element that the workgroup holds)
int rows_ring_bytes(const sdtw_distill_desc *d, RowsShape s)
{
    return (d->top * 12 + (s.waves - 1) * s.vectors * 8 * width_of(d->logit_type) + 15) / 16 * 16;
}

void launch_distill_rows(const sdtw_distill_desc *d, RowsShape s, const DistillParams &p, hipStream_t st)
{
    const int ring = rows_ring_bytes(d, s);
    const int resident = 256 * std::max(1, s.per_simd * 4 / s.waves);
    const unsigned grid = (unsigned)std::min(p.rows, resident), threads = 64 * s.waves;
    ProfScope ps("distill_rows", st);
    with_type(d->logit_type, [&](auto t) {
        using T = decltype(t);
        constexpr bool wide = sizeof(T) == 4;
        if (s.vectors == 8)
            distill_rows_kernel<T, 8, wide ? 5 : 4><<<grid, threads, 3 * ring, st>>>(p, ring);
        else if constexpr (wide)
            distill_rows_kernel<T, 12, 4><<<grid, threads, 3 * ring, st>>>(p, ring);
    });
}

bool forward_grid_ok(const sdtw_distill_desc *d, const DistillPlan &P) { return grid_ok(d->rows * (int64_t)P.slices, P.threads); }
bool backward_grid_ok(const sdtw_distill_desc *d, const DistillPlan &P) { return grid_ok(distill_backward_workgroups(P, d->rows, d->top), 256); }

// ---------------------------------------------------------------- position bias

bool power_at_least(int d, int m, int e, int k, int D);

// First distances of the buckets from e on: the smallest d with d^m >= e^(m-k) D^k.
void bucket_starts(int e, int m, int D, int32_t *start)
{
    start[0] = e;
    for (int k = 1; k < m; ++k) {
        const double x = (double)e * std::pow((double)D / e, (double)k / m);
        const double near = std::nearbyint(x);
        // The power is good to about 1e-13 of itself; nearer than that to a whole number the whole numbers decide.
        if (std::fabs(x - near) < 1e-9 * x)
            start[k] = (int32_t)near + (power_at_least((int)near, m, e, k, D) ? 0 : 1);
        else
            start[k] = (int32_t)std::ceil(x);
    }
}

// d^m >= e^(m-k) D^k in whole numbers of as many 32-bit digits as it takes (m <= 128 factors below 2^25).
bool power_at_least(int d, int m, int e, int k, int D)
{
    constexpr int kDigits = 128;
    uint32_t a[kDigits] = {1}, b[kDigits] = {1};
    const int digits = (25 * m + 31) / 32;  // (no factor is beyond 2^24, and m at most 128)
    auto times = [digits](uint32_t *x, uint32_t f) {
        uint64_t carry = 0;
        for (int i = 0; i < digits; ++i) {
            carry += (uint64_t)x[i] * f;
            x[i] = (uint32_t)carry;
            carry >>= 32;
        }
    };
    for (int i = 0; i < m; ++i) {
        times(a, (uint32_t)d);
        times(b, (uint32_t)(i < k ? D : e));
    }
    for (int i = digits - 1; i >= 0; --i)
        if (a[i] != b[i]) return a[i] > b[i];
    return true;
}

bool bias_ok(const sdtw_bias_desc *d)
{
    if (!d) return false;
    if (d->B < 0 || d->H < 0 || d->N < 0 || d->M < 0) return false;
    if (d->two_sided != 0 && d->two_sided != 1) return false;
    if (d->buckets < (d->two_sided ? 4 : 2) || d->buckets > kMaxBuckets || (d->two_sided && d->buckets % 2 != 0)) return false;
    const int n = d->two_sided ? d->buckets / 2 : d->buckets;
    if (d->max_distance <= n / 2 || d->max_distance > 1 << 24) return false;
    if (!type_ok(d->plane_type) || !type_ok(d->table_type) || d->flags != 0) return false;
    if (d->N >= 1 << 30 || d->M >= 1 << 30) return false;
    if (d->offset >= (int64_t)1 << 62 || d->offset <= -((int64_t)1 << 62)) return false;
    const int64_t most = (int64_t)1 << 59, size[3] = {d->B, d->H, d->N};
    for (int i = 0; i < 3; ++i)
        if (d->in_stride[i] < 0 || d->out_stride[i] < 0 || d->in_stride[i] > most / std::max<int64_t>(1, size[i]) ||
            d->out_stride[i] > most / std::max<int64_t>(1, size[i]))
            return false;
    return true;
}

// Whether different cells of `out` have different places: sorted by stride, each dimension steps over the ones inside it.
bool disjoint(const sdtw_bias_desc *d)
{
    struct Dim { int64_t size, stride; } dim[3] = {{d->B, d->out_stride[0]}, {d->H, d->out_stride[1]}, {d->N, d->out_stride[2]}};
    std::sort(dim, dim + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t span = d->M;  // elements from the first cell of what lies inside to behind its last one
    for (const Dim &x : dim) {
        if (x.size <= 1) continue;
        if (x.stride < span) return false;
        span += (x.size - 1) * x.stride;
    }
    return true;
}

BucketRule bucket_rule(const sdtw_bias_desc *d)
{
    BucketRule r{};
    r.two_sided = d->two_sided;
    r.n = d->two_sided ? d->buckets / 2 : d->buckets;
    r.e = r.n / 2;
    r.m = r.n - r.e;
    bucket_starts(r.e, r.m, d->max_distance, r.start);
    r.start[r.m] = 0x7fffffff;
    r.per_octave = (float)(r.m / std::log2((double)d->max_distance / r.e));
    r.shift = (float)(-(double)r.per_octave * std::log2((double)r.e));
    return r;
}

BiasParams bias_params(const sdtw_bias_desc *d, const void *in, const int32_t *offsets, const int32_t *row_len, const int32_t *col_len)
{
    BiasParams p{};
    p.B = d->B; p.H = d->H; p.N = d->N; p.M = d->M;
    p.buckets = d->buckets; p.table_type = d->table_type;
    // (|j - i| is below 2^30 and max_distance at most 2^24: beyond 2^32 every distance is in a last bucket, whatever the offset)
    p.offset = std::min(std::max(d->offset, -((int64_t)1 << 32)), (int64_t)1 << 32);
    for (int i = 0; i < 3; ++i) { p.in_stride[i] = d->in_stride[i]; p.out_stride[i] = d->out_stride[i]; }
    p.table_stride[0] = d->table_stride[0]; p.table_stride[1] = d->table_stride[1];
    p.in = in;
    p.offsets = offsets; p.row_len = row_len; p.col_len = col_len;
    return p;
}

bool begins_on_vectors(const void *plane, const int64_t (&stride)[3], int W)
{
    return reinterpret_cast<uintptr_t>(plane) % 16 == 0 && stride[0] % W == 0 && stride[1] % W == 0 && stride[2] % W == 0;
}

// How the backward pass is split (`fits`: into a grid that can be launched): tiles of the plane, then the batch, into 2048
// workgroups where it has them.  Measured with 1024, 2048, 8192: 32 x 1 x 8192 x 8192 float32 1294, 1286, 1294 us,
// 4 x 16 x 2048 x 2048 bfloat16 89, 88, 88 us.
struct BiasPlan { bool fits; int64_t wave_rows, across, col_tiles, tiles, batch_per_part, batch_parts, parts; };

BiasPlan bias_plan(const sdtw_bias_desc *d)
{
    BiasPlan P{};
    P.fits = grid_ok(d->H * (int64_t)d->buckets, 256);  // (the second kernel)
    if (!P.fits || d->B == 0 || d->H == 0 || d->N == 0 || d->M == 0) return P;
    const int64_t width = 64 * width_of(d->plane_type), want = 2048;
    P.across = d->M > 2 * width ? 4 : d->M > width ? 2 : 1;
    P.col_tiles = (d->M + P.across * width - 1) / (P.across * width);
    auto tile = [&](int64_t wave_rows) {
        const int64_t rows = wave_rows * (4 / P.across);
        P.wave_rows = wave_rows;
        P.tiles = P.col_tiles * ((d->N + rows - 1) / rows);
    };
    // A wavefront goes down 64 rows, 8 a step - or 16, where that makes no more than a workgroup for each compute unit, and the steps' latency
    // counts: 13.9 against 14.5 us at 4 x 1 x 64 x 64 float32, 15.5 and 19.9 at 16 x 8 x 300 x 300 bfloat16; but 33.7 against 28.7 at
    // 32 x 1 x 1024 x 1024 float32.
    tile(64);
    P.fits = P.tiles <= 0x7fffffff / d->H;  // (what follows stays within 64 bits)
    if (!P.fits) return P;
    if (P.tiles * d->H * d->B <= 256) tile(16);
    const int64_t units = P.tiles * d->H;
    P.batch_parts = std::min<int64_t>(d->B, (want + units - 1) / units);
    P.batch_per_part = (d->B + P.batch_parts - 1) / P.batch_parts;
    P.batch_parts = (d->B + P.batch_per_part - 1) / P.batch_per_part;
    P.parts = P.tiles * P.batch_parts;
    P.fits = grid_ok(P.parts * d->H, 256);
    return P;
}

}  // namespace

namespace sdtw {

int position_bias_add(const sdtw_bias_desc *desc, const void *table, bool penalty, const void *in, const int32_t *offsets,
                      const int32_t *row_len, const int32_t *col_len, void *out, hipStream_t st)
{
    if (!bias_ok(desc)) return SDTW_ERR_INVALID_ARG;
    if (desc->B == 0 || desc->H == 0 || desc->N == 0 || desc->M == 0) return SDTW_OK;
    if (!table || !out || !disjoint(desc)) return SDTW_ERR_INVALID_ARG;
    if (in == out)  // in place: a thread uses of what it reads exactly the cells that it writes
        for (int i = 0; i < 3; ++i)
            if (desc->in_stride[i] != desc->out_stride[i]) return SDTW_ERR_INVALID_ARG;
    BiasParams p = bias_params(desc, in, offsets, row_len, col_len);
    p.table = table;
    p.penalty = penalty;
    p.out = out;
    const int W = width_of(desc->plane_type);
    p.tx = 1;
    while (p.tx < 256 && p.tx * W < desc->M) p.tx *= 2;
    const int rows = 256 / p.tx * kBiasRows, cols = p.tx * W;
    p.col_tiles = (desc->M + cols - 1) / cols;
    p.row_tiles = (desc->N + rows - 1) / rows;
    const int64_t tiles = (int64_t)p.col_tiles * p.row_tiles, planes = (int64_t)desc->B * desc->H;
    if (!grid_ok(planes, 256) || !grid_ok(tiles, 256) || !grid_ok(tiles * planes, 256)) return SDTW_ERR_INVALID_ARG;
    (void)hipGetLastError();
    const BucketRule rule = bucket_rule(desc);
    {
        ProfScope ps("position_bias_forward", st);
        // Planes that the memory-side cache of 256 MB cannot hold are written past it: 357 against 387 us at 8 x 16 x 2048 x 2048
        // bfloat16.  (Just beyond its size that depends on what the cache held: 92 against 84 at 8 x 16 x 1100 x 960 float16 where the
        // output's memory is that of the call before.)  Others stay there for the next kernel: 67 against 83 us with a softmax
        // behind it at 8 x 4 x 1024 x 1024 bfloat16; alone 46 against 50 at 32 x 1 x 1024 x 1024 float32.
        // Rows that begin inside vectors share lines with their neighbours and go through the caches both ways: 382 against 391 us
        // (read past them) and 406 (both) at 8 x 16 x 2001 x 2003 bfloat16, 175, 175 and 170 at 4 x 16 x 1001 x 1501 float32; at 8 x 16 x
        // 1100 x 937 float16, which just fits the cache, 103, 89 and 108.
        const bool vectors = begins_on_vectors(in, desc->in_stride, W) && begins_on_vectors(out, desc->out_stride, W);
        const bool stream = vectors && planes * desc->N * desc->M * (16 / W) >= (int64_t)256 << 20;
        with_type(desc->plane_type, [&](auto t) {
            using T = decltype(t);
            const auto kernel = stream    ? position_bias_forward_kernel<T, true, true>
                                : vectors ? position_bias_forward_kernel<T, true, false>
                                          : position_bias_forward_kernel<T, false, false>;
            kernel<<<(unsigned)(tiles * planes), 256, (size_t)(rows + cols) * 4, st>>>(p, rule);
        });
    }
    return hip_ok();
}

int position_bias_table_grad(const sdtw_bias_desc *desc, const void *penalty_table, const void *grad, const float *scale,
                             bool scale_heads, const int32_t *offsets, const int32_t *row_len, const int32_t *col_len, float *dtable,
                             void *workspace, size_t workspace_bytes, hipStream_t st)
{
    if (!bias_ok(desc)) return SDTW_ERR_INVALID_ARG;
    if (desc->H == 0) return SDTW_OK;
    const BiasPlan P = bias_plan(desc);
    if (!dtable || (!grad && P.parts > 0)) return SDTW_ERR_INVALID_ARG;
    if (!P.fits) return SDTW_ERR_INVALID_ARG;
    if (int rc = check_ws(workspace, workspace_bytes, sdtw_position_bias_workspace_bytes(desc))) return rc;
    (void)hipGetLastError();
    BiasParams p = bias_params(desc, grad, offsets, row_len, col_len);
    p.scale = scale;
    p.scale_heads = scale_heads;
    p.table = penalty_table;
    p.dtable = dtable;
    p.partial = static_cast<double *>(workspace);
    p.wave_rows = (int32_t)P.wave_rows;
    p.across = (int32_t)P.across;
    p.col_tiles = (int32_t)P.col_tiles;
    p.tiles = (int32_t)P.tiles;
    p.batch_parts = (int32_t)P.batch_parts;
    p.batch_per_part = (int32_t)P.batch_per_part;
    p.parts = (int32_t)P.parts;
    const BucketRule rule = bucket_rule(desc);
    if (P.parts > 0) {
        ProfScope ps("position_bias_backward", st);
        with_type(desc->plane_type, [&](auto t) {
            position_bias_backward_kernel<decltype(t)><<<(unsigned)(P.parts * desc->H), 256, 0, st>>>(p, rule);
        });
    }
    {
        ProfScope ps("position_bias_table", st);
        position_bias_table_kernel<<<(unsigned)(desc->H * desc->buckets), 256, 0, st>>>(p);
    }
    return hip_ok();
}

}  // namespace sdtw

extern "C" {

size_t sdtw_distill_workspace_bytes(const sdtw_distill_desc *desc)
{
    if (!distill_ok(desc)) return 0;
    return distill_plan(desc).total;
}

int sdtw_distill_forward(const sdtw_distill_desc *desc, const void *logits, const void *teacher_logits, const void *teacher_ids,
                         const float *teacher_lse, const int32_t *teacher_row, float *loss, float *stats, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (!distill_ok(desc)) return SDTW_ERR_INVALID_ARG;
    if (desc->rows == 0) return SDTW_OK;
    if (!distill_args_ok(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row) || !loss || !stats) return SDTW_ERR_INVALID_ARG;
    const DistillPlan P = distill_plan(desc);
    const int vectors = short_vectors(desc, logits, false);
    if (!(vectors ? grid_ok(short_workgroups(desc), 256) : forward_grid_ok(desc, P))) return SDTW_ERR_INVALID_ARG;
    if (int rc = check_ws(workspace, workspace_bytes, P.total)) return rc;
    (void)hipGetLastError();  // what an earlier, unrelated call left behind is not this call's error
    DistillParams p = distill_params(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row);
    p.loss = loss;
    p.stats = reinterpret_cast<RowStats *>(stats);
    p.partial = reinterpret_cast<float4 *>(static_cast<char *>(workspace) + P.off_partial);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (vectors)
        launch_distill_short<false>(desc, vectors, p, st);
    else
        launch_distill_forward(P, p, desc->logit_type, true, st);
    return hip_ok();
}

int sdtw_distill_backward(const sdtw_distill_desc *desc, const void *logits, const void *teacher_logits, const void *teacher_ids,
                          const float *teacher_lse, const int32_t *teacher_row, const float *grad_loss, const float *stats,
                          void *dlogits, void *stream)
{
    if (!distill_ok(desc)) return SDTW_ERR_INVALID_ARG;
    if (desc->rows == 0) return SDTW_OK;
    if (!distill_args_ok(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row) || !stats || !dlogits) return SDTW_ERR_INVALID_ARG;
    if (dlogits == logits && desc->grad_stride != desc->logit_stride) return SDTW_ERR_INVALID_ARG;
    const DistillPlan P = distill_plan(desc);
    if (!backward_grid_ok(desc, P)) return SDTW_ERR_INVALID_ARG;
    (void)hipGetLastError();
    DistillParams p = distill_params(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row);
    p.grad_loss = grad_loss;
    p.stats = reinterpret_cast<RowStats *>(const_cast<float *>(stats));
    p.dlogits = dlogits;
    launch_distill_backward(P, p, desc->logit_type, static_cast<hipStream_t>(stream));
    return hip_ok();
}

int sdtw_distill_step(const sdtw_distill_desc *desc, const void *logits, const void *teacher_logits, const void *teacher_ids,
                      const float *teacher_lse, const int32_t *teacher_row, const float *grad_loss, float *loss, void *dlogits,
                      void *workspace, size_t workspace_bytes, void *stream)
{
    if (!distill_ok(desc)) return SDTW_ERR_INVALID_ARG;
    if (desc->rows == 0) return SDTW_OK;
    if (!distill_args_ok(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row) || !loss || !dlogits) return SDTW_ERR_INVALID_ARG;
    if (dlogits == logits && desc->grad_stride != desc->logit_stride) return SDTW_ERR_INVALID_ARG;
    const DistillPlan P = distill_plan(desc);
    const int vectors = short_vectors(desc, logits, true);
    const RowsShape shape = rows_shape(desc, logits);
    const bool one_read = shape.vectors > 0 && desc->top <= kRowsTop;  // (a grid of what is resident)
    if (!(vectors ? grid_ok(short_workgroups(desc), 256) : one_read || (forward_grid_ok(desc, P) && backward_grid_ok(desc, P))))
        return SDTW_ERR_INVALID_ARG;
    if (int rc = check_ws(workspace, workspace_bytes, P.total)) return rc;
    (void)hipGetLastError();
    DistillParams p = distill_params(desc, logits, teacher_logits, teacher_ids, teacher_lse, teacher_row);
    p.loss = loss;
    p.grad_loss = grad_loss;
    p.dlogits = dlogits;
    p.stats = reinterpret_cast<RowStats *>(static_cast<char *>(workspace) + P.off_stats);
    p.partial = reinterpret_cast<float4 *>(static_cast<char *>(workspace) + P.off_partial);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (vectors) {
        launch_distill_short<true>(desc, vectors, p, st);
        return hip_ok();
    }
    if (one_read) {
        launch_distill_rows(desc, shape, p, st);
        return hip_ok();
    }
    // Two passes.  Up to twice the memory-side cache of 256 MB the first one reads without the streaming hint, and the second
    // finds part of it there - 136 us at 1024 x 131072 bfloat16, with the hint 135 to 151 -; at 8192 x 65536 (1 GB) 545 against 513.
    const int64_t bytes = (int64_t)desc->rows * desc->vocab * (16 / width_of(desc->logit_type));
    launch_distill_forward(P, p, desc->logit_type, bytes > (int64_t)512 << 20, st);
    launch_distill_backward(P, p, desc->logit_type, st);
    return hip_ok();
}

int sdtw_position_bias_starts(const sdtw_bias_desc *desc, int32_t *starts)
{
    if (!bias_ok(desc) || !starts) return SDTW_ERR_INVALID_ARG;
    const BucketRule r = bucket_rule(desc);
    for (int u = 0; u < r.n; ++u) starts[u] = u < r.e ? u : r.start[u - r.e];
    return SDTW_OK;
}

int sdtw_position_bias_forward(const sdtw_bias_desc *desc, const void *table, const void *in, const int32_t *offsets,
                               const int32_t *row_len, const int32_t *col_len, void *out, void *stream)
{
    return position_bias_add(desc, table, false, in, offsets, row_len, col_len, out, static_cast<hipStream_t>(stream));
}

size_t sdtw_position_bias_workspace_bytes(const sdtw_bias_desc *desc)
{
    if (!bias_ok(desc)) return 0;
    const BiasPlan P = bias_plan(desc);
    return P.fits ? std::max<size_t>(256, align_up((size_t)desc->H * desc->buckets * (size_t)P.parts * sizeof(double), 256)) : 0;
}

int sdtw_position_bias_backward(const sdtw_bias_desc *desc, const void *grad, const float *scale, const int32_t *offsets,
                                const int32_t *row_len, const int32_t *col_len, float *dtable, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    return position_bias_table_grad(desc, nullptr, grad, scale, false, offsets, row_len, col_len, dtable, workspace, workspace_bytes,
                                    static_cast<hipStream_t>(stream));
}

}  // extern "C"
