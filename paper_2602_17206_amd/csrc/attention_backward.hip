// C entry points of attention's backward pass (declared in include/sdtw.h): checks, the split of the work, launches.
#include "attention_backward_kernels.h"
#include "attention_host.h"

namespace {

using namespace sdtw;

struct BackwardPlan {
    bool fits;
    int64_t row_tiles, key_tiles, parts;
    size_t off_table, off_keys, off_packed, total;
};

// delta from the rounded outputs is good enough where they are averages over many keys.  Over few of them - a row of one key has no gradient
// at all - it is not: float16 gradients of 68 rows and keys were twice as far from 64 bits as those of a chain in 32 bits.
bool few_keys(const sdtw_attention_desc *d) { return d->type != SDTW_TYPE_F32 && d->M <= 512; }

BackwardPlan backward_plan(const sdtw_attention_desc *d)
{
    BackwardPlan P{};
    P.row_tiles = ((int64_t)d->N + 127) / 128;
    P.key_tiles = ((int64_t)d->M + 127) / 128;
    // The keys' kernel is split over the rows, of which it walks `steps` tiles, until there are two workgroups for each compute unit, or
    // four where they still have 32 tiles each; with at least 8 tiles (4 where units are very few).  What it costs is parts in 32 bits and the
    // launch that adds them up.  bfloat16, us with and without a split:
    //   1 x 8 heads in groups of 4, 2048 x 64: 47 (8 parts) and 267; 32 parts 57   1 x 8 x 1024 x 64: 31 (4) and 40
    //   1 x 16 x 2048 x 64: 69 (2) and 74; 4 parts 79   2 x 16 heads in groups of 4, 4096 x 128, causal: 331 (4) and 772; 2 parts 458
    //   4 x 16 x 1024 x 64 (512 units): 82 (2) and 54   5 x 16 x 512 x 64 (8 tiles): 49 (2) and 33
    const int64_t units = (int64_t)d->B * d->Hk * P.key_tiles, steps = (int64_t)(d->H / d->Hk) * (((int64_t)d->N + 63) / 64);
    P.parts = 1;
    if (units > 0 && units < 512) {
        const int64_t two = (511 + units) / units, four = (1023 + units) / units;
        P.parts = steps >= 32 * four ? four : std::max<int64_t>(1, std::min(two, steps / (units < 128 ? 4 : 8)));
    }
    P.fits = (int64_t)d->B * d->H <= 0x7fffffff && attention_grid_ok((int64_t)d->B * d->H * std::max<int64_t>(1, P.row_tiles)) &&
             (int64_t)d->B * d->Hk <= 0x7fffffff &&
             attention_grid_ok((int64_t)d->B * d->Hk * std::max<int64_t>(1, P.key_tiles) * P.parts) && attention_grid_ok((int64_t)d->H * d->buckets);
    if (!P.fits) return P;
    P.off_table = align_up((size_t)d->B * d->H * d->N * sizeof(float), 256);
    P.off_keys = P.off_table + align_up((size_t)d->H * d->buckets * d->B * P.row_tiles * sizeof(float), 256);
    P.off_packed = P.off_keys + (P.parts > 1 ? align_up((size_t)P.parts * 2 * d->B * d->Hk * d->M * d->D * sizeof(float), 256) : 0);
    if (P.parts > 1) P.fits = attention_grid_ok(((int64_t)2 * d->B * d->Hk * d->M * d->D + 255) / 256);
    P.total = P.off_packed;
    for (const auto *stride : {&d->q_stride, &d->dout_stride}) P.total += packed_bytes(d, *stride, d->H, d->N);
    if (!few_keys(d)) P.total += packed_bytes(d, d->out_stride, d->H, d->N);
    for (const auto *stride : {&d->k_stride, &d->v_stride}) P.total += packed_bytes(d, *stride, d->Hk, d->M);
    P.total = std::max<size_t>(256, P.total);
    return P;
}

}  // namespace

extern "C" {

size_t sdtw_attention_backward_workspace_bytes(const sdtw_attention_desc *desc)
{
    BucketRule rule{};
    if (attention_check(desc, &rule) != SDTW_OK) return 0;
    const BackwardPlan P = backward_plan(desc);
    return P.fits ? P.total : 0;
}

int sdtw_attention_backward(const sdtw_attention_desc *desc, const void *q, const void *k, const void *v, const void *table,
                            const sdtw_attention_lists *lists, const void *out, const float *lse, const void *dout, void *dq,
                            void *dk, void *dv, float *dtable, void *workspace, size_t workspace_bytes, void *stream)
{
    BucketRule rule{};
    if (int rc = attention_check(desc, &rule)) return rc;
    if (!lists_ok(desc, lists)) return SDTW_ERR_INVALID_ARG;
    const bool rows = desc->B > 0 && desc->H > 0 && desc->N > 0, keys = desc->B > 0 && desc->M > 0;
    if (dtable && desc->buckets == 0) return SDTW_ERR_INVALID_ARG;
    if (!rows && !keys && (!dtable || desc->H == 0)) return SDTW_OK;
    if ((rows && (!q || !out || !lse || !dout || !dq)) || (keys && (!k || !v || !dk || !dv)) || !table == (desc->buckets != 0 && desc->H > 0))
        return SDTW_ERR_INVALID_ARG;
    if (!strides_ok(desc->out_stride, desc->B, desc->H, desc->N, desc->D) || !strides_ok(desc->dout_stride, desc->B, desc->H, desc->N, desc->D) ||
        !strides_ok(desc->dq_stride, desc->B, desc->H, desc->N, desc->D) || !strides_ok(desc->dk_stride, desc->B, desc->Hk, desc->M, desc->D) ||
        !strides_ok(desc->dv_stride, desc->B, desc->Hk, desc->M, desc->D))
        return SDTW_ERR_INVALID_ARG;
    if ((rows && !places_differ(desc->dq_stride, desc->B, desc->H, desc->N, desc->D)) ||
        (keys && (!places_differ(desc->dk_stride, desc->B, desc->Hk, desc->M, desc->D) ||
                  !places_differ(desc->dv_stride, desc->B, desc->Hk, desc->M, desc->D))))
        return SDTW_ERR_INVALID_ARG;
    if (!apart(dq, {q, k, v, table, out, lse, dout, dk, dv}) || !apart(dk, {q, k, v, table, out, lse, dout, dv}) ||
        !apart(dv, {q, k, v, table, out, lse, dout}))
        return SDTW_ERR_INVALID_ARG;
    const BackwardPlan P = backward_plan(desc);
    if (!P.fits) return SDTW_ERR_INVALID_ARG;
    if (int rc = check_ws(workspace, workspace_bytes, P.total)) return rc;
    if (!apart(dtable, {dq, dk, dv})) return SDTW_ERR_INVALID_ARG;
    (void)hipGetLastError();
    AttentionParams p = attention_params(desc, lists);
    p.q = q; p.k = k; p.v = v; p.table = table;
    p.out = const_cast<void *>(out);
    p.lse = const_cast<float *>(lse);
    p.dout = dout;
    p.dq = dq; p.dk = dk; p.dv = dv;
    p.dtable = dtable;
    p.row_tiles = (int32_t)P.row_tiles;
    p.near = near_diagonals(desc, rule);
    p.key_tiles = (int32_t)P.key_tiles;
    p.delta = static_cast<float *>(workspace);
    p.parts = (int32_t)P.parts;
    p.key_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + P.off_keys);
    p.table_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + P.off_table);
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *room = static_cast<char *>(workspace) + P.off_packed;
    const void *packed_out = p.out;
    p.close = few_keys(desc);
    const bool close_delta = dtable || p.close;  // (nothing reads the outputs then)
    if (rows) {
        pack(desc, p.q, p.q_stride, desc->H, desc->N, room, st);
        pack(desc, p.dout, p.dout_stride, desc->H, desc->N, room, st);
        if (!close_delta) pack(desc, packed_out, p.out_stride, desc->H, desc->N, room, st);
    }
    p.out = const_cast<void *>(packed_out);
    if (keys) {
        pack(desc, p.k, p.k_stride, desc->Hk, desc->M, room, st);
        pack(desc, p.v, p.v_stride, desc->Hk, desc->M, room, st);
    }
    with_shape(desc->type, desc->D, [&](auto t, auto features) {
        using T = decltype(t);
        constexpr int DP = decltype(features)::value;
        with_variant(desc, lists, [&](auto variant) {
            constexpr int F = decltype(variant)::value;
            const size_t bytes = 4 * TileShape<T, DP>::bytes(kKeys) + bias_bytes(4, p.near);
            const unsigned grid = (unsigned)((int64_t)p.B * p.H * p.row_tiles);
            // Few keys and workgroups: delta in the same kernel saves a launch; with more, its own one has more wavefronts on a SIMD.  us in
            // one kernel and in two, with the table's gradient: 4 x 2 x 96 x 96 x 16 float32 27 and 33; 4 x 16 x 256 x 256 x 64 bfloat16 34 and
            // 40; 8 x 16 x 512 x 512 67 and 72; 16 x 16 x 512 x 512 126 and 127; 2 x 16 x 2048 x 2048 141 and 136.
            p.together = kTogether<DP> && grid <= 512 && p.M <= 512;
            if (rows && close_delta && !p.together) {
                ProfScope ps("attention_delta", st);
                attention_rows_gradient_kernel<T, DP, F, kRowsDelta><<<grid, 256, bytes, st>>>(p, rule);
            }
            if (rows && dtable) {
                if constexpr ((F & kBias) != 0) {
                    ProfScope ps("attention_rows_gradient", st);
                    p.table_columns = 32;
                    const size_t tiles = TileShape<T, DP>::bytes(kKeys) >= 16384 ? 2 * TileShape<T, DP>::bytes(kKeys) : 0;  // (one buffer, see there)
                    auto need = [&] { return bytes - tiles + ((size_t)4 * p.buckets * p.table_columns + 4 * TableSum::kTile) * sizeof(float); };
                    while (need() + 2048 > kLdsBytes) p.table_columns /= 2;
                    attention_rows_gradient_kernel<T, DP, F, kRowsTable><<<grid, 256, need(), st>>>(p, rule);
                }
            } else if (rows && close_delta) {
                ProfScope ps("attention_rows_gradient", st);
                attention_rows_gradient_kernel<T, DP, F, kRowsGiven><<<grid, 256, bytes, st>>>(p, rule);
            } else if (rows) {
                ProfScope ps("attention_rows_gradient", st);
                attention_rows_gradient_kernel<T, DP, F, kRowsPlain><<<grid, 256, bytes, st>>>(p, rule);
            }
            if (keys) {
                ProfScope ps("attention_keys_gradient", st);
                attention_keys_gradient_kernel<T, DP, F><<<(unsigned)((int64_t)p.B * p.Hk * p.key_tiles * p.parts), 256, bytes, st>>>(p, rule);
            }
        });
        if (keys && p.parts > 1) {
            ProfScope ps("attention_keys_join", st);
            const int64_t elements = (int64_t)2 * p.B * p.Hk * p.M * p.D;
            if (p.D % 4 == 0) attention_keys_join_kernel<T, 4><<<(unsigned)((elements / 4 + 255) / 256), 256, 0, st>>>(p);
            else attention_keys_join_kernel<T, 1><<<(unsigned)((elements + 255) / 256), 256, 0, st>>>(p);
        }
    });
    if (dtable) {
        ProfScope ps("attention_table", st);
        if (!rows) p.row_tiles = 0;
        attention_table_kernel<<<(unsigned)(p.H * p.buckets), 64, 0, st>>>(p);
    }
    return hip_ok();
}

}  // extern "C"
