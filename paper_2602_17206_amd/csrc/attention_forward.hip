// C entry points of attention's forward pass (declared in include/sdtw.h): checks, the split of the work, launches.
#include "attention_forward_kernels.h"
#include "attention_host.h"

namespace {

using namespace sdtw;

struct ForwardPlan {
    bool fits, few;
    int64_t row_tiles, splits, workgroups;
    size_t off_packed, total;
};

size_t few_rows_lds(const sdtw_attention_desc *d)
{
    size_t bytes = 0;
    with_shape(d->type, d->D, [&](auto t, auto features) { bytes = (size_t)few_rows_bytes<decltype(t), decltype(features)::value>(); });
    return bytes + (d->buckets ? ((size_t)std::min(32, d->H / d->Hk) * d->buckets + kBiasStarts) * 4 + 2048 : 0);
}

ForwardPlan split_forward(const sdtw_attention_desc *d)
{
    ForwardPlan P{};
    P.fits = true;
    P.splits = 1;
    if (d->B == 0 || d->H == 0 || d->N == 0) return P;
    const int64_t tiles = (d->N + 127) / 128, G = d->H / d->Hk;
    // The kernel for few rows, where there are no 1024 wavefronts of 32 rows for the other one (the matrix cores have as many), or a group's
    // rows fill no more than two of its tiles; over few keys its joins cost more than they give.  bfloat16 (float32), D 64, one head a group, us
    // with it and with the other:
    //   64 rows of 16 x 16 heads, 8192 keys: 141 and 207; 128 rows: 228 and 198   4 x 1000 x 1000: 21 and 21 (29 and 78); 256: 116 and 59
    //   32 x 512 x 512: 14 and 14 (31 and 44)   32 x 256 x 256: 11 and 10 (15 and 25)   256 x 192 x 192: 23 and 12 (50 and 33)
    //   4 x 64 x 64: 10 and 8 (13 and 11)   8 x 4 groups of 8 heads, 32 rows, 8192 keys: 55 and 147
    // ... at D 128, and just below the 1024 wavefronts:
    //   64 rows of 16 x 16 heads, 8192 keys: 236 and 327 (739 and 1276)   8 heads, 512 x 8192: 50 and 219 (192 and 1179)
    //   4 x 16 heads, 480 x 4096: 129 and 131 (683 and 640); D 64: 77 and 85 (323 and 333)   480 x 480 causal: 37 and 21 (102 and 82)
    //   16 heads, 1984 x 1984 causal: 65 and 56 (238 and 293); D 64: 33 and 38 (129 and 150)   1000 x 1000 causal: 27 and 32 (92 and 148)
    const int64_t waves = (int64_t)d->B * d->H * ((d->N + 31) / 32);
    P.few = (d->N * G <= 64 || waves < 1024) && d->M > (d->type == SDTW_TYPE_F32 ? 64 : 256) && few_rows_lds(d) + 4096 <= kLdsBytes;
    if (!P.few) {
        P.row_tiles = tiles;
        P.workgroups = (int64_t)d->B * d->H * tiles;
        P.fits = (int64_t)d->B * d->H <= 0x7fffffff && attention_grid_ok(P.workgroups);
        return P;
    }
    P.row_tiles = ((int64_t)d->N * G + 31) / 32;
    const int64_t units = (int64_t)d->B * d->Hk * P.row_tiles;
    // Two workgroups for each compute unit, of two tiles of 128 keys at least; up to four tiles are walked through without a split, which
    // would take a second launch.
    const int64_t key_tiles = ((int64_t)d->M + 127) / 128;
    P.splits = key_tiles <= 4 ? 1 : std::max<int64_t>(1, std::min<int64_t>({(512 + units - 1) / units, key_tiles / 2, 1024}));
    P.workgroups = units * P.splits;
    P.fits = attention_grid_ok(P.workgroups) && attention_grid_ok((int64_t)d->B * d->H * d->N);
    if (P.splits > 1) P.off_packed = align_up((size_t)d->B * d->H * d->N * P.splits * (d->D + 2) * sizeof(float), 256);
    return P;
}

ForwardPlan forward_plan(const sdtw_attention_desc *d)
{
    ForwardPlan P = split_forward(d);
    P.total = std::max<size_t>(256, P.off_packed + packed_bytes(d, d->q_stride, d->H, d->N) + packed_bytes(d, d->k_stride, d->Hk, d->M) +
                                        packed_bytes(d, d->v_stride, d->Hk, d->M));
    return P;
}

}  // namespace

extern "C" {

size_t sdtw_attention_forward_workspace_bytes(const sdtw_attention_desc *desc)
{
    BucketRule rule{};
    if (attention_check(desc, &rule) != SDTW_OK) return 0;
    const ForwardPlan P = forward_plan(desc);
    return P.fits ? P.total : 0;
}

int sdtw_attention_forward(const sdtw_attention_desc *desc, const void *q, const void *k, const void *v, const void *table,
                           const sdtw_attention_lists *lists, void *out, float *lse, void *workspace, size_t workspace_bytes,
                           void *stream)
{
    BucketRule rule{};
    if (int rc = attention_check(desc, &rule)) return rc;
    if (!lists_ok(desc, lists)) return SDTW_ERR_INVALID_ARG;
    if (desc->B == 0 || desc->H == 0 || desc->N == 0) return SDTW_OK;
    if (!q || !out || !lse || (desc->M > 0 && (!k || !v)) || !table == (desc->buckets != 0)) return SDTW_ERR_INVALID_ARG;
    if (!strides_ok(desc->out_stride, desc->B, desc->H, desc->N, desc->D) ||
        !places_differ(desc->out_stride, desc->B, desc->H, desc->N, desc->D))
        return SDTW_ERR_INVALID_ARG;
    if (!apart(out, {q, k, v, table}) || !apart(lse, {q, k, v, table})) return SDTW_ERR_INVALID_ARG;
    const ForwardPlan P = forward_plan(desc);
    if (!P.fits) return SDTW_ERR_INVALID_ARG;
    if (int rc = check_ws(workspace, workspace_bytes, P.total)) return rc;
    if (!apart(lse, {out})) return SDTW_ERR_INVALID_ARG;
    (void)hipGetLastError();
    AttentionParams p = attention_params(desc, lists);
    p.q = q; p.k = k; p.v = v; p.table = table;
    p.out = out;
    p.lse = lse;
    p.row_tiles = (int32_t)P.row_tiles;
    p.near = near_diagonals(desc, rule);
    p.splits = (int32_t)P.splits;
    p.part = static_cast<float *>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *room = static_cast<char *>(workspace) + P.off_packed;
    pack(desc, p.q, p.q_stride, desc->H, desc->N, room, st);
    pack(desc, p.k, p.k_stride, desc->Hk, desc->M, room, st);
    pack(desc, p.v, p.v_stride, desc->Hk, desc->M, room, st);
    with_shape(desc->type, desc->D, [&](auto t, auto features) {
        using T = decltype(t);
        constexpr int DP = decltype(features)::value;
        with_variant(desc, lists, [&](auto variant) {
            constexpr int F = decltype(variant)::value;
            if (P.few) {
                ProfScope ps("attention_few_rows", st);
                attention_few_rows_kernel<T, DP, F><<<(unsigned)P.workgroups, 256, few_rows_lds(desc), st>>>(p, rule);
            } else {
                ProfScope ps("attention_forward", st);
                const size_t bytes = 4 * TileShape<T, DP>::bytes(kKeys) + bias_bytes(4, p.near);
                attention_forward_kernel<T, DP, F><<<(unsigned)P.workgroups, 256, bytes, st>>>(p, rule);
            }
        });
        if (P.splits > 1) {
            ProfScope ps("attention_join", st);
            attention_join_kernel<T><<<(unsigned)((int64_t)p.B * p.H * p.N), 256, 0, st>>>(p);
        }
    });
    return hip_ok();
}

}  // extern "C"
