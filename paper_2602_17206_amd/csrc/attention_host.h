// What the two attention entry points' host code shares: argument checks and kernel parameters.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "attention_tiles.h"
#include "host_common.h"
#include "layout.h"

namespace sdtw {

inline bool attention_type_ok(int t) { return t == SDTW_TYPE_F32 || t == SDTW_TYPE_F16 || t == SDTW_TYPE_BF16; }

// A grid has fewer than 2^32 threads, and these kernels number their workgroups in 31 bits.
inline bool attention_grid_ok(int64_t workgroups) { return workgroups <= 0xffffffffll / 256; }

constexpr int kMaxFeatures = 128;
constexpr size_t kLdsBytes = 160 << 10;

// D rounded up to whole 16-byte chunks
inline int loaded_features(const sdtw_attention_desc *d)
{
    const int W = d->type == SDTW_TYPE_F32 ? 4 : 8;
    return (d->D + W - 1) / W * W;
}

inline sdtw_bias_desc bias_of(const sdtw_attention_desc *d)
{
    sdtw_bias_desc b{};
    b.B = d->B; b.H = d->H; b.N = d->N; b.M = d->M;
    b.buckets = d->buckets; b.max_distance = d->max_distance; b.two_sided = d->two_sided;
    b.plane_type = SDTW_TYPE_F32; b.table_type = d->table_type;
    b.offset = d->offset;
    return b;
}

inline bool strides_ok(const int64_t (&stride)[4], int64_t a, int64_t b, int64_t c, int64_t d)
{
    const int64_t most = (int64_t)1 << 58, size[4] = {a, b, c, d};
    for (int i = 0; i < 4; ++i)
        if (stride[i] < 0 || stride[i] > most / std::max<int64_t>(1, size[i])) return false;
    return true;
}

// Whether different elements have different places: sorted by stride, each dimension steps over the ones inside it.
inline bool places_differ(const int64_t (&stride)[4], int64_t a, int64_t b, int64_t c, int64_t d)
{
    struct Dim { int64_t size, stride; } dim[3] = {{a, stride[0]}, {b, stride[1]}, {c, stride[2]}};
    if (stride[3] != 1 && d > 1) return false;
    std::sort(dim, dim + 3, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
    int64_t span = d;  // elements from the first of what lies inside to behind its last one
    for (const Dim &x : dim) {
        if (x.size <= 1) continue;
        if (x.stride < span) return false;
        span += (x.size - 1) * x.stride;
    }
    return true;
}

// SDTW_OK, or what is wrong with the descriptor; the rule of its buckets.
inline int attention_check(const sdtw_attention_desc *d, BucketRule *rule)
{
    if (!d || d->B < 0 || d->H < 0 || d->Hk < 1 || d->N < 0 || d->M < 0 || d->D < 1) return SDTW_ERR_INVALID_ARG;
    if (d->H % d->Hk != 0 || d->N > 1 << 28 || d->M > 1 << 28) return SDTW_ERR_INVALID_ARG;
    // (what follows stays within 64 bits)
    const int64_t heads = (int64_t)d->B * d->H, key_heads = (int64_t)d->B * d->Hk, most = (int64_t)1 << 48;
    if (heads > 0x7fffffff || key_heads > 0x7fffffff || heads * d->N > most || key_heads * d->M > most) return SDTW_ERR_INVALID_ARG;
    if (!attention_type_ok(d->type) || d->flags != 0 || (d->causal != 0 && d->causal != 1)) return SDTW_ERR_INVALID_ARG;
    if (!(d->scale >= 0x1p-26f && d->scale <= 0x1p26f)) return SDTW_ERR_INVALID_ARG;
    // (the kernels multiply by the cap, by 1 over it and by the scale over it: numbers below the normal ones would have few digits or none)
    if (!(d->cap >= 0.0f) || !std::isfinite(d->cap * kLog2e)) return SDTW_ERR_INVALID_ARG;
    if (d->cap != 0.0f && !(std::isnormal(d->cap) && std::isnormal(d->scale / d->cap))) return SDTW_ERR_INVALID_ARG;
    if (d->offset >= (int64_t)1 << 62 || d->offset <= -((int64_t)1 << 62)) return SDTW_ERR_INVALID_ARG;
    if (d->prefix < 0 || (d->prefix > 0 && !d->causal)) return SDTW_ERR_INVALID_ARG;
    if (!strides_ok(d->q_stride, d->B, d->H, d->N, d->D) || !strides_ok(d->k_stride, d->B, d->Hk, d->M, d->D) ||
        !strides_ok(d->v_stride, d->B, d->Hk, d->M, d->D))
        return SDTW_ERR_INVALID_ARG;
    if (d->buckets != 0) {
        const sdtw_bias_desc b = bias_of(d);
        if (!position_bias_rule(&b, rule)) return SDTW_ERR_INVALID_ARG;
        const int64_t most = (int64_t)1 << 40;
        for (const int64_t s : d->table_stride)
            if (s < 0 || s > most) return SDTW_ERR_INVALID_ARG;
    }
    return d->D > kMaxFeatures ? SDTW_ERR_UNSUPPORTED : SDTW_OK;
}

inline bool lists_ok(const sdtw_attention_desc *d, const sdtw_attention_lists *lists)
{
    if (!lists) return true;
    if (lists->prefixes && !d->causal) return false;
    // (an empty list may have no place)
    return !lists->row_document == !lists->col_document || d->B == 0 || d->N == 0 || d->M == 0;
}

// Whether an output is none of the inputs (a kernel behind the one that writes it may still read them).  Empty tensors have no place.
inline bool apart(const void *out, std::initializer_list<const void *> others)
{
    for (const void *x : others)
        if (out && out == x) return false;
    return true;
}

inline AttentionParams attention_params(const sdtw_attention_desc *d, const sdtw_attention_lists *lists)
{
    AttentionParams p{};
    p.B = d->B; p.H = d->H; p.Hk = d->Hk; p.N = d->N; p.M = d->M; p.D = d->D;
    p.loaded = loaded_features(d);
    p.buckets = d->buckets; p.table_type = d->table_type; p.causal = d->causal;
    p.offset = (int32_t)std::min<int64_t>(std::max<int64_t>(d->offset, -(1 << 29)), 1 << 29);
    p.prefix = (int32_t)std::min<int64_t>(d->prefix, 1 << 29);
    p.scale = d->scale;
    p.scale2 = d->scale * kLog2e;
    p.unscale = 1.0f / d->scale;
    p.cap = d->cap;
    if (d->cap > 0.0f) p.cap_in = d->scale / d->cap, p.cap_out = d->cap * kLog2e;
    if (lists) {
        p.offsets = lists->offsets; p.prefixes = lists->prefixes;
        p.row_len = lists->row_len; p.col_len = lists->col_len;
        p.row_document = lists->row_document; p.col_document = lists->col_document;
    }
    for (int i = 0; i < 4; ++i) {
        p.q_stride[i] = d->q_stride[i]; p.k_stride[i] = d->k_stride[i]; p.v_stride[i] = d->v_stride[i];
        p.out_stride[i] = d->out_stride[i]; p.dout_stride[i] = d->dout_stride[i];
        p.dq_stride[i] = d->dq_stride[i]; p.dk_stride[i] = d->dk_stride[i]; p.dv_stride[i] = d->dv_stride[i];
    }
    p.table_stride[0] = d->table_stride[0]; p.table_stride[1] = d->table_stride[1];
    return p;
}

// Inputs whose features are apart or do not fill 16-byte chunks, or whose rows are 2^22 elements and more apart (64 of them are a tile, whose
// bytes are counted in 31 bits): the kernels read a packed copy of them, [B, heads, rows, loaded].
inline bool packed(const sdtw_attention_desc *d, const int64_t (&stride)[4])
{
    return d->D != loaded_features(d) || (stride[3] != 1 && d->D > 1) || stride[2] >= (int64_t)1 << 22;
}
inline size_t packed_bytes(const sdtw_attention_desc *d, const int64_t (&stride)[4], int64_t heads, int64_t rows)
{
    return packed(d, stride) ? align_up((size_t)d->B * heads * rows * loaded_features(d) * (d->type == SDTW_TYPE_F32 ? 4 : 2), 256) : 0;
}

// Launches the copy where one is needed; `x` and its strides become those of the copy, `room` moves on behind it.
inline void pack(const sdtw_attention_desc *d, const void *&x, int64_t (&stride)[4], int64_t heads, int64_t rows, char *&room, hipStream_t st)
{
    const size_t bytes = packed_bytes(d, stride, heads, rows);
    if (bytes == 0) return;
    const int64_t loaded = loaded_features(d), vectors = (int64_t)d->B * heads * rows * loaded / (d->type == SDTW_TYPE_F32 ? 4 : 8);
    ProfScope ps("attention_pack", st);
    PackParams p{};
    p.in = x;
    p.out = room;
    for (int i = 0; i < 4; ++i) p.stride[i] = stride[i];
    p.heads = heads; p.rows = rows; p.D = d->D; p.loaded = (int32_t)loaded; p.vectors = vectors;
    const unsigned grid = (unsigned)std::min<int64_t>((vectors + 255) / 256, 8192);
    if (d->type == SDTW_TYPE_F32) attention_pack_kernel<uint32_t><<<grid, 256, 0, st>>>(p);
    else attention_pack_kernel<uint16_t><<<grid, 256, 0, st>>>(p);
    x = room;
    room += bytes;
    stride[3] = 1; stride[2] = loaded; stride[1] = loaded * rows; stride[0] = loaded * rows * heads;
}

// Diagonals from the last bucket's first distance on either side, and a margin; 0 beyond 2048 of them (10 KB of LDS).  Laid out once they save
// looking them up tile by tile: 4 x 16 x 2048 x 2048 x 64 bfloat16 causal, last distance 1024: forward 66 us and 68 without, delta 59 and 65, rows
// 229 and 242, keys 124 and 135; beyond 2048 there is nothing left to gain (4096: 69, 69, 255 and 126 either way).
inline int near_diagonals(const sdtw_attention_desc *d, const BucketRule &rule)
{
    if (!d->buckets) return 0;
    const int64_t last = rule.n - 1 < rule.e ? rule.n - 1 : rule.start[rule.n - 1 - rule.e];
    const int64_t all = last + kBiasMargin + 1 + (rule.two_sided ? last + kBiasMargin : kBiasMargin);
    return all <= 2048 ? (int)all : 0;
}

// Calls f with a value of the element type and, as a type, the features rounded up to 32, 64, 96 or 128.
template <int DP> struct Features { static constexpr int value = DP; };
template <int F> struct Variant { static constexpr int value = F; };
// ... and what the kernel has to be compiled for.  (A cap and documents are one variant: either pays for the other's tests.)
template <typename F> void with_variant(const sdtw_attention_desc *d, const sdtw_attention_lists *lists, F f)
{
    const bool more = d->cap > 0.0f || (lists && lists->row_document);
    if (d->buckets) {
        if (more) f(Variant<kBias | kCap | kDocuments>{});
        else f(Variant<kBias>{});
    } else {
        if (more) f(Variant<kCap | kDocuments>{});
        else f(Variant<0>{});
    }
}
template <typename F> void with_shape(int type, int D, F f)
{
    auto sized = [&](auto t) {
        if (D <= 32) f(t, Features<32>{});
        else if (D <= 64) f(t, Features<64>{});
        else if (D <= 96) f(t, Features<96>{});
        else f(t, Features<128>{});
    };
    if (type == SDTW_TYPE_F32) sized(float{});
    else if (type == SDTW_TYPE_F16) sized(_Float16{});
    else sized(Bf16{});
}

}  // namespace sdtw
