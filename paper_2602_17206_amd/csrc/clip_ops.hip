// C entry points of gradient clipping (declared in include/sdtw.h): checks, the split into launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "clip_kernels.h"
#include "host_common.h"
#include "layout.h"

namespace {

using namespace sdtw;

constexpr int32_t kMostGradients = 1 << 20;

int size_of(int type) { return type == SDTW_TYPE_F32 ? 4 : 2; }
bool clip_type_ok(int t) { return t == SDTW_TYPE_F32 || t == SDTW_TYPE_F16 || t == SDTW_TYPE_BF16; }

bool gradients_ok(const sdtw_gradient *g, int32_t count)
{
    if (count < 0 || count > kMostGradients || (count > 0 && !g)) return false;
    int64_t all = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].count < 0 || g[i].count >= (int64_t)1 << 48 || !clip_type_ok(g[i].type) || !clip_type_ok(g[i].out_type)) return false;
        if (g[i].count > 0 && (!g[i].data || !g[i].out)) return false;
        all += g[i].count;
        if (all >= (int64_t)1 << 48) return false;
        if (g[i].data == g[i].out && g[i].type != g[i].out_type && g[i].count > 0) return false;
    }
    return (all + (int64_t)kMostGradients * kClipChunk) / kClipChunk < 0x7fffffff;  // (chunks are counted in 32 bits)
}

// Whether what is written overlaps nothing else: SDTW_OK, SDTW_ERR_INVALID_ARG, or SDTW_ERR_WORKSPACE without host memory for it.
int check_overlap(const sdtw_gradient *g, int32_t count, const float *norm)
{
    struct Span { uintptr_t begin, end; bool written; };
    Span *span = new (std::nothrow) Span[2 * (size_t)count + 1];  // (the tensors', and the norm's)
    if (!span) return SDTW_ERR_WORKSPACE;
    const uintptr_t at = reinterpret_cast<uintptr_t>(norm);
    size_t n = 0;
    span[n++] = Span{at, at + sizeof(float), true};
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].count == 0) continue;
        const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].data), out = reinterpret_cast<uintptr_t>(g[i].out);
        span[n++] = Span{out, out + (uintptr_t)g[i].count * size_of(g[i].out_type), true};
        if (in != out) span[n++] = Span{in, in + (uintptr_t)g[i].count * size_of(g[i].type), false};
    }
    std::sort(span, span + n, [](const Span &a, const Span &b) { return a.begin < b.begin; });
    uintptr_t any = 0, written = 0;  // ends of what lies before
    int rc = SDTW_OK;
    for (size_t k = 0; k < n; ++k) {
        if (span[k].begin < (span[k].written ? any : written)) rc = SDTW_ERR_INVALID_ARG;
        any = std::max(any, span[k].end);
        if (span[k].written) written = std::max(written, span[k].end);
    }
    delete[] span;
    return rc;
}

int launches_of(int32_t count) { return std::max(1, (count + kClipTensors - 1) / kClipTensors); }

// Workgroups of a launch, so that all launches together leave about kClipParts sums behind.
int most_workgroups(int launches) { return std::max(256, kClipParts / launches); }

}  // namespace

extern "C" {

size_t sdtw_gradient_clip_workspace_bytes(const sdtw_gradient *gradients, int32_t count)
{
    if (!gradients_ok(gradients, count)) return 0;
    const int launches = launches_of(count);
    return align_up((size_t)launches * most_workgroups(launches) * sizeof(double), 256);
}

int sdtw_gradient_clip(const sdtw_gradient *gradients, int32_t count, float max_norm, float *norm, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    if (!gradients_ok(gradients, count) || !norm || !(max_norm >= 0.0f)) return SDTW_ERR_INVALID_ARG;
    if (int rc = check_overlap(gradients, count, norm)) return rc;
    const int launches = launches_of(count), most = most_workgroups(launches);
    if (int rc = check_ws(workspace, workspace_bytes, (size_t)launches * most * sizeof(double))) return rc;
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(stream);
    ClipParams p{};
    p.parts = static_cast<double *>(workspace);
    p.max_norm = max_norm;
    auto fill = [&](ClipList &list, int launch) {
        const int32_t from = launch * kClipTensors, to = std::min(count, from + kClipTensors);
        list.tensors = 0;
        int32_t chunks = 0;
        bool writes = std::isfinite(max_norm);
        for (int32_t i = from; i < to; ++i) {
            if (gradients[i].count == 0) continue;
            const int at = list.tensors++;
            list.data[at] = gradients[i].data;
            list.out[at] = gradients[i].out;
            list.count_types[at] = (uint64_t)gradients[i].count | (uint64_t)gradients[i].type << 56 | (uint64_t)gradients[i].out_type << 60;
            list.first[at] = chunks;
            chunks += (int32_t)((gradients[i].count + kClipChunk - 1) / kClipChunk);
            writes = writes || gradients[i].data != gradients[i].out;
        }
        list.first[list.tensors] = chunks;
        return writes;
    };
    ClipList list;
    if (launches == 1) {
        (void)fill(list, 0);
        int64_t elements = 0;
        for (int32_t i = 0; i < count; ++i) elements += gradients[i].count;
        // One launch for what its 16 wavefronts hold a chunk of each: 13 tensors of 1000 elements 8.8 us, in two launches 12.5; of 5000, 10.5 and
        // 12.6.  26 of 5000: 25.5 and 12.8; 60 of 1000: 30.7 and 13.3.
        if (list.first[list.tensors] <= 16 && elements <= 1 << 16) {
            p.norm = norm;
            ProfScope ps("clip_small", st);
            clip_small_kernel<<<1, 1024, 0, st>>>(list, p);
            return hip_ok();
        }
    }
    for (int l = 0; l < launches; ++l) {
        (void)fill(list, l);
        const int grid = std::min(list.first[list.tensors], most);
        if (grid == 0) continue;
        p.part = p.all_parts;
        p.all_parts += grid;
        ProfScope ps("clip_squares", st);
        clip_squares_kernel<<<(unsigned)grid, 256, 0, st>>>(list, p);
    }
    for (int l = launches - 1; l >= 0; --l) {
        const bool writes = fill(list, l);
        p.norm = l == 0 ? norm : nullptr;
        int grid = std::min(list.first[list.tensors], most);
        if (!writes) {
            if (l > 0) continue;
            grid = 1;
            list.tensors = 0;
            list.first[0] = 0;
        }
        if (grid == 0 && l > 0) continue;
        ProfScope ps("clip_scale", st);
        clip_scale_kernel<<<(unsigned)std::max(grid, 1), 256, 0, st>>>(list, p);
    }
    return hip_ok();
}

}  // extern "C"
