// C entry points of grouping, dispatch and combination of rows (group_rows.cuh).
#include "../../include/stmoe.h"

#include <algorithm>
#include <cmath>

#include "group_rows.cuh"
#include "host_utils.cuh"

using namespace stmoe_dev;
using namespace stmoe_host;

namespace {

bool pairs_ok(int64_t rows, int top_k) { return rows >= 0 && top_k >= 1 && rows <= INT32_MAX / top_k; }
bool group_ok(int64_t rows, int top_k) { return pairs_ok(rows, top_k) && rows * top_k <= 1 << 30; }     // a warp's last position stays an int
bool elem_ok(int dtype) { return dtype == STMOE_F32 || dtype == STMOE_BF16 || dtype == STMOE_F16; }
int elem_bytes(int dtype) { return dtype == STMOE_F32 ? 4 : 2; }
// One CTA, a cluster of up to eight, or CTAs on their own that count in a launch before.  A CTA by itself takes 4096 pairs, one of many 1024.
bool in_cluster(int64_t pairs) { return pairs <= kGrpCtaPairs * kGrpCluster; }
int group_ctas(int64_t pairs)
{
    if (in_cluster(pairs)) return pairs <= kGrpCtaPairs ? 1 : kGrpCluster;
    return (int)std::min<int64_t>(kGrpMaxCtas, (pairs + 1023) / 1024);
}
bool rows_ok(const void *p, int dtype, int64_t stride, int64_t rows, int64_t cols)
{
    return p && elem_ok(dtype) && (rows <= 1 || stride >= cols) && ((uintptr_t)p & (elem_bytes(dtype) - 1)) == 0;
}
bool rows_vec(const void *p, int dtype, int64_t stride) { return ((uintptr_t)p & 15) == 0 && stride * elem_bytes(dtype) % 16 == 0; }

// Pieces of 256 columns that a warp has: four, or one where that would leave SMs without work (fewer than a wave of 148 x 8 CTAs)
int64_t combine_parts(int64_t tokens, int64_t cols, int pieces) { return tokens * ((cols + pieces * 8 * kWarp - 1) / (pieces * 8 * kWarp)); }
int combine_pieces(int64_t tokens, int64_t cols) { return combine_parts(tokens, cols, 4) >= 148 * 8 * (kRowThreads / kWarp) ? 4 : 1; }

template <int DY, int DO> int launch_combine(const CombineArgs &a, cudaStream_t st)
{
    constexpr int kWarps = kRowThreads / kWarp;
    const int ctas = (int)(((int64_t)a.T * a.parts + kWarps - 1) / kWarps);
    if (combine_pieces(a.T, a.C) == 4) return launch_behind(combine_rows_kernel<DY, DO, 4>, ctas, kRowThreads, 0, 1, st, a);
    return launch_behind(combine_rows_kernel<DY, DO, 1>, ctas, kRowThreads, 0, 1, st, a);
}
template <int DY, int DG, int WPT> int launch_combine_backward_of(const CombineArgs &a, cudaStream_t st)
{
    constexpr int kTokens = kRowThreads / kWarp / WPT;
    const int ctas = (a.T + kTokens - 1) / kTokens;
    if (a.K <= 2) return launch_behind(combine_rows_backward_kernel<DY, DG, WPT, 2>, ctas, kRowThreads, 0, 1, st, a);
    return launch_behind(combine_rows_backward_kernel<DY, DG, WPT, 4>, ctas, kRowThreads, 0, 1, st, a);
}
// Eight warps a token where rows are long, four where tokens are too few to fill the GPU's 148 x 64 warps, else one.
template <int DY, int DG> int launch_combine_backward(const CombineArgs &a, cudaStream_t st)
{
    if (a.C > 4 * 8 * kWarp) return launch_combine_backward_of<DY, DG, 8>(a, st);
    if (a.C > 8 * kWarp && a.T < 148 * 64) return launch_combine_backward_of<DY, DG, 4>(a, st);
    return launch_combine_backward_of<DY, DG, 1>(a, st);
}
template <bool backward, int DY, int DO> int launch_as(const CombineArgs &a, cudaStream_t st)
{
    if constexpr (backward) return launch_combine_backward<DY, DO>(a, st);
    else return launch_combine<DY, DO>(a, st);
}
template <bool backward> int launch_typed(int y_dtype, int dtype, const CombineArgs &a, cudaStream_t st)
{
    if (y_dtype == STMOE_F32) return launch_as<backward, 0, 0>(a, st);
    if (y_dtype == STMOE_BF16) return dtype == STMOE_F32 ? launch_as<backward, 1, 0>(a, st) : launch_as<backward, 1, 1>(a, st);
    return dtype == STMOE_F32 ? launch_as<backward, 4, 0>(a, st) : launch_as<backward, 4, 4>(a, st);
}

}  // namespace

extern "C" {

size_t stmoe_group_rows_scratch_bytes(int64_t rows, int top_k, int n_groups)
{
    if (!group_ok(rows, top_k) || n_groups < 1 || n_groups > kGrpMaxGroups) return 0;
    const int ctas = group_ctas(rows * top_k);
    return in_cluster(rows * top_k) ? 0 : sizeof(int) * (size_t)ctas * (n_groups + 1);
}

int stmoe_group_rows(const int32_t *ids, int64_t rows, int top_k, int n_groups, int32_t *counts, int32_t *starts, int32_t *order,
                     int32_t *slots, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    if (!ids || !group_ok(rows, top_k) || n_groups < 1 || n_groups > kGrpMaxGroups || !counts || !starts || !order || !slots ||
        !aligned(ids, counts, starts, order, slots))
        return STMOE_ERR_BAD_ARG;
    const size_t need = stmoe_group_rows_scratch_bytes(rows, top_k, n_groups);
    if (need && (!scratch || ((uintptr_t)scratch & 3) || scratch_bytes < need)) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    GroupArgs a{};
    a.ids = ids, a.pairs = (int)(rows * top_k), a.G = n_groups;
    a.counts = counts, a.starts = starts, a.order = order, a.slots = slots;
    const int ctas = std::max(1, group_ctas(a.pairs));
    a.per_warp = (int)(((int64_t)a.pairs + (int64_t)ctas * kGrpWarps * kWarp - 1) / ((int64_t)ctas * kGrpWarps * kWarp)) * kWarp;
    const bool cluster = in_cluster(a.pairs);
    a.hist = cluster ? nullptr : (int *)scratch;
    const int smem = (int)sizeof(int) * (kGrpWarps + 2) * (n_groups + 1);
    static PerDevice<bool> asked;       // more than 48 KB of dynamic shared memory: asked for once per device
    bool done = false;
    if (const int rc = asked.get(dev, &done, [](bool &) {
            const int most = (int)sizeof(int) * (kGrpWarps + 2) * (kGrpMaxGroups + 1);
            if (const int rc = cuda_status(cudaFuncSetAttribute(group_count_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most))) return rc;
            return cuda_status(cudaFuncSetAttribute(group_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
        }))
        return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!cluster)
        if (const int rc = launch_behind(group_count_kernel, ctas, kGrpThreads, smem, 1, st, a)) return rc;
    return launch_behind(group_place_kernel, ctas, kGrpThreads, smem, cluster ? ctas : 1, st, a);
}

int stmoe_dispatch_rows(const void *x, int64_t row_bytes, int64_t x_stride, int64_t rows, int top_k, const int32_t *slots, const int32_t *n_rows,
                        void *out, int64_t out_rows, int64_t out_stride, void *cuda_stream)
{
    if (!x || !out || !slots || !pairs_ok(rows, top_k) || row_bytes < 1 || row_bytes > INT32_MAX || out_rows < 0 || out_rows > INT32_MAX ||
        (rows > 1 && x_stride < row_bytes) || (out_rows > 1 && out_stride < row_bytes) || !aligned(slots, n_rows))
        return STMOE_ERR_BAD_ARG;
    if (rows == 0) return STMOE_OK;
    if (overlap({x, x_stride, rows, row_bytes, 1}, {out, out_stride, out_rows, row_bytes, 1})) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    DispatchArgs a{};
    a.x = (const uint8_t *)x, a.x_stride = rows > 1 ? x_stride : 0, a.out = (uint8_t *)out, a.out_stride = out_rows > 1 ? out_stride : 0;
    a.row_bytes = row_bytes, a.slots = slots, a.rows = n_rows, a.T = (int)rows, a.K = top_k, a.out_rows = (int)out_rows;
    const uint64_t all = (uintptr_t)x | (uintptr_t)out | (uint64_t)a.x_stride | (uint64_t)a.out_stride | (uint64_t)row_bytes;
    const int unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : all % 2 == 0 ? 2 : 1;
    a.parts = (unsigned)((row_bytes / unit + 4 * kWarp - 1) / (4 * kWarp));
    if ((int64_t)a.T * a.parts >= INT32_MAX) return STMOE_ERR_TOO_LARGE;
    const int ctas = (int)(((int64_t)a.T * a.parts * kWarp + kRowThreads - 1) / kRowThreads);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (unit) {
    case 16: return launch_behind(dispatch_rows_kernel<uint4>, ctas, kRowThreads, 0, 1, st, a);
    case 4: return launch_behind(dispatch_rows_kernel<uint32_t>, ctas, kRowThreads, 0, 1, st, a);
    case 2: return launch_behind(dispatch_rows_kernel<uint16_t>, ctas, kRowThreads, 0, 1, st, a);
    default: return launch_behind(dispatch_rows_kernel<uint8_t>, ctas, kRowThreads, 0, 1, st, a);
    }
}

int stmoe_combine_rows(const void *y, int y_dtype, int64_t y_stride, int64_t y_rows, const int32_t *slots, const float *w, const void *residual,
                       int64_t residual_stride, float scale, int64_t tokens, int top_k, int64_t cols, void *out, int out_dtype,
                       int64_t out_stride, void *cuda_stream)
{
    if (!pairs_ok(tokens, top_k) || cols < 1 || cols > INT32_MAX / 2 || y_rows < 0 || y_rows > INT32_MAX || !slots || !aligned(slots, w) ||
        !rows_ok(y, y_dtype, y_stride, y_rows, cols) || !rows_ok(out, out_dtype, out_stride, tokens, cols) ||
        (residual && !rows_ok(residual, out_dtype, residual_stride, tokens, cols)) || (out_dtype != y_dtype && out_dtype != STMOE_F32))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    const int yb = elem_bytes(y_dtype), ob = elem_bytes(out_dtype);
    const Span to{out, out_stride, tokens, cols, ob};
    const bool same = residual == out && (tokens == 1 || residual_stride == out_stride);
    if (overlap({y, y_stride, y_rows, cols, yb}, to) || (residual && !same && overlap({residual, residual_stride, tokens, cols, ob}, to)))
        return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    CombineArgs a{};
    a.y = y, a.y_stride = y_stride, a.y_rows = (int)y_rows, a.slots = slots, a.w = w, a.res = residual, a.res_stride = residual_stride;
    a.scale = scale, a.T = (int)tokens, a.K = top_k, a.C = (int)cols, a.out = out, a.out_stride = out_stride;
    a.vec = rows_vec(y, y_dtype, y_stride) && rows_vec(out, out_dtype, out_stride) && (!residual || rows_vec(residual, out_dtype, residual_stride));
    a.parts = (unsigned)(combine_parts(tokens, cols, combine_pieces(tokens, cols)) / tokens);
    if ((int64_t)a.T * a.parts >= INT32_MAX) return STMOE_ERR_TOO_LARGE;
    return launch_typed<false>(y_dtype, out_dtype, a, (cudaStream_t)cuda_stream);
}

int stmoe_combine_rows_backward(const void *grad, int grad_dtype, int64_t grad_stride, const void *y, int y_dtype, int64_t y_stride, int64_t y_rows,
                                const int32_t *slots, const float *w, float scale, int64_t tokens, int top_k, int64_t cols, const int32_t *n_rows,
                                void *grad_y, int64_t grad_y_stride, float *grad_w, void *cuda_stream)
{
    if (!pairs_ok(tokens, top_k) || cols < 1 || cols > INT32_MAX / 2 || y_rows < 0 || y_rows > INT32_MAX || !slots || !aligned(slots, n_rows) ||
        !aligned(w, (const float *)grad_w) || !rows_ok(y, y_dtype, y_stride, y_rows, cols) || !rows_ok(grad, grad_dtype, grad_stride, tokens, cols) ||
        !rows_ok(grad_y, y_dtype, grad_y_stride, y_rows, cols) || (grad_dtype != y_dtype && grad_dtype != STMOE_F32))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    const int yb = elem_bytes(y_dtype), gb = elem_bytes(grad_dtype);
    const Span to{grad_y, grad_y_stride, y_rows, cols, yb};
    if (overlap({y, y_stride, y_rows, cols, yb}, to) || overlap({grad, grad_stride, tokens, cols, gb}, to)) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    CombineArgs a{};
    a.y = y, a.y_stride = y_stride, a.y_rows = (int)y_rows, a.slots = slots, a.w = w, a.res = grad, a.res_stride = grad_stride, a.rows = n_rows;
    a.scale = scale, a.T = (int)tokens, a.K = top_k, a.C = (int)cols, a.out = grad_y, a.out_stride = grad_y_stride, a.dw = grad_w;
    a.vec = rows_vec(y, y_dtype, y_stride) && rows_vec(grad, grad_dtype, grad_stride) && rows_vec(grad_y, y_dtype, grad_y_stride);
    return launch_typed<true>(y_dtype, grad_dtype, a, (cudaStream_t)cuda_stream);
}

}  // extern "C"
