// C entry points of the choice of experts (router_select.cuh).
#include "../../include/stmoe.h"

#include <algorithm>
#include <cmath>

#include "host_utils.cuh"
#include "router_select.cuh"

using namespace stmoe_dev;
using namespace stmoe_host;

namespace {

bool sel_args_ok(const void *logits, int dtype, int64_t stride, int64_t tokens, int n_experts, int top_k)
{
    return logits && (dtype == STMOE_F32 || dtype == STMOE_BF16 || dtype == STMOE_F16) && tokens >= 0 && n_experts >= 1 &&
           n_experts <= kSelMaxExperts && top_k >= 1 && top_k <= n_experts && top_k <= kSelMaxK && (tokens <= 1 || stride >= n_experts) &&
           tokens <= INT32_MAX / top_k && ((uintptr_t)logits & (dtype == STMOE_F32 ? 3 : 1)) == 0;
}
bool rows_vec(const void *p, int dtype, int64_t stride) { return ((uintptr_t)p & 15) == 0 && stride % (dtype == STMOE_F32 ? 4 : 8) == 0; }

template <int DT, int LPR> int launch(bool backward, const SelectArgs &a, cudaStream_t st)
{
    constexpr int rows = kSelThreads / LPR;
    void (*kernel)(SelectArgs) = backward ? router_select_backward_kernel<DT, LPR> : router_select_kernel<DT, LPR>;
    return launch_behind(kernel, (int)(((int64_t)a.T + rows - 1) / rows), kSelThreads, 0, 1, st, a);
}
// A warp a row, in turns: four CTAs an SM, as the kernel's registers allow.
template <int DT> int launch_wide(const SelectArgs &a, int sms, cudaStream_t st)
{
    const int64_t ctas = ((int64_t)a.T + kSelThreads / kWarp - 1) / (kSelThreads / kWarp);
    return launch_behind(router_select_wide_kernel<DT>, (int)std::min<int64_t>(ctas, sms * 4), kSelThreads, 0, 1, st, a);
}
// whether groups are whole lanes of a row of LPR = 32
bool whole_groups(const SelectArgs &a)
{
    const int gs = a.E / a.G, lg = gs / kSelN;
    return a.G == 1 || (gs % kSelN == 0 && (lg & (lg - 1)) == 0);
}
// a lane a choice: up to four rows a warp
template <int DT> int launch_sparse_backward(const SelectArgs &a, int sms, cudaStream_t st)
{
    int kp = 1;
    while (kp < a.K) kp *= 2;
    const int rows = std::min(4, kWarp / kp), per = kSelThreads / kWarp * rows;
    return launch_behind(router_select_sparse_backward_kernel<DT>, (int)std::min<int64_t>(((int64_t)a.T + per - 1) / per, sms * 6), kSelThreads, 0, 1, st, a, kp, rows);
}
// lanes that share a row: a power of two with eight logits each
template <int DT> int launch_lanes(bool backward, const SelectArgs &a, int sms, cudaStream_t st)
{
    if (backward && (a.sigmoid || a.renorm)) return launch_sparse_backward<DT>(a, sms, st);
    if (a.E <= 8) return launch<DT, 1>(backward, a, st);
    if (a.E <= 16) return launch<DT, 2>(backward, a, st);
    if (a.E <= 32) return launch<DT, 4>(backward, a, st);
    if (a.E <= 64) return launch<DT, 8>(backward, a, st);
    if (a.E <= 128) return launch<DT, 16>(backward, a, st);
    if (!backward && whole_groups(a)) return launch_wide<DT>(a, sms, st);
    return launch<DT, 32>(backward, a, st);
}
int launch_typed(int dtype, bool backward, const SelectArgs &a, int sms, cudaStream_t st)
{
    if (dtype == STMOE_F32) return launch_lanes<0>(backward, a, sms, st);
    if (dtype == STMOE_BF16) return launch_lanes<1>(backward, a, sms, st);
    return launch_lanes<4>(backward, a, sms, st);
}

}  // namespace

extern "C" {

int stmoe_router_select(const void *logits, int dtype, int64_t stride, const float *bias, const uint8_t *mask, int64_t tokens, int n_experts,
                        int top_k, int n_groups, int top_groups, int group_best, int flags, float scale, int32_t *ids, float *w, void *cuda_stream)
{
    if (!sel_args_ok(logits, dtype, stride, tokens, n_experts, top_k) || n_groups < 1 || n_groups > kSelMaxGroups || n_experts % n_groups ||
        top_groups < 1 || top_groups > n_groups || group_best < 1 || group_best > 2 || (flags & ~(STMOE_SELECT_SIGMOID | STMOE_SELECT_RENORM)) ||
        !std::isfinite(scale) || !ids || !w || !aligned(ids, w, bias))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    SelectArgs a{};
    a.logits = logits, a.stride = stride, a.bias = bias, a.mask = mask, a.T = (int)tokens, a.E = n_experts, a.K = top_k;
    // all groups stay: nothing to rank
    a.G = top_groups == n_groups ? 1 : n_groups, a.top_groups = top_groups, a.best = group_best;
    a.vec = rows_vec(logits, dtype, stride), a.sigmoid = flags & STMOE_SELECT_SIGMOID, a.renorm = flags & STMOE_SELECT_RENORM;
    a.exact = !bias && (a.G == 1 || group_best == 1);
    a.scale = scale, a.ids = ids, a.w = w;
    return launch_typed(dtype, false, a, sms, (cudaStream_t)cuda_stream);
}

int stmoe_router_select_backward(const void *logits, int dtype, int64_t stride, int64_t tokens, int n_experts, int top_k, int flags, float scale,
                                 const int32_t *ids, const float *w, const float *grad_w, void *grad_logits, int64_t grad_stride, void *cuda_stream)
{
    if (!sel_args_ok(logits, dtype, stride, tokens, n_experts, top_k) || !sel_args_ok(grad_logits, dtype, grad_stride, tokens, n_experts, top_k) ||
        (flags & ~(STMOE_SELECT_SIGMOID | STMOE_SELECT_RENORM)) || !std::isfinite(scale) || !ids || !w || !grad_w || !aligned(ids, w, grad_w))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    const int bytes = dtype == STMOE_F32 ? 4 : 2;
    if (overlap({logits, stride, tokens, n_experts, bytes}, {grad_logits, grad_stride, tokens, n_experts, bytes})) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    SelectArgs a{};
    a.logits = logits, a.stride = stride, a.T = (int)tokens, a.E = n_experts, a.K = top_k;
    a.vec = rows_vec(logits, dtype, stride) && rows_vec(grad_logits, dtype, grad_stride);
    a.sigmoid = flags & STMOE_SELECT_SIGMOID, a.renorm = flags & STMOE_SELECT_RENORM, a.scale = scale;
    a.ids = (int *)ids, a.w = (float *)w, a.grad = grad_w, a.dlogits = grad_logits, a.dstride = grad_stride;
    return launch_typed(dtype, true, a, sms, (cudaStream_t)cuda_stream);
}

}  // extern "C"
