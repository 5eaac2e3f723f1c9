// C entry points of the router's balance loss (router_balance.cuh).
#include "../../include/stmoe.h"

#include <algorithm>

#include "host_utils.cuh"
#include "router_balance.cuh"

using namespace stmoe_dev;
using namespace stmoe_host;

namespace {

bool bal_args_ok(const void *logits, int dtype, int64_t stride, int64_t tokens, int n_experts, int top_k)
{
    return logits && (dtype == STMOE_F32 || dtype == STMOE_BF16 || dtype == STMOE_F16) && tokens >= 0 && n_experts >= 1 &&
           n_experts <= kBalMaxExperts && top_k >= 1 && top_k <= n_experts && (tokens <= 1 || stride >= n_experts) &&
           tokens <= INT32_MAX / top_k && ((uintptr_t)logits & (dtype == STMOE_F32 ? 3 : 1)) == 0;
}
bool rows_vec(const void *p, int dtype, int64_t stride, int n_experts)
{
    const int v = dtype == STMOE_F32 ? 4 : 8;
    return ((uintptr_t)p & 15) == 0 && stride % v == 0 && n_experts % v == 0;
}
bool overlap(const void *p, int64_t p_stride, const void *q, int64_t q_stride, int64_t tokens, int n_experts, int dtype)
{
    const int64_t eb = dtype == STMOE_F32 ? 4 : 2;
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    const uintptr_t a_end = a + eb * ((tokens - 1) * p_stride + n_experts), b_end = b + eb * ((tokens - 1) * q_stride + n_experts);
    return a < b_end && b < a_end;
}
// lanes that share a row: a power of two with sixteen logits each (one lane with eight for up to eight)
int lanes_per_row(int n_experts)
{
    int l = 1;
    while (l * 16 < n_experts) l *= 2;
    return l;
}
// steps of rows that one CTA would take
int64_t bal_steps(int64_t tokens, int lpr)
{
    const int64_t rows = (int64_t)(kBalThreads / kWarp) * (kWarp / lpr) * kBalRows;
    return (tokens + rows - 1) / rows;
}
// CTAs that a batch is spread over where each has few steps: rows of the workspace, which knows no device
constexpr int kBalOnceCtas = 592;
// Up to kBalAlone steps are left to one CTA, which needs no second launch to add partial sums up.
constexpr int64_t kBalAlone = 2;
// CTAs that it takes for no lane to add more than kBalLaneSteps steps of rows in fp32
int64_t bal_least_ctas(int64_t steps) { return (steps + kBalLaneSteps - 1) / kBalLaneSteps; }
// three CTAs an SM (launch bounds); forward: whole multiples of that where rows are many
int bal_grid(int64_t tokens, int lpr, int sms, bool backward)
{
    const int64_t steps = bal_steps(tokens, lpr);
    if (steps <= kBalAlone) return 1;
    const int64_t once = std::min<int64_t>(steps, std::min(sms * 3, kBalOnceCtas));
    return (int)(backward ? once : (bal_least_ctas(steps) + once - 1) / once * once);
}

template <int DT, int LPR, int N, int kRead> int launch_as(bool backward, const BalanceArgs &a, int grid, int dev, cudaStream_t st)
{
    // more than the default 48 KB of dynamic shared memory: asked for once per device
    static PerDevice<bool> asked[2];
    void (*kernel)(BalanceArgs) = backward ? router_balance_backward_kernel<DT, LPR, N, kRead> : router_balance_kernel<DT, LPR, N, kRead>;
    const int stage = backward ? BalWalk<DT, LPR, N, kRead, false>::stage_bytes() : BalWalk<DT, LPR, N, kRead, true>::stage_bytes();
    const int smem = kRead == kBalScalar ? 0 : kBalDepth * stage;
    bool done = false;
    if (smem)
        if (const int rc = asked[backward].get(dev, &done, [=](bool &) {
                return cuda_status(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            }))
            return rc;
    return launch_behind(kernel, grid, kBalThreads, smem, 1, st, a);
}
template <int DT, int LPR, int N> int launch(bool backward, const BalanceArgs &a, int grid, int dev, cudaStream_t st)
{
    if (!a.vec) return launch_as<DT, LPR, N, kBalScalar>(backward, a, grid, dev, st);
    return a.E == LPR * N ? launch_as<DT, LPR, N, kBalFull>(backward, a, grid, dev, st) : launch_as<DT, LPR, N, kBalVec>(backward, a, grid, dev, st);
}
template <int DT> int launch_lanes(int lpr, bool backward, const BalanceArgs &a, int grid, int dev, cudaStream_t st)
{
    switch (lpr) {
    case 1: return a.E <= 8 ? launch<DT, 1, 8>(backward, a, grid, dev, st) : launch<DT, 1, 16>(backward, a, grid, dev, st);
    case 2: return launch<DT, 2, 16>(backward, a, grid, dev, st);
    case 4: return launch<DT, 4, 16>(backward, a, grid, dev, st);
    case 8: return launch<DT, 8, 16>(backward, a, grid, dev, st);
    default: return launch<DT, 16, 16>(backward, a, grid, dev, st);
    }
}
int launch_typed(int dtype, int lpr, bool backward, const BalanceArgs &a, int grid, int dev, cudaStream_t st)
{
    if (dtype == STMOE_F32) return launch_lanes<0>(lpr, backward, a, grid, dev, st);
    if (dtype == STMOE_BF16) return launch_lanes<1>(lpr, backward, a, grid, dev, st);
    return launch_lanes<4>(lpr, backward, a, grid, dev, st);
}

}  // namespace

extern "C" {

size_t stmoe_router_balance_scratch_bytes(int64_t tokens, int n_experts)
{
    if (n_experts < 1 || n_experts > kBalMaxExperts || tokens < 1 || bal_steps(tokens, lanes_per_row(n_experts)) <= kBalAlone) return 0;
    // the multiple that the grid is rounded up to depends on the device
    const int64_t rows = bal_least_ctas(bal_steps(tokens, lanes_per_row(n_experts))) + kBalOnceCtas;
    return sizeof(float) * (size_t)rows * bal_part_words(n_experts);
}

int stmoe_router_balance(const void *logits, int dtype, int64_t stride, const int32_t *ids, const uint8_t *mask, int64_t tokens,
                         int n_experts, int top_k, float *loss, int32_t *counts, int32_t *rows, void *scratch,
                         size_t scratch_bytes, void *cuda_stream)
{
    if (!bal_args_ok(logits, dtype, stride, tokens, n_experts, top_k) || !ids || !loss || !counts || !rows ||
        !aligned(ids, loss, counts, rows))
        return STMOE_ERR_BAD_ARG;
    const size_t need = stmoe_router_balance_scratch_bytes(tokens, n_experts);
    if (need && (!scratch || ((uintptr_t)scratch & 3) || scratch_bytes < need)) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    const int lpr = lanes_per_row(n_experts), grid = bal_grid(tokens, lpr, sms, false);
    BalanceArgs a{};
    a.logits = logits, a.stride = stride, a.ids = ids, a.mask = mask, a.T = (int)tokens, a.E = n_experts, a.K = top_k;
    a.vec = rows_vec(logits, dtype, stride, n_experts);
    a.part = (float *)scratch, a.ctas = grid, a.loss = loss, a.counts = counts, a.rows = rows;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int rc = launch_typed(dtype, lpr, false, a, grid, dev, st);
    if (rc != STMOE_OK || grid == 1) return rc;
    return launch_behind(router_balance_finish_kernel, kBalFinish, 1024, 0, kBalFinish, st, a);
}

int stmoe_router_balance_backward(const void *logits, int dtype, int64_t stride, const uint8_t *mask, int64_t tokens,
                                  int n_experts, int top_k, const int32_t *counts, const int32_t *rows, const float *grad_loss,
                                  void *grad_logits, int64_t grad_stride, void *cuda_stream)
{
    if (!bal_args_ok(logits, dtype, stride, tokens, n_experts, top_k) || !counts || !rows || !grad_loss ||
        !bal_args_ok(grad_logits, dtype, grad_stride, tokens, n_experts, top_k) || !aligned(counts, rows, grad_loss))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    if (overlap(logits, stride, grad_logits, grad_stride, tokens, n_experts, dtype)) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    const int lpr = lanes_per_row(n_experts), grid = bal_grid(tokens, lpr, sms, true);
    BalanceArgs a{};
    a.logits = logits, a.stride = stride, a.mask = mask, a.T = (int)tokens, a.E = n_experts, a.K = top_k;
    a.vec = rows_vec(logits, dtype, stride, n_experts) && rows_vec(grad_logits, dtype, grad_stride, n_experts);
    a.counts = (int *)counts, a.rows = (int *)rows, a.grad = grad_loss;
    a.dlogits = grad_logits, a.dstride = grad_stride;
    return launch_typed(dtype, lpr, true, a, grid, dev, (cudaStream_t)cuda_stream);
}

}  // extern "C"
