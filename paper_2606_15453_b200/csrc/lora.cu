// C entry points of the adapters of many requests (lora.cuh).
#include "../../include/stmoe.h"

#include <algorithm>
#include <cmath>

#include "host_utils.cuh"
#include "lora_tile.cuh"

using namespace stmoe_dev;
using namespace stmoe_host;

namespace {

bool half_ok(int dtype) { return dtype == STMOE_BF16 || dtype == STMOE_F16; }
int elem_bytes(int dtype) { return dtype == STMOE_F32 ? 4 : 2; }
bool rows_ok(const void *p, int dtype, int64_t stride, int64_t rows, int64_t cols)
{
    return p && (rows <= 1 || stride >= cols) && ((uintptr_t)p & (elem_bytes(dtype) - 1)) == 0;
}
bool rows_vec(const void *p, int dtype, int64_t stride) { return ((uintptr_t)p & 15) == 0 && stride * elem_bytes(dtype) % 16 == 0; }
int64_t up_to(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

constexpr int kMaxLength = 1 << 22;       // of inner and outer: blocks of both are one grid dimension
bool sizes_ok(int64_t tokens, int n, int rank, int inner, int outer)
{
    return tokens >= 0 && tokens <= INT32_MAX / 2 && n >= 1 && n <= kLoraMaxAdapters && rank >= 1 && rank <= kLoraMaxRank && inner >= 1 &&
           inner <= kMaxLength && outer >= 1 && outer <= kMaxLength;
}
// The tile kernels' share.  In a graph, rank 16, 4096 -> 4096 (rank 64, 2048 -> 2816), they take 13 us and half of one for every adapter that has rows, however
// few; the kernels for few rows 7 us and 3 for every 100 rows.  The host does not know which adapters have rows, so the rule takes all of them to
// have some: rows enough for tiles beside a large table that few of them use take the kernels for few rows.  Tiles against few, every adapter with rows: 256 rows of 1 adapter 13.8 : 14.2 (13.4 : 17.1), of 8
// adapters 17.9 : 14.2 (17.3 : 17.1), 384 of 8 18.0 : 19.6 (17.4 : 23.8), 1024 of 8 19 : 35 (19 : 38), 1024 of 64 46 : 35 (42 : 38), 1024 of 256
// 149 : 48 (132 : 63).
bool by_tiles(int64_t tokens, int n_adapters, int rank) { return tokens >= 20 * ((int64_t)n_adapters + 10) && rank <= kTileMaxRank; }
// Parts of the inner dimension: enough CTAs for the GPU where rows are few, two steps to a warp (four to a tile) at least.
int down_splits(int64_t tokens, int n_adapters, int rank, int inner)
{
    if (by_tiles(tokens, n_adapters, rank)) {
        const int64_t most = std::min<int64_t>(kDownMaxSplits, (inner + 255) / 256);
        return (int)std::max<int64_t>(1, std::min<int64_t>(most, 296 / ((tokens + kTileRows - 1) / kTileRows)));
    }
    const int64_t steps = (inner + kLoraStep - 1) / kLoraStep;
    const int64_t most = std::min<int64_t>(16, (steps + 2 * kLoraWarps - 1) / (2 * kLoraWarps));
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, 592 / std::max<int64_t>(1, tokens)));
}
// parts times rows is never more than this, which does not fall as rows grow
int64_t part_bytes(int64_t tokens, int rank) { return up_to((int64_t)sizeof(float) * std::max<int64_t>(tokens, 592) * up_to(rank, 8), 256); }
int grad_task_rows(int64_t tokens) { return (int)std::max<int64_t>(256, up_to((tokens + 15) / 16, kGradPos)); }
int grad_parts(int64_t tokens) { return (int)std::min<int64_t>(32, 2 * tokens / 256); }     // 2 tokens / task rows at most, and does not fall

// more than the default 48 KB of shared memory: asked for once per device
template <typename K> int smem_of(PerDevice<bool> &asked, int dev, K kernel, int bytes)
{
    bool done = false;
    return asked.get(dev, &done, [=](bool &) { return cuda_status(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)); });
}
template <int DT, bool XVEC, bool WVEC> int launch_down_tiles(const LoraArgs &a, int dev, cudaStream_t st)
{
    static PerDevice<bool> asked;
    if (const int rc = smem_of(asked, dev, lora_down_tile_kernel<DT, XVEC, WVEC>, 97 * 1024)) return rc;
    const int tiles = (int)std::min<int64_t>(a.T, a.T / kTileRows + a.n);
    if ((int64_t)tiles * a.splits > INT32_MAX) return STMOE_ERR_TOO_LARGE;
    // the parts of a tile are a cluster, which adds them up: one part is left in memory
    return launch_behind(lora_down_tile_kernel<DT, XVEC, WVEC>, tiles * a.splits, kDownTileThreads, 1024 + down_stages(a.r) * down_stage_bytes(a.r), a.splits, st, a);
}
template <int DT> int launch_down_as(const LoraArgs &a, bool xvec, bool wvec, int dev, cudaStream_t st)
{
    if (by_tiles(a.T, a.n, a.r)) {
        if (xvec) return wvec ? launch_down_tiles<DT, true, true>(a, dev, st) : launch_down_tiles<DT, true, false>(a, dev, st);
        return wvec ? launch_down_tiles<DT, false, true>(a, dev, st) : launch_down_tiles<DT, false, false>(a, dev, st);
    }
    const dim3 grid(a.T, a.splits, (a.r + kLoraRankBlock - 1) / kLoraRankBlock);
    return xvec && wvec ? launch_behind(lora_down_kernel<DT, true>, grid, kLoraThreads, 0, 1, st, a) : launch_behind(lora_down_kernel<DT, false>, grid, kLoraThreads, 0, 1, st, a);
}
int launch_down(LoraArgs &a, int dtype, int dev, cudaStream_t st)
{
    a.splits = down_splits(a.T, a.n, a.r, a.I);
    const int step = by_tiles(a.T, a.n, a.r) ? 64 : kLoraStep, steps = (a.I + step - 1) / step;
    a.steps = (steps + a.splits - 1) / a.splits;
    a.splits = (steps + a.steps - 1) / a.steps;
    const bool xvec = rows_vec(a.x, dtype, a.T > 1 ? a.x_stride : 0) && a.I % 8 == 0;
    const bool wvec = rows_vec(a.a, dtype, a.r > 1 ? a.a_row : 0) && (a.n == 1 || a.a_group % 8 == 0) && a.I % 8 == 0;
    return dtype == STMOE_BF16 ? launch_down_as<1>(a, xvec, wvec, dev, st) : launch_down_as<4>(a, xvec, wvec, dev, st);
}
template <int DT, int DO, int PL, bool WVEC, bool OVEC> int launch_up_tiles(const LoraArgs &a, int dev, int sms, cudaStream_t st)
{
    static PerDevice<bool> asked;
    constexpr auto kernel = lora_up_tile_kernel<DT, DO, PL, WVEC, OVEC>;
    if (const int rc = smem_of(asked, dev, kernel, std::max(up_smem<DO, PL>(64), up_smem<DO, PL>(kTileMaxRank)))) return rc;
    const int64_t units = std::min<int64_t>(a.T, a.T / kTileRows + a.n + 1) * ((a.O + up_cols<DO>() - 1) / up_cols<DO>());
    if (units > INT32_MAX) return STMOE_ERR_TOO_LARGE;
    return launch_behind(kernel, (int)std::min<int64_t>(units, sms), kUpTileThreads, up_smem<DO, PL>(a.r), 1, st, a);
}
template <int DT, int DO, int PL, bool WVEC> int launch_up_tiles(const LoraArgs &a, int dev, int sms, cudaStream_t st)
{
    const bool ovec = a.out_vec && a.O % Elem<DO>::kVec == 0;
    return ovec ? launch_up_tiles<DT, DO, PL, WVEC, true>(a, dev, sms, st) : launch_up_tiles<DT, DO, PL, WVEC, false>(a, dev, sms, st);
}
template <int DT, int DO, int PL> int launch_up_as(const LoraArgs &a, bool vec, int dev, int sms, cudaStream_t st)
{
    if (by_tiles(a.T, a.n, a.r)) return vec ? launch_up_tiles<DT, DO, PL, true>(a, dev, sms, st) : launch_up_tiles<DT, DO, PL, false>(a, dev, sms, st);
    const dim3 grid(a.T, (a.O + kLoraOutBlock - 1) / kLoraOutBlock);
    return vec ? launch_behind(lora_up_kernel<DT, DO, PL, true>, grid, kLoraThreads, 0, 1, st, a)
               : launch_behind(lora_up_kernel<DT, DO, PL, false>, grid, kLoraThreads, 0, 1, st, a);
}
int launch_up(LoraArgs &a, int dtype, int out_dtype, int dev, int sms, cudaStream_t st)
{
    const int64_t tall = a.T > 1;
    a.out_vec = rows_vec(a.out, out_dtype, tall * a.out_stride) && (!a.base || rows_vec(a.base, out_dtype, tall * a.base_stride));
    const bool vec = rows_vec(a.b, dtype, a.O > 1 ? a.b_row : 0) && (a.n == 1 || a.b_group % 8 == 0) && (a.r % 8 == 0 || a.b_padded);
    if (dtype == STMOE_BF16) return out_dtype == STMOE_F32 ? launch_up_as<1, 0, 3>(a, vec, dev, sms, st) : launch_up_as<1, 1, 2>(a, vec, dev, sms, st);
    return out_dtype == STMOE_F32 ? launch_up_as<4, 0, 3>(a, vec, dev, sms, st) : launch_up_as<4, 4, 2>(a, vec, dev, sms, st);
}
// Adds a matrix to a launch of lora_pack_kernel.
void pack(LoraPackArgs &p, int w, const void *from, int64_t group, int64_t row, int64_t groups, int64_t rows, int cols, uint16_t *to)
{
    LoraPackArgs::Matrix &m = p.m[w];
    m.from = (const uint16_t *)from, m.to = to, m.group = group, m.row = row, m.rows = (int)rows, m.cols = cols, m.ld = (int)up_to(cols, 8);
    m.parts = (m.ld + kPackCols - 1) / kPackCols, m.tasks = groups * rows * m.parts;
}
int launch_pack(const LoraPackArgs &p, cudaStream_t st)
{
    const int64_t ctas = (p.m[0].tasks + p.m[1].tasks + p.m[2].tasks + kLoraWarps - 1) / kLoraWarps;
    if (ctas > INT32_MAX) return STMOE_ERR_TOO_LARGE;
    return launch_behind(lora_pack_kernel, (int)ctas, kLoraThreads, 0, 1, st, p);
}
// room for packed rows of `cols`, none where they can be aligned as they are
int64_t pack_bytes(int64_t rows, int cols) { return cols % 8 ? up_to(2 * rows * up_to(cols, 8), 256) : 0; }

template <int DT> int launch_grad(LoraGradPair &p, int dev, cudaStream_t st)
{
    static PerDevice<bool> asked;
    if (const int rc = smem_of(asked, dev, lora_grad_kernel<DT>, kGradSmem)) return rc;
    const LoraGradArgs &a = p.g[p.g[0].grad ? 0 : 1];
    int blocks[2];
    for (int w = 0; w < 2; ++w) blocks[w] = p.g[w].grad ? (p.g[w].C + kGradCols - 1) / kGradCols : 0;
    p.blocks = blocks[0];
    const dim3 grid(a.n + a.T / a.task_rows, blocks[0] + blocks[1], (a.r + kLoraRankBlock - 1) / kLoraRankBlock);
    if (const int rc = launch_behind(lora_grad_kernel<DT>, grid, kLoraThreads, kGradSmem, 1, st, p)) return rc;
    if (a.T <= a.task_rows) return STMOE_OK;    // no adapter has several tasks
    const int64_t size = (int64_t)a.r * std::max(blocks[0] ? p.g[0].C : 0, blocks[1] ? p.g[1].C : 0);
    const dim3 sums(a.n, (unsigned)std::min<int64_t>(256, (size + kLoraThreads - 1) / kLoraThreads), (blocks[0] > 0) + (blocks[1] > 0));
    return launch_behind(lora_grad_sum_kernel<DT>, sums, kLoraThreads, 0, 1, st, p);
}

}  // namespace

extern "C" {

size_t stmoe_lora_scratch_bytes(int64_t tokens, int n_adapters, int rank, int inner, int outer)
{
    if (!sizes_ok(tokens, n_adapters, rank, inner, outer)) return 0;
    return (size_t)(part_bytes(tokens, rank) + pack_bytes(tokens, inner) + pack_bytes((int64_t)n_adapters * rank, inner) + pack_bytes((int64_t)n_adapters * outer, rank));
}

int stmoe_lora(const void *x, int dtype, int64_t x_stride, int64_t tokens, const void *a, int64_t a_group, int64_t a_row, const void *b, int64_t b_group,
               int64_t b_row, int n_adapters, int rank, int inner, int outer, const int32_t *ids, const int32_t *order,
               const int32_t *counts, const int32_t *starts, const float *scale, float alpha, const void *base, int64_t base_stride, void *out, int out_dtype, int64_t out_stride, float *hidden, void *scratch,
               size_t scratch_bytes, void *cuda_stream)
{
    if (!half_ok(dtype) || (out_dtype != dtype && out_dtype != STMOE_F32) || !sizes_ok(tokens, n_adapters, rank, inner, outer) ||
        !rows_ok(x, dtype, x_stride, tokens, inner) || !rows_ok(a, dtype, a_row, rank, inner) || !rows_ok(b, dtype, b_row, outer, rank) ||
        (n_adapters > 1 && (a_group < 0 || b_group < 0)) || !rows_ok(out, out_dtype, out_stride, tokens, outer) ||
        (base && !rows_ok(base, out_dtype, base_stride, tokens, outer)) || !ids || !order || !counts || !starts ||
        !aligned(ids, order, counts, starts) || !aligned(scale, (const float *)hidden))
        return STMOE_ERR_BAD_ARG;
    if (tokens == 0) return STMOE_OK;
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < stmoe_lora_scratch_bytes(tokens, n_adapters, rank, inner, outer)) return STMOE_ERR_BAD_ARG;
    const int xb = elem_bytes(dtype), ob = elem_bytes(out_dtype);
    const bool same = base == out && (tokens == 1 || base_stride == out_stride);
    const Span to{out, out_stride, tokens, outer, ob};
    if (overlap({x, x_stride, tokens, inner, xb}, to) || (base && !same && overlap({base, base_stride, tokens, outer, ob}, to))) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    LoraArgs k{};
    k.x = x, k.x_stride = x_stride, k.a = a, k.b = b, k.a_group = a_group, k.a_row = a_row, k.b_group = b_group, k.b_row = b_row;
    k.order = order, k.ids = ids, k.scale = scale, k.alpha = alpha, k.T = (int)tokens, k.n = n_adapters, k.r = rank, k.I = inner, k.O = outer;
    k.counts = counts, k.starts = starts, k.polls = g_mx4_polls.load(std::memory_order_relaxed), k.rp = (int)up_to(rank, 8), k.part = (float *)scratch;
    k.base = base, k.base_stride = base_stride, k.out = out, k.out_stride = out_stride, k.keep = same, k.hidden = hidden;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (by_tiles(tokens, n_adapters, rank) && (inner % 8 || rank % 8)) {
        LoraPackArgs p{};
        uint8_t *at = (uint8_t *)scratch + part_bytes(tokens, rank);
        const int64_t i8 = up_to(inner, 8), r8 = up_to(rank, 8);
        if (inner % 8) {
            uint16_t *const xs = (uint16_t *)at, *const as = (uint16_t *)(at += pack_bytes(tokens, inner));
            at += pack_bytes((int64_t)n_adapters * rank, inner);
            pack(p, 0, x, 0, x_stride, 1, tokens, inner, xs), pack(p, 1, a, a_group, a_row, n_adapters, rank, inner, as);
            k.x = xs, k.x_stride = i8, k.a = as, k.a_row = i8, k.a_group = rank * i8, k.I = (int)i8;
        }
        if (rank % 8) {
            pack(p, 2, b, b_group, b_row, n_adapters, outer, rank, (uint16_t *)at);
            k.b = at, k.b_row = r8, k.b_group = outer * r8, k.b_padded = true;
        }
        if (const int rc = launch_pack(p, st)) return rc;
    }
    if (const int rc = launch_down(k, dtype, dev, st)) return rc;
    return launch_up(k, dtype, out_dtype, dev, sms, st);
}

size_t stmoe_lora_backward_scratch_bytes(int64_t tokens, int n_adapters, int rank, int inner, int outer)
{
    if (!sizes_ok(tokens, n_adapters, rank, inner, outer)) return 0;
    int64_t n = up_to((int64_t)2 * n_adapters * rank * up_to(outer, 8), 256) + up_to((int64_t)2 * n_adapters * inner * up_to(rank, 8), 256);
    n += part_bytes(tokens, rank) + up_to((int64_t)sizeof(float) * tokens * rank, 256) + pack_bytes(tokens, inner) + pack_bytes(tokens, outer);
    return (size_t)(n + (int64_t)sizeof(float) * grad_parts(tokens) * rank * ((int64_t)inner + outer));
}

int stmoe_lora_backward(const void *grad, int dtype, int64_t grad_stride, const void *x, int64_t x_stride, int64_t tokens, const void *a, int64_t a_group,
                        int64_t a_row, const void *b, int64_t b_group, int64_t b_row, int n_adapters, int rank, int inner, int outer,
                        const int32_t *ids, const int32_t *order, const int32_t *counts, const int32_t *starts, const float *scale, float alpha,
                        const float *hidden, void *grad_x, int64_t grad_x_stride, void *grad_a, void *grad_b, void *scratch, size_t scratch_bytes,
                        void *cuda_stream)
{
    if (!half_ok(dtype) || !sizes_ok(tokens, n_adapters, rank, inner, outer) || !rows_ok(grad, dtype, grad_stride, tokens, outer) ||
        !rows_ok(x, dtype, x_stride, tokens, inner) || !rows_ok(a, dtype, a_row, rank, inner) || !rows_ok(b, dtype, b_row, outer, rank) ||
        (n_adapters > 1 && (a_group < 0 || b_group < 0)) || !rows_ok(grad_x, dtype, grad_x_stride, tokens, inner) ||
        !ids || !order || !counts || !starts || (grad_b && !hidden) || !aligned(ids, order, counts, starts) || !aligned(scale, hidden) ||
        !aligned((const uint16_t *)grad_a, (const uint16_t *)grad_b))
        return STMOE_ERR_BAD_ARG;
    const size_t need = stmoe_lora_backward_scratch_bytes(tokens, n_adapters, rank, inner, outer);
    if (!scratch || ((uintptr_t)scratch & 255) || scratch_bytes < need) return STMOE_ERR_BAD_ARG;
    const Span to{grad_x, grad_x_stride, tokens, inner, 2};
    if (overlap({x, x_stride, tokens, inner, 2}, to) || overlap({grad, grad_stride, tokens, outer, 2}, to)) return STMOE_ERR_BAD_ARG;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (tokens == 0) {
        // lora_grad_kernel would write the zeros too, but it reads the counts ahead of its wait, which only a kernel of this call before it makes right
        if (grad_a)
            if (const int rc = cuda_status(cudaMemsetAsync(grad_a, 0, (size_t)2 * n_adapters * rank * inner, st))) return rc;
        return grad_b ? cuda_status(cudaMemsetAsync(grad_b, 0, (size_t)2 * n_adapters * rank * outer, st)) : STMOE_OK;
    }
    uint8_t *at = (uint8_t *)scratch;
    auto take = [&](int64_t bytes) { uint8_t *p = at; at += up_to(bytes, 256); return p; };
    const int64_t outer8 = up_to(outer, 8), rank8 = up_to(rank, 8);
    uint16_t *const bt = (uint16_t *)take((int64_t)2 * n_adapters * rank * outer8), *const a_t = (uint16_t *)take((int64_t)2 * n_adapters * inner * rank8);
    float *const part = (float *)take(part_bytes(tokens, rank)), *const u = (float *)take((int64_t)sizeof(float) * tokens * rank);
    const bool tiles = by_tiles(tokens, n_adapters, rank), packed = tiles && outer % 8;
    if (tiles && (inner % 8 || outer % 8)) {
        LoraPackArgs p{};
        if (packed) {
            uint16_t *const to = (uint16_t *)take(pack_bytes(tokens, outer));
            pack(p, 0, grad, 0, grad_stride, 1, tokens, outer, to);
            grad = to, grad_stride = outer8;
        }
        if (inner % 8) {
            uint16_t *const to = (uint16_t *)take(pack_bytes(tokens, inner));
            pack(p, 1, x, 0, x_stride, 1, tokens, inner, to);
            x = to, x_stride = up_to(inner, 8);
        }
        if (const int rc = launch_pack(p, st)) return rc;
    }
    float *const parts = (float *)at;
    LoraTransposeArgs t{{(const uint16_t *)b, (const uint16_t *)a}, {bt, a_t}, {b_group, a_group}, {b_row, a_row}, {outer8, rank8}, {outer, rank}, {rank, inner}, {}};
    for (int w = 0; w < 2; ++w) t.tiles[w] = ((t.rows[w] + 31) / 32) * ((t.cols[w] + 31) / 32);
    if (const int rc = launch_behind(lora_transpose_kernel, dim3(t.tiles[0] + t.tiles[1], n_adapters), kLoraThreads, 0, 1, st, t)) return rc;
    // the forward kernels with the roles of A and B exchanged
    LoraArgs k{};
    k.x = grad, k.x_stride = grad_stride, k.a = bt, k.a_row = outer8, k.a_group = rank * outer8, k.b = a_t, k.b_row = rank8, k.b_group = inner * rank8;
    k.order = order, k.ids = ids, k.scale = scale, k.alpha = alpha, k.T = (int)tokens, k.n = n_adapters, k.r = rank, k.O = inner;
    k.I = packed ? (int)outer8 : outer, k.b_padded = true;       // zeros behind the rows of bt and a_t, and of grad where it was packed
    k.counts = counts, k.starts = starts, k.polls = g_mx4_polls.load(std::memory_order_relaxed), k.rp = (int)up_to(rank, 8), k.part = part;
    k.out = grad_x, k.out_stride = grad_x_stride, k.hidden = u, k.early = true;
    if (const int rc = launch_down(k, dtype, dev, st)) return rc;
    if (const int rc = launch_up(k, dtype, dtype, dev, sms, st)) return rc;
    if (!grad_a && !grad_b) return STMOE_OK;
    LoraGradPair p{};
    for (int w = 0; w < 2; ++w) {
        LoraGradArgs &g = p.g[w];
        g.order = order, g.counts = counts, g.starts = starts, g.scale = scale, g.alpha = alpha, g.T = (int)tokens, g.n = n_adapters, g.r = rank;
        g.task_rows = grad_task_rows(tokens), g.parts = grad_parts(tokens), g.by_col = w == 1;
        g.u = w ? hidden : u, g.z = w ? grad : x, g.z_stride = w ? grad_stride : x_stride, g.C = w ? outer : inner, g.grad = w ? grad_b : grad_a;
        g.part = parts + (w ? (int64_t)g.parts * rank * inner : 0);
        g.u_vec = rank % 4 == 0 && ((uintptr_t)g.u & 15) == 0, g.vec = rows_vec(g.z, dtype, tokens > 1 ? g.z_stride : 0);
    }
    return dtype == STMOE_BF16 ? launch_grad<1>(p, dev, st) : launch_grad<4>(p, dev, st);
}

}  // extern "C"
