// C entry points of the MX4 operators (mx4.cuh, mx4_matmul.cuh).
#include "../../include/stmoe.h"

#include <algorithm>

#include "host_utils.cuh"
#include "mx4.cuh"
#include "mx4_matmul.cuh"

using namespace stmoe_dev;
using namespace stmoe_host;

namespace {

bool elem_type(int dtype) { return dtype == STMOE_F32 || dtype == STMOE_BF16 || dtype == STMOE_F16; }
long long elem_bytes(int dtype) { return dtype == STMOE_F32 ? 4 : 2; }

template <int DT, bool kVec, bool kPack> int launch_rows_as(bool quantize, const Mx4Rows &a, int64_t warps, int sms, cudaStream_t st)
{
    const int64_t ctas = (warps + kMxThreads / kWarp - 1) / (kMxThreads / kWarp);
    const int grid = (int)std::min<int64_t>(ctas, (int64_t)sms * (quantize ? mx4_quantize_ctas<DT, kVec>() : 8));
    return launch_behind(quantize ? mx4_quantize_kernel<DT, kVec, kPack> : mx4_dequantize_kernel<DT, kVec, kPack>, grid, kMxThreads, 0, 1, st, a);
}
template <int DT> int launch_rows(bool quantize, const Mx4Rows &a, int64_t warps, int sms, cudaStream_t st)
{
    if (a.vec)
        return a.pack > 1 ? launch_rows_as<DT, true, true>(quantize, a, warps, sms, st) : launch_rows_as<DT, true, false>(quantize, a, warps, sms, st);
    return a.pack > 1 ? launch_rows_as<DT, false, true>(quantize, a, warps, sms, st) : launch_rows_as<DT, false, false>(quantize, a, warps, sms, st);
}

int mx4_rows(bool quantize, void *x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, uint8_t *codes,
             int64_t code_stride, uint8_t *scales, int64_t scale_stride, void *cuda_stream)
{
    if (!x || !codes || !scales || !elem_type(dtype) || rows < 0 || cols < 1) return STMOE_ERR_BAD_ARG;
    const int64_t nb = (cols - 1) / kMxBlock + 1;
    if ((rows > 1 && (x_stride < cols || code_stride < nb * 16 || code_stride % 4 || scale_stride < nb)) ||
        ((uintptr_t)codes & 3) || ((uintptr_t)x & (elem_bytes(dtype) - 1)))
        return STMOE_ERR_BAD_ARG;
    if (rows == 0) return STMOE_OK;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    Mx4Rows a{};
    a.x = x, a.codes = codes, a.scales = scales, a.rows = rows, a.cols = cols;
    a.x_stride = x_stride, a.code_stride = code_stride, a.scale_stride = scale_stride;
    // rows without gaps whose blocks do not straddle them are one long row: short rows then fill
    // their warps (a warp takes 1024 elements)
    if (rows > 1 && cols % kMxBlock == 0 && x_stride == cols && code_stride == nb * 16 && scale_stride == nb)
        a.rows = 1, a.cols = rows * cols;
    a.vec = ((uintptr_t)x & 15) == 0 && (a.rows == 1 || (x_stride * elem_bytes(dtype)) % 16 == 0);
    const int64_t padded = (a.cols + kMxBlock - 1) / kMxBlock * kMxBlock;
    a.pack = padded <= kMxSeg / 2 ? (int)(kMxSeg / padded) : 1;
    const int64_t tasks = (a.rows + a.pack - 1) / a.pack * ((a.cols - 1) / kMxSeg + 1);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == STMOE_F32) return launch_rows<0>(quantize, a, tasks, sms, st);
    if (dtype == STMOE_BF16) return launch_rows<1>(quantize, a, tasks, sms, st);
    return launch_rows<4>(quantize, a, tasks, sms, st);
}

// codes [rows][row_bytes]: boxes of 128 bytes x box_rows rows, 128-byte swizzle, zeros outside
int encode_codes(EncodeTiledFn fn, CUtensorMap *m, const uint8_t *base, int64_t rows, int64_t row_bytes, int64_t stride, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, es[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void *)base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? STMOE_OK
               : STMOE_ERR_CUDA;
}

// once per device: the kernels' shared memory, and how many of their clusters run at a time (the same for
// the three output types)
int matmul_clusters(int dev, MmClusters *c)
{
    static PerDevice<MmClusters> kept;
    return kept.get(dev, c, [](MmClusters &m) {
        for (const void *k : {(const void *)mx4_matmul_kernel<0>, (const void *)mx4_matmul_kernel<1>, (const void *)mx4_matmul_kernel<4>})
            if (const int rc = cuda_status(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmSmemBytes))) return rc;
        return mm_clusters(mx4_matmul_kernel<0>, kMmThreads, &m) ? STMOE_OK : STMOE_ERR_CUDA;
    });
}

template <int ODT>
int launch_matmul(const CUtensorMap &ma, const CUtensorMap &mb, const Mx4MatmulArgs &a, int grid, cudaStream_t st)
{
    return launch_behind(mx4_matmul_kernel<ODT>, grid, kMmThreads, kMmSmemBytes, a.splits, st, ma, mb, a);
}

}  // namespace

extern "C" {

int stmoe_mx4_quantize(const void *x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, uint8_t *codes,
                       int64_t code_stride, uint8_t *scales, int64_t scale_stride, void *cuda_stream)
{
    return mx4_rows(true, (void *)x, dtype, rows, cols, x_stride, codes, code_stride, scales, scale_stride, cuda_stream);
}

int stmoe_mx4_dequantize(const uint8_t *codes, int64_t code_stride, const uint8_t *scales, int64_t scale_stride, int64_t rows,
                         int64_t cols, void *x, int dtype, int64_t x_stride, void *cuda_stream)
{
    return mx4_rows(false, x, dtype, rows, cols, x_stride, (uint8_t *)codes, code_stride, (uint8_t *)scales, scale_stride,
                    cuda_stream);
}

int stmoe_mx4_matmul(const uint8_t *a_codes, int64_t a_code_stride, const uint8_t *a_scales, int64_t a_scale_stride, int64_t m,
                     const uint8_t *b_codes, int64_t b_code_stride, const uint8_t *b_scales, int64_t b_scale_stride,
                     int n_groups, int n, int k_blocks, const int32_t *counts, void *out, int out_dtype,
                     int64_t out_stride, uint32_t *flags, void *cuda_stream)
{
    const int64_t row_bytes = (int64_t)k_blocks * 16;
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out || !elem_type(out_dtype) || m < 0 || m > INT32_MAX - 256 ||
        n < 1 || n > (1 << 24) || k_blocks < 1 || k_blocks > (1 << 20) || n_groups < 1 || n_groups > kMmMaxGroups ||
        (n_groups > 1 && !counts) || (int64_t)n_groups * n > INT32_MAX - 256 || ((uintptr_t)a_codes & 15) ||
        ((uintptr_t)b_codes & 15) || (m > 1 && (a_code_stride % 16 || a_code_stride < row_bytes)) ||
        ((int64_t)n_groups * n > 1 && (b_code_stride % 16 || b_code_stride < row_bytes)) || (m > 1 && a_scale_stride < k_blocks) ||
        ((int64_t)n_groups * n > 1 && b_scale_stride < k_blocks) || (m > 1 && out_stride < n) || ((uintptr_t)out & (elem_bytes(out_dtype) - 1)) ||
        !aligned(counts, flags))
        return STMOE_ERR_BAD_ARG;
    if (m == 0) return STMOE_OK;
    int dev = 0, sms = 0;
    if (const int rc = current_device(&dev, &sms)) return rc;
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return STMOE_ERR_CUDA;

    Mx4MatmulArgs a{};
    a.a_scales = a_scales, a.b_scales = b_scales, a.a_scale_stride = a_scale_stride, a.b_scale_stride = b_scale_stride;
    a.counts = counts, a.groups = n_groups, a.m = (int)m, a.n = n, a.blocks = k_blocks;
    a.out = out, a.out_stride = out_stride, a.err = flags, a.polls = g_mx4_polls.load(std::memory_order_relaxed);
    a.out_wide = ((uintptr_t)out & 15) == 0 && (m == 1 || (out_stride * elem_bytes(out_dtype)) % 16 == 0);
    const auto align = [](const void *p, int64_t stride) {
        const uint64_t bits = (uint64_t)(uintptr_t)p | (uint64_t)stride;
        return bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 1;
    };
    a.a_align = align(a_scales, m > 1 ? a_scale_stride : 0), a.b_align = align(b_scales, b_scale_stride);
    const int64_t mean = (m + n_groups - 1) / n_groups;
    a.bn = mean <= 16 ? 16 : mean <= 32 ? 32 : mean <= 64 ? 64 : mean <= 128 ? 128 : kMmMaxTokens;
    const int64_t row_tiles = (n + kMmRows - 1) / kMmRows;
    // token tiles: at most one part-filled tile per group beyond the full ones
    const int64_t tok_tiles = std::min<int64_t>(m, m / a.bn + n_groups);
    const int64_t tasks = row_tiles * tok_tiles;
    if (tasks > INT32_MAX - 4096) return STMOE_ERR_TOO_LARGE;
    const int steps = (k_blocks + kMmStageBlocks - 1) / kMmStageBlocks;
    MmClusters clusters;
    const int rc = matmul_clusters(dev, &clusters);
    if (rc != STMOE_OK) return rc;
    a.splits = mm_splits(tasks, steps, clusters);   // too few tiles for the SMs: a cluster shares a tile's reduction
    const int grid = a.splits > 1 ? (int)tasks * a.splits : (int)std::min<int64_t>(tasks, sms);

    CUtensorMap ma, mb;
    // a single row has no stride
    const int64_t b_rows = (int64_t)n_groups * n;
    if (encode_codes(fn, &ma, a_codes, m, row_bytes, m > 1 ? a_code_stride : row_bytes, a.bn) != STMOE_OK ||
        encode_codes(fn, &mb, b_codes, b_rows, row_bytes, b_rows > 1 ? b_code_stride : row_bytes, kMmRows) != STMOE_OK)
        return STMOE_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (out_dtype == STMOE_F32) return launch_matmul<0>(ma, mb, a, grid, st);
    if (out_dtype == STMOE_BF16) return launch_matmul<1>(ma, mb, a, grid, st);
    return launch_matmul<4>(ma, mb, a, grid, st);
}

}  // extern "C"
