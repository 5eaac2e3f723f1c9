// Host side that the operators' entry points share: error codes of CUDA calls, the current device, launches
// behind the kernel before, the driver's tensor-map encoder.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/stmoe.h"
#include "per_device.h"

namespace stmoe_host {

inline int cuda_status(cudaError_t e)
{
    if (e == cudaSuccess) return STMOE_OK;
    (void)cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? STMOE_ERR_OOM : STMOE_ERR_CUDA;
}

// whether every one of these is NULL or on a boundary of its element type's size
template <typename... T> bool aligned(const T *...p) { return ((((uintptr_t)p & (sizeof(T) - 1)) == 0) && ...); }

// A matrix in memory (stride in elements of so many bytes), and whether two of them share some, seen from their first to
// their last element.
struct Span {
    const void *p;
    int64_t stride, rows, cols;
    int bytes;
    uintptr_t end() const { return (uintptr_t)p + bytes * ((rows > 1 ? (rows - 1) * stride : 0) + cols); }
};
inline bool overlap(const Span &a, const Span &b) { return a.rows && b.rows && (uintptr_t)a.p < b.end() && (uintptr_t)b.p < a.end(); }

// ordinal of the current device, and how many SMs it has
inline int current_device(int *dev, int *sms)
{
    static PerDevice<int> kept;
    if (const int rc = cuda_status(cudaGetDevice(dev))) return rc;
    if (*dev < 0 || *dev >= kMaxDevices) return STMOE_ERR_CUDA;
    const int d = *dev;
    return kept.get(d, sms, [d](int &n) { return cuda_status(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, d)); });
}

// Launch that may start while the kernel before it in the stream drains (programmatic dependent
// launch; the kernels wait for it themselves), in clusters of `cluster` CTAs.
template <typename... P, typename... A>
int launch_behind(void (*kernel)(P...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t st, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid, cfg.blockDim = dim3(block), cfg.dynamicSmemBytes = smem, cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, args...));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled, or nullptr where the driver has none
inline EncodeTiledFn encode_tiled_fn()
{
    static std::atomic<EncodeTiledFn> kept{nullptr};   // the same value whoever fills it
    EncodeTiledFn fn = kept.load(std::memory_order_relaxed);
    if (!fn) {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)sym;
        (void)cudaGetLastError();
        kept.store(fn, std::memory_order_relaxed);
    }
    return fn;
}

}  // namespace stmoe_host
