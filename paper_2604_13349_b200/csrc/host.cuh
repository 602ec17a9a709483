// Host-side helpers that the library's entry points share: error returns, launches, device properties, tensor maps.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstdio>

#include "obf.h"

namespace obf {

// Kernels that the last call of this thread enqueued (obf_last_launch_count).
inline thread_local int32_t g_last_launches = 0;

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Streaming multiprocessors of the current device (148 on a B200 when no device can be asked).
inline int sm_count()
{
    static int cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return 148; }
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
            cudaGetLastError();
            n = 148;
        }
        cached[dev] = n;
    }
    return cached[dev];
}

inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

#define OBF_CUDA_TRY(expr)                                                        \
    do {                                                                          \
        cudaError_t e_ = (expr);                                                  \
        if (e_ != cudaSuccess) {                                                  \
            std::fprintf(stderr, "obf: %s failed: %s\n", #expr, cudaGetErrorString(e_)); \
            (void)cudaGetLastError();      /* reported here: not the next call's */       \
            return OBF_ERR_CUDA;                                                  \
        }                                                                         \
    } while (0)

// The limit belongs to the kernel, not to the launch, and host threads share it: a kernel whose use of shared memory varies
// is given the most it can ever need, the same in every call, so that no call lowers it between another's limit and launch.
template <typename K>
inline obf_status_t set_smem(K kernel, size_t bytes)
{
    OBF_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    OBF_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, (int)cudaSharedmemCarveoutMaxShared));
    return OBF_OK;
}

#define OBF_TRY(expr)                        \
    do {                                     \
        const obf_status_t s_ = (expr);      \
        if (s_ != OBF_OK) return s_;         \
    } while (0)

// Launch that may be set up while the stream's kernel before it still runs.  The first kernel of a call launched so begins with
// pdl_wait(), before it lets the next one be set up; a later one does, too, unless it reads nothing that the one before writes: then it
// may wait at its end instead, so that whatever follows it follows both.  Between two kernels of a call that is about a
// microsecond less.  `cluster`: blocks of a thread-block cluster, at most
// eight, in the grid's first dimension.
template <typename... P, typename... A>
inline obf_status_t launch_clusters(int cluster, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A &...args)
{
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = cluster;
        at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    OBF_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    return OBF_OK;
}

template <typename... P, typename... A>
inline obf_status_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const A &...args)
{
    return launch_clusters(1, kernel, grid, threads, smem, st, args...);
}

// cuTensorMapEncodeTiled, looked up through the runtime so that the library does not link the driver.
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn tensor_map_encoder()
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || !ptr) {
            cudaGetLastError();
            return nullptr;
        }
        fn = reinterpret_cast<EncodeTiledFn>(ptr);
    }
    return fn;
}

}  // namespace obf
