// Host side shared by the stand-alone operators (scores.cu, mxfp4.cu): error text, argument checks, launches.
//
// These operators keep nothing between calls: no context, no scratch of their own.  Two calls may run at the same
// time on different streams or in different captured graphs, and every call is asynchronous.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <utility>

#include "../../include/s2d2.h"

namespace s2d2 {
namespace ops {

// Sets the text of s2d2_ops_last_error() for this host thread and returns `code`.
int fail(int code, const char* fmt, ...);
void clear_error();

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct Device {
    int id = -1;
    int n_sms = 0;
    int* timeouts = nullptr;          // device word: CTAs whose bounded waits ran out so far; never cleared, so that no reader takes it from another
    EncodeTiledFn encode = nullptr;
};
// The current device, set up on first use; S2D2_OK or a failure with its text.  The set-up loads every kernel of these operators
// (kernels are otherwise loaded at their first launch, which a stream capture may not allow) and raises its limits.
int device(const Device** out);
cudaError_t load_score_kernels();      // scores.cu
cudaError_t load_mxfp4_kernels();      // mxfp4.cu

// Loads a kernel and allows it `smem` bytes of dynamic shared memory.
template <typename... P>
inline cudaError_t load(void (*kernel)(P...), int smem = 0) {
    cudaFuncAttributes a;
    cudaError_t e = cudaFuncGetAttributes(&a, kernel);
    if (e == cudaSuccess && smem) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return e;
}

// `p` must be device (or managed) memory of the current device, aligned to `align` bytes.
int check_ptr(const Device* d, const void* p, size_t align, const char* what);

// Launch with an optional cluster and with programmatic stream serialisation: the kernel may begin its set-up while the
// kernel in front of it on the stream drains; it waits (griddepcontrol.wait) before it touches global memory.
template <typename... P, typename... A>
inline cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = cluster;
        at[1].val.clusterDim.y = 1;
        at[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = at;
    return cudaLaunchKernelEx(&cfg, kernel, P(std::forward<A>(args))...);
}

}  // namespace ops

#ifdef __CUDACC__
// Programmatic dependent launch: everything before pdl_wait() touches no global memory that another kernel writes.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// Thread-block clusters
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Address of `smem` (this CTA's shared::cta address) in the CTA of rank `rank` of the cluster
__device__ __forceinline__ uint32_t cluster_map(uint32_t smem, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem), "r"(rank));
    return a;
}
#endif

}  // namespace s2d2
