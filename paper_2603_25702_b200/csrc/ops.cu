// Error text, device set-up and the time-out status of the stand-alone operators.
#include <stdarg.h>
#include <stdio.h>

#include <atomic>
#include <mutex>

#include "ops_host.h"

namespace s2d2 {
namespace ops {

namespace {
constexpr int MAX_DEVICES = 64;
thread_local char g_err[256];
std::mutex g_setup;
std::atomic<bool> g_ready[MAX_DEVICES];
Device g_dev[MAX_DEVICES];
__device__ int g_timeouts;
thread_local int g_seen[MAX_DEVICES];
}  // namespace

void clear_error() { g_err[0] = 0; }

int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

int device(const Device** out) {
    int id = 0;
    cudaError_t e = cudaGetDevice(&id);
    if (e != cudaSuccess) return fail(S2D2_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(e));
    if (id < 0 || id >= MAX_DEVICES) return fail(S2D2_ERR_UNSUPPORTED, "device index too large");
    if (!g_ready[id].load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(g_setup);
        if (!g_ready[id].load(std::memory_order_relaxed)) {
            Device d;
            d.id = id;
            int major = 0;
            if ((e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, id)) != cudaSuccess ||
                (e = cudaDeviceGetAttribute(&d.n_sms, cudaDevAttrMultiProcessorCount, id)) != cudaSuccess)
                return fail(S2D2_ERR_CUDA, "cudaDeviceGetAttribute: %s", cudaGetErrorString(e));
            if (major != 10) return fail(S2D2_ERR_UNSUPPORTED, "built for sm_100a only");
            if ((e = cudaGetSymbolAddress((void**)&d.timeouts, g_timeouts)) != cudaSuccess)
                return fail(S2D2_ERR_CUDA, "cudaGetSymbolAddress: %s", cudaGetErrorString(e));
            void* fn = nullptr;
            cudaDriverEntryPointQueryResult q;
            if ((e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q)) != cudaSuccess || !fn)
                return fail(S2D2_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
            d.encode = (EncodeTiledFn)fn;
            if ((e = load_score_kernels()) != cudaSuccess || (e = load_mxfp4_kernels()) != cudaSuccess) {
                cudaGetLastError();
                return fail(S2D2_ERR_CUDA, "loading the kernels: %s", cudaGetErrorString(e));
            }
            g_dev[id] = d;
            g_ready[id].store(true, std::memory_order_release);
        }
    }
    *out = &g_dev[id];
    return S2D2_OK;
}

int check_ptr(const Device* d, const void* p, size_t align, const char* what) {
    if (!p) return fail(S2D2_ERR_INVALID, "%s: null pointer", what);
    if ((uintptr_t)p % align) return fail(S2D2_ERR_INVALID, "%s: must be aligned to %d bytes", what, (int)align);
    cudaPointerAttributes a;
    cudaError_t e = cudaPointerGetAttributes(&a, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(S2D2_ERR_INVALID, "%s: not a device pointer (%s)", what, cudaGetErrorString(e));
    }
    if (a.type == cudaMemoryTypeManaged) return S2D2_OK;
    if (a.type != cudaMemoryTypeDevice) return fail(S2D2_ERR_INVALID, "%s: not a device pointer", what);
    if (a.device != d->id) return fail(S2D2_ERR_INVALID, "%s: memory of device %d, the current device is %d", what, a.device, d->id);
    return S2D2_OK;
}

}  // namespace ops
}  // namespace s2d2

using namespace s2d2;

extern "C" const char* s2d2_ops_last_error(void) { return ops::g_err; }

extern "C" int s2d2_ops_status(void* cuda_stream) {
    ops::clear_error();
    const ops::Device* d;
    if (int rc = ops::device(&d)) return rc;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    int n = 0;
    cudaError_t e = cudaMemcpyAsync(&n, d->timeouts, sizeof(int), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return ops::fail(S2D2_ERR_CUDA, "%s", cudaGetErrorString(e));
    if (n == ops::g_seen[d->id]) return S2D2_OK;
    ops::g_seen[d->id] = n;
    return ops::fail(S2D2_ERR_TIMEOUT, "a bounded wait inside a kernel ran out; its outputs are NaN");
}
