// What the serving operators' host code shares: argument checks, the workspace, launches.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdlib>

#include "bcast_serve.h"
#include "exec_internal.h"

#define SERVE_TRY(expr)                                                              \
    do {                                                                             \
        const cudaError_t e_ = (expr);                                               \
        if (e_ != cudaSuccess) return bcast_internal_cuda_failed((int)e_);           \
    } while (0)

namespace bcast_serve {

constexpr int64_t kMaxDim = (1ll << 31) - 1;       // largest length of one dimension
constexpr int64_t kMaxStride = 1ll << 38;          // largest stride, in elements (a tensor map's limit is 2^40 bytes)

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// One array as an operator sees it: its pointer must be memory of the current device (a host pointer
// handed to a kernel would fault the GPU) and aligned to `align` bytes.
inline int check_array(const void *p, uintptr_t align, int device)
{
    if (!p || ((uintptr_t)p & (align - 1))) return BCAST_ERR_INVAL;
    cudaPointerAttributes attr;
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess) {
        cudaGetLastError();                        // not a sticky error: clear it
        return BCAST_ERR_INVAL;
    }
    if (attr.type == cudaMemoryTypeManaged) return BCAST_OK;
    return attr.type == cudaMemoryTypeDevice && attr.device == device ? BCAST_OK : BCAST_ERR_INVAL;
}

inline bool stride_ok(int64_t stride, int64_t least, int64_t multiple)
{
    return stride >= least && stride <= kMaxStride && stride % multiple == 0;
}

inline int check_workspace(void *ws, uint64_t have, int64_t need, int device)
{
    if (need < 0) return (int)need;
    if (have < (uint64_t)need) return BCAST_ERR_CAPACITY;
    return check_array(ws, 256, device);
}

// Are the kernels to begin as if one of their bounded waits had run out?  (For tests of what they do then.)
inline int give_up_at_once()
{
    static const int yes = [] {
        const char *v = std::getenv("BCAST_SERVE_GIVE_UP");
        return v && *v && std::atoi(v) ? 1 : 0;
    }();
    return yes;
}

// The SM count that workspace sizes are computed with: they must not depend on whether a device is
// there, so it is the B200's.
constexpr int kSms = 148;

// Let a kernel have `bytes` of dynamic shared memory; the driver is told once per device.
template <auto *kernel>
int allow_smem(size_t bytes)
{
    static std::atomic<uint64_t> told{0};
    int device = 0;
    SERVE_TRY(cudaGetDevice(&device));
    const uint64_t bit = device < 64 ? 1ull << device : 0;
    if (told.load(std::memory_order_relaxed) & bit) return BCAST_OK;
    SERVE_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    told.fetch_or(bit, std::memory_order_relaxed);
    return BCAST_OK;
}

// Launch `kernel`; `after`: it may start while the kernel before it on the stream is still running (it
// then waits for it with griddepcontrol.wait before touching what that kernel wrote).
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool after, unsigned cluster, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    unsigned n = 0;
    if (after) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = cluster;
        at[n].val.clusterDim.y = 1;
        at[n++].val.clusterDim.z = 1;
    }
    cfg.attrs = at;
    cfg.numAttrs = n;
    SERVE_TRY(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
    return BCAST_OK;
}

}  // namespace bcast_serve
