// Helpers of the host side of libmlkv, shared by its translation units: error texts, the device of a
// call, driver entry points.  Internal; not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "mlkv.h"
#include "mlkv_internal.h"

namespace mlkv {

// Sets mlkv_last_error() and returns the code.
inline int fail(int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

inline int fail_cuda(cudaError_t e, const char *what)
{
    return fail(MLKV_ERR_CUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                   const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
using CtxGetCurrentFn = CUresult (*)(CUcontext *);
using CtxGetDeviceFn = CUresult (*)(CUdevice *);

template <typename Fn>
Fn driver_entry(const char *name)
{
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion(name, &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
        return nullptr;
    return reinterpret_cast<Fn>(fn);
}

// The device of the CUDA context current on this thread (e.g. the one PyTorch made current);
// falls back to this runtime's current device.
inline int current_device()
{
    static CtxGetCurrentFn get_ctx = driver_entry<CtxGetCurrentFn>("cuCtxGetCurrent");
    static CtxGetDeviceFn get_dev = driver_entry<CtxGetDeviceFn>("cuCtxGetDevice");
    CUcontext ctx = nullptr;
    if (get_ctx != nullptr && get_dev != nullptr && get_ctx(&ctx) == CUDA_SUCCESS && ctx) {
        CUdevice dev;
        if (get_dev(&dev) == CUDA_SUCCESS)
            return static_cast<int>(dev);
    }
    int d = 0;
    cudaGetDevice(&d);
    return d;
}

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess)
            prev = -1;
        if (prev != dev)
            ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        int now = -1;
        if (prev >= 0 && cudaGetDevice(&now) == cudaSuccess && now != prev)
            cudaSetDevice(prev);
    }
};

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether [a, a + na) and [b, b + nb) share a byte.
inline bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
    return x < y + nb && y < x + na;
}

// Refuses a cache of `rows` times `row_bytes` bytes that no device holds: 64 bits would wrap, and the
// allocation would be of what is left.
inline int check_cache_bytes(long long rows, long long row_bytes)
{
    if (rows > (1LL << 62) / row_bytes)
        return fail(MLKV_ERR_OOM, "a cache of %lld rows of %lld bytes exceeds any device's memory", rows,
                    row_bytes);
    return MLKV_OK;
}

// The checks of a cache's sizes and layer-to-owner map (mlkv_cache_create).
int validate_map(int l, int h, int d, const int *owner, int g, int b, int max_seq);

// One layer's causal prefill over K and V of its own (kv_direct) or of a cache slot, with every
// argument checked already: the tensor maps of the queries (and, direct, of K and V), the work units
// and the launches.
struct PrefillCall {
    const void *Q, *K, *V;      // K, V: only with direct
    void *out;
    const int *prompt_lens;
    int *err;
    int b, h, g, d, s_max, slot, sm_count;
    bool direct;
    const CUtensorMap *tmap_kv; // the cache in boxes of 128 positions; only without direct
    int window, sinks;          // window 0: every earlier position is visible
};
int issue_prefill(const PrefillCall &a, cudaStream_t stream);
// The checks of a prompt's sizes, lengths, queries and outputs shared by the prefill calls.
int check_prefill_args(const void *Q, const void *out, const int *prompt_lens, int b, int h, int d,
                       int s_max, int max_seq);
// The checks of a window (0: none) and its sinks.
int check_window(int window, int sinks);
// A window that no length up to `most` outgrows is none; more sinks than positions are all positions.
inline void clamp_window(int most, int *window, int *sinks)
{
    if (*window >= most)
        *window = 0;
    if (*sinks > most)
        *sinks = most;
}

}  // namespace mlkv
