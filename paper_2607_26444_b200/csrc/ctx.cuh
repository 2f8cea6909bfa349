// The context behind the opaque handle of the C ABI, and the checks that every entry point shares (host only).
#pragma once

#include <mutex>
#include <vector>

#include "common.cuh"

struct strata_region {
    uint64_t id;
    uintptr_t base;
    size_t bytes;
    size_t used;      // bump pointer of strata_pool_carve
};

struct strata_ctx {
    strata_moe_shape shape;
    int device;
    int n_sm;             // SMs the persistent kernels size their grids for (the device's, or the caller's budget)
    int n_sm_device;
    int x_early;          // the caller's promise about x (strata_ctx_set_x_early)
    int* ws;              // device workspace (header + tile counts)
    size_t ws_bytes;
    uint64_t next_region;
    uint64_t launches;
    strata::TraceBuf trace;
    // host round trip only: copy streams and events, created on first use (no device memory)
    cudaStream_t s_in = nullptr, s_out = nullptr;
    std::vector<cudaEvent_t> ev_in, ev_done;
    cudaEvent_t ev_entry = nullptr, ev_out = nullptr;
    std::vector<strata_region> regions;
    std::mutex mu;
};

namespace strata {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
        if (prev == dev) prev = -1;
    }
    ~DeviceGuard()
    {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

inline bool region_contains(const strata_ctx* c, const void* p, size_t bytes)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    for (const strata_region& r : c->regions)
        if (a >= r.base && bytes <= r.bytes && a - r.base <= r.bytes - bytes) return true;
    return false;
}

// One more kernel on the context's account; the C entries return what this returns.
inline strata_status launched(strata_ctx* c, cudaError_t err, uint64_t kernels = 1)
{
    {
        std::lock_guard<std::mutex> lk(c->mu);
        c->launches += kernels;
    }
    if (err == cudaSuccess) return STRATA_OK;
    cudaGetLastError();
    return STRATA_ERR_CUDA;
}

}  // namespace strata
