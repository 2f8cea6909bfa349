// Shared by the kernels of strata_layer.h: element access and the launchers.
#pragma once

#include "common.cuh"
#include "strata_layer.h"

namespace strata {

cudaError_t launch_route(const strata_moe_shape& s, const strata_route_params& r, const void* logits, int type,
                         long long stride, const float* bias, int32_t* ids, float* w, int n_sm, cudaStream_t st);
cudaError_t launch_route_grad(const strata_moe_shape& s, const strata_route_params& r, const void* logits, int type,
                              long long stride, const int32_t* ids, const float* dw, void* dlogits, long long dstride,
                              int* status, cudaStream_t st);
cudaError_t configure_norm_kernels();
cudaError_t launch_norm(const strata_norm_args& a, cudaStream_t st);
size_t norm_grad_scratch_bytes(long long rows, int cols, int n_sm);
cudaError_t launch_norm_grad(const strata_norm_grad_args& a, int* status, int n_sm, cudaStream_t st, int* n_launches);
cudaError_t launch_quantize(const void* x, long long x_stride, long long rows, int cols, int q_type, void* q,
                            long long q_stride, float* q_scale, long long q_scale_stride, const int32_t* n_valid,
                            cudaStream_t st);
cudaError_t configure_matmul_kernels();
cudaError_t launch_expert_matmul(const strata_moe_shape& s, const strata_moe_layout_t& L, const strata_matmul_args& a,
                                 int* status, WorkQueue wq, int n_sm, cudaStream_t st);

#ifdef __CUDACC__
// A wait with a limit.  False if it ran out, here or in another thread of the block (`dead`, in shared memory): the status then
// tells that the results are void, and every role of the block leaves its loop.
__device__ __forceinline__ bool wait_or_dead(uint64_t* bar, uint32_t parity, volatile int* dead, int* status)
{
    for (uint32_t it = 0; it < (uint32_t)(STRATA_WAIT_LIMIT); ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*dead) return false;
    }
    *dead = 1;
    report_status(status, STRATA_ERR_TIMEOUT);
    return false;
}

__device__ __forceinline__ void unpack_bf16x8(uint4 v, float* f)
{
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint4 pack_bf16x8(const float* f)
{
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
template <bool BF16>
__device__ __forceinline__ float load_as_float(const void* base, long long i)
{
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(base)[i] << 16);
    else return static_cast<const float*>(base)[i];
}
// VPL values at elements off+e0 .. of a row of E; vec_ok: rows start on 16 bytes
template <int VPL, bool BF16>
__device__ __forceinline__ void store_row(const float (&g)[VPL], void* base, long long off, int e0, int E, bool vec_ok)
{
    constexpr int VW = BF16 ? 8 : 4;
    if constexpr (VPL >= VW) {
#pragma unroll
        for (int j = 0; j < VPL; j += VW) {
            if (vec_ok && e0 + j + VW <= E) {
                if constexpr (BF16) st_stream16(static_cast<uint16_t*>(base) + off + e0 + j, pack_bf16x8(&g[j]));
                else
                    st_stream16(static_cast<float*>(base) + off + e0 + j,
                                make_uint4(__float_as_uint(g[j]), __float_as_uint(g[j + 1]), __float_as_uint(g[j + 2]),
                                           __float_as_uint(g[j + 3])));
            } else {
#pragma unroll
                for (int i = 0; i < VW; ++i)
                    if (e0 + j + i < E) {
                        if constexpr (BF16)
                            static_cast<uint16_t*>(base)[off + e0 + j + i] = (uint16_t)pack_bf16x2(g[j + i], 0.0f);
                        else static_cast<float*>(base)[off + e0 + j + i] = g[j + i];
                    }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (e0 + i < E) {
                if constexpr (BF16) static_cast<uint16_t*>(base)[off + e0 + i] = (uint16_t)pack_bf16x2(g[i], 0.0f);
                else static_cast<float*>(base)[off + e0 + i] = g[i];
            }
    }
}
#endif

}  // namespace strata
