// What the kernels over router logits share: one warp owns a token, a lane VPL logits of neighbouring experts.
#pragma once

#include "layer.cuh"

namespace strata {

constexpr unsigned kFull = 0xffffffffu;

// The sum is pinned to its own rounding: a contraction into the exponential's last multiply would move scores by an
// ulp, and with them the order of near-ties.
__device__ __forceinline__ float sigmoid_f(float l) { return __frcp_rn(__fadd_rn(1.0f, expf(-l))); }
// exp(l - m) for l <= m; infinities at the maximum count as equal to it
__device__ __forceinline__ float softmax_term(float l, float m) { return l == m ? 1.0f : expf(l - m); }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// VPL logits of experts e0 .. e0+VPL-1.  RAW: experts beyond E read as zero and NaN stays; otherwise both read as -inf.
template <int VPL, bool BF16, bool RAW = false>
__device__ __forceinline__ void load_logits(float (&l)[VPL], const void* base, long long row_off, int e0, int E, bool vec_ok)
{
    constexpr int VW = BF16 ? 8 : 4;                              // logits in 16 bytes
    if constexpr (VPL >= VW) {
#pragma unroll
        for (int j = 0; j < VPL; j += VW) {
            if (vec_ok && e0 + j + VW <= E) {
                if constexpr (BF16) {
                    const uint4 v = ld_stream16(static_cast<const uint16_t*>(base) + row_off + e0 + j);
                    unpack_bf16x8(v, &l[j]);
                } else {
                    const uint4 v = ld_stream16(static_cast<const float*>(base) + row_off + e0 + j);
                    l[j] = __uint_as_float(v.x);
                    l[j + 1] = __uint_as_float(v.y);
                    l[j + 2] = __uint_as_float(v.z);
                    l[j + 3] = __uint_as_float(v.w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < VW; ++i)
                    l[j + i] = e0 + j + i < E ? load_as_float<BF16>(base, row_off + e0 + j + i) : RAW ? 0.0f : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            l[i] = e0 + i < E ? load_as_float<BF16>(base, row_off + e0 + i) : RAW ? 0.0f : -INFINITY;
    }
    if constexpr (!RAW) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;
    }
}

// registers per lane for runs of `lanes` lanes over `n` experts
inline int lanes_width(int n, int lanes = 32)
{
    int v = 1;
    while (lanes * v < n) v *= 2;
    return v;
}

inline bool rows_on_16(const void* base, long long stride, int type)
{
    const int size = type == STRATA_T_F32 ? 4 : 2;
    return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && stride * size % 16 == 0;
}

}  // namespace strata
