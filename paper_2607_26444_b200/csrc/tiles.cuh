// What the experts' products share, in 8 and in 4 bits: loads by TMA, descriptors, TMEM, the tiles that a claim stands for, and
// the epilogue's stores.
#pragma once

#include <cuda.h>

#include "layer.cuh"

namespace strata {

__device__ __forceinline__ void mbar_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
        : "memory");
}

// Shared-memory descriptor of a K-major operand with 128-byte swizzle: start address, 1024 bytes between groups of
// eight rows, descriptor version 1.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void mma_commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                 : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t (&r)[16], uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}
// the loaded registers are tied to the wait, so that no use of them moves in front of it
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Row tiles of `height` over `rows` rows, without the sum that passes 2^31 - 1 where one expert holds nearly as many.
__host__ __device__ constexpr int tiles_of(int rows, int height) { return rows / height + (rows % height != 0 ? 1 : 0); }
static_assert(tiles_of(0, 256) == 0 && tiles_of(1, 64) == 1 && tiles_of(64, 64) == 1 && tiles_of(65, 64) == 2, "");
static_assert(tiles_of(2147483647, 256) == 8388608 && tiles_of(2147483647, 64) == 33554432, "");

struct Work {
    int e, m, row0, rows;               // expert, channel tile, first receive row, rows of the tile
};

// Tiles are dealt by an ordered claim (common.cuh): their costs differ, since an expert's last row tile is partial, and
// a static round robin left the SMs between 79 % and 100 % of the kernel's time at work (prefill chunk of 16,384 rows).
// Tiles are numbered expert by expert, inside an expert channel tile by channel tile, row tiles fastest: CTAs that run
// together read the same weights (once from HBM) and the same few row tiles.
template <int BN>
__device__ __forceinline__ Work find_work(unsigned t, const int* s_base, const int* s_off, const int* s_cnt, int E,
                                          int m_tiles)
{
    const int key = (int)(t / (unsigned)m_tiles);
    int a = 0, b = E;                   // s_base[a] <= key < s_base[b]
    while (b - a > 1) {
        const int mid = (a + b) >> 1;
        if (s_base[mid] <= key) a = mid;
        else b = mid;
    }
    const unsigned nt = (unsigned)(s_base[a + 1] - s_base[a]);
    const unsigned local = t - (unsigned)s_base[a] * (unsigned)m_tiles;
    Work w;
    w.e = a;
    w.m = (int)(local / nt);
    const int n = (int)(local - (unsigned)w.m * nt);
    w.row0 = s_off[a] + n * BN;
    w.rows = min(BN, s_cnt[a] - n * BN);
    return w;
}

// Whether both warps of an exchanging pair go on: one vote for all 64 threads, so that neither waits for the other in vain.
// The vote asks for converged warps, which lanes that left a wait one by one need not be.
__device__ __forceinline__ bool pair_all(bool ok, int pair)
{
    uint32_t r;
    __syncwarp();
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)ok), "r"(1 + pair)
        : "memory");
    return r != 0;
}

// silu(g) * u.  The exponential is within 2 + 1.2 |g| ulp (CUDA's bound for __expf), 2^-16 at the most, and the division within 2, against
// the result's own 2^-9; where 1 + exp(-g) passes 2^126 (g < -87.3) the quotient is zero instead of below 2^-119.
__device__ __forceinline__ float gate_mul(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

// N columns of 32 channels, lane = channel `ch`: neighbouring lanes exchange, so that one holds two channels of column c and
// the other two channels of column c + 1, and each writes them with one 4-byte store (64 bytes per row and warp).  Where
// rows of out do not all start on 4 bytes, or the channels are odd in number, the two are stored one by one.
template <int N>
__device__ __forceinline__ void store_pairs(const float (&y)[N], int lane, uint16_t* out, long long stride, int rows, int ch,
                                            int limit, bool words)
{
    const int odd = lane & 1;
    ch &= ~1;
    out += odd * stride + ch;
#pragma unroll
    for (int c = 0; c < N; c += 2) {
        const float other = __shfl_xor_sync(0xffffffffu, odd ? y[c] : y[c + 1], 1);
        const uint32_t v = odd ? pack_bf16x2(other, y[c + 1]) : pack_bf16x2(y[c], other);
        uint16_t* at = out + c * stride;
        if (words) {
            if (ch < limit && c + odd < rows) *reinterpret_cast<uint32_t*>(at) = v;
        } else if (c + odd < rows) {
            if (ch < limit) at[0] = (uint16_t)v;
            if (ch + 1 < limit) at[1] = (uint16_t)(v >> 16);
        }
    }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_fn()
{
    static EncodeFn fn = []() -> EncodeFn {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}

// A map of bytes.
inline bool encode(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                   const cuuint32_t* box, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    EncodeFn fn = encode_fn();
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Row tiles of height bn, at most: every expert may end in one partial tile.
inline long long row_tiles(const strata_moe_shape& s, long long a_rows, int bn)
{
    const long long items = min((long long)s.R * s.T * s.K, a_rows);
    const long long rows = s.slot_capacity > 0 ? (long long)s.E * s.R * s.slot_capacity : items;
    return rows / bn + min((long long)s.E, rows);
}

}  // namespace strata
