// Residual addition with root-mean-square norm (bf16 and / or 8-bit output), its backward pass, and the row
// quantiser (strata_layer.h has the formulas).  All three stream rows of bf16 through registers: a row is read
// once, its statistics are formed across the threads that hold it, and its results are written once.
#include "layer.cuh"

namespace strata {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kVpt = 4;                // 16-byte vectors of a row per thread
constexpr int kGradCtasPerSm = 4;

enum QKind { kNoCodes = 0, kInt8 = 1, kE4m3 = 2 };

// coherent load (outputs may alias inputs row by row) that leaves L1 to the weights
__device__ __forceinline__ uint4 ld_row16(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

__device__ __forceinline__ void load_weight8(const void* w, bool f32, int col, float* out)
{
    if (f32) {
        const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(w) + col);
        const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(w) + col + 4);
        out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w;
        out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
    } else {
        unpack_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + col), out);
    }
}

// Sum of a and maximum (or sum) of b over the threads of one row.  Rows of one warp need no barrier; otherwise the
// partials of the warps meet in shared memory, in a buffer that alternates from row to row, so one barrier is enough.
template <bool B_IS_MAX>
__device__ __forceinline__ void row_reduce(float& a, float& b, float2* buf, bool one_warp, int phase)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(kFull, a, o);
        const float t = __shfl_xor_sync(kFull, b, o);
        b = B_IS_MAX ? fmaxf(b, t) : b + t;
    }
    if (one_warp) return;
    const int warp = (int)threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    float2* mine = buf + (phase & 1) * 32;
    if ((threadIdx.x & 31) == 0) mine[warp] = make_float2(a, b);
    __syncthreads();
    a = mine[0].x;
    b = mine[0].y;
    for (int q = 1; q < warps; ++q) {
        a += mine[q].x;
        b = B_IS_MAX ? fmaxf(b, mine[q].y) : b + mine[q].y;
    }
}

// 8 codes of y * limit / top (top = max|y| of the row), one correctly rounded binary32 quotient each, so that a
// quotient half-way between two codes is seen as such.  The quotient: inv = 1/top correctly rounded, q0 = n * inv, the
// exact remainder n - q0 * top by one fused multiply-add, and q0 + remainder * inv (Markstein, IBM J. Res. Dev. 34,
// 1990).  n = y * limit has at most 24 significant bits (y from bf16 values and bf16 weights), top at most 16: a quotient
// that binary32 holds is returned exactly, and none lies close enough to a midpoint to round the other way.  Rows
// with extreme magnitudes are moved into range by a power of two first (row_range), so the remainder stays exact.
// Three instructions instead of the division's ten: the division made the quantiser bound by instruction issue.
template <int QK>
__device__ __forceinline__ uint2 codes8(const float* y, float range, float top, float inv)
{
    constexpr float kLimit = QK == kInt8 ? 127.0f : 448.0f;
    const float f = kLimit * range;
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float n = y[i] * f;
        const float q0 = n * inv;
        q[i] = fmaf(fmaf(-q0, top, n), inv, q0);
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float* p = q + 4 * h;
        if constexpr (QK == kInt8) {
            // adding 1.5 * 2^23 rounds to an integer, ties to even, and leaves it in the low bits
            constexpr float kRound = 12582912.0f;
            const uint32_t lo = __byte_perm(__float_as_uint(p[0] + kRound), __float_as_uint(p[1] + kRound), 0x0040);
            const uint32_t hi = __byte_perm(__float_as_uint(p[2] + kRound), __float_as_uint(p[3] + kRound), 0x0040);
            w[h] = __byte_perm(lo, hi, 0x5410);
        } else {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(p[1]), "f"(p[0]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(p[3]), "f"(p[2]));
            w[h] = (uint32_t)lo | ((uint32_t)hi << 16);
        }
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ float row_range(float top)
{
    return top < 0x1p-60f ? 0x1p80f : top > 0x1p100f ? 0x1p-30f : 1.0f;
}

struct RowParams {
    const uint16_t* x;
    const uint16_t* res;
    const void* weight;
    uint16_t* res_out;
    uint16_t* out;
    uint8_t* q;
    float* q_scale;
    const int32_t* n_valid;
    int* status;
    long long x_stride, res_stride, res_out_stride, out_stride, q_stride, q_scale_stride;
    long long rows;
    int vecs;              // 16-byte vectors in a row
    int tpr;               // threads of one row: the whole block, or 32 (several rows per block)
    int stages;            // rows in flight per row group (ring)
    int weight_f32;
    float eps, inv_cols;
};

constexpr int kMaxStages = 4, kMaxGroups = 8;

// A wait that runs out marks the block dead: later waits return at once, the block finishes its rows with whatever its
// buffers hold and the status tells that the results are void.
__device__ __forceinline__ void ring_wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status)
{
    for (uint32_t it = 0; it < (uint32_t)(STRATA_WAIT_LIMIT); ++it)
        if (mbar_try_wait(bar, parity) || *dead) return;
    *dead = 1;
    report_status(status, STRATA_ERR_TIMEOUT);
}

// Forward pass.  NORM: y = (h * w) * rstd; otherwise y = x (row quantiser).  max|y| follows from max|h * w|, because
// multiplying by rstd keeps the order, so both statistics come out of one reduction, and the codes need no rstd at all.
//
// A row belongs to one block (rows of up to 1024 columns: to one warp of eight), which keeps it packed in registers
// between the two passes.  RING: bulk copies keep the next rows of the group in flight in shared memory whatever the
// threads do (a stage is free again after the reduction's barrier); without it, two blocks of 224 threads held too
// few loads in flight: 837 us for 65,536 x 7168 with residual to e4m3.  Launches with one row per group at most load
// directly: there is nothing to run ahead of.
template <bool NORM, bool RES, int QK, bool RING, int MAXT>
__global__ void __launch_bounds__(MAXT) row_kernel(const RowParams p)
{
    extern __shared__ __align__(128) unsigned char ring[];            // [groups][stages][1 or 2 rows]
    __shared__ float2 s_part[64];
    __shared__ uint64_t s_full[kMaxGroups][kMaxStages];
    __shared__ int s_dead;
    const bool one_warp = p.tpr == 32;
    const int sub = one_warp ? (int)threadIdx.x >> 5 : 0;            // row group inside the block
    const int tid = one_warp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const int groups = one_warp ? (int)blockDim.x >> 5 : 1;
    const uint32_t row_bytes = (uint32_t)p.vecs * 16u, stage_bytes = RES ? 2u * row_bytes : row_bytes;
    unsigned char* my_ring = ring + (size_t)sub * p.stages * stage_bytes;
    if constexpr (RING) {
        if (threadIdx.x == 0) {
            s_dead = 0;
            for (int g = 0; g < groups; ++g)
                for (int s = 0; s < p.stages; ++s) mbar_init(&s_full[g][s], 1);
            mbar_fence_init();
        }
        __syncthreads();
    }
    griddep_wait();
    long long rows = p.rows;
    if (p.n_valid) rows = min(rows, (long long)max(0, *p.n_valid));
    const long long first = (long long)blockIdx.x * groups + sub, step = (long long)gridDim.x * groups;
    auto fetch = [&](long long row, int stage) {
        uint64_t* bar = &s_full[sub][stage];
        unsigned char* dst = my_ring + (size_t)stage * stage_bytes;
        mbar_expect_tx(bar, stage_bytes);
        bulk_g2s_plain(dst, p.x + row * p.x_stride, row_bytes, bar);
        if constexpr (RES) bulk_g2s_plain(dst + row_bytes, p.res + row * p.res_stride, row_bytes, bar);
    };
    if (RING && tid == 0)
        for (int s = 0; s < p.stages; ++s)
            if (first + s * step < rows) fetch(first + s * step, s);
    int phase = 0, stage = 0;
    uint32_t parity = 0;
    for (long long row = first; row < rows; row += step, ++phase) {
        const unsigned char* src = my_ring + (size_t)stage * stage_bytes;
        uint4 h[kVpt];                                               // the row, as stored
        if constexpr (RING) {
            ring_wait(&s_full[sub][stage], parity, &s_dead, p.status);
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs) h[j] = *reinterpret_cast<const uint4*>(src + (size_t)c * 16);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs) h[j] = ld_row16(p.x + row * p.x_stride + (size_t)c * 8);
            }
        }
        uint4 r[kVpt];
        if constexpr (RES) {
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs)
                    r[j] = RING ? *reinterpret_cast<const uint4*>(src + row_bytes + (size_t)c * 16)
                                : ld_row16(p.res + row * p.res_stride + (size_t)c * 8);
            }
        }
        float sum = 0.0f, top = 0.0f;
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                float f[8];
                unpack_bf16x8(h[j], f);
                if constexpr (RES) {
                    float t[8];
                    unpack_bf16x8(r[j], t);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] += t[i];
                    h[j] = pack_bf16x8(f);
                    *reinterpret_cast<uint4*>(p.res_out + row * p.res_out_stride + (size_t)c * 8) = h[j];
                    unpack_bf16x8(h[j], f);                          // what is stored is what is normed
                }
                if constexpr (NORM) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
                    if constexpr (QK != kNoCodes) {
                        float w[8];
                        load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
#pragma unroll
                        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i] * w[i]));
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
                }
            }
        }
        row_reduce<true>(sum, top, s_part, one_warp, phase);
        if constexpr (RING) {
            if (tid == 0 && row + p.stages * step < rows) fetch(row + p.stages * step, stage);
            if (++stage == p.stages) {
                stage = 0;
                parity ^= 1;
            }
        }
        float rstd = 1.0f;
        if constexpr (NORM) rstd = __frcp_rn(__fsqrt_rn(fmaf(sum, p.inv_cols, p.eps)));
        const float range = row_range(top), in_range = top == 0.0f ? 1.0f : top * range, inv = __frcp_rn(in_range);
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                float f[8];
                unpack_bf16x8(h[j], f);
                if constexpr (NORM) {
                    float w[8];
                    load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] *= w[i];
                }
                if constexpr (QK != kNoCodes)
                    *reinterpret_cast<uint2*>(p.q + row * p.q_stride + (size_t)c * 8) = codes8<QK>(f, range, in_range, inv);
                if constexpr (NORM) {
                    if (QK == kNoCodes || p.out) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] *= rstd;
                        *reinterpret_cast<uint4*>(p.out + row * p.out_stride + (size_t)c * 8) = pack_bf16x8(f);
                    }
                }
            }
        }
        if (QK != kNoCodes && tid == 0)
            p.q_scale[row * p.q_scale_stride] = __fdiv_rn(top * rstd, QK == kInt8 ? 127.0f : 448.0f);
    }
    griddep_launch_dependents();
    if constexpr (RING) {                                            // a block that gave up lets its copies land first
        if (tid == 0 && s_dead)
            for (int s = 0; s < p.stages; ++s) {
                const long long last = rows > first ? (rows - 1 - first) / step : -1;       // uses of the ring: 0 .. last
                const long long use = last - ((last - s) % p.stages + p.stages) % p.stages;
                if (use >= 0) mbar_wait_bounded(&s_full[sub][s], (uint32_t)(use / p.stages) & 1u);
            }
    }
}

struct GradParams {
    const uint16_t* dy;
    const uint16_t* h;
    const void* weight;
    const uint16_t* dres;
    uint16_t* dx;
    float* part;           // [gridDim.x * rows per block, 8 * vecs]
    long long dy_stride, h_stride, dres_stride, dx_stride;
    long long rows;
    int vecs, tpr, weight_f32;
    float eps, inv_cols;
};

// Backward pass.  A thread keeps the same columns for every row it meets, so its share of dweight stays in
// registers; each row-owner writes one partial row, and a second kernel adds the partial rows in a fixed order.
template <bool RES, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_grad_kernel(const GradParams p)
{
    __shared__ float2 s_part[64];
    const bool one_warp = p.tpr == 32;
    const int sub = one_warp ? (int)threadIdx.x >> 5 : 0;
    const int tid = one_warp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const int rows_per_block = one_warp ? (int)blockDim.x >> 5 : 1;
    griddep_wait();
    float dw[kVpt][8];
#pragma unroll
    for (int j = 0; j < kVpt; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f;
    const long long owner = (long long)blockIdx.x * rows_per_block + sub, owners = (long long)gridDim.x * rows_per_block;
    int phase = 0;
    for (long long row = owner; row < p.rows; row += owners, ++phase) {
        uint4 hv[kVpt], dv[kVpt], rv[kVpt];
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                hv[j] = ld_row16(p.h + row * p.h_stride + (size_t)c * 8);
                dv[j] = ld_row16(p.dy + row * p.dy_stride + (size_t)c * 8);
            }
        }
        if constexpr (RES) {
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs) rv[j] = ld_row16(p.dres + row * p.dres_stride + (size_t)c * 8);
            }
        }
        float sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                float h[8], d[8], w[8];
                unpack_bf16x8(hv[j], h);
                unpack_bf16x8(dv[j], d);
                load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum = fmaf(h[i], h[i], sum);
                    dot = fmaf(d[i] * w[i], h[i], dot);
                }
            }
        }
        row_reduce<false>(sum, dot, s_part, one_warp, phase);
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(sum, p.inv_cols, p.eps)));
        const float mean = dot * rstd * p.inv_cols;                  // mean(g * hat)
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                float h[8], d[8], w[8], o[8];
                unpack_bf16x8(hv[j], h);
                unpack_bf16x8(dv[j], d);
                load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
                if constexpr (RES) unpack_bf16x8(rv[j], o);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float hat = h[i] * rstd;
                    dw[j][i] = fmaf(d[i], hat, dw[j][i]);
                    const float t = fmaf(-hat, mean, d[i] * w[i]);
                    o[i] = RES ? fmaf(rstd, t, o[i]) : rstd * t;
                }
                *reinterpret_cast<uint4*>(p.dx + row * p.dx_stride + (size_t)c * 8) = pack_bf16x8(o);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kVpt; ++j) {
        const int c = tid + j * p.tpr;
        if (c < p.vecs) {
            float4* o = reinterpret_cast<float4*>(p.part + (size_t)owner * p.vecs * 8 + (size_t)c * 8);
            o[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
            o[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
        }
    }
    griddep_launch_dependents();
}

// dweight[c] = sum of the partial rows: 8 columns x 32 row lanes per block, each lane adding every 32nd partial row,
// then a tree over the lanes.
constexpr int kSumCols = 8, kSumLanes = 32;
__global__ void __launch_bounds__(kSumCols* kSumLanes) weight_sum_kernel(const float* part, long long owners, int cols,
                                                                         float* dweight)
{
    __shared__ float s[kSumLanes][kSumCols + 1];
    griddep_wait();
    griddep_launch_dependents();
    const int cx = (int)threadIdx.x % kSumCols, lane = (int)threadIdx.x / kSumCols;
    const int col = (int)blockIdx.x * kSumCols + cx;                 // cols is a multiple of 8
    float a = 0.0f;
    for (long long r = lane; r < owners; r += kSumLanes) a += part[(size_t)r * cols + col];
    s[lane][cx] = a;
    __syncthreads();
#pragma unroll
    for (int o = kSumLanes / 2; o > 0; o >>= 1) {
        if (lane < o) s[lane][cx] += s[lane + o][cx];
        __syncthreads();
    }
    if (lane == 0) dweight[col] = s[0][cx];
}

struct RowGeom {
    int tpr, threads, groups;          // threads per row, threads per block, rows per block at a time
};
RowGeom row_geom(int cols)
{
    RowGeom g;
    const int vecs = cols / 8;
    g.tpr = ((vecs + kVpt - 1) / kVpt + 31) / 32 * 32;
    g.groups = g.tpr == 32 ? kMaxGroups : 1;
    g.threads = g.tpr * g.groups;
    return g;
}

template <bool NORM, bool RES, int QK>
cudaError_t run_rows(RowParams& p, const RowGeom& g, int n_sm, cudaStream_t st)
{
    const long long blocks = (p.rows + g.groups - 1) / g.groups;
    const size_t row = (size_t)p.vecs * (RES ? 32 : 16) * (size_t)g.groups;       // bytes a block reads per round
    // blocks per SM: up to 1,024 threads, with two rows per group in flight in 200 KB of shared memory
    constexpr size_t kRing = 200 * 1024;
    const int per_sm = (int)max(1ll, min((long long)(1024 / g.threads), (long long)(kRing / (2 * row))));
    if (blocks <= (long long)n_sm * per_sm) {
        return g.threads <= 256 ? launch_pdl(row_kernel<NORM, RES, QK, false, 256>, (unsigned)blocks, g.threads, 0, st, p)
                                : launch_pdl(row_kernel<NORM, RES, QK, false, 1024>, (unsigned)blocks, g.threads, 0, st, p);
    }
    p.stages = (int)max(1ll, min((long long)kMaxStages, (long long)(kRing / (per_sm * row))));
    const size_t smem = row * p.stages;
    const unsigned grid = (unsigned)(n_sm * per_sm);
    return g.threads <= 256 ? launch_pdl(row_kernel<NORM, RES, QK, true, 256>, grid, g.threads, smem, st, p)
                            : launch_pdl(row_kernel<NORM, RES, QK, true, 1024>, grid, g.threads, smem, st, p);
}

long long grad_owners(long long rows, const RowGeom& g, int n_sm)
{
    const long long blocks = min((rows + g.groups - 1) / g.groups, (long long)n_sm * kGradCtasPerSm);
    return blocks * g.groups;
}

}  // namespace

// Attributes of the kernels that use more than 48 KB of shared memory.
namespace {
template <bool NORM, bool RES, int QK>
cudaError_t configure_rows()
{
    cudaError_t e = cudaFuncSetAttribute(row_kernel<NORM, RES, QK, true, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         200 * 1024);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(row_kernel<NORM, RES, QK, true, 1024>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 200 * 1024);
    return e;
}
}  // namespace
cudaError_t configure_norm_kernels()
{
    cudaError_t e = configure_rows<true, true, kNoCodes>();
    if (e == cudaSuccess) e = configure_rows<true, true, kInt8>();
    if (e == cudaSuccess) e = configure_rows<true, true, kE4m3>();
    if (e == cudaSuccess) e = configure_rows<true, false, kNoCodes>();
    if (e == cudaSuccess) e = configure_rows<true, false, kInt8>();
    if (e == cudaSuccess) e = configure_rows<true, false, kE4m3>();
    if (e == cudaSuccess) e = configure_rows<false, false, kInt8>();
    if (e == cudaSuccess) e = configure_rows<false, false, kE4m3>();
    return e;
}

cudaError_t launch_norm(const strata_norm_args& a, int* status, int n_sm, cudaStream_t st)
{
    const RowGeom g = row_geom(a.cols);
    RowParams p{};
    p.x = static_cast<const uint16_t*>(a.x);
    p.res = static_cast<const uint16_t*>(a.residual);
    p.weight = a.weight;
    p.res_out = static_cast<uint16_t*>(a.residual_out);
    p.out = static_cast<uint16_t*>(a.out);
    p.q = static_cast<uint8_t*>(a.q);
    p.q_scale = a.q_scale;
    p.x_stride = a.x_stride;
    p.res_stride = a.residual_stride;
    p.res_out_stride = a.residual_out_stride;
    p.out_stride = a.out_stride;
    p.q_stride = a.q_stride;
    p.q_scale_stride = a.q_scale_stride;
    p.status = status;
    p.rows = a.rows;
    p.vecs = a.cols / 8;
    p.tpr = g.tpr;
    p.weight_f32 = a.weight_type == STRATA_T_F32;
    p.eps = a.eps;
    p.inv_cols = 1.0f / (float)a.cols;
    const int qk = !a.q ? kNoCodes : a.q_type == STRATA_T_INT8 ? kInt8 : kE4m3;
    if (a.residual)
        return qk == kNoCodes ? run_rows<true, true, kNoCodes>(p, g, n_sm, st)
               : qk == kInt8  ? run_rows<true, true, kInt8>(p, g, n_sm, st)
                              : run_rows<true, true, kE4m3>(p, g, n_sm, st);
    return qk == kNoCodes ? run_rows<true, false, kNoCodes>(p, g, n_sm, st)
           : qk == kInt8  ? run_rows<true, false, kInt8>(p, g, n_sm, st)
                          : run_rows<true, false, kE4m3>(p, g, n_sm, st);
}

cudaError_t launch_quantize(const void* x, long long x_stride, long long rows, int cols, int q_type, void* q,
                            long long q_stride, float* q_scale, long long q_scale_stride, const int32_t* n_valid,
                            int* status, int n_sm, cudaStream_t st)
{
    const RowGeom g = row_geom(cols);
    RowParams p{};
    p.x = static_cast<const uint16_t*>(x);
    p.q = static_cast<uint8_t*>(q);
    p.q_scale = q_scale;
    p.n_valid = n_valid;
    p.status = status;
    p.x_stride = x_stride;
    p.q_stride = q_stride;
    p.q_scale_stride = q_scale_stride;
    p.rows = rows;
    p.vecs = cols / 8;
    p.tpr = g.tpr;
    return q_type == STRATA_T_INT8 ? run_rows<false, false, kInt8>(p, g, n_sm, st)
                                   : run_rows<false, false, kE4m3>(p, g, n_sm, st);
}

size_t norm_grad_scratch_bytes(long long rows, int cols, int n_sm)
{
    return (size_t)grad_owners(rows, row_geom(cols), n_sm) * (size_t)cols * sizeof(float);
}

cudaError_t launch_norm_grad(const strata_norm_grad_args& a, int n_sm, cudaStream_t st, int* n_launches)
{
    const RowGeom g = row_geom(a.cols);
    const long long owners = grad_owners(a.rows, g, n_sm);
    GradParams p{};
    p.dy = static_cast<const uint16_t*>(a.dy);
    p.h = static_cast<const uint16_t*>(a.h);
    p.weight = a.weight;
    p.dres = static_cast<const uint16_t*>(a.dresidual);
    p.dx = static_cast<uint16_t*>(a.dx);
    p.part = static_cast<float*>(a.scratch);
    p.dy_stride = a.dy_stride;
    p.h_stride = a.h_stride;
    p.dres_stride = a.dresidual_stride;
    p.dx_stride = a.dx_stride;
    p.rows = a.rows;
    p.vecs = a.cols / 8;
    p.tpr = g.tpr;
    p.weight_f32 = a.weight_type == STRATA_T_F32;
    p.eps = a.eps;
    p.inv_cols = 1.0f / (float)a.cols;
    *n_launches = 0;
    cudaError_t err = cudaSuccess;
    if (owners > 0) {
        const unsigned grid = (unsigned)(owners / g.groups);
#define STRATA_GRAD(MAXT)                                                                                              \
    (a.dresidual ? launch_pdl(norm_grad_kernel<true, MAXT>, grid, g.threads, 0, st, p)                                 \
                 : launch_pdl(norm_grad_kernel<false, MAXT>, grid, g.threads, 0, st, p))
        err = g.threads <= 256 ? STRATA_GRAD(256) : g.threads <= 512 ? STRATA_GRAD(512) : STRATA_GRAD(1024);
#undef STRATA_GRAD
        *n_launches = 1;
        if (err != cudaSuccess) return err;
    }
    *n_launches += 1;
    return launch_pdl(weight_sum_kernel, (unsigned)(a.cols / kSumCols), kSumCols * kSumLanes, 0, st, p.part, owners,
                      a.cols, a.dweight);
}

}  // namespace strata
