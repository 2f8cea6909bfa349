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

// 8 codes of y / scale (IEEE binary32 division, as the e4m3 dispatch divides)
template <int QK>
__device__ __forceinline__ uint2 codes8(const float* y, float scale)
{
    const float s = scale == 0.0f ? 1.0f : scale;
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = __fdiv_rn(y[4 * h + i], s);
        if constexpr (QK == kInt8) {
            const uint32_t lo = __byte_perm((uint32_t)__float2int_rn(q[0]), (uint32_t)__float2int_rn(q[1]), 0x0040);
            const uint32_t hi = __byte_perm((uint32_t)__float2int_rn(q[2]), (uint32_t)__float2int_rn(q[3]), 0x0040);
            w[h] = __byte_perm(lo, hi, 0x5410);
        } else {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(q[1]), "f"(q[0]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(q[3]), "f"(q[2]));
            w[h] = (uint32_t)lo | ((uint32_t)hi << 16);
        }
    }
    return make_uint2(w[0], w[1]);
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
    long long x_stride, res_stride, res_out_stride, out_stride, q_stride, q_scale_stride;
    long long rows;
    int vecs;              // 16-byte vectors in a row
    int tpr;               // threads of one row: the whole block, or 32 (several rows per block)
    int weight_f32;
    float eps, inv_cols;
};

// Forward pass.  NORM: y = (h * w) * rstd; otherwise y = x (row quantiser).  max|y| follows from max|h * w|, because
// multiplying by rstd keeps the order, so both statistics come out of one reduction.
template <bool NORM, bool RES, int QK, int MAXT>
__global__ void __launch_bounds__(MAXT) row_kernel(const RowParams p)
{
    __shared__ float2 s_part[64];
    const bool one_warp = p.tpr == 32;
    const int sub = one_warp ? (int)threadIdx.x >> 5 : 0;            // row inside the block
    const int tid = one_warp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const int rows_per_block = one_warp ? (int)blockDim.x >> 5 : 1;
    griddep_wait();
    long long rows = p.rows;
    if (p.n_valid) rows = min(rows, (long long)max(0, *p.n_valid));
    int phase = 0;
    for (long long row = (long long)blockIdx.x * rows_per_block + sub; row < rows;
         row += (long long)gridDim.x * rows_per_block, ++phase) {
        const uint16_t* x = p.x + row * p.x_stride;
        uint4 v[kVpt], r[kVpt];
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) v[j] = ld_row16(x + (size_t)c * 8);
        }
        if constexpr (RES) {
            const uint16_t* rp = p.res + row * p.res_stride;
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs) r[j] = ld_row16(rp + (size_t)c * 8);
            }
        }
        float h[kVpt][8], sum = 0.0f, top = 0.0f;
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                unpack_bf16x8(v[j], h[j]);
                if constexpr (RES) {
                    float t[8];
                    unpack_bf16x8(r[j], t);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[j][i] += t[i];
                    const uint4 stored = pack_bf16x8(h[j]);
                    *reinterpret_cast<uint4*>(p.res_out + row * p.res_out_stride + (size_t)c * 8) = stored;
                    unpack_bf16x8(stored, h[j]);                     // what is stored is what is normed
                }
                if constexpr (NORM) {
                    float w[8];
                    load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sum = fmaf(h[j][i], h[j][i], sum);
                        h[j][i] *= w[i];
                    }
                }
                if constexpr (QK != kNoCodes) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(h[j][i]));
                }
            }
        }
        row_reduce<true>(sum, top, s_part, one_warp, phase);
        float rstd = 1.0f;
        if constexpr (NORM) rstd = __frcp_rn(__fsqrt_rn(fmaf(sum, p.inv_cols, p.eps)));
        const float scale = QK == kNoCodes ? 0.0f : __fdiv_rn(top * rstd, QK == kInt8 ? 127.0f : 448.0f);
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                if constexpr (NORM) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[j][i] *= rstd;
                    if (p.out)
                        *reinterpret_cast<uint4*>(p.out + row * p.out_stride + (size_t)c * 8) = pack_bf16x8(h[j]);
                }
                if constexpr (QK != kNoCodes)
                    *reinterpret_cast<uint2*>(p.q + row * p.q_stride + (size_t)c * 8) = codes8<QK>(h[j], scale);
            }
        }
        if (QK != kNoCodes && tid == 0) p.q_scale[row * p.q_scale_stride] = scale;
    }
    griddep_launch_dependents();
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
    int tpr, threads, rows_per_block, maxt;
};
RowGeom row_geom(int cols)
{
    RowGeom g;
    const int vecs = cols / 8;
    g.tpr = ((vecs + kVpt - 1) / kVpt + 31) / 32 * 32;
    g.threads = g.tpr == 32 ? 128 : g.tpr;
    g.rows_per_block = g.tpr == 32 ? 4 : 1;
    g.maxt = g.threads <= 256 ? 256 : g.threads <= 512 ? 512 : 1024;
    return g;
}

template <bool NORM, bool RES, int QK>
cudaError_t run_rows(const RowParams& p, const RowGeom& g, int n_sm, cudaStream_t st)
{
    const long long blocks = (p.rows + g.rows_per_block - 1) / g.rows_per_block;
    const unsigned grid = (unsigned)min(blocks, (long long)n_sm * 16);
    switch (g.maxt) {
        case 256: return launch_pdl(row_kernel<NORM, RES, QK, 256>, grid, g.threads, 0, st, p);
        case 512: return launch_pdl(row_kernel<NORM, RES, QK, 512>, grid, g.threads, 0, st, p);
        default: return launch_pdl(row_kernel<NORM, RES, QK, 1024>, grid, g.threads, 0, st, p);
    }
}

long long grad_owners(long long rows, const RowGeom& g, int n_sm)
{
    const long long blocks = min((rows + g.rows_per_block - 1) / g.rows_per_block, (long long)n_sm * kGradCtasPerSm);
    return blocks * g.rows_per_block;
}

}  // namespace

cudaError_t launch_norm(const strata_norm_args& a, int n_sm, cudaStream_t st)
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
                            int n_sm, cudaStream_t st)
{
    const RowGeom g = row_geom(cols);
    RowParams p{};
    p.x = static_cast<const uint16_t*>(x);
    p.q = static_cast<uint8_t*>(q);
    p.q_scale = q_scale;
    p.n_valid = n_valid;
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
        const unsigned grid = (unsigned)(owners / g.rows_per_block);
#define STRATA_GRAD(MAXT)                                                                                              \
    (a.dresidual ? launch_pdl(norm_grad_kernel<true, MAXT>, grid, g.threads, 0, st, p)                                 \
                 : launch_pdl(norm_grad_kernel<false, MAXT>, grid, g.threads, 0, st, p))
        err = g.maxt == 256 ? STRATA_GRAD(256) : g.maxt == 512 ? STRATA_GRAD(512) : STRATA_GRAD(1024);
#undef STRATA_GRAD
        *n_launches = 1;
        if (err != cudaSuccess) return err;
    }
    *n_launches += 1;
    return launch_pdl(weight_sum_kernel, (unsigned)(a.cols / kSumCols), kSumCols * kSumLanes, 0, st, p.part, owners,
                      a.cols, a.dweight);
}

}  // namespace strata
