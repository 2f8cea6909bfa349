// Residual addition with root-mean-square norm (bf16 and / or 8-bit output), its backward pass, and the row
// quantiser (strata_layer.h has the formulas).  All three stream rows of bf16 through registers: a row is read
// once, its statistics are formed across the threads that hold it, and its results are written once.
#include "layer.cuh"

#ifdef STRATA_TEST_HOOKS
#include <atomic>
#endif

namespace strata {

namespace {

#ifdef STRATA_TEST_HOOKS
// Test builds only: block 0 of the next launch with a ring expects 16 bytes more than its first row delivers (see matmul.cu).
std::atomic<int> g_inject_short_row{0};
#define STRATA_TEST_EXTRA(first) (p.test_flags && blockIdx.x == 0 && (first) ? 16u : 0u)
#else
#define STRATA_TEST_EXTRA(first) 0u
#endif

constexpr unsigned kFull = 0xffffffffu;
constexpr int kVpt = 4;                // 16-byte vectors of a row per thread
constexpr size_t kRingBytes = 200 * 1024;  // shared memory of an SM that rows in flight may take

enum QKind { kNoCodes = 0, kInt8 = 1, kE4m3 = 2 };

// Two binary32 values in one register pair: sm_100 multiplies and adds them with one instruction, and these kernels are
// bound by instruction issue before they are bound by memory (the norm of 65,536 x 7168 to e4m3 with scalar arithmetic took 206
// warp instructions per 32 vectors and 590 us; with pairs 146, and the bytes at the copy rate are 502 us).
using Pair = unsigned long long;
__device__ __forceinline__ Pair make_pair(float lo, float hi)
{
    Pair d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ float2 split(Pair p)
{
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(p));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair widen(uint32_t u) { return make_pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
__device__ __forceinline__ void widen8(uint4 v, Pair* p)
{
    p[0] = widen(v.x);
    p[1] = widen(v.y);
    p[2] = widen(v.z);
    p[3] = widen(v.w);
}
__device__ __forceinline__ uint32_t narrow(Pair p)
{
    const float2 f = split(p);
    return pack_bf16x2(f.x, f.y);
}
__device__ __forceinline__ uint4 narrow8(const Pair* p) { return make_uint4(narrow(p[0]), narrow(p[1]), narrow(p[2]), narrow(p[3])); }
// bf16 sums, rounded once
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

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

__device__ __forceinline__ void load_weight8(const void* w, bool f32, int col, Pair* out)
{
    if (f32) {
        const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(static_cast<const float*>(w) + col);
        const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(static_cast<const float*>(w) + col + 4);
        out[0] = a.x;
        out[1] = a.y;
        out[2] = b.x;
        out[3] = b.y;
    } else {
        widen8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + col), out);
    }
}

// a load from shared memory that is not merged with an earlier one (to keep the registers free in between)
__device__ __forceinline__ uint4 lds16(const void* p)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_addr(p)) : "memory");
    return v;
}

// Sum of a and maximum (or sum) of b over the tpr threads of row group `sub`.  Rows of one warp need no barrier; otherwise the
// partials of the warps meet in shared memory (the group's own part of buf, not reused before its next barrier but one:
// callers with several rows alternate between two buffers), behind a barrier of the group.
template <bool B_IS_MAX>
__device__ __forceinline__ void row_reduce(float& a, float& b, float2* buf, int sub, int tpr)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(kFull, a, o);
        const float t = __shfl_xor_sync(kFull, b, o);
        b = B_IS_MAX ? fmaxf(b, t) : b + t;
    }
    if (tpr == 32) return;
    const int warps = tpr >> 5, warp = (int)threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) buf[warp] = make_float2(a, b);
    asm volatile("bar.sync %0, %1;" ::"r"(sub), "r"(tpr) : "memory");
    const float2* mine = buf + sub * warps;
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
// that binary32 holds is returned exactly, and none lies close enough to a midpoint to round the other way.  With binary32
// weights y is rounded to 24 bits, and so is n: a correctly rounded quotient of a rounded numerator.  Rows
// with extreme magnitudes are moved into range by a power of two first (row_range), so the remainder stays exact.
// Three instructions instead of the division's ten: the division made the quantiser bound by instruction issue.
template <int QK>
__device__ __forceinline__ uint2 codes8(const Pair* y, Pair factor, Pair neg_top, Pair inv)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float2 q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const Pair n = mul2(y[2 * h + i], factor);
            const Pair q0 = mul2(n, inv);
            q[i] = split(fma2(fma2(q0, neg_top, n), inv, q0));
        }
        if constexpr (QK == kInt8) {
            // adding 1.5 * 2^23 rounds to an integer, ties to even, and leaves it in the low bits
            constexpr float kRound = 12582912.0f;
            const uint32_t lo = __byte_perm(__float_as_uint(q[0].x + kRound), __float_as_uint(q[0].y + kRound), 0x0040);
            const uint32_t hi = __byte_perm(__float_as_uint(q[1].x + kRound), __float_as_uint(q[1].y + kRound), 0x0040);
            w[h] = __byte_perm(lo, hi, 0x5410);
        } else {
            uint16_t lo, hi;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(q[0].y), "f"(q[0].x));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(q[1].y), "f"(q[1].x));
            asm("mov.b32 %0, {%1, %2};" : "=r"(w[h]) : "h"(lo), "h"(hi));
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
    long long x_stride, res_stride, res_out_stride, out_stride, q_stride, q_scale_stride;
    long long rows;
    int vecs;              // 16-byte vectors in a row
    int tpr;               // threads of one row, a multiple of 32; a block holds blockDim.x / tpr rows
    int weight_f32;
    float eps, inv_cols;
};

// y = h * weight for eight columns (vector c of the row)
__device__ __forceinline__ void weigh8(const RowParams& p, int c, Pair* y)
{
    Pair w[4];
    load_weight8(p.weight, p.weight_f32 != 0, c * 8, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], w[i]);
}

// Forward pass.  NORM: y = (h * w) * rstd; otherwise y = x (row quantiser).  max|y| follows from max|h * w|, because
// multiplying by rstd keeps the order, so both statistics come out of one reduction, and the codes need no rstd at all.
//
// One row per group of threads, no loop: the hardware deals blocks of up to 256 threads to SMs as they free up, which keeps
// every SM busy to the end.  The row waits in registers between the two passes, as h * w where the codes need that and the
// registers allow it.  65,536 x 7168 with residual to e4m3: 487 us, 520 once the power limit slows the clocks (6.3 TB/s);
// widening and weighing again in the second pass: 501 and 550; persistent blocks with a ring of bulk copies and ordered
// claims: 526 and 569 (and 90, not 82 us, at 16,384 x 4096 to bf16); several rows per block, the next one fetched ahead:
// 157 to 171 us, not 148, at 131,072 x 2048.  Three blocks per SM (80 registers) with a residual, four (64) without: 178,
// not 200 us, at 65,536 x 4096 to e4m3.
template <bool NORM, bool RES, int QK, int VPT, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT > 256 ? 1 : VPT == 8 || (NORM && RES) ? 3 : 4) row_kernel(const RowParams p)
{
    __shared__ float2 s_part[32];
    const int sub = (int)threadIdx.x / p.tpr, tid = (int)threadIdx.x - sub * p.tpr;
    const long long row = (long long)blockIdx.x * ((int)blockDim.x / p.tpr) + sub;
    griddep_wait();
    griddep_launch_dependents();
    if (row >= p.rows || (p.n_valid && row >= *p.n_valid)) return;
    uint4 h[VPT];                                                   // the row, as stored
    {
        const uint16_t* x = p.x + row * p.x_stride;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) h[j] = ld_row16(x + (size_t)c * 8);
        }
    }
    if constexpr (RES) {
        const uint16_t* res = p.res + row * p.res_stride;
        uint16_t* res_out = p.res_out + row * p.res_out_stride;
        uint4 r[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) r[j] = ld_row16(res + (size_t)c * 8);
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {                                        // what is stored is what is normed
                h[j] = make_uint4(add_bf16x2(h[j].x, r[j].x), add_bf16x2(h[j].y, r[j].y), add_bf16x2(h[j].z, r[j].z),
                                  add_bf16x2(h[j].w, r[j].w));
                *reinterpret_cast<uint4*>(res_out + (size_t)c * 8) = h[j];
            }
        }
    }
    constexpr bool kKeep = QK != kNoCodes && VPT == 4;               // h * w waits in registers, not h
    Pair squares = 0, kept[kKeep ? VPT : 1][4];
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tid + j * p.tpr;
        if (c < p.vecs) {
            Pair* y = kept[kKeep ? j : 0];
            widen8(h[j], y);
            if constexpr (NORM) {
#pragma unroll
                for (int i = 0; i < 4; ++i) squares = fma2(y[i], y[i], squares);
                if constexpr (QK != kNoCodes) weigh8(p, c, y);
            }
            if constexpr (QK != kNoCodes) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = split(y[i]);
                    top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
                }
            }
        }
    }
    const float2 sq = split(squares);
    float sum = sq.x + sq.y;
    row_reduce<true>(sum, top, s_part, sub, p.tpr);
    float rstd = 1.0f;
    if constexpr (NORM) rstd = __frcp_rn(__fsqrt_rn(fmaf(sum, p.inv_cols, p.eps)));
    const float range = row_range(top), in_range = top == 0.0f ? 1.0f : top * range, inv = __frcp_rn(in_range);
    const float factor = (QK == kInt8 ? 127.0f : 448.0f) * range;
    const Pair factor2 = make_pair(factor, factor), neg_top2 = make_pair(-in_range, -in_range), inv2 = make_pair(inv, inv);
    const Pair rstd2 = make_pair(rstd, rstd);
    uint8_t* q = p.q + row * p.q_stride;
    uint16_t* out = p.out + row * p.out_stride;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tid + j * p.tpr;
        if (c < p.vecs) {
            Pair* y = kept[kKeep ? j : 0];
            if constexpr (!kKeep) {
                widen8(h[j], y);
                if constexpr (NORM) weigh8(p, c, y);
            }
            if constexpr (QK != kNoCodes) *reinterpret_cast<uint2*>(q + (size_t)c * 8) = codes8<QK>(y, factor2, neg_top2, inv2);
            if constexpr (NORM) {
                if (QK == kNoCodes || p.out) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], rstd2);
                    *reinterpret_cast<uint4*>(out + (size_t)c * 8) = narrow8(y);
                }
            }
        }
    }
    if (QK != kNoCodes && tid == 0)                                  // a zero row has scale 0 also where eps = 0 makes rstd infinite
        p.q_scale[row * p.q_scale_stride] = top == 0.0f && rstd == INFINITY ? 0.0f : __fdiv_rn(top * rstd, QK == kInt8 ? 127.0f : 448.0f);
}

constexpr int kMaxStages = 4, kMaxGroups = 8;

struct GradParams {
    const uint16_t* dy;
    const uint16_t* h;
    const void* weight;
    const uint16_t* dres;
    uint16_t* dx;
    float* part;           // [gridDim.x * rows per block, 8 * vecs]
    int* status;
    long long dy_stride, h_stride, dres_stride, dx_stride;
    long long rows;
    int vecs, tpr, stages, weight_f32;
    float eps, inv_cols;
#ifdef STRATA_TEST_HOOKS
    int test_flags;
#endif
};

// Backward pass.  A thread keeps the same columns for every row it meets, so its share of dweight stays in
// registers; each row group writes one partial row, and a second kernel adds the partial rows in a fixed order.
// (Rows are dealt in equal shares: with claims the order of the sum would change from call to call.)
// 16,384 x 4096 with residual: 88 us (6.1 TB/s).  Rows of more than 16,384 columns take blocks of 544 to 1024 threads, whose 64
// registers do not hold a thread's share (64 to 496 bytes are spilled), and beyond 17,064 columns (25,600 without a residual) not
// even two rows fit the ring: 2^27 elements with residual and bf16 weights take 202 us at 16,384 columns, 320 at 16,640, 418 at 20,000, 385 at
// 32,768, where the bytes are 164.
// RING: rows arrive by bulk copies ahead of their turn.  A stage is read in both passes over its row; it is refilled after the next
// row's reduction, behind a barrier of the row's threads (of the warp, where a row has one) that each reaches only when it
// is done with the stage.
template <bool RES, bool RING, bool WF32, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 128 ? 4 : 1) norm_grad_kernel(const GradParams p)
{
    extern __shared__ __align__(128) unsigned char ring[];            // [groups][stages][2 or 3 rows]: h, dy, dresidual
    __shared__ float2 s_part[64];
    __shared__ uint64_t s_full[kMaxGroups][kMaxStages];
    __shared__ int s_dead;
    const bool one_warp = p.tpr == 32;
    const int sub = one_warp ? (int)threadIdx.x >> 5 : 0;
    const int tid = one_warp ? (int)threadIdx.x & 31 : (int)threadIdx.x;
    const int groups = one_warp ? (int)blockDim.x >> 5 : 1;
    const uint32_t row_bytes = (uint32_t)p.vecs * 16u, stage_bytes = (RES ? 3u : 2u) * row_bytes;
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
    Pair dw[kVpt][4];
#pragma unroll
    for (int j = 0; j < kVpt; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[j][i] = 0;
    uint4 wv[kVpt];                                                  // bf16 weights stay in registers, as they come
    if constexpr (!WF32) {
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) wv[j] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.weight) + c * 8);
        }
    }
    const long long owner = (long long)blockIdx.x * groups + sub, owners = (long long)gridDim.x * groups;
    int fetched = 0;
    auto fetch = [&] {
        const long long row = owner + fetched * owners;
        if (row >= p.rows) return;
        const int stage = fetched % p.stages;
        uint64_t* bar = &s_full[sub][stage];
        unsigned char* dst = my_ring + (size_t)stage * stage_bytes;
        mbar_expect_tx(bar, stage_bytes + STRATA_TEST_EXTRA(fetched == 0));
        bulk_g2s_plain(dst, p.h + row * p.h_stride, row_bytes, bar);
        bulk_g2s_plain(dst + row_bytes, p.dy + row * p.dy_stride, row_bytes, bar);
        if constexpr (RES) bulk_g2s_plain(dst + 2 * row_bytes, p.dres + row * p.dres_stride, row_bytes, bar);
        ++fetched;
    };
    if (RING && tid == 0)
        for (int s = 0; s < p.stages; ++s) fetch();
    volatile int* dead = &s_dead;                                    // a block that gave up fetches nothing more
    int phase = 0, stage = 0;
    uint32_t parity = 0;
    for (long long row = owner; row < p.rows; row += owners, ++phase) {
        const unsigned char* src = my_ring + (size_t)stage * stage_bytes;
        uint4 hv[kVpt], dv[kVpt], rv[kVpt];                          // without a ring; with one they are read where they lie
        if constexpr (RING) {
            wait_or_dead(&s_full[sub][stage], parity, &s_dead, p.status);
        } else {
#pragma unroll
            for (int j = 0; j < kVpt; ++j) {
                const int c = tid + j * p.tpr;
                if (c < p.vecs) {
                    hv[j] = ld_row16(p.h + row * p.h_stride + (size_t)c * 8);
                    dv[j] = ld_row16(p.dy + row * p.dy_stride + (size_t)c * 8);
                    if constexpr (RES) rv[j] = ld_row16(p.dres + row * p.dres_stride + (size_t)c * 8);
                }
            }
        }
        Pair squares = 0, dots = 0;
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                if constexpr (RING) {
                    hv[j] = *reinterpret_cast<const uint4*>(src + (size_t)c * 16);
                    dv[j] = *reinterpret_cast<const uint4*>(src + row_bytes + (size_t)c * 16);
                }
                Pair h[4], d[4], w[4];
                widen8(hv[j], h);
                widen8(dv[j], d);
                if constexpr (WF32) load_weight8(p.weight, true, c * 8, w);
                else widen8(wv[j], w);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    squares = fma2(h[i], h[i], squares);
                    dots = fma2(mul2(d[i], w[i]), h[i], dots);
                }
            }
        }
        const float2 sq = split(squares), dt = split(dots);
        float sum = sq.x + sq.y, dot = dt.x + dt.y;
        row_reduce<false>(sum, dot, s_part + (phase & 1) * 32, sub, p.tpr);
        if constexpr (RING) {
            __syncwarp();                                            // a row of one warp has met no barrier, and shuffles order no memory
            if (tid == 0 && phase > 0 && !*dead) fetch();            // into the stage of the row before this one
        }
        const float rstd = rsqrtf(fmaf(sum, p.inv_cols, p.eps));     // within 2 ulp: dx is rounded to bf16, dweight sums it over the rows
        const float mean = dot * rstd * p.inv_cols;                  // mean(g * hat)
        const Pair rstd2 = make_pair(rstd, rstd), neg_mean2 = make_pair(-mean, -mean);
#pragma unroll
        for (int j = 0; j < kVpt; ++j) {
            const int c = tid + j * p.tpr;
            if (c < p.vecs) {
                if constexpr (RING) {
                    hv[j] = lds16(src + (size_t)c * 16);
                    dv[j] = lds16(src + row_bytes + (size_t)c * 16);
                    if constexpr (RES) rv[j] = *reinterpret_cast<const uint4*>(src + 2 * row_bytes + (size_t)c * 16);
                }
                Pair h[4], d[4], w[4], o[4];
                widen8(hv[j], h);
                widen8(dv[j], d);
                if constexpr (WF32) load_weight8(p.weight, true, c * 8, w);
                else widen8(wv[j], w);
                if constexpr (RES) widen8(rv[j], o);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Pair hat = mul2(h[i], rstd2);
                    dw[j][i] = fma2(d[i], hat, dw[j][i]);
                    const Pair t = fma2(hat, neg_mean2, mul2(d[i], w[i]));
                    o[i] = RES ? fma2(rstd2, t, o[i]) : mul2(rstd2, t);
                }
                *reinterpret_cast<uint4*>(p.dx + row * p.dx_stride + (size_t)c * 8) = narrow8(o);
            }
        }
        if constexpr (RING)
            if (++stage == p.stages) {
                stage = 0;
                parity ^= 1;
            }
    }
#pragma unroll
    for (int j = 0; j < kVpt; ++j) {
        const int c = tid + j * p.tpr;
        if (c < p.vecs) {
            ulonglong2* o = reinterpret_cast<ulonglong2*>(p.part + (size_t)owner * p.vecs * 8 + (size_t)c * 8);
            o[0] = make_ulonglong2(dw[j][0], dw[j][1]);
            o[1] = make_ulonglong2(dw[j][2], dw[j][3]);
        }
    }
    griddep_launch_dependents();
    if constexpr (RING) {
        if (tid == 0 && s_dead)
            for (int u = max(0, fetched - p.stages); u < fetched; ++u)
                mbar_wait_bounded(&s_full[sub][u % p.stages], (uint32_t)(u / p.stages) & 1u);
    }
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
// Backward pass: one row per block, or eight rows of one warp each.
RowGeom row_geom(int cols)
{
    RowGeom g;
    const int vecs = cols / 8;
    g.tpr = ((vecs + kVpt - 1) / kVpt + 31) / 32 * 32;
    g.groups = g.tpr == 32 ? kMaxGroups : 1;
    g.threads = g.tpr * g.groups;
    return g;
}

template <bool NORM, bool RES, int QK, int VPT>
cudaError_t run_rows_v(RowParams& p, cudaStream_t st)
{
    p.tpr = ((p.vecs + VPT - 1) / VPT + 31) / 32 * 32;
    const int groups = p.tpr <= 128 ? 256 / p.tpr : 1, threads = p.tpr * groups;
    const long long blocks = (p.rows + groups - 1) / groups;
    if (blocks >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    constexpr int kLong = VPT == 8 ? 512 : 1024;
    return threads <= 256 ? launch_pdl(row_kernel<NORM, RES, QK, VPT, 256>, (unsigned)blocks, threads, 0, st, p)
                          : launch_pdl(row_kernel<NORM, RES, QK, VPT, kLong>, (unsigned)blocks, threads, 0, st, p);
}

// Vectors per thread.  Eight put twice the loads of a thread in flight and need fewer warps per row (one up to 2048 columns), four
// spread a row over more threads and leave room to keep h * w between the passes.  Measured, four against eight, us:
//   quantiser, eight above 1024 columns: 65,280 x 2056: 119, 87 (half of eight's places hold anything, two thirds of four's);
//     51,622 x 2600: 100, 77; 32,768 x 4096: 78, 63; 32,704 x 4104: 118, 84; 16,368 x 8200: 97, 85; 4096 x 32768: 110, 70
//   norm without residual to bf16, the same except from 8200 to 10,240 columns: 65,280 x 2056: 138, 100; 32,768 x 4096: 93, 82;
//     18,724 x 7168: 98, 81; 16,368 x 8200: 100, 102; 2048 x 8200: 14, 15; 13,107 x 10,240: 89, 90; 10,922 x 12,288: 96, 85
//   norm without residual to e4m3, four: 65,536 x 2048: 90, 97; 16,384 x 8192: 93, 102
//   norm with residual to bf16, four: 16,368 x 8200: 162, 179; 8065 x 16,640: 160, 209; 8192 x 16,384: 160, 162
//   norm with residual to e4m3, eight from 10,248 to 16,384 columns: 4096 x 12,288: 68, 62; 8192 x 12,288: 130, 114; 8192 x 16,384: 160, 152;
//     outside four: 16,368 x 8200: 175, 174; 2048 x 8200: 24, 26; 18,724 x 7168: 147, 160; 8065 x 16,640: 230, 251
//   few rows, four: 128 rows of 7168 with residual to e4m3 (one wave of blocks, latency): 3.6, 5.3; with residual to e4m3 2048 x 16,384:
//     46.0, 46.5; from 2048 rows without one: 2048 x 7168: 10.7, 9.0 (quantiser), 12.6, 11.0 (norm); 2048 x 1032: 8.2, 8.4 and 7.0, 7.1
template <bool NORM, bool RES, int QK>
cudaError_t run_rows(RowParams& p, cudaStream_t st)
{
    if constexpr (NORM && RES && QK != kNoCodes) {
        if (p.vecs > 10240 / 8 && p.vecs <= 16384 / 8 && p.rows >= 4096) return run_rows_v<NORM, RES, QK, 8>(p, st);
    } else if constexpr (!NORM || (!RES && QK == kNoCodes)) {
        const bool four = NORM && p.vecs > 8192 / 8 && p.vecs <= 10240 / 8;
        if (p.vecs > 1024 / 8 && p.rows >= 2048 && !four) return run_rows_v<NORM, RES, QK, 8>(p, st);
    }
    return run_rows_v<NORM, RES, QK, 4>(p, st);
}

// Row groups of the backward pass: up to four blocks per SM, as long as two rounds of rows (three operands) of each fit
// the ring; more groups mean more partial rows, fewer mean less in flight.
long long grad_owners(long long rows, const RowGeom& g, int cols, int n_sm)
{
    const long long round = (long long)cols * 6 * g.groups;
    const long long per_sm = max(1ll, min(4ll, (long long)kRingBytes / (2 * round)));
    return min((rows + g.groups - 1) / g.groups, (long long)n_sm * per_sm) * g.groups;
}

}  // namespace

// Attributes of the kernels that use more than 48 KB of shared memory.
namespace {
template <bool RES>
cudaError_t configure_grad()
{
    const void* f[6] = {(const void*)norm_grad_kernel<RES, true, true, 128>,  (const void*)norm_grad_kernel<RES, true, true, 512>,
                        (const void*)norm_grad_kernel<RES, true, true, 1024>, (const void*)norm_grad_kernel<RES, true, false, 128>,
                        (const void*)norm_grad_kernel<RES, true, false, 512>, (const void*)norm_grad_kernel<RES, true, false, 1024>};
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < 6 && e == cudaSuccess; ++i)
        e = cudaFuncSetAttribute(f[i], cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingBytes);
    return e;
}

template <bool RES, bool RING, bool WF32>
cudaError_t run_grad_w(const GradParams& p, const RowGeom& g, unsigned grid, size_t smem, cudaStream_t st)
{
    if (g.threads <= 128) return launch_pdl(norm_grad_kernel<RES, RING, WF32, 128>, grid, g.threads, smem, st, p);
    if (g.threads <= 512) return launch_pdl(norm_grad_kernel<RES, RING, WF32, 512>, grid, g.threads, smem, st, p);
    return launch_pdl(norm_grad_kernel<RES, RING, WF32, 1024>, grid, g.threads, smem, st, p);
}
template <bool RES, bool RING>
cudaError_t run_grad(const GradParams& p, const RowGeom& g, unsigned grid, size_t smem, cudaStream_t st)
{
    return p.weight_f32 ? run_grad_w<RES, RING, true>(p, g, grid, smem, st) : run_grad_w<RES, RING, false>(p, g, grid, smem, st);
}
}  // namespace
cudaError_t configure_norm_kernels()
{
    cudaError_t e = cudaSuccess;
    e = configure_grad<true>();
    if (e == cudaSuccess) e = configure_grad<false>();
    return e;
}

cudaError_t launch_norm(const strata_norm_args& a, cudaStream_t st)
{
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
    p.weight_f32 = a.weight_type == STRATA_T_F32;
    p.eps = a.eps;
    p.inv_cols = 1.0f / (float)a.cols;
    const int qk = !a.q ? kNoCodes : a.q_type == STRATA_T_INT8 ? kInt8 : kE4m3;
    if (a.residual)
        return qk == kNoCodes ? run_rows<true, true, kNoCodes>(p, st)
               : qk == kInt8  ? run_rows<true, true, kInt8>(p, st)
                              : run_rows<true, true, kE4m3>(p, st);
    return qk == kNoCodes ? run_rows<true, false, kNoCodes>(p, st)
           : qk == kInt8  ? run_rows<true, false, kInt8>(p, st)
                          : run_rows<true, false, kE4m3>(p, st);
}

cudaError_t launch_quantize(const void* x, long long x_stride, long long rows, int cols, int q_type, void* q,
                            long long q_stride, float* q_scale, long long q_scale_stride, const int32_t* n_valid,
                            cudaStream_t st)
{
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
    return q_type == STRATA_T_INT8 ? run_rows<false, false, kInt8>(p, st)
                                   : run_rows<false, false, kE4m3>(p, st);
}

size_t norm_grad_scratch_bytes(long long rows, int cols, int n_sm)
{
    return (size_t)grad_owners(rows, row_geom(cols), cols, n_sm) * (size_t)cols * sizeof(float);
}

cudaError_t launch_norm_grad(const strata_norm_grad_args& a, int* status, int n_sm, cudaStream_t st, int* n_launches)
{
    const RowGeom g = row_geom(a.cols);
    const long long owners = grad_owners(a.rows, g, a.cols, n_sm);
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
        p.status = status;
        const size_t round = (size_t)p.vecs * 16 * (a.dresidual ? 3 : 2) * (size_t)g.groups;     // bytes of a block's rows
        const int per_sm = (int)((grid + n_sm - 1) / n_sm);
        p.stages = (int)min((long long)kMaxStages, (long long)(kRingBytes / (per_sm * round)));
        const bool use_ring = p.stages >= 2 && a.rows > owners;
        const size_t smem = use_ring ? round * p.stages : 0;
#ifdef STRATA_TEST_HOOKS
        p.test_flags = use_ring ? g_inject_short_row.exchange(0) : 0;
#endif
        err = a.dresidual ? (use_ring ? run_grad<true, true>(p, g, grid, smem, st) : run_grad<true, false>(p, g, grid, smem, st))
                          : (use_ring ? run_grad<false, true>(p, g, grid, smem, st) : run_grad<false, false>(p, g, grid, smem, st));
        *n_launches = 1;
        if (err != cudaSuccess) return err;
    }
    *n_launches += 1;
    return launch_pdl(weight_sum_kernel, (unsigned)(a.cols / kSumCols), kSumCols * kSumLanes, 0, st, p.part, owners,
                      a.cols, a.dweight);
}

}  // namespace strata

#ifdef STRATA_TEST_HOOKS
extern "C" void strata_test_inject_short_row(int on) { strata::g_inject_short_row.store(on); }
#endif
