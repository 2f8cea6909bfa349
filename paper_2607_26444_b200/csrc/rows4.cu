// bf16 rows to 4-bit codes with block scales, and back (strata_layer.h has the formulas).  Both stream: a row's values are read
// once and written once.
#include "layer.cuh"

namespace strata {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr uint32_t kInfBits = 0x7f80u;  // bf16: magnitudes from here on are infinite or NaN

// Two binary32 values in one register pair, multiplied and added by one instruction.
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
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair widen(uint32_t u) { return make_pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }

// Nearest e2m1 codes (ties to even, 6 at the most) of eight values, the first in the lowest bits.
__device__ __forceinline__ uint32_t codes_of(const Pair* v)
{
    uint32_t d;
    const float2 a = split(v[0]), b = split(v[1]), c = split(v[2]), e = split(v[3]);
    asm("{\n\t.reg .b8 x, y, z, w;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 x, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 y, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 z, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 w, %8, %7;\n\t"
        "mov.b32 %0, {x, y, z, w};\n\t}"
        : "=r"(d)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y), "f"(e.x), "f"(e.y));
    return d;
}
// The values of eight codes, as four pairs of halves.
__device__ __forceinline__ void values_of(uint32_t codes, uint32_t* h)
{
    asm("{\n\t.reg .b8 x, y, z, w;\n\tmov.b32 {x, y, z, w}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, x;\n\tcvt.rn.f16x2.e2m1x2 %1, y;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, z;\n\tcvt.rn.f16x2.e2m1x2 %3, w;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}
__device__ __forceinline__ float low_half(uint32_t h)
{
    float f;
    asm("{\n\t.reg .f16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(f) : "r"(h));
    return f;
}
__device__ __forceinline__ float high_half(uint32_t h)
{
    float f;
    asm("{\n\t.reg .f16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, u;\n\t}" : "=f"(f) : "r"(h));
    return f;
}
__device__ __forceinline__ uint32_t e4m3_of(float v)
{
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.0f), "f"(v));
    return d;
}
__device__ __forceinline__ float e4m3_value(uint32_t b)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
    return low_half(h);
}

// largest of the two magnitudes in a word, over four words; NaN and infinities are the largest patterns
__device__ __forceinline__ uint32_t top_of(uint4 v)
{
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
}

struct Rows4Params {
    const uint16_t* x;
    uint8_t* codes;
    uint8_t* block;
    float* scale;
    void* out;
    const int32_t* n_valid;
    long long x_stride, code_stride, block_stride, scale_stride, out_stride;
    long long rows;
    int vecs;              // units of eight values in a row
    int tpr;               // threads of one row: 4, 8, 16 or a multiple of 32; a block holds blockDim.x / tpr rows
    int out_f32;
};

// One row per group of threads, eight values (16 bytes in, 4 out) per thread and step.  NV needs the row's largest magnitude
// before any code, so a row waits in registers.
//
// mxfp4, per block of 32 (four lanes): with u the bits of the largest magnitude, its exponent raised where the fraction is
// 0.75 or more, less two, is the scale's exponent (log2 M - 2, one more from 7 * 2^s on, where the largest code, 6, would be farther
// off than the next binade's 8): (u + 32) >> 7, less two; 2^125 at the most, beyond which 4 * 2^126 would be infinite.  x / 2^s is exact.
// nvfp4, per block of 16 (two lanes): b = e4m3(448 M / A) from one correctly rounded quotient (Markstein's correction, as in
// norm.cu): 11 and 8 bits, so a quotient half-way between two scales is seen as such.  Codes are of q = 2688 x / (A b).  A
// quotient is half-way between two codes, T / 4 with T = 1, 3, 5, 7, 10, 14, 20, or at least 2^-16.4 away from it: with x = X 2^i and
// A b = D 2^j (X below 2^8, D below 2^12) the distance is |84 X 2^k - T D| / (4 D) for a whole k, and D 2^-k is at most about 84 X / T
// where the two are close.  So q is rounded to multiples of 2^-17 (by adding 96 and taking it away): its error before that, 2^-19.4 (a reciprocal
// within 2^-23, a product, one fused multiply-add), is gone where q is half-way, and moves nothing else across.
template <bool NV, int VPT, int MAXT>
__global__ void __launch_bounds__(MAXT) quantize4_kernel(const Rows4Params p)
{
    __shared__ uint32_t s_top[32];
    const int sub = (int)threadIdx.x / p.tpr, tid = (int)threadIdx.x - sub * p.tpr;
    const long long row = (long long)blockIdx.x * ((int)blockDim.x / p.tpr) + sub;
    griddep_wait();
    griddep_launch_dependents();
    const bool live = row < p.rows && !(p.n_valid && row >= *p.n_valid);
    if (!live && p.tpr >= 32) return;                               // rows that share a warp stay for its exchanges
    const int vecs = live ? p.vecs : 0;
    const uint16_t* x = p.x + row * p.x_stride;
    uint8_t* codes = p.codes + row * p.code_stride;
    uint8_t* block = p.block + row * p.block_stride;
    uint4 v[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tid + j * p.tpr;
        v[j] = c < vecs ? ld_stream16(x + (size_t)c * 8) : make_uint4(0, 0, 0, 0);
    }
    if constexpr (!NV) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int c = tid + j * p.tpr;
            uint32_t m = top_of(v[j]);
            m = max(m, __shfl_xor_sync(kFull, m, 1));
            m = max(m, __shfl_xor_sync(kFull, m, 2));
            const uint32_t e = m >= kInfBits ? 255u : (uint32_t)min(max((int)((m + 32) >> 7) - 2, 0), 252);
            const float mult = __uint_as_float(e == 255u ? 0u : (254u - e) << 23);
            const Pair mult2 = make_pair(mult, mult);
            Pair q[4] = {mul2(widen(v[j].x), mult2), mul2(widen(v[j].y), mult2), mul2(widen(v[j].z), mult2), mul2(widen(v[j].w), mult2)};
            if (c < vecs) {
                *reinterpret_cast<uint32_t*>(codes + (size_t)c * 4) = codes_of(q);
                if ((c & 3) == 0) block[c >> 2] = (uint8_t)e;
            }
        }
    } else {
        uint32_t m[VPT], top = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            m[j] = top_of(v[j]);
            top = max(top, m[j]);
        }
        if (p.tpr >= 32) top = __reduce_max_sync(kFull, top);
        else
            for (int o = p.tpr >> 1; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
        if (p.tpr > 32) {
            const int warps = p.tpr >> 5;
            if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
            asm volatile("bar.sync %0, %1;" ::"r"(sub), "r"(p.tpr) : "memory");
            for (int w = 0; w < warps; ++w) top = max(top, s_top[sub * warps + w]);
        }
        const float a = __uint_as_float(top << 16);
        const float range = a < 0x1p-60f ? 0x1p80f : a > 0x1p100f ? 0x1p-30f : 1.0f;
        const float ar = top == 0 ? 1.0f : a * range, inv = __frcp_rn(ar);
        const Pair range2 = make_pair(range, range), big = make_pair(96.0f, 96.0f), neg_big = make_pair(-96.0f, -96.0f);
        // Two lanes hold a block of every vector: the even lane works out the scale of their first, the odd one of their second.
        static_assert(VPT % 2 == 0, "");
#pragma unroll
        for (int j = 0; j < VPT; j += 2) {
            const uint32_t odd = threadIdx.x & 1u;
            const uint32_t sent = odd ? m[j] : m[j + 1], kept = odd ? m[j + 1] : m[j];
            const uint32_t mb = max(kept, __shfl_xor_sync(kFull, sent, 1));
            const float n = __uint_as_float(mb << 16) * range * 448.0f, q0 = n * inv;
            uint32_t b = e4m3_of(fmaf(fmaf(q0, -ar, n), inv, q0));
            float r;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(ar * e4m3_value(b)));
            const float own = b == 0 ? 0.0f : 2688.0f * r, other = __shfl_xor_sync(kFull, own, 1);
            const int at = tid + (j + (int)odd) * p.tpr;             // the vector whose block this lane did
            if (at < vecs) block[at >> 1] = (uint8_t)b;
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
                const int c = tid + (j + i2) * p.tpr;
                const float mult = (i2 == 0) == (odd == 0) ? own : other;
                const Pair mult2 = make_pair(mult, mult);
                const uint4 u = v[j + i2];
                Pair q[4] = {widen(u.x), widen(u.y), widen(u.z), widen(u.w)};
                if (range != 1.0f) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[i] = mul2(q[i], range2);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = add2(fma2(q[i], mult2, big), neg_big);
                if (c < vecs) *reinterpret_cast<uint32_t*>(codes + (size_t)c * 4) = codes_of(q);
            }
        }
        if (tid == 0 && live) p.scale[row * p.scale_stride] = top >= kInfBits ? __uint_as_float(0x7fc00000u) : __fdiv_rn(a, 2688.0f);
    }
}

template <bool NV, int VPT, int MAXT>
__global__ void __launch_bounds__(MAXT) dequantize4_kernel(const Rows4Params p)
{
    const int sub = (int)threadIdx.x / p.tpr, tid = (int)threadIdx.x - sub * p.tpr;
    const long long row = (long long)blockIdx.x * ((int)blockDim.x / p.tpr) + sub;
    griddep_wait();
    griddep_launch_dependents();
    if (row >= p.rows || (p.n_valid && row >= *p.n_valid)) return;
    const uint8_t* codes = p.codes + row * p.code_stride;
    const uint8_t* block = p.block + row * p.block_stride;
    const float scale = p.scale ? p.scale[row * p.scale_stride] : 1.0f;
    uint32_t v[VPT], b[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tid + j * p.tpr;
        if (c < p.vecs) {
            v[j] = *reinterpret_cast<const uint32_t*>(codes + (size_t)c * 4);
            b[j] = block[NV ? c >> 1 : c >> 2];
        }
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int c = tid + j * p.tpr;
        if (c >= p.vecs) continue;
        float unit;
        if constexpr (NV) unit = e4m3_value(b[j]);
        else unit = __uint_as_float(b[j] == 255u ? 0x7fc00000u : b[j] == 0 ? 0x00400000u : b[j] << 23);
        if (p.scale) unit *= scale;
        uint32_t h[4];
        values_of(v[j], h);
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = low_half(h[i]) * unit;
            f[2 * i + 1] = high_half(h[i]) * unit;
        }
        if (p.out_f32) {
            float* o = static_cast<float*>(p.out) + row * p.out_stride + (size_t)c * 8;
            *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4*>(o + 4) = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + row * p.out_stride + (size_t)c * 8) = pack_bf16x8(f);
        }
    }
}

template <int VPT, typename F>
cudaError_t run_rows4(Rows4Params& p, F launch)
{
    const int least = (p.vecs + VPT - 1) / VPT;
    p.tpr = least > 16 ? (least + 31) / 32 * 32 : least > 8 ? 16 : least > 4 ? 8 : 4;
    const int groups = p.tpr <= 128 ? 256 / p.tpr : 1, threads = p.tpr * groups;
    const long long blocks = (p.rows + groups - 1) / groups;
    if (blocks >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    return launch((unsigned)blocks, (unsigned)threads);
}

// Vectors per thread of the quantiser: eight put more loads in flight and need fewer warps per row (one up to 2048 columns: no
// barrier).  Measured with two, four and eight, us, mxfp4 then nvfp4: 131,072 x 2048: 124, 108, 105; 217, 156, 122 (the bytes at the
// measured copy rate: 107, 110); 16,411 x 7200: 61, 53, 50; 94, 80, 66; 65,536 x 1024: 32, 28, 27; 55, 38, 33; 100,000 x 160: 13,
// 11, 10; 21, 16, 13.  Sixteen: 172 and 196 at 2048 columns, 59 and 64 at 7200.  Of the inverse, two and four: 131,072 x 2048 118, 102;
// 100,000 x 160 13, 10.
template <bool NV>
cudaError_t quantize4(Rows4Params& p, cudaStream_t st)
{
    return run_rows4<8>(p, [&](unsigned blocks, unsigned threads) {
        return threads <= 256 ? launch_pdl(quantize4_kernel<NV, 8, 256>, blocks, threads, 0, st, p)
                              : launch_pdl(quantize4_kernel<NV, 8, 512>, blocks, threads, 0, st, p);
    });
}
template <bool NV>
cudaError_t dequantize4(Rows4Params& p, cudaStream_t st)
{
    return run_rows4<4>(p, [&](unsigned blocks, unsigned threads) {
        return threads <= 256 ? launch_pdl(dequantize4_kernel<NV, 4, 256>, blocks, threads, 0, st, p)
                              : launch_pdl(dequantize4_kernel<NV, 4, 1024>, blocks, threads, 0, st, p);
    });
}

Rows4Params params_of(const strata_rows4& q, long long rows, int cols, const int32_t* n_valid)
{
    Rows4Params p{};
    p.codes = static_cast<uint8_t*>(q.codes);
    p.block = static_cast<uint8_t*>(q.block);
    p.scale = q.scale;
    p.code_stride = q.code_stride;
    p.block_stride = q.block_stride;
    p.scale_stride = q.scale_stride;
    p.n_valid = n_valid;
    p.rows = rows;
    p.vecs = cols / 8;
    return p;
}

}  // namespace

cudaError_t launch_quantize4(const void* x, long long x_stride, long long rows, int cols, int type, const strata_rows4& q,
                             const int32_t* n_valid, cudaStream_t st)
{
    Rows4Params p = params_of(q, rows, cols, n_valid);
    p.x = static_cast<const uint16_t*>(x);
    p.x_stride = x_stride;
    return type == STRATA_T_NVF4 ? quantize4<true>(p, st) : quantize4<false>(p, st);
}

cudaError_t launch_dequantize4(const strata_rows4& q, long long rows, int cols, int type, void* out, int out_type,
                               long long out_stride, const int32_t* n_valid, cudaStream_t st)
{
    Rows4Params p = params_of(q, rows, cols, n_valid);
    p.out = out;
    p.out_f32 = out_type == STRATA_T_F32;
    p.out_stride = out_stride;
    return type == STRATA_T_NVF4 ? dequantize4<true>(p, st) : dequantize4<false>(p, st);
}

}  // namespace strata
