// The experts' products over the receive buffer: 8-bit rows, grouped by expert as the routing layout orders them, times
// each expert's 8-bit weights (strata_layer.h has the formulas).  tcgen05 matrix instructions, operands brought by TMA
// into 128-byte-swizzled shared memory, accumulators in TMEM, persistent CTAs over tiles found on the device.
//
// The weights are the M operand and the rows the N operand: out^T = W * A^T.  An instruction then always has 128
// channels, and its N (16 .. 256) follows the number of rows that the expert really has, so a decoding step with a
// handful of rows per expert neither multiplies nor fetches 128 rows of padding; it streams the weights.
#include "tiles.cuh"

#ifdef STRATA_TEST_HOOKS
#include <atomic>
#endif

namespace strata {

namespace {

#ifdef STRATA_TEST_HOOKS
// Test builds only: CTA 0 of the next launch expects 16 bytes more than its first loads deliver, so that its bounded wait runs
// out and the error path runs without any fault, trap or unbounded spin.
std::atomic<int> g_inject_short_load{0};
#endif

constexpr int kM = 128;                 // channels of a matrix instruction
constexpr int kKBytes = 128;            // inner extent of a stage: one swizzle span
constexpr int kUmmaK = 32;              // bytes of K per matrix instruction
constexpr int kBlock = kM * kKBytes;    // one 128-row block of weights of a stage

// A tile is MB blocks of 128 weight rows by up to BN rows of the N operand.
//   MB = 1: one accumulator.  Gated: its rows 0..63 are 64 gate channels, rows 64..127 the same channels of up, and the
//           epilogue warps of the two halves exchange columns through shared memory.
//   MB = 2: two accumulators that share the N operand.  Gated: 128 gate channels and the same of up, which then meet in
//           one thread; otherwise 256 channels.
// Accumulators are doubled (one pair is filled while the other is read) wherever TMEM's 512 columns allow it.
template <int MB, int BN>
struct Tile {
    static constexpr int box_rows = BN >= 128 ? 64 : 32;            // rows of one TMA box of the N operand
    static constexpr int w_stage = MB * kBlock, a_stage = BN * kKBytes;
    static constexpr int stages = 192 * 1024 / (w_stage + a_stage);
    static constexpr int bufs = MB * BN * 2 <= 512 ? 2 : 1;
    static constexpr int tmem_cols = bufs * MB * BN;
    static constexpr int epi_warps = MB == 2 ? 8 : 4;               // a multiple of four: warp & 3 selects the TMEM lanes
    static constexpr int threads = 64 + 32 * epi_warps;             // warp 0: loads, warp 1: matrix instructions
    static constexpr int cols = BN / (epi_warps / 4);               // columns of a tile that one epilogue warp reads
    static constexpr int swap_floats = MB == 1 ? epi_warps * 2 * 8 * 32 : 0;   // exchange of a gated tile
    static constexpr size_t data_bytes = (size_t)stages * (w_stage + a_stage);
    static_assert(stages <= 8 && tmem_cols <= 512 && data_bytes % 1024 == 0, "");
};

struct MatParams {
    CUtensorMap map_w, map_a;
    const int32_t* expert_count;        // NULL: segments are full (fixed-capacity layout)
    const int32_t* expert_offset;
    const float* a_scale;
    const float* w_scale;
    uint16_t* out;
    int* status;
    WorkQueue wq;
    long long a_rows, a_scale_stride, out_stride;
    int E, k_blocks, channels, m_tiles; // channels: rows of w per expert
    int out_words;                      // pairs of channels of out lie on 4 bytes
#ifdef STRATA_TEST_HOOKS
    int test_flags;
#endif
};

constexpr int kClaims = 4;              // tiles that the loading warp may be ahead of the epilogue

struct SmemTail {                       // behind the operand stages
    uint64_t full[8], empty[8], tmem_full[2], tmem_empty[2], drain;
    uint64_t claim_full[kClaims], claim_empty[kClaims];
    unsigned claim[kClaims];
    uint32_t tmem_base, issued;
    int dead, pad[3];
};
static_assert(sizeof(SmemTail) % 16 == 0, "the scales behind it are read in vectors");

template <bool INT8>
__device__ __forceinline__ uint32_t instr_desc(int n)
{
    const uint32_t types = INT8 ? (2u << 4) | (1u << 7) | (1u << 10)     // D int32, A and B signed 8-bit
                                : (1u << 4);                             // D float, A and B e4m3
    return types | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kM >> 4) << 24);
}
template <bool INT8>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (INT8)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
template <bool INT8>
__device__ __forceinline__ float acc_value(uint32_t v)
{
    return INT8 ? __int2float_rn((int)v) : __uint_as_float(v);
}
// The n-th tile that the loading warp handed over.
__device__ __forceinline__ bool next_tile(SmemTail& tail, uint32_t n, unsigned& t, volatile int* dead, int* status)
{
    if (!wait_or_dead(&tail.claim_full[n % kClaims], (n / kClaims) & 1, dead, status)) return false;
    t = *reinterpret_cast<volatile unsigned*>(&tail.claim[n % kClaims]);
    return true;
}

template <bool INT8, bool GATED, int MB, int BN>
__global__ void __launch_bounds__(Tile<MB, BN>::threads, 1) expert_matmul_kernel(const __grid_constant__ MatParams p)
{
    using T = Tile<MB, BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_w = smem;                                       // [stages][MB * 128][128]
    unsigned char* s_a = smem + T::stages * T::w_stage;              // [stages][BN][128]
    SmemTail* tail = reinterpret_cast<SmemTail*>(smem + T::data_bytes);
    float* s_scale = reinterpret_cast<float*>(tail + 1);             // [epilogue warps][cols]
    float* s_swap = s_scale + T::epi_warps * T::cols;                // [epilogue warps][2][8][32]
    int* s_base = reinterpret_cast<int*>(s_swap + T::swap_floats);   // [E + 1]
    int* s_off = s_base + p.E + 1;                                   // [E]
    int* s_cnt = s_off + p.E;                                        // [E]
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < T::stages; ++s) {
            mbar_init(&tail->full[s], 1);
            mbar_init(&tail->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tail->tmem_full[b], 1);
            mbar_init(&tail->tmem_empty[b], T::epi_warps);
        }
        for (int c = 0; c < kClaims; ++c) {
            mbar_init(&tail->claim_full[c], 1);
            mbar_init(&tail->claim_empty[c], 1 + T::epi_warps);
        }
        mbar_init(&tail->drain, 1);
        tail->dead = 0;
        mbar_fence_init();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_w) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_a) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tail->tmem_base)),
                     "n"(T::tmem_cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    griddep_wait();
    // segments, kept inside the buffer whatever the offsets hold
    for (int e = (int)threadIdx.x; e < p.E; e += T::threads) {
        const long long off = p.expert_offset[e];
        const long long cnt = p.expert_count ? (long long)p.expert_count[e] : (long long)p.expert_offset[e + 1] - off;
        const bool ok = off >= 0 && off <= p.a_rows;
        s_off[e] = ok ? (int)off : 0;
        s_cnt[e] = ok ? (int)max(0ll, min(cnt, p.a_rows - off)) : 0;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == 0) {                                                 // prefix of row tiles
        int carry = 0;
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            const int own = e0 + lane < p.E ? tiles_of(s_cnt[e0 + lane], BN) : 0;
            int v = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (e0 + lane < p.E) s_base[e0 + lane] = carry + v - own;
            carry += __shfl_sync(0xffffffffu, v, 31);
        }
        if (lane == 0) s_base[p.E] = carry;
    }
    __syncthreads();
    const uint32_t tmem = tail->tmem_base;
    const unsigned n_tiles = (unsigned)s_base[p.E] * (unsigned)p.m_tiles;
    volatile int* dead = &tail->dead;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true, exhausted = false;
            unsigned t = blockIdx.x < n_tiles ? blockIdx.x : kNoUnit;
            for (uint32_t n = 0; ok; ++n) {
                // hand the tile to the other warps (kNoUnit ends their loops), then claim the next one
                if (!wait_or_dead(&tail->claim_empty[n % kClaims], ((n / kClaims) & 1) ^ 1, dead, p.status)) break;
                tail->claim[n % kClaims] = t;
                mbar_arrive(&tail->claim_full[n % kClaims]);
                if (t == kNoUnit) break;
                const unsigned next = claim_unit(p.wq, n_tiles, gridDim.x, exhausted);
                const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
                const int boxes = (w.rows + T::box_rows - 1) / T::box_rows;
                const uint32_t bytes = (uint32_t)(T::w_stage + boxes * T::box_rows * kKBytes);
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages;
                    if (!wait_or_dead(&tail->empty[s], ((it / T::stages) & 1) ^ 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    uint32_t expect = bytes;
#ifdef STRATA_TEST_HOOKS
                    if (p.test_flags && blockIdx.x == 0 && it == 0) expect += 16;
#endif
                    mbar_expect_tx(&tail->full[s], expect);
                    unsigned char* dw = s_w + s * T::w_stage;
                    if constexpr (GATED) {                           // [2E][channels / 2][inner]: gate, up
                        constexpr int kRows = MB * kM / 2;
#pragma unroll
                        for (int g = 0; g < 2; ++g)
                            tma_load_3d(dw + g * kRows * kKBytes, &p.map_w, kb * kKBytes, w.m * kRows, 2 * w.e + g, &tail->full[s]);
                    } else {
#pragma unroll
                        for (int b = 0; b < MB; ++b)
                            tma_load_3d(dw + b * kBlock, &p.map_w, kb * kKBytes, (w.m * MB + b) * kM, w.e, &tail->full[s]);
                    }
                    for (int b = 0; b < boxes; ++b)
                        tma_load_2d(s_a + s * T::a_stage + b * T::box_rows * kKBytes, &p.map_a, kb * kKBytes,
                                    w.row0 + b * T::box_rows, &tail->full[s]);
                }
                t = next;
            }
            tail->issued = it;
        }
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t it = 0, use = 0;
            bool ok = true;
            for (; ok; ++use) {
                unsigned t;
                if (!next_tile(*tail, use, t, dead, p.status)) break;
                mbar_arrive(&tail->claim_empty[use % kClaims]);
                if (t == kNoUnit) break;
                const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
                const uint32_t idesc = instr_desc<INT8>((w.rows + 15) & ~15);
                const uint32_t buf = use % T::bufs;
                if (!wait_or_dead(&tail->tmem_empty[buf], ((use / T::bufs) & 1) ^ 1, dead, p.status)) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * MB * BN;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages;
                    if (!wait_or_dead(&tail->full[s], (it / T::stages) & 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    const uint64_t dw = smem_desc(smem_addr(s_w + s * T::w_stage));
                    const uint64_t da = smem_desc(smem_addr(s_a + s * T::a_stage));
#pragma unroll
                    for (int k = 0; k < kKBytes / kUmmaK; ++k)
#pragma unroll
                        for (int b = 0; b < MB; ++b)
                            mma<INT8>(d + b * BN, dw + b * (kBlock >> 4) + k * (kUmmaK >> 4), da + k * (kUmmaK >> 4), idesc,
                                      (kb | k) != 0);
                    mma_commit(&tail->empty[s]);
                }
                if (ok) mma_commit(&tail->tmem_full[buf]);
            }
            if (*dead) {                                             // instructions in flight must end before TMEM is freed
                mma_commit(&tail->drain);
                mbar_wait_bounded(&tail->drain, 0);
            }
        }
    } else {
        const int ew = warp - 2, quad = warp & 3;                    // TMEM lanes 32*quad .. of this warp
        const int col0 = (ew >> 2) * T::cols;                        // first column of this warp
        float* scale = s_scale + ew * T::cols;
        const int half = p.channels / 2;
        uint32_t use = 0;
        for (;; ++use) {
            unsigned t;
            const bool got = next_tile(*tail, use, t, dead, p.status);
            if constexpr (GATED && MB == 1) {                        // the two warps of an exchange leave together
                if (!pair_all(got, quad & 1)) break;
            } else if (!__all_sync(0xffffffffu, got)) {
                break;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&tail->claim_empty[use % kClaims]);
            if (t == kNoUnit) break;
            const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
            const uint32_t buf = use % T::bufs;
            const int rows = min(T::cols, w.rows - col0);            // of this warp; may be negative
            const float* ws = p.w_scale + (size_t)w.e * p.channels;
            // channel(s) of w that this lane holds, and the first channel of out
            int ch[2], out_ch[2];
            if constexpr (GATED && MB == 1) {
                out_ch[0] = w.m * (kM / 2) + (quad & 1) * 32 + lane;
                ch[0] = out_ch[0] + (quad >> 1) * half;
            } else if constexpr (GATED) {
                out_ch[0] = ch[0] = w.m * kM + quad * 32 + lane;
                ch[1] = ch[0] + half;
            } else {
#pragma unroll
                for (int b = 0; b < MB; ++b) out_ch[b] = ch[b] = (w.m * MB + b) * kM + quad * 32 + lane;
            }
            const int limit = GATED ? half : p.channels;
            const bool words = p.out_words != 0;
            float wsc[2];
#pragma unroll
            for (int b = 0; b < MB; ++b) wsc[b] = out_ch[GATED ? 0 : b] < limit ? ws[ch[b]] : 0.0f;
            __syncwarp();
            for (int c = lane; c < T::cols; c += 32)
                scale[c] = c < rows ? p.a_scale[(long long)(w.row0 + col0 + c) * p.a_scale_stride] : 0.0f;
            __syncwarp();
            const bool ok = wait_or_dead(&tail->tmem_full[buf], (use / T::bufs) & 1, dead, p.status);
            if constexpr (GATED && MB == 1) {
                if (!pair_all(ok, quad & 1)) break;
            } else if (!__all_sync(0xffffffffu, ok)) {
                break;
            }
            tmem_fence_after();
            const uint32_t addr = tmem + buf * MB * BN + ((uint32_t)(quad * 32) << 16) + col0;
            uint16_t* out = p.out + (long long)(w.row0 + col0) * p.out_stride;
            int phase = 0;
            for (int c0 = 0; c0 < rows; c0 += 16, phase ^= 1) {
                __syncwarp();                                        // loads from TMEM ask for converged warps: waits and stores part them
                float sc[16];
#pragma unroll
                for (int c = 0; c < 16; c += 4) *reinterpret_cast<float4*>(&sc[c]) = *reinterpret_cast<const float4*>(&scale[c0 + c]);
                if constexpr (GATED && MB == 1) {
                    uint32_t v[16];
                    tmem_ld16(v, addr + c0);
                    tmem_ld_wait(v);
                    float y[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) y[c] = acc_value<INT8>(v[c]) * (sc[c] * wsc[0]);
                    // the gate's warp finishes columns 0..7, up's warp columns 8..15
                    const bool up = quad >> 1;
                    float* mine = s_swap + (ew * 2 + phase) * 8 * 32 + lane;
                    const float* theirs = s_swap + ((ew ^ 2) * 2 + phase) * 8 * 32 + lane;
#pragma unroll
                    for (int c = 0; c < 8; ++c) mine[c * 32] = up ? y[c] : y[8 + c];
                    asm volatile("bar.sync %0, 64;" ::"r"(1 + (quad & 1)) : "memory");
                    float o[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float other = theirs[c * 32];
                        o[c] = up ? gate_mul(other, y[8 + c]) : gate_mul(y[c], other);
                    }
                    const int shift = up ? 8 : 0;
                    store_pairs<8>(o, lane, out + (long long)(c0 + shift) * p.out_stride, p.out_stride, rows - c0 - shift, out_ch[0],
                                   limit, words);
                } else if constexpr (GATED) {
                    uint32_t g[16], u[16];
                    tmem_ld16(g, addr + c0);
                    tmem_ld16(u, addr + BN + c0);
                    tmem_ld_wait(g);
                    tmem_ld_wait(u);
                    float y[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        y[c] = gate_mul(acc_value<INT8>(g[c]) * (sc[c] * wsc[0]), acc_value<INT8>(u[c]) * (sc[c] * wsc[1]));
                    store_pairs<16>(y, lane, out + (long long)c0 * p.out_stride, p.out_stride, rows - c0, out_ch[0], limit, words);
                } else {
#pragma unroll
                    for (int b = 0; b < MB; ++b) {
                        uint32_t v[16];
                        tmem_ld16(v, addr + b * BN + c0);
                        tmem_ld_wait(v);
                        float y[16];
#pragma unroll
                        for (int c = 0; c < 16; ++c) y[c] = acc_value<INT8>(v[c]) * (sc[c] * wsc[b]);
                        store_pairs<16>(y, lane, out + (long long)c0 * p.out_stride, p.out_stride, rows - c0, out_ch[b], limit, words);
                    }
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tail->tmem_empty[buf]);
        }
    }
    __syncwarp();
    griddep_launch_dependents();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (threadIdx.x == 0 && *dead) {                                 // loads in flight must land before the CTA leaves
        const uint32_t it = tail->issued, first = it > (uint32_t)T::stages ? it - T::stages : 0;
        for (uint32_t u = first; u < it; ++u) mbar_wait_bounded(&tail->full[u % T::stages], (u / T::stages) & 1);
    }
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(T::tmem_cols) : "memory");
}

template <int MB, int BN>
size_t smem_bytes(int E)
{
    using T = Tile<MB, BN>;
    return 1024 + T::data_bytes + sizeof(SmemTail) + (size_t)(T::epi_warps * T::cols + T::swap_floats) * sizeof(float) +
           (size_t)(3 * E + 1) * sizeof(int);
}

template <int MB, int BN>
cudaError_t run(const strata_moe_shape& s, const strata_matmul_args& a, MatParams& p, int n_sm, cudaStream_t st)
{
    using T = Tile<MB, BN>;
    {
        const cuuint64_t dims[2] = {(cuuint64_t)a.inner, (cuuint64_t)a.a_rows};
        const cuuint64_t strides[1] = {(cuuint64_t)a.a_stride};
        const cuuint32_t box[2] = {(cuuint32_t)kKBytes, (cuuint32_t)T::box_rows};
        if (!encode(&p.map_a, a.a, 2, dims, strides, box)) return cudaErrorInvalidValue;
    }
    {   // [E][channels][inner]; gated: [2E][channels / 2][inner], gate and up of an expert in turn
        const cuuint64_t k = (cuuint64_t)a.inner, rows = (cuuint64_t)a.channels / (a.gated ? 2 : 1);
        const cuuint64_t dims[3] = {k, rows, (cuuint64_t)s.E * (a.gated ? 2 : 1)};
        const cuuint64_t strides[2] = {k, rows * k};
        const cuuint32_t box[3] = {(cuuint32_t)kKBytes, (cuuint32_t)(a.gated ? MB * kM / 2 : kM), 1};
        if (!encode(&p.map_w, a.w, 3, dims, strides, box)) return cudaErrorInvalidValue;
    }
    const int per_tile = MB * kM / (a.gated ? 2 : 1), wide = a.channels / (a.gated ? 2 : 1);
    p.m_tiles = (wide + per_tile - 1) / per_tile;
    const long long tiles = row_tiles(s, a.a_rows, BN) * p.m_tiles;
    if (tiles >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)min(tiles, (long long)n_sm);
    const size_t smem = smem_bytes<MB, BN>(s.E);
    if (a.type == STRATA_T_INT8)
        return a.gated ? launch_pdl(expert_matmul_kernel<true, true, MB, BN>, grid, T::threads, smem, st, p)
                       : launch_pdl(expert_matmul_kernel<true, false, MB, BN>, grid, T::threads, smem, st, p);
    return a.gated ? launch_pdl(expert_matmul_kernel<false, true, MB, BN>, grid, T::threads, smem, st, p)
                   : launch_pdl(expert_matmul_kernel<false, false, MB, BN>, grid, T::threads, smem, st, p);
}

template <int MB, int BN>
cudaError_t configure()
{
    const void* fns[4] = {(const void*)expert_matmul_kernel<true, true, MB, BN>,
                          (const void*)expert_matmul_kernel<true, false, MB, BN>,
                          (const void*)expert_matmul_kernel<false, true, MB, BN>,
                          (const void*)expert_matmul_kernel<false, false, MB, BN>};
    for (const void* f : fns) {
        const cudaError_t e =
            cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<MB, BN>(kMaxExperts));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_matmul_kernels()
{
    cudaError_t e = configure<1, 64>();
    if (e == cudaSuccess) e = configure<2, 128>();
    if (e == cudaSuccess) e = configure<2, 256>();
    return e;
}

cudaError_t launch_expert_matmul(const strata_moe_shape& s, const strata_moe_layout_t& L, const strata_matmul_args& a,
                                 int* status, WorkQueue wq, int n_sm, cudaStream_t st)
{
    MatParams p;
    p.expert_count = s.slot_capacity > 0 ? nullptr : L.expert_count;
    p.expert_offset = L.expert_offset;
    p.a_scale = a.a_scale;
    p.w_scale = a.w_scale;
    p.out = static_cast<uint16_t*>(a.out);
    p.status = status;
    p.wq = wq;
#ifdef STRATA_TEST_HOOKS
    p.test_flags = g_inject_short_load.exchange(0);
#endif
    p.a_rows = a.a_rows;
    p.a_scale_stride = a.a_scale_stride;
    p.out_stride = a.out_stride;
    p.E = s.E;
    p.k_blocks = (a.inner + kKBytes - 1) / kKBytes;
    p.channels = a.channels;
    p.out_words = a.channels % (a.gated ? 4 : 2) == 0 && a.out_stride % 2 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 3u) == 0;
    // Which tile: the shortest estimate of rounds * (inner blocks * c + f) over the GPU, where c is what one inner block of a
    // tile takes and f what a tile adds (its epilogue where the accumulators are not doubled, the ring's refill).  The
    // constants were fitted to 116 measured shapes (8 and 32 experts, 2 .. 2048 mean rows, inner 512 .. 7168, 512 .. 4096
    // channels, even and Zipf routing); the choice is on average 2 % above the best of the three, and 30 % above at
    // worst, where a skewed routing has other tiles than the mean.  At 7168 -> 4096 gated, 32 experts: one token
    // <1,64> 45 us, <2,128> 42 us; 32 rows each 149, 156 (<2,256> 163); 128 rows 337, 185, 178; 512 rows 1149, 469, 396.
    // Where the weights' way from HBM takes longer than that, smaller tiles spread it better over the SMs: 1.03, 1.08 and 1.13
    // of the bytes at the measured copy rate (149, 156, 163 us against 144 us at 32 rows each).
    // What the estimate does not see: rows spread around their mean (at a multiple of the height half of the experts spill into one
    // more tile), that a partly filled tile takes fewer matrix cycles (at 128 rows each it says 155 and 259 us for the two larger
    // ones, and takes the one that is 4 % slower), and slots that are masked or unrouted (a call's rows are known on the device only).
    struct Cost { int mb, bn; float c, f, hbm; };
    static const Cost costs[3] = {{1, 64, 0.37f, 0.65f, 1.03f}, {2, 128, 0.66f, 1.06f, 1.08f}, {2, 256, 1.22f, 2.78f, 1.13f}};
    constexpr float kHbmBytesPerUs = 6.55e6f;
    const long long items = s.slot_capacity > 0 ? (long long)s.E * s.R * s.slot_capacity : (long long)s.R * s.T * s.K;
    const long long used = min(items, (long long)s.E), mean = (items + s.E - 1) / s.E;
    int v = 0;
    float least = 0.0f;
    for (int i = 0; i < 3; ++i) {
        const int per_tile = costs[i].mb * kM / (a.gated ? 2 : 1), wide = a.channels / (a.gated ? 2 : 1);
        const float tiles = (float)(used * ((mean + costs[i].bn - 1) / costs[i].bn) * ((wide + per_tile - 1) / per_tile));
        const float rounds = tiles > (float)n_sm ? tiles / (float)n_sm + 0.19f : 1.0f;
        const float bytes_us = (float)used * (float)a.channels * (float)a.inner / kHbmBytesPerUs;
        const float cost = max(rounds * ((float)p.k_blocks * costs[i].c + costs[i].f), bytes_us * costs[i].hbm);
        if (i == 0 || cost < least) {
            least = cost;
            v = i;
        }
    }
    v = (int)tune("STRATA_MM", v);
    switch (v) {
        case 0: return run<1, 64>(s, a, p, n_sm, st);
        case 1: return run<2, 128>(s, a, p, n_sm, st);
        default: return run<2, 256>(s, a, p, n_sm, st);
    }
}

}  // namespace strata

#ifdef STRATA_TEST_HOOKS
extern "C" void strata_test_inject_short_load(int on) { strata::g_inject_short_load.store(on); }
#endif
