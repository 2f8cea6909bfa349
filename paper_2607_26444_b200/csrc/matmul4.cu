// The experts' products over the receive buffer in 4 bits: e2m1 codes with a scale per block of 32 (a power of two) or 16 (e4m3)
// values of a row, grouped by expert as the routing layout orders them, times each expert's 4-bit weights (strata_layer.h has the
// formulas).  The matrix instructions take the block scales themselves, from TMEM.
//
// As in 8 bits the weights are the M operand and the rows the N operand (matmul.cu).  A stage is 128 bytes of codes of every row, 256
// values, which is one swizzle span, and a box of 16 scale bytes of every row.  The instructions want the scales of 128 rows as
// 32 lines of 4 words, one word (4 scales) of rows l, l + 32, l + 64 and l + 96 per line: TMA brings 128 rows of 4 words, and a
// warp turns them in place, lane l the 4 x 4 words of its four rows.
#include "tiles.cuh"

namespace strata {

namespace {

constexpr int kM = 128;                 // channels of a matrix instruction
constexpr int kKBytes = 128;            // bytes of codes of a row in a stage: one swizzle span, 256 values
constexpr int kUmmaK = 32;              // the same of a matrix instruction: 64 values
constexpr int kBlock = kM * kKBytes;    // codes of one 128-row block of weights in a stage
constexpr int kScaleBox = 16;           // scale bytes of a row in a stage
constexpr int kScales = kM * kScaleBox; // scales of 128 rows

// A tile is MB blocks of 128 weight rows by up to BN rows of the N operand (see matmul.cu for the gated forms).
template <bool NV, int MB, int BN>
struct Tile4 {
    static constexpr int box_rows = BN >= 192 ? 64 : 32;            // rows of one TMA box of the N operand
    static constexpr int n_blocks = (BN + 127) / 128;
    static constexpr int w_stage = MB * kBlock, a_stage = BN * kKBytes;
    static constexpr int ws_stage = MB * kScales, as_stage = n_blocks * kScales;
    static constexpr int stage_bytes = w_stage + a_stage + ws_stage + as_stage;
    static constexpr int stages = 208 * 1024 / stage_bytes < 8 ? 208 * 1024 / stage_bytes : 8;
    static constexpr int words = NV ? 4 : 2;                        // scale words of a row that a stage uses
    static constexpr int sw_cols = MB * words * 4, sa_cols = n_blocks * words * 4;    // TMEM columns of a stage's scales
    static constexpr int scale_cols = 2 * (sw_cols + sa_cols);      // two stages in turn
    static constexpr int bufs = 2 * MB * BN + scale_cols <= 512 ? 2 : 1;
    static constexpr int acc_cols = bufs * MB * BN;
    static constexpr int used_cols = acc_cols + scale_cols;
    static constexpr int tmem_cols = used_cols <= 128 ? 128 : used_cols <= 256 ? 256 : 512;
    static constexpr int epi_warps = MB == 2 ? 8 : 4;
    static constexpr int threads = 128 + 32 * epi_warps;            // warps 0: loads, 1: matrix instructions, 2 and 3: scales
    static constexpr int cols = BN / (epi_warps / 4);
    static constexpr int swap_floats = MB == 1 ? epi_warps * 2 * 8 * 32 : 0;
    static constexpr size_t data_bytes = (size_t)stages * stage_bytes;
    static_assert(used_cols <= 512 && stages >= 2 && cols % 16 == 0 && a_stage % 1024 == 0 && data_bytes % 1024 == 0, "");
};

struct Mat4Params {
    CUtensorMap map_w, map_a, map_ws, map_as;
    const int32_t* expert_count;        // NULL: segments are full (fixed-capacity layout)
    const int32_t* expert_offset;
    const float* a_scale;               // NULL: 1
    const float* w_scale;               // NULL: 1
    uint16_t* out;
    int* status;
    WorkQueue wq;
    long long a_rows, a_scale_stride, w_scale_stride, out_stride;
    int E, k_blocks, channels, m_tiles; // channels: rows of w per expert
    int last_steps;                     // matrix instructions of the last inner block
    int out_words;                      // pairs of channels of out lie on 4 bytes
};

constexpr int kClaims = 4;              // tiles that the loading warp may be ahead of the epilogue

struct Smem4Tail {                      // behind the operand stages
    uint64_t full[8], ready[8], empty[8], tmem_full[2], tmem_empty[2], drain;
    uint64_t claim_full[kClaims], claim_empty[kClaims];
    unsigned claim[kClaims];
    uint32_t tmem_base, issued;
    int dead, pad[3];
};
static_assert(sizeof(Smem4Tail) % 16 == 0, "the scales behind it are read in vectors");

// Descriptor of 32 lines of 16 bytes without a swizzle: 128 bytes between groups of eight lines.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// Instruction descriptor: A and B e2m1, K-major; scales e8m0 or e4m3; `id`: first of the instruction's scales in their word.
template <bool NV>
__device__ __forceinline__ uint32_t instr_desc4(int n, int id)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (NV ? 0u : 1u << 23) | ((uint32_t)(kM >> 7) << 27) |
           ((uint32_t)id << 4) | ((uint32_t)id << 29);
}
template <bool NV>
__device__ __forceinline__ void mma4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                     uint32_t accumulate)
{
    if constexpr (NV)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
}

// 128 rows of four words become, for each of the four, 32 lines of one word of rows l, l + 32, l + 64 and l + 96.  A lane reads
// and writes the same 64 bytes.
__device__ __forceinline__ void turn_scales(unsigned char* block, int lane)
{
    uint4* at = reinterpret_cast<uint4*>(block) + lane;
    const uint4 a = at[0], b = at[32], c = at[64], d = at[96];
    at[0] = make_uint4(a.x, b.x, c.x, d.x);
    at[32] = make_uint4(a.y, b.y, c.y, d.y);
    at[64] = make_uint4(a.z, b.z, c.z, d.z);
    at[96] = make_uint4(a.w, b.w, c.w, d.w);
}

__device__ __forceinline__ bool next_tile(Smem4Tail& tail, uint32_t n, unsigned& t, volatile int* dead, int* status)
{
    if (!wait_or_dead(&tail.claim_full[n % kClaims], (n / kClaims) & 1, dead, status)) return false;
    t = *reinterpret_cast<volatile unsigned*>(&tail.claim[n % kClaims]);
    return true;
}

template <bool NV, bool GATED, int MB, int BN>
__global__ void __launch_bounds__(Tile4<NV, MB, BN>::threads, 1) expert_matmul4_kernel(const __grid_constant__ Mat4Params p)
{
    using T = Tile4<NV, MB, BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_w = smem;                                       // [stages][MB * 128][128]
    unsigned char* s_a = s_w + T::stages * T::w_stage;               // [stages][BN][128]
    unsigned char* s_ws = s_a + T::stages * T::a_stage;              // [stages][MB * 128][16]
    unsigned char* s_as = s_ws + T::stages * T::ws_stage;            // [stages][n_blocks * 128][16]
    Smem4Tail* tail = reinterpret_cast<Smem4Tail*>(smem + T::data_bytes);
    float* s_scale = reinterpret_cast<float*>(tail + 1);             // [epilogue warps][cols]
    float* s_swap = s_scale + T::epi_warps * T::cols;                // [epilogue warps][2][8][32]
    int* s_base = reinterpret_cast<int*>(s_swap + T::swap_floats);   // [E + 1]
    int* s_off = s_base + p.E + 1;                                   // [E]
    int* s_cnt = s_off + p.E;                                        // [E]
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < T::stages; ++s) {
            mbar_init(&tail->full[s], 1);
            mbar_init(&tail->ready[s], 2);
            mbar_init(&tail->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tail->tmem_full[b], 1);
            mbar_init(&tail->tmem_empty[b], T::epi_warps);
        }
        for (int c = 0; c < kClaims; ++c) {
            mbar_init(&tail->claim_full[c], 1);
            mbar_init(&tail->claim_empty[c], 3 + T::epi_warps);
        }
        mbar_init(&tail->drain, 1);
        tail->dead = 0;
        mbar_fence_init();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_w) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_ws) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_as) : "memory");
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
                const uint32_t bytes = (uint32_t)(T::w_stage + T::ws_stage + boxes * T::box_rows * (kKBytes + kScaleBox));
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages;
                    if (!wait_or_dead(&tail->empty[s], ((it / T::stages) & 1) ^ 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    mbar_expect_tx(&tail->full[s], bytes);
                    unsigned char* dw = s_w + s * T::w_stage;
                    unsigned char* ds = s_ws + s * T::ws_stage;
                    const int sx = (NV ? kb : kb >> 1) * kScaleBox;  // two blocks of 256 values share a box of 16 scales of 32
                    if constexpr (GATED) {                           // [2E][channels / 2][inner]: gate, up
                        constexpr int kRows = MB * kM / 2;
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            tma_load_3d(dw + g * kRows * kKBytes, &p.map_w, kb * kKBytes, w.m * kRows, 2 * w.e + g, &tail->full[s]);
                            tma_load_3d(ds + g * kRows * kScaleBox, &p.map_ws, sx, w.m * kRows, 2 * w.e + g, &tail->full[s]);
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < MB; ++b) {
                            tma_load_3d(dw + b * kBlock, &p.map_w, kb * kKBytes, (w.m * MB + b) * kM, w.e, &tail->full[s]);
                            tma_load_3d(ds + b * kScales, &p.map_ws, sx, (w.m * MB + b) * kM, w.e, &tail->full[s]);
                        }
                    }
                    for (int b = 0; b < boxes; ++b) {
                        tma_load_2d(s_a + s * T::a_stage + b * T::box_rows * kKBytes, &p.map_a, kb * kKBytes,
                                    w.row0 + b * T::box_rows, &tail->full[s]);
                        tma_load_2d(s_as + s * T::as_stage + b * T::box_rows * kScaleBox, &p.map_as, sx, w.row0 + b * T::box_rows,
                                    &tail->full[s]);
                    }
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
                const int n = (w.rows + 15) & ~15;
                const uint32_t buf = use % T::bufs;
                if (!wait_or_dead(&tail->tmem_empty[buf], ((use / T::bufs) & 1) ^ 1, dead, p.status)) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * MB * BN;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages, parity = (it / T::stages) & 1;
                    if (!wait_or_dead(&tail->full[s], parity, dead, p.status) || !wait_or_dead(&tail->ready[s], parity, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    const uint64_t dw = smem_desc(smem_addr(s_w + s * T::w_stage));
                    const uint64_t da = smem_desc(smem_addr(s_a + s * T::a_stage));
                    const uint32_t sw = tmem + T::acc_cols + (it & 1) * (T::sw_cols + T::sa_cols), sa = sw + T::sw_cols;
                    const int first = NV ? 0 : (kb & 1) * 2;         // word of the box that this stage begins with
                    const uint64_t qw = scale_desc(smem_addr(s_ws + s * T::ws_stage) + first * 512);
                    const uint64_t qa = scale_desc(smem_addr(s_as + s * T::as_stage) + first * 512);
#pragma unroll
                    for (int i = 0; i < T::words; ++i) {
#pragma unroll
                        for (int b = 0; b < MB; ++b) copy_scales(sw + (b * T::words + i) * 4, qw + b * (kScales >> 4) + i * (512 >> 4));
#pragma unroll
                        for (int b = 0; b < T::n_blocks; ++b)
                            copy_scales(sa + (i * T::n_blocks + b) * 4, qa + b * (kScales >> 4) + i * (512 >> 4));
                    }
                    const int steps = kb == p.k_blocks - 1 ? p.last_steps : kKBytes / kUmmaK;
#pragma unroll
                    for (int k = 0; k < kKBytes / kUmmaK; ++k) {
                        if (k < steps) {
                            const int i = NV ? k : k >> 1;
                            const uint32_t idesc = instr_desc4<NV>(n, NV ? 0 : (k & 1) * 2);
#pragma unroll
                            for (int b = 0; b < MB; ++b)
                                mma4<NV>(d + b * BN, dw + b * (kBlock >> 4) + k * (kUmmaK >> 4), da + k * (kUmmaK >> 4), idesc,
                                         sw + (b * T::words + i) * 4, sa + i * T::n_blocks * 4, (kb | k) != 0);
                        }
                    }
                    mma_commit(&tail->empty[s]);
                }
                if (ok) mma_commit(&tail->tmem_full[buf]);
            }
            if (*dead) {                                             // instructions in flight must end before TMEM is freed
                mma_commit(&tail->drain);
                mbar_wait_bounded(&tail->drain, 0);
            }
        }
    } else if (warp < 4) {                                           // warp 2: scales of the weights, warp 3: of the rows
        uint32_t it = 0, use = 0;
        bool ok = true;
        unsigned char* base = warp == 2 ? s_ws : s_as;
        const int stage = warp == 2 ? T::ws_stage : T::as_stage;
        for (; ok; ++use) {
            unsigned t;
            if (!__all_sync(0xffffffffu, next_tile(*tail, use, t, dead, p.status))) break;
            if (lane == 0) mbar_arrive(&tail->claim_empty[use % kClaims]);
            if (t == kNoUnit) break;
            for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                const uint32_t s = it % T::stages;
                ok = __all_sync(0xffffffffu, wait_or_dead(&tail->full[s], (it / T::stages) & 1, dead, p.status));
                if (!ok) break;
                for (int b = 0; b < stage; b += kScales) turn_scales(base + s * stage + b, lane);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&tail->ready[s]);
            }
        }
    } else {
        const int ew = warp - 4, quad = warp & 3;                    // TMEM lanes 32*quad .. of this warp
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
            for (int b = 0; b < MB; ++b)
                wsc[b] = p.w_scale && out_ch[GATED ? 0 : b] < limit
                             ? p.w_scale[((long long)w.e * p.channels + ch[b]) * p.w_scale_stride]
                             : 1.0f;
            __syncwarp();
            for (int c = lane; c < T::cols; c += 32)
                scale[c] = p.a_scale && c < rows ? p.a_scale[(long long)(w.row0 + col0 + c) * p.a_scale_stride] : 1.0f;
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
                    for (int c = 0; c < 16; ++c) y[c] = __uint_as_float(v[c]) * (sc[c] * wsc[0]);
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
                        y[c] = gate_mul(__uint_as_float(g[c]) * (sc[c] * wsc[0]), __uint_as_float(u[c]) * (sc[c] * wsc[1]));
                    store_pairs<16>(y, lane, out + (long long)c0 * p.out_stride, p.out_stride, rows - c0, out_ch[0], limit, words);
                } else {
#pragma unroll
                    for (int b = 0; b < MB; ++b) {
                        uint32_t v[16];
                        tmem_ld16(v, addr + b * BN + c0);
                        tmem_ld_wait(v);
                        float y[16];
#pragma unroll
                        for (int c = 0; c < 16; ++c) y[c] = __uint_as_float(v[c]) * (sc[c] * wsc[b]);
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

template <bool NV, int MB, int BN>
size_t smem_bytes4(int E)
{
    using T = Tile4<NV, MB, BN>;
    return 1024 + T::data_bytes + sizeof(Smem4Tail) + (size_t)(T::epi_warps * T::cols + T::swap_floats) * sizeof(float) +
           (size_t)(3 * E + 1) * sizeof(int);
}

template <bool NV, int MB, int BN>
cudaError_t run4(const strata_moe_shape& s, const strata_matmul4_args& a, Mat4Params& p, int n_sm, cudaStream_t st)
{
    using T = Tile4<NV, MB, BN>;
    const cuuint64_t groups = (cuuint64_t)s.E * (a.gated ? 2 : 1), rows = (cuuint64_t)a.channels / (a.gated ? 2 : 1);
    const cuuint32_t w_rows = (cuuint32_t)(a.gated ? MB * kM / 2 : kM);
    const cuuint64_t bytes[2] = {(cuuint64_t)a.inner / 2, (cuuint64_t)a.inner / (NV ? 16 : 32)};
    const cuuint32_t box[2] = {kKBytes, kScaleBox};
    const strata_rows4* ops[2] = {&a.w, &a.a};
    CUtensorMap* maps[2][2] = {{&p.map_w, &p.map_ws}, {&p.map_a, &p.map_as}};
    for (int o = 0; o < 2; ++o)
        for (int i = 0; i < 2; ++i) {                                // codes, block scales
            const void* base = i == 0 ? ops[o]->codes : ops[o]->block;
            const cuuint64_t stride = (cuuint64_t)(i == 0 ? ops[o]->code_stride : ops[o]->block_stride);
            // weights: [E][channels]; gated: [2E][channels / 2], gate and up of an expert in turn
            const cuuint64_t dims[3] = {bytes[i], o == 0 ? rows : (cuuint64_t)a.a_rows, groups};
            const cuuint64_t strides[2] = {stride, rows * stride};
            const cuuint32_t boxes[3] = {box[i], o == 0 ? w_rows : (cuuint32_t)T::box_rows, 1};
            if (!encode(maps[o][i], base, o == 0 ? 3 : 2, dims, strides, boxes,
                        i == 0 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE))
                return cudaErrorInvalidValue;
        }
    const int per_tile = MB * kM / (a.gated ? 2 : 1), wide = a.channels / (a.gated ? 2 : 1);
    p.m_tiles = (wide + per_tile - 1) / per_tile;
    const long long tiles = row_tiles(s, a.a_rows, BN) * p.m_tiles;
    if (tiles >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)min(tiles, (long long)n_sm);
    const size_t smem = smem_bytes4<NV, MB, BN>(s.E);
    return a.gated ? launch_pdl(expert_matmul4_kernel<NV, true, MB, BN>, grid, T::threads, smem, st, p)
                   : launch_pdl(expert_matmul4_kernel<NV, false, MB, BN>, grid, T::threads, smem, st, p);
}

template <bool NV, int MB, int BN>
cudaError_t configure4()
{
    const void* fns[2] = {(const void*)expert_matmul4_kernel<NV, true, MB, BN>, (const void*)expert_matmul4_kernel<NV, false, MB, BN>};
    for (const void* f : fns) {
        const cudaError_t e =
            cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes4<NV, MB, BN>(kMaxExperts));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
template <bool NV>
cudaError_t configure4_all()
{
    cudaError_t e = configure4<NV, 1, 64>();
    if (e == cudaSuccess) e = configure4<NV, 2, 96>();
    if (e == cudaSuccess) e = configure4<NV, 2, 192>();
    return e;
}

template <bool NV>
cudaError_t pick4(int v, const strata_moe_shape& s, const strata_matmul4_args& a, Mat4Params& p, int n_sm, cudaStream_t st)
{
    switch (v) {
        case 0: return run4<NV, 1, 64>(s, a, p, n_sm, st);
        case 1: return run4<NV, 2, 96>(s, a, p, n_sm, st);
        default: return run4<NV, 2, 192>(s, a, p, n_sm, st);
    }
}

}  // namespace

cudaError_t configure_matmul4_kernels()
{
    const cudaError_t e = configure4_all<false>();
    return e == cudaSuccess ? configure4_all<true>() : e;
}

cudaError_t launch_expert_matmul4(const strata_moe_shape& s, const strata_moe_layout_t& L, const strata_matmul4_args& a,
                                  int* status, WorkQueue wq, int n_sm, cudaStream_t st)
{
    Mat4Params p;
    p.expert_count = s.slot_capacity > 0 ? nullptr : L.expert_count;
    p.expert_offset = L.expert_offset;
    p.a_scale = a.a.scale;
    p.w_scale = a.w.scale;
    p.out = static_cast<uint16_t*>(a.out);
    p.status = status;
    p.wq = wq;
    p.a_rows = a.a_rows;
    p.a_scale_stride = a.a.scale_stride;
    p.w_scale_stride = a.w.scale_stride;
    p.out_stride = a.out_stride;
    p.E = s.E;
    p.k_blocks = (a.inner / 2 + kKBytes - 1) / kKBytes;
    p.last_steps = (a.inner / 2 - (p.k_blocks - 1) * kKBytes + kUmmaK - 1) / kUmmaK;
    p.channels = a.channels;
    p.out_words = a.channels % (a.gated ? 4 : 2) == 0 && a.out_stride % 2 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 3u) == 0;
    const long long items = s.slot_capacity > 0 ? (long long)s.E * s.R * s.slot_capacity : (long long)s.R * s.T * s.K;
    const long long mean = (items + s.E - 1) / s.E;
    const int v = (int)tune("STRATA_MM4", mean <= 64 ? 0 : mean <= 192 ? 1 : 2);
    return a.type == STRATA_T_NVF4 ? pick4<true>(v, s, a, p, n_sm, st) : pick4<false>(v, s, a, p, n_sm, st);
}

}  // namespace strata
