// The experts' products over the receive buffer: 8-bit rows, grouped by expert as the routing layout orders them, times
// each expert's 8-bit weights (strata_layer.h has the formulas).  tcgen05 matrix instructions, operands brought by TMA
// into 128-byte-swizzled shared memory, accumulators in TMEM, persistent CTAs over tiles found on the device.
//
// The weights are the M operand and the rows the N operand: out^T = W * A^T.  An instruction then always has 128
// channels, and its N (16 .. 256) follows the number of rows that the expert really has, so a decoding step with a
// handful of rows per expert neither multiplies nor fetches 128 rows of padding; it streams the weights.
#include <cuda.h>

#include "layer.cuh"

namespace strata {

namespace {

constexpr int kM = 128;                 // weight rows of a tile (gated: 64 gate rows and 64 up rows, see kGateRows)
constexpr int kGateRows = 16;           // gated: every 32 rows of the tile are 16 of the gate, then the same 16 of up
constexpr int kKBytes = 128;            // inner extent of a stage: one swizzle span
constexpr int kUmmaK = 32;              // bytes of K per matrix instruction
constexpr int kThreads = 192;           // warp 0: loads, warp 1: matrix instructions, warps 2..5: epilogue
constexpr int kAStage = kM * kKBytes;

template <int BN>
struct Tile {
    static constexpr int box_rows = BN >= 128 ? 64 : 32;            // rows of one TMA box of the N operand
    static constexpr int b_stage = BN * kKBytes;
    static constexpr int stages = BN == 256 ? 4 : BN == 128 ? 6 : 8;
    static constexpr int tmem_cols = 2 * BN;                        // two accumulators: one is filled while one is read
    static constexpr size_t data_bytes = (size_t)stages * (kAStage + b_stage);
};

struct MatParams {
    CUtensorMap map_w, map_a;
    const int32_t* expert_count;        // NULL: segments are full (fixed-capacity layout)
    const int32_t* expert_offset;
    const float* a_scale;
    const float* w_scale;
    uint16_t* out;
    int* status;
    long long a_rows, a_scale_stride, out_stride;
    int E, k_blocks, channels, m_tiles; // channels: rows of w per expert
};

struct SmemTail {                       // behind the operand stages
    uint64_t full[8], empty[8], tmem_full[2], tmem_empty[2], drain;
    uint32_t tmem_base, issued;
    int dead, pad[3];
};
static_assert(sizeof(SmemTail) % 16 == 0, "the scales behind it are read in vectors");

// ---- waits with a limit: a wait that runs out sets the status and makes every role of the CTA leave its loop ----
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
__device__ __forceinline__ void mma_commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                 : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t (&r)[32], uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

struct Work {
    int e, m, row0, rows;               // expert, channel tile, first receive row, rows of the tile
};

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

template <bool INT8, bool GATED, int BN>
__global__ void __launch_bounds__(kThreads, 1) expert_matmul_kernel(const __grid_constant__ MatParams p)
{
    using T = Tile<BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_w = smem;                                       // [stages][128][128]
    unsigned char* s_a = smem + T::stages * kAStage;                 // [stages][BN][128]
    SmemTail* tail = reinterpret_cast<SmemTail*>(smem + T::data_bytes);
    float* s_scale = reinterpret_cast<float*>(tail + 1);             // [4][BN]
    int* s_base = reinterpret_cast<int*>(s_scale + 4 * BN);          // [E + 1]
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
            mbar_init(&tail->tmem_empty[b], 4);
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
    for (int e = (int)threadIdx.x; e < p.E; e += kThreads) {
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
            const int own = e0 + lane < p.E ? (s_cnt[e0 + lane] + BN - 1) / BN : 0;
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
            bool ok = true;
            for (unsigned t = blockIdx.x; t < n_tiles && ok; t += gridDim.x) {
                const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
                const int boxes = (w.rows + T::box_rows - 1) / T::box_rows;
                const uint32_t bytes = (uint32_t)(kAStage + boxes * T::box_rows * kKBytes);
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages;
                    if (!wait_or_dead(&tail->empty[s], ((it / T::stages) & 1) ^ 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    mbar_expect_tx(&tail->full[s], bytes);
                    if constexpr (GATED) {
#pragma unroll
                        for (int b = 0; b < kM / kGateRows; ++b)
                            tma_load_3d(s_w + s * kAStage + b * kGateRows * kKBytes, &p.map_w, kb * kKBytes,
                                        w.m * (kM / 2) + (b >> 1) * kGateRows, 2 * w.e + (b & 1), &tail->full[s]);
                    } else
                        tma_load_2d(s_w + s * kAStage, &p.map_w, kb * kKBytes, w.e * p.channels + w.m * kM, &tail->full[s]);
                    for (int b = 0; b < boxes; ++b)
                        tma_load_2d(s_a + s * T::b_stage + b * T::box_rows * kKBytes, &p.map_a, kb * kKBytes,
                                    w.row0 + b * T::box_rows, &tail->full[s]);
                }
            }
            tail->issued = it;
        }
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t it = 0, use = 0;
            bool ok = true;
            for (unsigned t = blockIdx.x; t < n_tiles && ok; t += gridDim.x, ++use) {
                const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
                const uint32_t idesc = instr_desc<INT8>((w.rows + 15) & ~15);
                const uint32_t buf = use & 1;
                if (!wait_or_dead(&tail->tmem_empty[buf], ((use >> 1) & 1) ^ 1, dead, p.status)) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * BN;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const uint32_t s = it % T::stages;
                    if (!wait_or_dead(&tail->full[s], (it / T::stages) & 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    tmem_fence_after();
                    const uint64_t da = smem_desc(smem_addr(s_w + s * kAStage));
                    const uint64_t db = smem_desc(smem_addr(s_a + s * T::b_stage));
#pragma unroll
                    for (int k = 0; k < kKBytes / kUmmaK; ++k)
                        mma<INT8>(d, da + k * (kUmmaK >> 4), db + k * (kUmmaK >> 4), idesc, (kb | k) != 0);
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
        const int quad = warp & 3;                                   // TMEM lanes 32*quad .. of this warp
        float* scale = s_scale + quad * BN;
        const int half = p.channels / 2;
        uint32_t use = 0;
        for (unsigned t = blockIdx.x; t < n_tiles; t += gridDim.x, ++use) {
            const Work w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
            const uint32_t buf = use & 1;
            // Channel of w that this lane holds.  Gated: lanes q and q + 16 hold gate and up of one output channel.
            int ch, out_ch;
            bool in;
            if constexpr (GATED) {
                out_ch = w.m * (kM / 2) + quad * kGateRows + (lane & 15);
                in = out_ch < half;
                ch = out_ch + (lane >> 4) * half;
            } else {
                ch = w.m * kM + quad * 32 + lane;
                out_ch = ch & ~1;
                in = ch < p.channels;
            }
            const float ws = in ? p.w_scale[(size_t)w.e * p.channels + ch] : 0.0f;
            __syncwarp();
            for (int c = lane; c < BN; c += 32)
                scale[c] = c < w.rows ? p.a_scale[(long long)(w.row0 + c) * p.a_scale_stride] : 0.0f;
            __syncwarp();
            const bool ok = wait_or_dead(&tail->tmem_full[buf], (use >> 1) & 1, dead, p.status);
            if (!__all_sync(0xffffffffu, ok)) break;
            tmem_fence_after();
            const uint32_t addr = tmem + buf * BN + ((uint32_t)(quad * 32) << 16);
            constexpr int kPair = GATED ? 16 : 1;                    // the partner is lane ^ kPair
            const int odd = (lane & kPair) ? 1 : 0;
            uint16_t* out = p.out + out_ch;
            for (int c0 = 0; c0 < w.rows; c0 += 32) {
                uint32_t v[32];
                tmem_ld32(v, addr + c0);
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float a0 = INT8 ? __int2float_rn((int)v[c]) : __uint_as_float(v[c]);
                    const float a1 = INT8 ? __int2float_rn((int)v[c + 1]) : __uint_as_float(v[c + 1]);
                    const float y0 = a0 * (scale[c0 + c] * ws), y1 = a1 * (scale[c0 + c + 1] * ws);
                    // the two partners hold two channels (gated: gate and up of one channel) of rows c and c + 1;
                    // after the exchange one has both of row c, the other both of row c + 1
                    const float other = __shfl_xor_sync(0xffffffffu, odd ? y0 : y1, kPair);
                    const float lo = odd ? other : y0, hi = odd ? y1 : other;
                    const int col = c0 + c + odd;
                    uint16_t* at = out + (long long)(w.row0 + col) * p.out_stride;
                    if constexpr (GATED) {
                        const float g = __fdividef(lo, 1.0f + __expf(-lo)) * hi;
                        if (in && col < w.rows) *at = (uint16_t)pack_bf16x2(g, 0.0f);
                    } else {
                        if (in && col < w.rows) *reinterpret_cast<uint32_t*>(at) = pack_bf16x2(lo, hi);
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

template <int BN>
size_t smem_bytes(int E)
{
    return 1024 + Tile<BN>::data_bytes + sizeof(SmemTail) + 4 * BN * sizeof(float) + (size_t)(3 * E + 1) * sizeof(int);
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn()
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

bool encode(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box)
{
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    EncodeFn fn = encode_fn();
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, (cuuint32_t)rank, const_cast<void*>(base), dims, strides, box, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN>
cudaError_t run(const strata_moe_shape& s, const strata_matmul_args& a, MatParams& p, int n_sm, cudaStream_t st)
{
    {
        const cuuint64_t dims[2] = {(cuuint64_t)a.inner, (cuuint64_t)a.a_rows};
        const cuuint64_t strides[1] = {(cuuint64_t)a.a_stride};
        const cuuint32_t box[2] = {(cuuint32_t)kKBytes, (cuuint32_t)Tile<BN>::box_rows};
        if (!encode(&p.map_a, a.a, 2, dims, strides, box)) return cudaErrorInvalidValue;
    }
    // no more CTAs than tiles can exist: every expert may end in one partial row tile
    const long long items = min((long long)s.R * s.T * s.K, (long long)a.a_rows);
    const long long rows = s.slot_capacity > 0 ? (long long)s.E * s.R * s.slot_capacity : items;
    const long long row_tiles = rows / BN + min((long long)s.E, rows);
    if (row_tiles * p.m_tiles >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    const unsigned grid = (unsigned)min(row_tiles * p.m_tiles, (long long)n_sm);
    const size_t smem = smem_bytes<BN>(s.E);
    if (a.type == STRATA_T_INT8)
        return a.gated ? launch_pdl(expert_matmul_kernel<true, true, BN>, grid, kThreads, smem, st, p)
                       : launch_pdl(expert_matmul_kernel<true, false, BN>, grid, kThreads, smem, st, p);
    return a.gated ? launch_pdl(expert_matmul_kernel<false, true, BN>, grid, kThreads, smem, st, p)
                   : launch_pdl(expert_matmul_kernel<false, false, BN>, grid, kThreads, smem, st, p);
}

template <int BN>
cudaError_t configure()
{
    const void* fns[4] = {(const void*)expert_matmul_kernel<true, true, BN>, (const void*)expert_matmul_kernel<true, false, BN>,
                          (const void*)expert_matmul_kernel<false, true, BN>,
                          (const void*)expert_matmul_kernel<false, false, BN>};
    for (const void* f : fns) {
        const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<BN>(kMaxExperts));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_matmul_kernels()
{
    cudaError_t e = configure<64>();
    if (e == cudaSuccess) e = configure<128>();
    if (e == cudaSuccess) e = configure<256>();
    return e;
}

cudaError_t launch_expert_matmul(const strata_moe_shape& s, const strata_moe_layout_t& L, const strata_matmul_args& a,
                                 int* status, int n_sm, cudaStream_t st)
{
    MatParams p;
    const cuuint64_t k = (cuuint64_t)a.inner, ch = (cuuint64_t)a.channels;
    if (a.gated) {                       // [2E][channels/2][inner]: boxes alternate between gate and up
        const cuuint64_t dims[3] = {k, ch / 2, 2 * (cuuint64_t)s.E};
        const cuuint64_t strides[2] = {k, ch / 2 * k};
        const cuuint32_t box[3] = {(cuuint32_t)kKBytes, (cuuint32_t)kGateRows, 1};
        if (!encode(&p.map_w, a.w, 3, dims, strides, box)) return cudaErrorInvalidValue;
    } else {
        const cuuint64_t dims[2] = {k, ch * (cuuint64_t)s.E};
        const cuuint64_t strides[1] = {k};
        const cuuint32_t box[2] = {(cuuint32_t)kKBytes, (cuuint32_t)kM};
        if (!encode(&p.map_w, a.w, 2, dims, strides, box)) return cudaErrorInvalidValue;
    }
    p.expert_count = s.slot_capacity > 0 ? nullptr : L.expert_count;
    p.expert_offset = L.expert_offset;
    p.a_scale = a.a_scale;
    p.w_scale = a.w_scale;
    p.out = static_cast<uint16_t*>(a.out);
    p.status = status;
    p.a_rows = a.a_rows;
    p.a_scale_stride = a.a_scale_stride;
    p.out_stride = a.out_stride;
    p.E = s.E;
    p.k_blocks = (a.inner + kKBytes - 1) / kKBytes;
    p.channels = a.channels;
    p.m_tiles = a.gated ? (a.channels / 2 + kM / 2 - 1) / (kM / 2) : (a.channels + kM - 1) / kM;
    const long long rows = s.slot_capacity > 0 ? (long long)s.R * s.slot_capacity : (long long)s.R * s.T * s.K / s.E;
    if (rows > 128) return run<256>(s, a, p, n_sm, st);
    if (rows > 64) return run<128>(s, a, p, n_sm, st);
    return run<64>(s, a, p, n_sm, st);
}

}  // namespace strata
