// The experts' products over the receive buffer in 4 bits: e2m1 codes with a scale per block of 32 (a power of two) or 16 (e4m3)
// values of a row, grouped by expert as the routing layout orders them, times each expert's 4-bit weights (strata_layer.h has the
// formulas).  The matrix instructions take the block scales themselves, from TMEM.
//
// As in 8 bits the weights are the M operand and the rows the N operand (matmul.cu).  A span is 128 bytes of codes of every row, 256
// values, one swizzle span; a stage is one or two of them.  Scales come in groups of 32 or 64 bytes of every row, for several
// spans: a box of 16 bytes per span took as many requests of the copy engine as the codes themselves.  The instructions want
// the scales of 128 rows as 32 lines, word (4 scales) by word, of rows l, l + 32, l + 64 and l + 96, in each of TMEM's four quarters:
// warps read the rows from shared memory and store them to their quarters, a chunk of four words at a time.  (tcgen05.cp from
// lines prepared in shared memory took about 60 cycles each in which the matrix unit did nothing: 324 us with, 251 without the
// copies at 512 rows per expert, 405 and 262 with e4m3 scales.)
//
// CG = 2: two CTAs share a tile.  Each holds its own weight rows and half of the tile's rows, and one instruction of the leader
// multiplies for both; an SM then reads 7 KB of shared memory for what takes it 10 KB alone, and fetches half the rows from L2.
//
// What bounds it (7168 -> 2 x 2048, 32 experts): few rows, the weights' way from HBM (32 rows each: 498 MB in 86 us, 5.9 TB/s); many,
// the way from L2 to an SM: a pair of <2,1,192> needs 32 KB a span and SM, at the 52 bytes a cycle that loads alone reach 600 cycles, where
// the instructions take 400; <2,2,192> needs 47 KB for twice the instructions, 900 for 800, but has no second set of accumulators,
// and its epilogue (28 of 217 us) stands alone.
#include <type_traits>

#include "tiles.cuh"

#ifdef STRATA_TEST_HOOKS
#include <atomic>
#endif

namespace strata {

namespace {

#ifdef STRATA_TEST_HOOKS
std::atomic<int> g_inject_short_load4{0};    // see matmul.cu
std::atomic<int> g_tile4{-1}, g_last_tile4{-1};    // the tile to take instead of the estimate's (-1: none); the one taken last
#endif

constexpr int kM = 128;                 // channels of a matrix instruction, in one CTA
constexpr int kKBytes = 128;            // bytes of codes of a row in a stage: one swizzle span, 256 values
constexpr int kUmmaK = 32;              // the same of a matrix instruction: 64 values
constexpr int kBlock = kM * kKBytes;    // codes of one 128-row block of weights in a stage
constexpr int kChunk = 16;              // scale bytes of a row that TMEM takes at a time: 4 words
constexpr int kChunks = 2;              // chunks of scales in TMEM
constexpr int kMaxGroups = 3;           // groups of scales in shared memory, at most
constexpr int kBoxRows = 32;            // rows of a TMA box of the N operand where it is not the whole height of a tile

// A tile of a CTA is MB blocks of 128 weight rows by up to BN rows of the N operand, of which it holds BN / CG.
// Gated, MB = 1: eight gate channels, the same eight of up, and so on: TMEM hands 16 lanes at a time to a warp, a thread the
//                lanes i and i + 8, so that gate and up of a channel meet in a thread.
// Gated, MB = 2: two accumulators that share the rows, 128 gate channels and the same of up.
template <bool NV, int CG, int MB, int BN>
struct Tile4 {
    static constexpr int own_rows = BN / CG;                        // rows of the N operand in this CTA
    static constexpr int w_span = MB * kBlock, a_span = own_rows * kKBytes;
    static constexpr int spans = MB == 1 ? 2 : 1;                   // of a stage
    static constexpr int stage_bytes = spans * (w_span + a_span);
    static constexpr int group_bytes = BN <= 64 ? 64 : 32;          // scale bytes of a row in a group
    static constexpr int per_group = group_bytes / (NV ? 16 : 8);   // spans that a group serves
    static constexpr int per_chunk = kChunk / (NV ? 16 : 8);
    static constexpr int words = 4 / per_chunk;                     // scale words of a row that a span uses
    static constexpr int groups = NV && BN > 96 && MB == 1 ? 3 : 2;            // as many spans as the ring of codes, at least
    static constexpr int ws_group = MB * kM * group_bytes, as_group = BN * group_bytes;
    static constexpr int a_cols = (BN / 32 + 3) / 4 * 4;            // TMEM columns of a word of the rows' scales
    static constexpr int chunk_cols = 4 * (MB * 4 + a_cols), scale_cols = kChunks * chunk_cols;
    static constexpr int bufs = 2 * MB * BN + scale_cols <= 512 ? 2 : 1;
    static constexpr int acc_cols = bufs * MB * BN;
    static constexpr int used_cols = acc_cols + scale_cols;
    static constexpr int tmem_cols = used_cols <= 128 ? 128 : used_cols <= 256 ? 256 : 512;
    static constexpr int epi_warps = BN > 64 ? 8 : 4;               // a multiple of four: warp & 3 selects the TMEM lanes
    // Warps that bring scales to TMEM, in sets of four that take the chunks in turn: one set works about 550 cycles on a chunk, which
    // at 16 values per scale is one span, 400 cycles of matrix instructions.
    static constexpr int scale_warps = MB == 1 ? 8 : 4;
    static constexpr int load_warp = scale_warps + epi_warps, mma_warp = load_warp + 2, deal_warp = load_warp + 3;
    static constexpr int threads = 32 * (deal_warp + 1);
    static constexpr int cols = BN / (epi_warps / 4);               // columns of a tile that one epilogue warp reads
    static constexpr int stage_out = epi_warps * 1024;              // bytes: 32 rows of 16 channels or 16 of 32 of every warp
    static constexpr int max_experts = CG * MB == 4 ? 512 : kMaxExperts;     // whose tables shared memory has room for
    static constexpr int ring = (CG * MB == 4 ? 204 : 202) * 1024 - groups * (ws_group + as_group);
    static constexpr int stages = ring / stage_bytes < 8 ? ring / stage_bytes : 8;
    static constexpr size_t data_bytes = (size_t)stages * stage_bytes + (size_t)groups * (ws_group + as_group);
    static_assert(used_cols <= 512 && stages >= 2 && cols % 16 == 0 && a_span % 1024 == 0 && own_rows % kBoxRows == 0 && per_group % spans == 0, "");
};

struct Mat4Params {
    CUtensorMap map_w, map_ws;          // weights: codes, scales
    CUtensorMap map_a[2], map_as[2];    // rows: boxes of kBoxRows, and of a tile's whole height
    const int32_t* expert_count;        // NULL: segments are full (fixed-capacity layout)
    const int32_t* expert_offset;
    const float* a_scale;               // NULL: 1
    const float* w_scale;               // NULL: 1
    uint16_t* out;
    int* status;
    WorkQueue wq;
    long long a_rows, a_scale_stride, w_scale_stride, out_stride;
    int E, k_spans, channels, m_tiles;  // channels: rows of w per expert
    int last_steps;                     // matrix instructions of the last span
    int out_piece;                      // 16, 8, 4 or 2 bytes: what every row of out starts on
#ifdef STRATA_TEST_HOOKS
    int test_flags;
#endif
};

constexpr int kClaims = 4;              // tiles that the dealing warp may be ahead of the epilogue

struct Smem4Tail {                      // behind the operand stages
    uint64_t full[8], empty[8], tmem_full[2], tmem_empty[2], drain;
    uint64_t group_full[kMaxGroups], group_empty[kMaxGroups];    // scales in shared memory
    uint64_t chunk_full[kChunks], chunk_empty[kChunks];          // scales in TMEM
    uint64_t work_full[kClaims], work_empty[kClaims];            // tiles, inside a CTA
    uint64_t claim_full[kClaims], claim_empty[kClaims];          // tiles, from the leader to the other CTA
    int4 work[kClaims];                 // expert (-1: no more), channel tile, first row, rows
    unsigned claim[kClaims];
    uint32_t tmem_base, issued[2], issued_groups[2];
    int dead;
};
static_assert(sizeof(Smem4Tail) % 16 == 0, "the scales behind it are read in vectors");

// Instruction descriptor: A and B e2m1, K-major; scales e8m0 or e4m3; `id`: first of the instruction's scales in their word.
template <bool NV, int CG>
__device__ __forceinline__ uint32_t instr_desc4(int n, int id)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (NV ? 0u : 1u << 23) | ((uint32_t)(CG * kM >> 7) << 27) |
           ((uint32_t)id << 4) | ((uint32_t)id << 29);
}
// Low words of operand descriptors (tiles.cuh: smem_desc); their high word is the same everywhere.
constexpr uint32_t kDescHigh = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return ((addr & 0x3ffffu) >> 4) | (1u << 16); }
#define STRATA_MMA4(group, kind, vec)                                                                                           \
    asm volatile(                                                                                                               \
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %6, 0;\n\tmov.b64 a, {%1, %7};\n\tmov.b64 b, {%2, %7};\n\t"       \
        "tcgen05.mma.cta_group::" group ".kind::" kind ".block_scale.scale_vec::" vec " [%0], a, b, %3, [%4], [%5], p;\n\t}" ::"r"( \
            d),                                                                                                                 \
        "r"(a), "r"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "n"(kDescHigh)                                           \
        : "memory")
template <bool NV, int CG>
__device__ __forceinline__ void mma4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                     uint32_t accumulate)
{
    if constexpr (CG == 1 && NV) STRATA_MMA4("1", "mxf4nvf4", "4X");
    else if constexpr (CG == 1) STRATA_MMA4("1", "mxf4", "2X");
    else if constexpr (NV) STRATA_MMA4("2", "mxf4nvf4", "4X");
    else STRATA_MMA4("2", "mxf4", "2X");
}
// One lane of a converged warp, always the same.  The warps that issue loads and matrix instructions stay together but for the
// instruction itself: their operands must lie in uniform registers, and where a single thread runs the loop each one is
// moved there every time (90 cycles per load and 100 per matrix instruction).
__device__ __forceinline__ bool elected()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// Arrives at the barrier (of both CTAs of a pair) when all instructions issued so far are done.
template <int CG>
__device__ __forceinline__ void commit4(uint64_t* bar)
{
    if constexpr (CG == 1) {
        mma_commit(bar);
    } else {
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
            "h"((uint16_t)3)
            : "memory");
    }
}

// The same place in the shared memory of CTA `rank` of the pair.
__device__ __forceinline__ uint32_t in_cta(const void* p, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
// Arrives at the leader's barrier.  No data in memory is handed over with it (TMEM has its own fences), so the arrival releases at
// CTA scope only: at cluster scope it waits for all that the warp has in flight, 1,300 cycles.
template <int CG>
__device__ __forceinline__ void arrive_leader(uint64_t* bar)
{
    if constexpr (CG == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_cta(bar, 0)) : "memory");
}
// A wait by all lanes of a converged warp, which stay together.  `peeked`: what `peek` said earlier; its answer is first looked at
// here, so that it comes while other instructions issue.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status, uint32_t peeked = 0)
{
    return __all_sync(0xffffffffu, peeked != 0) || __all_sync(0xffffffffu, wait_or_dead(bar, parity, dead, status));
}
__device__ __forceinline__ uint32_t peek(uint64_t* bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return ok;
}
// Loads of codes count at the leader's barrier.
template <int CG>
__device__ __forceinline__ void load4_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar, uint32_t leader_bar)
{
    if constexpr (CG == 1) tma_load_2d(dst, map, x, y, bar);
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
            "[%4];" ::"r"(smem_addr(dst)),
            "l"(map), "r"(x), "r"(y), "r"(leader_bar)
            : "memory");
}
// Weights: rows from y, or groups of eight of the interleaved gate and up from z, of expert e.
__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, int x, int y, int z, int e, uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], "
        "[%7];" ::"r"(smem_addr(dst)),
        "l"(map), "r"(x), "r"(y), "r"(0), "r"(z), "r"(e), "r"(smem_addr(bar))
        : "memory");
}
template <int CG>
__device__ __forceinline__ void load4_5d(void* dst, const CUtensorMap* map, int x, int y, int z, int e, uint64_t* bar, uint32_t leader_bar)
{
    if constexpr (CG == 1) tma_load_5d(dst, map, x, y, z, e, bar);
    else
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, "
            "%5, %6}], [%7];" ::"r"(smem_addr(dst)),
            "l"(map), "r"(x), "r"(y), "r"(0), "r"(z), "r"(e), "r"(leader_bar)
            : "memory");
}

// 16 lanes of TMEM by 8 * N columns: thread i holds lanes i / 4 (v[.][0], v[.][1]) and i / 4 + 8 (v[.][2], v[.][3]), of every eight
// columns the two from 2 * (i % 4) on.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t (&v)[4][4], uint32_t addr)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0][0]), "=r"(v[0][1]), "=r"(v[0][2]), "=r"(v[0][3]), "=r"(v[1][0]), "=r"(v[1][1]), "=r"(v[1][2]), "=r"(v[1][3]),
          "=r"(v[2][0]), "=r"(v[2][1]), "=r"(v[2][2]), "=r"(v[2][3]), "=r"(v[3][0]), "=r"(v[3][1]), "=r"(v[3][2]), "=r"(v[3][3])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_ld_16x32(uint32_t (&v)[2][4], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0][0]), "=r"(v[0][1]), "=r"(v[0][2]), "=r"(v[0][3]), "=r"(v[1][0]), "=r"(v[1][1]), "=r"(v[1][2]),
                   "=r"(v[1][3])
                 : "r"(addr));
}
// the loaded registers are tied to the wait, so that no use of them moves in front of it
template <int N>
__device__ __forceinline__ void tmem_ld_wait4(uint32_t (&v)[N][4])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+r"(v[j][0]), "+r"(v[j][1]), "+r"(v[j][2]), "+r"(v[j][3])::"memory");
}
// N matrices of eight channels (a thread's lane) by eight rows of out (its columns), stored row by row of out: 16 bytes at the
// address that lane 8 * j + i gives for row i of matrix j.
__device__ __forceinline__ void store_turned(uint32_t addr, const uint32_t (&r)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3])
                 : "memory");
}
__device__ __forceinline__ void store_turned(uint32_t addr, const uint32_t (&r)[2])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x2.trans.shared.b16 [%0], {%1,%2};" ::"r"(addr), "r"(r[0]), "r"(r[1]) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Four words (16 bytes at byte `at`) of the scales of up to 128 rows, lane l those of rows l, l + 32, l + 64 and l + 96.  TMA swizzles
// the rows, so that eight lanes meet eight different places of the banks: without, they meet two or four times.
template <int ROW_BYTES>
__device__ __forceinline__ void read_scales(const unsigned char* rows, int at, int n, int lane, uint4 (&v)[4])
{
    const int turned = at ^ (ROW_BYTES == 32 ? (lane >> 2 & 1) << 4 : (lane >> 1 & 3) << 4);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (32 * j < n) v[j] = *reinterpret_cast<const uint4*>(rows + (lane + 32 * j) * ROW_BYTES + turned);
        else v[j] = make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void by_word(const uint4 (&v)[4], uint32_t (&r)[16])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r[j] = v[j].x;
        r[4 + j] = v[j].y;
        r[8 + j] = v[j].z;
        r[12 + j] = v[j].w;
    }
}

// The n-th tile that the dealing warp handed over, by all lanes of a warp.  False: there is none, or a wait ran out.
__device__ __forceinline__ bool next_tile(Smem4Tail& tail, uint32_t n, Work& w, int lane, volatile int* dead, int* status)
{
    if (!warp_wait(&tail.work_full[n % kClaims], (n / kClaims) & 1, dead, status)) return false;
    int4 v;
    asm volatile("ld.shared.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_addr(&tail.work[n % kClaims])) : "memory");
    w.e = __shfl_sync(0xffffffffu, v.x, 0);
    w.m = __shfl_sync(0xffffffffu, v.y, 0);
    w.row0 = __shfl_sync(0xffffffffu, v.z, 0);
    w.rows = __shfl_sync(0xffffffffu, v.w, 0);
    if (lane == 0) mbar_arrive(&tail.work_empty[n % kClaims]);
    return w.e >= 0;
}
// claim_unit of common.cuh for `claimers` CTAs, which start on the first tiles, in two steps: the counter's answer takes up to a
// microsecond and a half under load, and is needed a tile later.
__device__ __forceinline__ unsigned claimed_tile(const WorkQueue& q, unsigned drawn, unsigned n_units, unsigned claimers, bool& exhausted)
{
    if (exhausted) return kNoUnit;
    if (drawn < n_units - claimers) return claimers + drawn;
    exhausted = true;
    if (drawn == n_units - 1) *q.next = 0;                           // the last of the failed claims, one per claimer
    return kNoUnit;
}

template <bool NV, bool GATED, int CG, int MB, int BN>
__global__ void __launch_bounds__(Tile4<NV, CG, MB, BN>::threads, 1) expert_matmul4_kernel(const __grid_constant__ Mat4Params p)
{
    using T = Tile4<NV, CG, MB, BN>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_w = smem;                                       // [stages][spans][MB * 128][128]
    unsigned char* s_a = s_w + T::stages * T::spans * T::w_span;     // [stages][spans][own rows][128]
    unsigned char* s_ws = s_a + T::stages * T::spans * T::a_span;    // [groups][MB * 128][group bytes]
    unsigned char* s_as = s_ws + T::groups * T::ws_group;              // [groups][BN][group bytes]
    Smem4Tail* tail = reinterpret_cast<Smem4Tail*>(smem + T::data_bytes);
    float* s_scale = reinterpret_cast<float*>(tail + 1);             // [epilogue warps][cols]
    unsigned char* s_out = reinterpret_cast<unsigned char*>(s_scale + T::epi_warps * T::cols);    // [epilogue warps][1024]
    int* s_base = reinterpret_cast<int*>(s_out + T::stage_out);      // [E + 1]
    int* s_off = s_base + p.E + 1;                                   // [E]
    int* s_cnt = s_off + p.E;                                        // [E]
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = (int)threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0u : blockIdx.x & 1u;            // place in the pair; 0: the leader
    const unsigned team = blockIdx.x / CG, teams = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < T::stages; ++s) {
            mbar_init(&tail->full[s], 2);                            // both loading warps
            mbar_init(&tail->empty[s], 1);
        }
        for (int g = 0; g < T::groups; ++g) {
            mbar_init(&tail->group_full[g], 2);
            mbar_init(&tail->group_empty[g], T::scale_warps);
        }
        for (int c = 0; c < kChunks; ++c) {
            mbar_init(&tail->chunk_full[c], CG * 4);
            mbar_init(&tail->chunk_empty[c], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tail->tmem_full[b], 1);
            mbar_init(&tail->tmem_empty[b], CG * T::epi_warps);
        }
        for (int c = 0; c < kClaims; ++c) {
            mbar_init(&tail->work_full[c], 1);
            mbar_init(&tail->work_empty[c], 2 + (rank == 0 ? 1 : 0) + T::scale_warps + T::epi_warps);   // only the leader multiplies
            mbar_init(&tail->claim_full[c], 1);
            mbar_init(&tail->claim_empty[c], 1);
        }
        mbar_init(&tail->drain, 1);
        tail->dead = 0;
        mbar_fence_init();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_w) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_ws) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_a[0]) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_as[0]) : "memory");
    }
    if (warp == T::mma_warp) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tail->tmem_base)),
                         "n"(T::tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tail->tmem_base)),
                         "n"(T::tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
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
    if constexpr (CG == 2) {                                         // both have their barriers before either touches the other's
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_base, 0);
    const unsigned n_tiles = (unsigned)s_base[p.E] * (unsigned)p.m_tiles;
    volatile int* dead = &tail->dead;

    if (warp == T::deal_warp) {
        // The leader claims a tile and hands it to the other CTA of the pair; each looks its place up and hands that to its warps.
        bool exhausted = teams >= n_tiles;
        unsigned t = team < n_tiles ? team : kNoUnit;
        for (uint32_t n = 0;; ++n) {
            const uint32_t c = n % kClaims, parity = (n / kClaims) & 1;
            unsigned drawn = 0;
            if (rank == 0) {
                if constexpr (CG == 2) {
                    if (!warp_wait(&tail->claim_empty[c], parity ^ 1, dead, p.status)) break;
                    if (lane == 0)
                        asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];" ::"r"(
                                         in_cta(&tail->claim[c], 1)),
                                     "r"(t), "r"(in_cta(&tail->claim_full[c], 1))
                                     : "memory");
                }
                if (lane == 0 && t != kNoUnit && !exhausted) drawn = atomicAdd(p.wq.next, 1u);
            } else {
                if (lane == 0) mbar_expect_tx(&tail->claim_full[c], sizeof(unsigned));    // st.async completes it
                __syncwarp();
                if (!warp_wait(&tail->claim_full[c], parity, dead, p.status)) break;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(t) : "r"(smem_addr(&tail->claim[c])) : "memory");
                t = __shfl_sync(0xffffffffu, t, 0);
                if (lane == 0) arrive_leader<CG>(&tail->claim_empty[c]);
            }
            Work w = {-1, 0, 0, 0};
            if (t != kNoUnit) w = find_work<BN>(t, s_base, s_off, s_cnt, p.E, p.m_tiles);
            if (!warp_wait(&tail->work_empty[c], parity ^ 1, dead, p.status)) break;
            if (lane == 0) {
                tail->work[c] = make_int4(w.e, w.m, w.row0, w.rows);
                mbar_arrive(&tail->work_full[c]);
            }
            if (t == kNoUnit) break;
            if (rank == 0 && lane == 0) t = claimed_tile(p.wq, drawn, n_tiles, teams, exhausted);
            t = __shfl_sync(0xffffffffu, t, 0);
        }
    } else if (warp == T::load_warp || warp == T::load_warp + 1) {   // weights, rows: a load takes its warp about 100 cycles
        const bool weights = warp == T::load_warp;
        uint32_t it = 0, git = 0, s = 0, phase = 0, peeked = 0;
        bool ok = true;
        Work w;
        for (uint32_t use = 0; ok && next_tile(*tail, use, w, lane, dead, p.status); ++use) {
            const int half_n = ((w.rows + 15) & ~15) / CG;           // rows of the tile in each CTA
            const int boxes = (half_n + kBoxRows - 1) / kBoxRows, all_boxes = (w.rows + kBoxRows - 1) / kBoxRows;
            const bool whole = boxes * kBoxRows == T::own_rows, all_whole = all_boxes * kBoxRows == BN;
            const int row0 = w.row0 + (int)rank * half_n;
            const int m = w.m * CG + (int)rank;
            const int w_row = GATED && MB == 1 ? 0 : m * MB * kM / (GATED ? 2 : 1), w_group = GATED && MB == 1 ? m * 8 : 0;
            const uint32_t span_bytes = (uint32_t)(CG * (weights ? T::w_span : boxes * kBoxRows * kKBytes));
            const uint32_t scale_bytes = (uint32_t)(weights ? T::ws_group : all_boxes * kBoxRows * T::group_bytes);
            for (int kb = 0; kb < p.k_spans; kb += T::spans, ++it) {
                if (kb % T::per_group == 0) {
                    const uint32_t g = git % T::groups;
                    if (!warp_wait(&tail->group_empty[g], ((git / T::groups) & 1) ^ 1, dead, p.status)) {
                        ok = false;
                        break;
                    }
                    ++git;
                    uint64_t* bar = &tail->group_full[g];
                    unsigned char* to = s_as + g * T::as_group;
                    const int x = kb / T::per_group * T::group_bytes;
                    if (elected()) {
                        mbar_expect_tx(bar, scale_bytes);
                        if (weights) tma_load_5d(s_ws + g * T::ws_group, &p.map_ws, x, w_row, w_group, w.e, bar);
                        else if (all_whole) tma_load_2d(to, &p.map_as[1], x, w.row0, bar);
                        else
                            for (int b = 0; b < all_boxes; ++b)
                                tma_load_2d(to + b * kBoxRows * T::group_bytes, &p.map_as[0], x, w.row0 + b * kBoxRows, bar);
                    }
                    __syncwarp();
                }
                if (!warp_wait(&tail->empty[s], phase ^ 1, dead, p.status, peeked)) {
                    ok = false;
                    break;
                }
                const uint32_t next_s = s + 1 == T::stages ? 0 : s + 1;
                if (next_s == 0) phase ^= 1;
                peeked = peek(&tail->empty[next_s], phase ^ 1);
                uint64_t* bar = &tail->full[s];
                const uint32_t leader_bar = CG == 1 ? 0u : in_cta(bar, 0);
                unsigned char* dw = s_w + s * (T::spans * T::w_span);
                unsigned char* da = s_a + s * (T::spans * T::a_span);
                const int spans = min(T::spans, p.k_spans - kb);
                if (elected()) {
                    if (rank == 0) {
                        uint32_t expect = span_bytes * (uint32_t)spans;
#ifdef STRATA_TEST_HOOKS
                        if (p.test_flags && blockIdx.x == 0 && it == 0 && weights) expect += 16;
#endif
                        mbar_expect_tx(bar, expect);
                    }
#pragma unroll
                    for (int i = 0; i < T::spans; ++i) {
                        if (i >= spans) break;
                        const int x = (kb + i) * kKBytes;
                        if (weights) load4_5d<CG>(dw + i * T::w_span, &p.map_w, x, w_row, w_group, w.e, bar, leader_bar);
                        else if (whole) load4_2d<CG>(da + i * T::a_span, &p.map_a[1], x, row0, bar, leader_bar);
                        else
                            for (int b = 0; b < boxes; ++b)
                                load4_2d<CG>(da + i * T::a_span + b * kBoxRows * kKBytes, &p.map_a[0], x, row0 + b * kBoxRows, bar,
                                             leader_bar);
                    }
                }
                __syncwarp();
                s = next_s;
            }
        }
        if (lane == 0) {
            tail->issued[warp - T::load_warp] = it;
            tail->issued_groups[warp - T::load_warp] = git;
        }
    } else if (warp == T::mma_warp) {
        if (rank == 0) {
            uint32_t s = 0, phase = 0, cit = 0, stage_peeked = 0, chunk_peeked = 0;
            bool ok = true;
            Work w;
            const uint32_t w_desc = desc_low(smem_addr(s_w)), a_desc = desc_low(smem_addr(s_a));
            for (uint32_t use = 0; ok && next_tile(*tail, use, w, lane, dead, p.status); ++use) {
                const int n = (w.rows + 15) & ~15;
                const uint32_t buf = use % T::bufs;
                if (!warp_wait(&tail->tmem_empty[buf], ((use / T::bufs) & 1) ^ 1, dead, p.status)) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * MB * BN;
                const uint32_t idesc0 = instr_desc4<NV, CG>(n, 0), idesc1 = instr_desc4<NV, CG>(n, NV ? 0 : 2);
                for (int kb0 = 0; ok && kb0 < p.k_spans; kb0 += T::spans) {
                    ok = warp_wait(&tail->full[s], phase, dead, p.status, stage_peeked);
                    if (!ok) break;
                    // whether the next stage is there is asked before this one's instructions, which take longer to issue than the
                    // answer to come
                    const uint32_t next_s = s + 1 == T::stages ? 0 : s + 1;
                    if (next_s == 0) phase ^= 1;
                    stage_peeked = peek(&tail->full[next_s], phase);
                    constexpr int kPart = T::spans < T::per_chunk ? T::spans : T::per_chunk;     // spans of one stage and one chunk
#pragma unroll
                    for (int i0 = 0; i0 < T::spans; i0 += kPart) {
                        const int kb1 = kb0 + i0;
                        if (kb1 >= p.k_spans) break;
                        const uint32_t c = cit % kChunks;
                        if (kb1 % T::per_chunk == 0) {
                            ok = warp_wait(&tail->chunk_full[c], (cit / kChunks) & 1, dead, p.status, chunk_peeked);
                            if (!ok) break;
                            tmem_fence_after();
                        }
                        const bool last = kb1 + kPart >= p.k_spans;
                        const bool chunk_ends = (kb1 + kPart) % T::per_chunk == 0 || last;
                        if (chunk_ends) {
                            ++cit;
                            chunk_peeked = peek(&tail->chunk_full[cit % kChunks], (cit / kChunks) & 1);
                        }
                        const uint32_t dw = w_desc + (s * T::spans + i0) * (T::w_span >> 4), da = a_desc + (s * T::spans + i0) * (T::a_span >> 4);
                        const int word = kb1 % T::per_chunk * T::words;                  // of the chunk, where these spans begin
                        const uint32_t sw = tmem + T::acc_cols + c * T::chunk_cols + word * 4;
                        const uint32_t sa = tmem + T::acc_cols + c * T::chunk_cols + MB * 16 + word * T::a_cols;
                        auto multiply = [&](int k) {                 // the k-th 64 values of these spans
                            const int i = k / 4, j = k % 4, at = NV ? k : k >> 1;        // span, step inside it, word of scales
#pragma unroll
                            for (int b = 0; b < MB; ++b)
                                mma4<NV, CG>(d + b * BN, dw + i * (T::w_span >> 4) + b * (kBlock >> 4) + j * (kUmmaK >> 4),
                                             da + i * (T::a_span >> 4) + j * (kUmmaK >> 4), (k & 1) ? idesc1 : idesc0, sw + b * 16 + at * 4,
                                             sa + at * T::a_cols, (kb1 | k) != 0);
                        };
                        if (elected()) {
                            if (!last) {
#pragma unroll
                                for (int k = 0; k < 4 * kPart; ++k) multiply(k);
                            } else {
                                const int steps = (p.k_spans - 1 - kb1) * 4 + p.last_steps;
#pragma unroll
                                for (int k = 0; k < 4 * kPart; ++k)
                                    if (k < steps) multiply(k);
                            }
                            if (i0 + kPart == T::spans || last) commit4<CG>(&tail->empty[s]);
                            if (chunk_ends) commit4<CG>(&tail->chunk_empty[c]);
                            if (last) commit4<CG>(&tail->tmem_full[buf]);
                        }
                        __syncwarp();
                    }
                    s = next_s;
                }
            }
            if (__any_sync(0xffffffffu, *dead) && elected()) {       // instructions in flight must end before TMEM is freed
                commit4<CG>(&tail->drain);
                mbar_wait_bounded(&tail->drain, 0);
            }
            __syncwarp();
        }
    } else if (warp < T::scale_warps) {                                 // scales to this warp's quarter of TMEM
        uint32_t git = 0, cit = 0;
        bool ok = true;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        constexpr uint32_t kSets = T::scale_warps / 4;
        const uint32_t set = (uint32_t)warp >> 2;
        Work w;
        uint4 vw[MB][4], va[T::a_cols / 4][4];
        // the chunk that begins with span kb, from its group in shared memory; `mine`: it is this set's
        auto fetch = [&](int kb, bool mine) {
            const uint32_t g = git % T::groups;
            const int at = kb % T::per_group / T::per_chunk * kChunk;        // of the chunk in its group's rows
            if (at == 0 && !warp_wait(&tail->group_full[g], (git / T::groups) & 1, dead, p.status)) return false;
            if (mine) {
#pragma unroll
                for (int b = 0; b < MB; ++b)
                    read_scales<T::group_bytes>(s_ws + g * T::ws_group + b * kM * T::group_bytes, at, kM, lane, vw[b]);
#pragma unroll
                for (int b = 0; b < T::a_cols / 4; ++b)
                    read_scales<T::group_bytes>(s_as + g * T::as_group + b * kM * T::group_bytes, at, BN - b * kM, lane, va[b]);
            }
            if (at == T::group_bytes - kChunk || kb + T::per_chunk >= p.k_spans) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&tail->group_empty[g]);
                ++git;
            }
            return true;
        };
        for (uint32_t use = 0; ok && next_tile(*tail, use, w, lane, dead, p.status); ++use) {
            for (int kb = 0; ok && kb < p.k_spans; kb += T::per_chunk, ++cit) {
                const bool mine = cit % kSets == set;
                ok = fetch(kb, mine);
                if (!ok || !mine) continue;
                const uint32_t c = cit % kChunks;
                ok = warp_wait(&tail->chunk_empty[c], ((cit / kChunks) & 1) ^ 1, dead, p.status);
                if (!ok) break;
                tmem_fence_after();
                const uint32_t to = tmem + T::acc_cols + c * T::chunk_cols + lanes;
                uint32_t r[16];
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    by_word(vw[b], r);
                    tmem_st16(to + b * 16, r);
                }
                if constexpr (T::a_cols == 4) {
                    by_word(va[0], r);
                    tmem_st16(to + MB * 16, r);
                } else {                                             // two words of up to 256 rows at a time
                    uint32_t q[16];
                    by_word(va[0], r);
                    by_word(va[T::a_cols / 4 - 1], q);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t x[16] = {r[8 * h],     r[8 * h + 1], r[8 * h + 2], r[8 * h + 3], q[8 * h],     q[8 * h + 1],
                                                q[8 * h + 2], q[8 * h + 3], r[8 * h + 4], r[8 * h + 5], r[8 * h + 6], r[8 * h + 7],
                                                q[8 * h + 4], q[8 * h + 5], q[8 * h + 6], q[8 * h + 7]};
                        tmem_st16(to + MB * 16 + h * 16, x);
                    }
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) arrive_leader<CG>(&tail->chunk_full[c]);
            }
        }
    } else {
        const int ew = warp - T::scale_warps, quad = warp & 3;          // TMEM lanes 32*quad .. of this warp
        const int col0 = (ew >> 2) * T::cols;                        // first column of this warp
        // A step: 32 columns of 16 channels, or 16 of 32; OB blocks of out per step and accumulators
        constexpr bool kTight = GATED && MB == 1;
        constexpr int kStep = kTight ? 32 : 16, kEights = kStep / 8, kPitch = kTight ? 32 : 64, OB = GATED ? 1 : MB;
        float* scale = s_scale + ew * T::cols;
        unsigned char* mine = s_out + ew * 1024;
        // 16-byte places of a row of the staged step, turned so that eight rows meet eight different places of the banks
        auto place = [&](int row, int chunk) {
            return row * kPitch + ((kTight ? chunk ^ (row >> 2 & 1) : chunk ^ (row >> 1 & 3)) << 4);
        };
        const int half = p.channels / 2, limit = GATED ? half : p.channels;
        const bool scaled = p.a_scale || p.w_scale;
        Work w;
        for (uint32_t use = 0; next_tile(*tail, use, w, lane, dead, p.status); ++use) {
            const int m = w.m * CG + (int)rank;
            const uint32_t buf = use % T::bufs;
            const int rows = min(T::cols, w.rows - col0);            // of this warp; may be negative
            const int ch0 = kTight ? m * (kM / 2) + quad * 16 : GATED ? m * kM + quad * 32 : m * MB * kM + quad * 32;   // of out
            float wsc[MB][2][2];                                     // of lanes 16 * h + i / 4 and + 8 of accumulator b
            if (scaled) {
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int c = ch0 + (kTight ? h * 8 : h * 16 + u * 8) + (GATED ? 0 : b * kM) + (lane >> 2);
                            const int up = kTight ? u : GATED ? b : 0;
                            wsc[b][h][u] = p.w_scale && c < limit
                                               ? p.w_scale[((long long)w.e * p.channels + c + up * half) * p.w_scale_stride]
                                               : 1.0f;
                        }
                __syncwarp();
                for (int c = lane; c < T::cols; c += 32)
                    scale[c] = p.a_scale && c < rows ? p.a_scale[(long long)(w.row0 + col0 + c) * p.a_scale_stride] : 1.0f;
                __syncwarp();
            }
            if (!warp_wait(&tail->tmem_full[buf], (use / T::bufs) & 1, dead, p.status)) break;
            tmem_fence_after();
            const uint32_t addr = tmem + buf * MB * BN + ((uint32_t)(quad * 32) << 16) + col0;
            uint16_t* out = p.out + (long long)(w.row0 + col0) * p.out_stride;
            uint32_t v[MB][2][kEights][4];                           // the step to come: loaded while the one before is worked on
            auto load = [&](int c0) {
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) tmem_ld_16x32(v[b][h], addr + b * BN + ((uint32_t)(16 * h) << 16) + c0);
            };
            // the staged step to out, in pieces of W bytes that every row starts on, neighbouring lanes along a row (16,384 rows,
            // 2048 -> 7164 nvfp4, 8 bytes: 201 us; element by element from 16-byte pieces 557; 7168 channels 178)
            auto flush = [&](auto piece, int c0, int block) {
                constexpr int W = decltype(piece)::value, kPieces = kPitch / W, kRowsAt = 32 / kPieces;
#pragma unroll 4
                for (int i = 0; i < kStep / kRowsAt; ++i) {
                    const int row = i * kRowsAt + lane / kPieces, at = lane % kPieces * W;
                    const int ch = ch0 + block + at / 2;
                    if (c0 + row >= rows || ch >= limit) continue;
                    const unsigned char* from = mine + place(row, at >> 4) + (at & 15);
                    uint16_t* to = out + (long long)(c0 + row) * p.out_stride + ch;
                    if (ch + W / 2 <= limit) {
                        if constexpr (W == 16) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
                        else if constexpr (W == 8) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(from);
                        else if constexpr (W == 4) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
                        else *to = *reinterpret_cast<const uint16_t*>(from);
                    } else {
                        for (int e = 0; ch + e < limit; ++e) to[e] = reinterpret_cast<const uint16_t*>(from)[e];
                    }
                }
            };
            __syncwarp();
            if (rows > 0) load(0);
            for (int c0 = 0; c0 < rows; c0 += kStep) {
                float y[MB][2][kEights][4];
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        tmem_ld_wait4(v[b][h]);
#pragma unroll
                        for (int j = 0; j < kEights; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[b][h][j][i] = __uint_as_float(v[b][h][j][i]);
                    }
                if (c0 + kStep < rows) load(c0 + kStep);
                if (scaled) {
#pragma unroll
                    for (int j = 0; j < kEights; ++j) {
                        const float2 sc = *reinterpret_cast<const float2*>(&scale[c0 + j * 8 + (lane & 3) * 2]);
#pragma unroll
                        for (int b = 0; b < MB; ++b)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int i = 0; i < 4; ++i) y[b][h][j][i] *= (i & 1 ? sc.y : sc.x) * wsc[b][h][i >> 1];
                    }
                }
#pragma unroll
                for (int b = 0; b < OB; ++b) {
                    // stage: lane 8 * j + i gives the place of row i of the j-th eight rows
                    const int row = lane % kStep;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (kTight) {
                            uint32_t r[kEights];
#pragma unroll
                            for (int j = 0; j < kEights; ++j)
                                r[j] = pack_bf16x2(gate_mul(y[0][h][j][0], y[0][h][j][2]), gate_mul(y[0][h][j][1], y[0][h][j][3]));
                            store_turned(smem_addr(mine + place(row, h)), r);
                        } else {
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                uint32_t r[kEights];
#pragma unroll
                                for (int j = 0; j < kEights; ++j) {
                                    if constexpr (GATED)
                                        r[j] = pack_bf16x2(gate_mul(y[0][h][j][2 * u], y[MB - 1][h][j][2 * u]),
                                                           gate_mul(y[0][h][j][2 * u + 1], y[MB - 1][h][j][2 * u + 1]));
                                    else r[j] = pack_bf16x2(y[b][h][j][2 * u], y[b][h][j][2 * u + 1]);
                                }
                                store_turned(smem_addr(mine + place(row, h * 2 + u)), r);
                            }
                        }
                    }
                    __syncwarp();
                    if (p.out_piece == 16) flush(std::integral_constant<int, 16>(), c0, b * kM);
                    else if (p.out_piece == 8) flush(std::integral_constant<int, 8>(), c0, b * kM);
                    else if (p.out_piece == 4) flush(std::integral_constant<int, 4>(), c0, b * kM);
                    else flush(std::integral_constant<int, 2>(), c0, b * kM);
                    __syncwarp();
                }
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader<CG>(&tail->tmem_empty[buf]);
        }
    }
    __syncwarp();
    griddep_launch_dependents();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (threadIdx.x == 0 && *dead) {                                 // loads in flight must land before the CTA leaves
        // the other CTA of a pair may have issued loads that the leader does not expect: it waits out the limit for them
        const uint32_t it = max(tail->issued[0], tail->issued[1]), first = it > (uint32_t)T::stages ? it - T::stages : 0;
        for (uint32_t u = first; u < it + (CG == 2 ? 1u : 0u); ++u)
            mbar_wait_bounded(&tail->full[u % T::stages], (u / T::stages) & 1);
        const uint32_t groups = max(tail->issued_groups[0], tail->issued_groups[1]);
        for (uint32_t u = groups > T::groups ? groups - T::groups : 0; u < groups; ++u)
            mbar_wait_bounded(&tail->group_full[u % T::groups], (u / T::groups) & 1);
    }
    if constexpr (CG == 2) {                                         // neither leaves while the other may still reach into it
        __syncthreads();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (warp == T::mma_warp) {
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(T::tmem_cols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(T::tmem_cols) : "memory");
    }
}

template <bool NV, int CG, int MB, int BN>
constexpr size_t smem_bytes4(int E)
{
    using T = Tile4<NV, CG, MB, BN>;
    return 1024 + T::data_bytes + sizeof(Smem4Tail) + (size_t)(T::epi_warps * T::cols) * sizeof(float) + T::stage_out +
           (size_t)(3 * E + 1) * sizeof(int);
}

template <bool NV, int CG, int MB, int BN>
cudaError_t run4(const strata_moe_shape& s, const strata_matmul4_args& a, Mat4Params& p, int n_sm, cudaStream_t st)
{
    using T = Tile4<NV, CG, MB, BN>;
    const cuuint64_t parts = a.gated ? 2 : 1, rows = (cuuint64_t)a.channels / parts;
    for (int i = 0; i < 2; ++i) {                                    // codes, block scales
        const cuuint64_t bytes = (cuuint64_t)a.inner / (i == 0 ? 2 : NV ? 16 : 32);
        const cuuint32_t box = i == 0 ? kKBytes : T::group_bytes;
        const CUtensorMapSwizzle swizzle = i == 0                  ? CU_TENSOR_MAP_SWIZZLE_128B
                                           : T::group_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                                                  : CU_TENSOR_MAP_SWIZZLE_32B;
        {   // weights: [E][channels]; gated: [E][2][channels / 2], gate and up in one box, in turn by eights where MB is 1
            const cuuint64_t stride = (cuuint64_t)(i == 0 ? a.w.code_stride : a.w.block_stride);
            const bool eights = a.gated && MB == 1;
            const cuuint64_t dims[5] = {bytes, eights ? 8 : rows, parts, eights ? rows / 8 : 1, (cuuint64_t)s.E};
            const cuuint64_t strides[4] = {stride, rows * stride, eights ? 8 * stride : stride, parts * rows * stride};
            const cuuint32_t boxes[5] = {box, (cuuint32_t)(eights ? 8 : MB * kM / parts), (cuuint32_t)parts, eights ? 8u : 1u, 1};
            if (!encode(i == 0 ? &p.map_w : &p.map_ws, i == 0 ? a.w.codes : a.w.block, 5, dims, strides, boxes, swizzle))
                return cudaErrorInvalidValue;
        }
        const cuuint64_t dims[2] = {bytes, (cuuint64_t)a.a_rows};
        const cuuint64_t strides[1] = {(cuuint64_t)(i == 0 ? a.a.code_stride : a.a.block_stride)};
        for (int whole = 0; whole < 2; ++whole) {
            const cuuint32_t boxes[2] = {box, (cuuint32_t)(!whole ? kBoxRows : i == 0 ? T::own_rows : BN)};
            if (!encode(i == 0 ? &p.map_a[whole] : &p.map_as[whole], i == 0 ? a.a.codes : a.a.block, 2, dims, strides, boxes, swizzle))
                return cudaErrorInvalidValue;
        }
    }
    const int per_tile = CG * MB * kM / (a.gated ? 2 : 1), wide = a.channels / (a.gated ? 2 : 1);
    p.m_tiles = (wide + per_tile - 1) / per_tile;
    const long long tiles = row_tiles(s, a.a_rows, BN) * p.m_tiles;
    if (tiles >= (1ll << 31)) return cudaErrorInvalidConfiguration;
    const unsigned grid = CG * (unsigned)min(tiles, (long long)max(1, n_sm / CG));
    const size_t smem = smem_bytes4<NV, CG, MB, BN>(s.E);
    return a.gated ? launch_pdl_cluster(expert_matmul4_kernel<NV, true, CG, MB, BN>, grid, T::threads, smem, CG, st, p)
                   : launch_pdl_cluster(expert_matmul4_kernel<NV, false, CG, MB, BN>, grid, T::threads, smem, CG, st, p);
}

template <bool NV, int CG, int MB, int BN>
cudaError_t configure4()
{
    static_assert(smem_bytes4<NV, CG, MB, BN>(Tile4<NV, CG, MB, BN>::max_experts) <= 227 * 1024, "");
    const void* fns[2] = {(const void*)expert_matmul4_kernel<NV, true, CG, MB, BN>, (const void*)expert_matmul4_kernel<NV, false, CG, MB, BN>};
    for (const void* f : fns) {
        const cudaError_t e =
            cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes4<NV, CG, MB, BN>(Tile4<NV, CG, MB, BN>::max_experts));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
template <bool NV>
cudaError_t configure4_all()
{
    cudaError_t e = configure4<NV, 1, 1, 64>();
    if (e == cudaSuccess) e = configure4<NV, 1, 2, 96>();
    if (e == cudaSuccess) e = configure4<NV, 2, 1, 192>();
    if (e == cudaSuccess) e = configure4<NV, 2, 2, 192>();
    return e;
}

template <bool NV>
cudaError_t pick4(int v, const strata_moe_shape& s, const strata_matmul4_args& a, Mat4Params& p, int n_sm, cudaStream_t st)
{
    switch (v) {
        case 0: return run4<NV, 1, 1, 64>(s, a, p, n_sm, st);
        case 1: return run4<NV, 1, 2, 96>(s, a, p, n_sm, st);
        case 2: return run4<NV, 2, 1, 192>(s, a, p, n_sm, st);
        default: return run4<NV, 2, 2, 192>(s, a, p, n_sm, st);
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
#ifdef STRATA_TEST_HOOKS
    p.test_flags = g_inject_short_load4.exchange(0);
#endif
    p.a_rows = a.a_rows;
    p.a_scale_stride = a.a.scale_stride;
    p.w_scale_stride = a.w.scale_stride;
    p.out_stride = a.out_stride;
    p.E = s.E;
    p.k_spans = (a.inner / 2 + kKBytes - 1) / kKBytes;
    p.last_steps = (a.inner / 2 - (p.k_spans - 1) * kKBytes + kUmmaK - 1) / kUmmaK;
    p.channels = a.channels;
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.out);
    p.out_piece = 16;
    while (p.out_piece > 2 && (a.out_stride * 2 % p.out_piece != 0 || at % p.out_piece != 0)) p.out_piece /= 2;
    // Which tile: the shortest estimate of rounds * (spans * (c + n * filled) + f + g * filled) over the GPU, where c + n is what one span
    // of a full tile takes and f + g what a tile adds, n and g the parts that grow with the rows in it (g is the epilogue where the
    // accumulators are not doubled); at least the weights' way from HBM.  The constants were fitted to 65 measured shapes of
    // each kind (8, 32 and 60 experts, 1 .. 2048 mean rows, inner 256 .. 7168, 512 .. 7168 channels, even and Zipf routing); the choice is on average
    // 1.9 % above the best of the four (one tile for all: 6 to 44 %), and 25 % at worst.  At 7168 -> 4096 gated, 32 experts,
    // mxfp4, us for <1,1,64>, <1,2,96>, <2,1,192>, <2,2,192>: one token 27, 25, 28, 26; 32 rows each 86, 88, 88, 89; 128 rows 153, 117, 97, 100;
    // 256 rows 276, 178, 155, 141; 512 rows 502, 338, 234, 217; nvfp4 700, 384, 291, 248; 2048 -> 7168, 512 rows, mxfp4 299, 196, 143, 157.
    // What the estimate does not see: rows spread around their mean, and slots that are masked or unrouted.  7,422 rows over 60 experts, 1440 ->
    // 2040 nvfp4, us for the four: even 58, 45, 40, 45, Zipf 60, 45, 46, 49; it takes <2,2,192> for both and expects 23 of it: some rounds of
    // tiles of unlike height, dealt in the order of the experts.  What a tile is does not show in the results: all four sum in the same order.
    struct Cost { int cg, mb, bn; float c, n, f, g, hbm; };
    static const Cost costs[2][4] = {{{1, 1, 64, 0.03f, 0.28f, 0.84f, 0.0f, 1.15f}, {1, 2, 96, 0.29f, 0.29f, 0.82f, 0.0f, 1.00f},
                                      {2, 1, 192, 0.12f, 0.25f, 1.17f, 0.10f, 1.17f}, {2, 2, 192, 0.26f, 0.39f, 1.24f, 2.36f, 1.17f}},
                                     {{1, 1, 64, 0.12f, 0.28f, 0.88f, 0.31f, 1.39f}, {1, 2, 96, 0.33f, 0.29f, 1.04f, 0.49f, 1.06f},
                                      {2, 1, 192, 0.25f, 0.20f, 1.12f, 1.09f, 1.23f}, {2, 2, 192, 0.35f, 0.35f, 1.26f, 3.24f, 1.23f}}};
    constexpr float kHbmBytesPerUs = 6.55e6f;
    const bool nv = a.type == STRATA_T_NVF4;
    const long long items = s.slot_capacity > 0 ? (long long)s.E * s.R * s.slot_capacity : (long long)s.R * s.T * s.K;
    const long long used = min(items, (long long)s.E), mean = (items + s.E - 1) / s.E;
    const float bytes_us = (float)used * (float)a.channels * (float)a.inner * (nv ? 0.5625f : 0.53125f) / kHbmBytesPerUs;
    int v = 1;                                                       // one CTA alone, any number of channels and experts
    float least = 0.0f;
    auto takes = [&](const Cost& k) {
        if (a.gated && k.mb == 1 && a.channels % 16 != 0) return false;      // takes gate and up by eights
        return k.cg <= n_sm && (k.cg * k.mb < 4 || s.E <= Tile4<false, 2, 2, 192>::max_experts);
    };
    for (int i = 0; i < 4; ++i) {
        const Cost& k = costs[nv][i];
        if (!takes(k)) continue;
        const int per_tile = k.cg * k.mb * kM / (a.gated ? 2 : 1), wide = a.channels / (a.gated ? 2 : 1), teams = n_sm / k.cg;
        const long long heights = (mean + k.bn - 1) / k.bn;
        const float tiles = (float)(used * heights * ((wide + per_tile - 1) / per_tile));
        const float rounds = tiles > (float)teams ? tiles / (float)teams + 0.19f : 1.0f;
        const float filled = (float)mean / (float)(heights * k.bn);
        const float cost = max(rounds * ((float)p.k_spans * (k.c + k.n * filled) + k.f + k.g * filled), bytes_us * k.hbm);
        if (least == 0.0f || cost < least) {
            least = cost;
            v = i;
        }
    }
    v = (int)tune("STRATA_MM4", v);
#ifdef STRATA_TEST_HOOKS
    if (const int forced = g_tile4.load(); forced >= 0) {
        if (forced > 3 || !takes(costs[nv][forced])) return cudaErrorInvalidValue;
        v = forced;
    }
    g_last_tile4.store(v);
#endif
    return nv ? pick4<true>(v, s, a, p, n_sm, st) : pick4<false>(v, s, a, p, n_sm, st);
}

}  // namespace strata

#ifdef STRATA_TEST_HOOKS
extern "C" void strata_test_inject_short_load4(int on) { strata::g_inject_short_load4.store(on); }
extern "C" void strata_test_tile4(int tile) { strata::g_tile4.store(tile); }
extern "C" int strata_test_last_tile4(void) { return strata::g_last_tile4.load(); }
#endif
