// Balance loss of the router with the counts per expert, and its gradient (strata_layer.h has the formulas).  LPT lanes of a warp own a
// token, 4 to 32 by the number of experts, each VPL logits in vectors of 16 bytes in turn (scores.cuh gives a lane its experts in one
// run: two loads of half a sector each).  All sums run in an order that the shape fixes: the tokens of a run of lanes, the runs of
// a block, the blocks of a group, the groups.
#include "scores.cuh"

namespace strata {

namespace {

constexpr int kWarps = 8;
constexpr int kSumCols = 8;            // experts of a block of balance_sum_kernel, one per warp
// Tokens of a run of lanes, at least.  More slices finish sooner and are more to add up: 16,384 x 128 takes 15.8, 15.2, 13.1 and 14.0 us
// with 1, 2, 4 and 8, the gradient, which adds nothing up, 7.1, 7.1, 9.5 and 12.1.
constexpr int kLossTokens = 4, kGradTokens = 2;
// Logits per lane and lanes per token.  Several tokens in a warp share its exchanges: 65,536 x 64, loss and gradient, 24 + 16 us with a
// warp per token, 17 + 11 with eight lanes.
constexpr int width_of(int E) { return E <= 256 ? 8 : E <= 512 ? 16 : 32; }
constexpr int lanes_of(int E) { return E <= 32 ? 4 : E <= 64 ? 8 : E <= 128 ? 16 : 32; }
// Blocks that an SM holds at a time, by the registers that VPL logits per lane take: grids are one wave of them.
constexpr int loss_blocks(int vpl) { return vpl == 8 ? 4 : vpl == 16 ? 2 : 1; }
constexpr int grad_blocks(int vpl) { return vpl == 8 ? 3 : vpl == 16 ? 2 : 1; }

struct BalanceGeom {
    int groups, slices, col_blocks;
    long long group_tokens;
};
// At least `tokens` of them for every run of lanes.
BalanceGeom balance_geom(const strata_moe_shape& s, const strata_balance_params& b, int blocks, int tokens)
{
    BalanceGeom g;
    g.groups = b.per_rank ? s.R : 1;
    g.group_tokens = b.per_rank ? s.T : (long long)s.R * s.T;
    const int least = tokens * kWarps * (32 / lanes_of(s.E));
    g.slices = (int)min((long long)max(1, blocks / g.groups), (g.group_tokens + least - 1) / least);
    g.col_blocks = (s.E + kSumCols - 1) / kSumCols;
    return g;
}

struct BalanceParams {
    const void* logits;
    long long stride, group_tokens;
    const int32_t* ids;
    float* part_p;         // [groups, E, slices]   sums of scores
    int32_t* part_c;       // [groups, E, slices]   slots
    int32_t* part_n;       // [groups * slices]     tokens that take part
    float* part_z;         // [groups * slices]     sums of squares
    float* part_loss;      // [groups * col_blocks]
    int32_t* count;
    int32_t* tokens;
    float* prob;
    float* loss;
    int* status;
    unsigned* ticket;
    int E, K, groups, slices, vec_ok;
    int finish;            // the first kernel adds the slices up itself
    float weight, z_weight;
};

// Sum and maximum over the LPT lanes of a token.
template <int LPT>
__device__ __forceinline__ float token_sum(float v)
{
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
template <int LPT>
__device__ __forceinline__ float token_max(float v)
{
#pragma unroll
    for (int o = LPT / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}
// Expert of register r of the token's lane `at`.
template <int LPT, bool BF16>
__device__ __forceinline__ int expert_of(int at, int r)
{
    constexpr int VW = BF16 ? 8 : 4;
    return r / VW * (LPT * VW) + at * VW + r % VW;
}
// A token's logits (NaN and places beyond E: -inf), or RAW values (places beyond E: 0).
template <int LPT, int VPL, bool BF16, bool RAW = false>
__device__ __forceinline__ void load_token(float (&l)[VPL], const void* base, long long row_off, int at, int E, bool vec_ok)
{
    constexpr int VW = BF16 ? 8 : 4;
#pragma unroll
    for (int j = 0; j < VPL; j += VW) {
        float(&part)[VW] = *reinterpret_cast<float(*)[VW]>(&l[j]);
        const int e0 = expert_of<LPT, BF16>(at, j);
        load_logits<VW, BF16, true>(part, base, row_off, e0, E, vec_ok);
        if constexpr (!RAW) {
#pragma unroll
            for (int i = 0; i < VW; ++i) part[i] = e0 + i < E ? fmaxf(part[i], -INFINITY) : -INFINITY;    // the other operand for NaN
        }
    }
}
template <int LPT, int VPL, bool BF16>
__device__ __forceinline__ void store_token(const float (&g)[VPL], void* base, long long row_off, int at, int E, bool vec_ok)
{
    constexpr int VW = BF16 ? 8 : 4;
#pragma unroll
    for (int j = 0; j < VPL; j += VW) {
        const float(&part)[VW] = *reinterpret_cast<const float(*)[VW]>(&g[j]);
        store_row<VW, BF16>(part, base, row_off, expert_of<LPT, BF16>(at, j), E, vec_ok);
    }
}
// A token's ids, up to 32 / LPT in each of its lanes.
template <int LPT>
__device__ __forceinline__ void load_ids(int (&id)[32 / LPT], const int32_t* ids, int at, int K)
{
#pragma unroll
    for (int s = 0; s < 32 / LPT; ++s) id[s] = s * LPT + at < K ? ids[s * LPT + at] : -1;
}
// Whether any of a token's lanes says so.
template <int LPT>
__device__ __forceinline__ bool token_any(bool v, int lane)
{
    const unsigned all = __ballot_sync(kFull, v);
    return LPT == 32 ? all != 0 : (all >> (lane / LPT * LPT) & ((1u << (LPT & 31)) - 1u)) != 0;
}

// within 2^-23
__device__ __forceinline__ float approx_rcp(float v)
{
    float d;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
    return d;
}

// The normalised scores p of a token; rest: 1 - s of the sigmoid, without the cancellation; where they are asked for, the softmax and
// the logarithm of its sum.  One exponential per logit gives the sigmoid on both sides, 1 / (1 + e) and e / (1 + e) with e = exp(-|l|),
// and exp(l) itself, which the softmax takes as long as no logit of the token passes 60.  Reciprocals are within 2^-23.  Sigmoid scores
// that add up to less than 2^-100 are their exponentials to within that, so their quotients are the softmax, whose sum is at least 1: the
// reciprocal of their own would pass binary32, or they would have vanished.
// Tokens that share a warp choose together; those that are not routed have no vote, and their results, whatever they are, are not used.
// FAST, for gradients in bf16: the exponential is the hardware's power of two (within 2 + 1.2 |x| ulp by CUDA's bound: 2^-16 where the
// score is still a normal number), against 2^-9 of the gradient's own rounding.  The loss and the mean scores are binary32 and take expf.
template <bool FAST>
__device__ __forceinline__ float exp_of(float x) { return FAST ? __expf(x) : expf(x); }

template <int LPT, int VPL, bool FAST, bool SIGMOID>
__device__ __forceinline__ void token_scores(const float (&l)[VPL], bool routed, bool want_soft, float (&p)[VPL], float (&rest)[VPL],
                                             float (&soft)[VPL], float& lse)
{
    lse = 0.0f;
    bool tiny = false;
    if constexpr (SIGMOID) {
        float s = 0.0f, total = 0.0f, top = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const float e = exp_of<FAST>(-fabsf(l[i])), r = approx_rcp(1.0f + e), small = e * r;
            p[i] = l[i] >= 0.0f ? r : small;
            rest[i] = l[i] >= 0.0f ? small : r;
            soft[i] = l[i] >= 0.0f ? approx_rcp(e) : e;
            s += p[i];
            total += soft[i];
            top = fmaxf(top, l[i] == -INFINITY ? 0.0f : fabsf(l[i]));
        }
        s = token_sum<LPT>(s);
        tiny = routed && s < 0x1p-100f;
        const float inv = tiny ? 0.0f : __frcp_rn(s);
#pragma unroll
        for (int i = 0; i < VPL; ++i) p[i] *= inv;
        const bool any_tiny = __any_sync(kFull, tiny);
        if (!want_soft && !any_tiny) return;
        if (!any_tiny && __all_sync(kFull, top <= 60.0f || !routed)) {
            total = token_sum<LPT>(total);
            const float inv_total = total > 0.0f ? __frcp_rn(total) : 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) soft[i] *= inv_total;
            if (total > 0.0f) lse = logf(total);
            return;
        }
    }
    float m = l[0];
#pragma unroll
    for (int i = 1; i < VPL; ++i) m = fmaxf(m, l[i]);
    m = token_max<LPT>(m);
    float s = 0.0f;
    if (fabsf(m) < INFINITY) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) soft[i] = exp_of<FAST>(l[i] - m);
    } else {                                                      // infinities at the maximum count as equal to it
#pragma unroll
        for (int i = 0; i < VPL; ++i) soft[i] = l[i] == -INFINITY ? 0.0f : softmax_term(l[i], m);
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) s += soft[i];
    s = token_sum<LPT>(s);
    const float inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) soft[i] *= inv;
    if (s > 0.0f) lse = m + logf(s);
    if (!SIGMOID || tiny) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) p[i] = soft[i];
    }
}

__device__ __forceinline__ int warp_count(int v) { return __reduce_add_sync(kFull, v); }

// The two losses from the groups' sum (`loss`, of this thread) and the blocks' squares, by a whole block; the ticket is returned.
__device__ __forceinline__ void finish_losses(const BalanceParams& p, float loss)
{
    __shared__ float s_f[kWarps], s_z[kWarps];
    __shared__ int s_alive[kWarps], s_total[kWarps];
    const int t = (int)threadIdx.x, lane = t & 31, warp = t >> 5;
    float z = 0.0f;
    int alive = 0, total = 0;
#pragma unroll 4
    for (int i = t; i < p.groups * p.slices; i += kWarps * 32) z += __ldcg(p.part_z + i);
    for (int i = t; i < p.groups; i += kWarps * 32) {
        const int m = __ldcg(p.tokens + i);
        alive += m > 0;
        total += m;
    }
    loss = warp_sum(loss);
    z = warp_sum(z);
    alive = warp_count(alive);
    total = warp_count(total);
    if (lane == 0) {
        s_f[warp] = loss;
        s_z[warp] = z;
        s_alive[warp] = alive;
        s_total[warp] = total;
    }
    __syncthreads();
    if (t != 0) return;
    for (int w = 1; w < kWarps; ++w) {
        loss += s_f[w];
        z += s_z[w];
        alive += s_alive[w];
        total += s_total[w];
    }
    p.loss[0] = alive > 0 ? p.weight * __fdiv_rn(loss, (float)alive) : 0.0f;
    p.loss[1] = total > 0 && p.z_weight != 0.0f ? p.z_weight * __fdiv_rn(z, (float)total) : 0.0f;
    *p.ticket = 0;
}
// Whether this block is the last of the grid to come here; what the others wrote before is visible to it.
__device__ __forceinline__ bool last_block(const BalanceParams& p)
{
    __shared__ bool s_last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (s_last) __threadfence();
    return s_last;
}
static_assert(kSumCols == kWarps, "both kernels finish with blocks of as many warps");

// Bound by issue and latency: at 65,536 x 256 (sigmoid, per rank) 31 us on the device for 67 MB, 295 instructions a token, and 8 us for the sums.
// expf instead of the hardware's power of two for bf16 logits: 34.2 and 35.5 us there with the sums, softmax 28.8 and 30.5.  64 registers spill
// 24 bytes a thread for fp32 logits with four lanes per token.
template <int LPT, int VPL, bool BF16, bool SIGMOID>
__global__ void __launch_bounds__(kWarps * 32, loss_blocks(VPL)) balance_kernel(const BalanceParams p)
{
    constexpr int kRuns = 32 / LPT, kSlots = LPT * VPL;           // runs of lanes of a warp; places for experts
    extern __shared__ float s_sum[];                              // [warps * runs][slots]
    __shared__ int s_count[kMaxExperts];
    __shared__ float s_z[kWarps * kRuns];
    __shared__ int s_n[kWarps * kRuns];
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, at = lane % LPT, run = warp * kRuns + lane / LPT;
    const int group = (int)blockIdx.x / p.slices, slice = (int)blockIdx.x - group * p.slices;
    for (int e = (int)threadIdx.x; e < p.E; e += kWarps * 32) s_count[e] = 0;
    __syncthreads();
    griddep_wait();
    float sum[VPL], z = 0.0f;
    int n = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) sum[i] = 0.0f;
    const long long step = (long long)p.slices * kWarps * kRuns, first = (long long)group * p.group_tokens;
    long long t = (long long)(slice * kWarps + warp) * kRuns;     // the warp's first token; run r has t + r
    float next[VPL];
    int next_id[kRuns];
    auto load = [&] {                                             // a token ahead: its way from memory is longer than one token's work
        const long long mine = t + lane / LPT, tok = first + min(mine, p.group_tokens - 1);
        load_ids<LPT>(next_id, p.ids + tok * p.K, at, mine < p.group_tokens ? p.K : 0);
        load_token<LPT, VPL, BF16>(next, p.logits, tok * p.stride, at, p.E, p.vec_ok != 0);
    };
    if (t < p.group_tokens) load();
    while (t < p.group_tokens) {
        float l[VPL], q[VPL], rest[VPL], soft[VPL], lse;
        int id[kRuns];
#pragma unroll
        for (int i = 0; i < VPL; ++i) l[i] = next[i];
#pragma unroll
        for (int s = 0; s < kRuns; ++s) id[s] = next_id[s];
        t += step;
        if (t < p.group_tokens) load();
        bool routed = false;
#pragma unroll
        for (int s = 0; s < kRuns; ++s) {
            if (id[s] < -1 || id[s] >= p.E) {
                report_status(p.status, STRATA_ERR_BAD_EXPERT_ID);
                id[s] = -1;
            }
            if (id[s] >= 0) {
                atomicAdd(&s_count[id[s]], 1);
                routed = true;
            }
        }
        __syncwarp();
        routed = token_any<LPT>(routed, lane);
        if (!__any_sync(kFull, routed)) continue;
        token_scores<LPT, VPL, false, SIGMOID>(l, routed, p.z_weight != 0.0f, q, rest, soft, lse);
        if (routed) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) sum[i] += q[i];
            z = fmaf(lse, lse, z);
            ++n;
        }
        __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) s_sum[run * kSlots + expert_of<LPT, BF16>(at, i)] = sum[i];
    if (at == 0) {
        s_z[run] = z;
        s_n[run] = n;
    }
    __syncthreads();
    griddep_launch_dependents();
    for (int e = (int)threadIdx.x; e < p.E; e += kWarps * 32) {
        float a = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps * kRuns; ++w) a += s_sum[w * kSlots + e];
        const size_t to = ((size_t)group * p.E + e) * p.slices + slice;
        p.part_p[to] = a;
        p.part_c[to] = s_count[e];
    }
    if (threadIdx.x == 0) {
        float a = 0.0f;
        int c = 0;
        for (int w = 0; w < kWarps * kRuns; ++w) {
            a += s_z[w];
            c += s_n[w];
        }
        p.part_z[blockIdx.x] = a;
        p.part_n[blockIdx.x] = c;
    }
    if (!p.finish) return;
    // small batches: the last block adds the slices up, a thread per group and expert
    __threadfence();
    if (!last_block(p)) return;
    float loss = 0.0f;
    for (int i = (int)threadIdx.x; i < p.groups * p.E; i += kWarps * 32) {
        const int g = i / p.E, e = i - g * p.E;
        float a = 0.0f;
        int c = 0, m = 0;
        for (int s = 0; s < p.slices; ++s) {
            a += __ldcg(p.part_p + (size_t)i * p.slices + s);
            c += __ldcg(p.part_c + (size_t)i * p.slices + s);
            m += __ldcg(p.part_n + g * p.slices + s);
        }
        const float prob = m > 0 ? __fdiv_rn(a, (float)m) : 0.0f;
        p.prob[i] = prob;
        p.count[i] = c;
        if (e == 0) p.tokens[g] = m;
        if (m > 0) loss += (float)c * prob * __fdiv_rn((float)p.E, (float)p.K * (float)m);
    }
    __threadfence();
    __syncthreads();                                              // the tokens of the groups
    finish_losses(p, loss);
}

// Slices to groups: 8 experts of one group per block, one per warp, whose lanes add every 32nd slice.  The block that draws the
// last ticket adds up the losses.
__global__ void __launch_bounds__(kSumCols * 32) balance_sum_kernel(const BalanceParams p, int col_blocks)
{
    __shared__ float s_f[kSumCols];
    const int t = (int)threadIdx.x, lane = t & 31, warp = t >> 5;
    const int group = (int)blockIdx.x / col_blocks, e = ((int)blockIdx.x - group * col_blocks) * kSumCols + warp;
    griddep_wait();
    griddep_launch_dependents();
    const size_t first = (size_t)group * p.slices;
    float a = 0.0f;
    int c = 0, n = 0;
    const size_t from = ((size_t)group * p.E + min(e, p.E - 1)) * p.slices;
#pragma unroll 10
    for (int i = lane; i < p.slices; i += 32) {
        n += p.part_n[first + i];
        a += p.part_p[from + i];
        c += p.part_c[from + i];
    }
    n = warp_count(n);
    c = warp_count(c);
    a = warp_sum(a);
    if (lane == 0) {
        const float prob = n > 0 ? __fdiv_rn(a, (float)n) : 0.0f;
        if (e < p.E) {
            p.prob[(size_t)group * p.E + e] = prob;
            p.count[(size_t)group * p.E + e] = c;
        }
        s_f[warp] = e < p.E && n > 0 ? (float)c * prob * __fdiv_rn((float)p.E, (float)p.K * (float)n) : 0.0f;
    }
    __syncthreads();
    if (t == 0) {
        float part = 0.0f;
        for (int w = 0; w < kSumCols; ++w) part += s_f[w];
        p.part_loss[blockIdx.x] = part;
        if (blockIdx.x % (unsigned)col_blocks == 0) p.tokens[group] = n;
    }
    if (!last_block(p)) return;
    float loss = 0.0f;
#pragma unroll 4
    for (int i = t; i < (int)gridDim.x; i += kSumCols * 32) loss += __ldcg(p.part_loss + i);
    finish_losses(p, loss);
}

struct BalanceGradParams {
    const void* logits;
    const void* add;
    void* dlogits;
    long long stride, add_stride, dstride, group_tokens;
    const int32_t* ids;
    const int32_t* count;
    const int32_t* tokens;
    const float* dloss;
    int E, K, groups, slices, vec_ok, add_vec_ok, dvec_ok;
    float weight, z_weight;
};

// The same case: 43 us, 400 instructions a token, 134 MB (21 us of HBM); a third block per SM keeps it at 80 registers.  That spills 20 to 48
// bytes a thread for a sigmoid, or with four lanes per token; at 1024 experts 255 registers spill 24 to 88 for a sigmoid.
template <int LPT, int VPL, bool BF16, bool SIGMOID>
__global__ void __launch_bounds__(kWarps * 32, grad_blocks(VPL)) balance_grad_kernel(const BalanceGradParams p)
{
    constexpr int kRuns = 32 / LPT;
    __shared__ int s_alive, s_total;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, at = lane % LPT;
    const int group = (int)blockIdx.x / p.slices, slice = (int)blockIdx.x - group * p.slices;
    if (threadIdx.x == 0) s_alive = s_total = 0;
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();
    for (int i = (int)threadIdx.x; i < p.groups; i += kWarps * 32) {
        const int m = p.tokens[i];
        if (m > 0) {
            atomicAdd(&s_alive, 1);
            atomicAdd(&s_total, m);
        }
    }
    __syncthreads();
    const int n = p.tokens[group];
    const float d0 = p.dloss ? p.dloss[0] : 1.0f, d1 = p.dloss ? p.dloss[1] : 1.0f;
    // d balance / d p[t, e] = c[e]
    const float unit = n > 0 ? d0 * p.weight * __fdiv_rn((float)p.E, (float)s_alive * (float)p.K * (float)n) / (float)n : 0.0f;
    const float unit_z = n > 0 ? d1 * p.z_weight * 2.0f / (float)s_total : 0.0f;
    const bool want_z = p.z_weight != 0.0f;
    float c[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = expert_of<LPT, BF16>(at, i);
        c[i] = e < p.E ? unit * (float)p.count[(size_t)group * p.E + e] : 0.0f;
    }
    const long long step = (long long)p.slices * kWarps * kRuns, first = (long long)group * p.group_tokens;
    long long t = (long long)(slice * kWarps + warp) * kRuns;
    float next[VPL];
    int next_id[kRuns];
    auto load = [&] {                                             // a token ahead, as above
        const long long mine = t + lane / LPT, tok = first + min(mine, p.group_tokens - 1);
        load_ids<LPT>(next_id, p.ids + tok * p.K, at, mine < p.group_tokens ? p.K : 0);
        load_token<LPT, VPL, BF16>(next, p.logits, tok * p.stride, at, p.E, p.vec_ok != 0);
    };
    if (t < p.group_tokens) load();
    while (t < p.group_tokens) {
        const long long mine = t + lane / LPT, tok = first + mine;
        const bool live = mine < p.group_tokens;
        float l[VPL], q[VPL], rest[VPL], soft[VPL], g[VPL], lse;
        bool routed = false;
#pragma unroll
        for (int i = 0; i < VPL; ++i) l[i] = next[i];
#pragma unroll
        for (int s = 0; s < kRuns; ++s) routed |= next_id[s] >= 0 && next_id[s] < p.E;
        if (p.add && live) load_token<LPT, VPL, BF16, true>(g, p.add, tok * p.add_stride, at, p.E, p.add_vec_ok != 0);
        else {
#pragma unroll
            for (int i = 0; i < VPL; ++i) g[i] = 0.0f;
        }
        t += step;
        if (t < p.group_tokens) load();
        __syncwarp();
        routed = token_any<LPT>(routed, lane);
        if (__any_sync(kFull, routed)) {
            token_scores<LPT, VPL, BF16, SIGMOID>(l, routed, want_z, q, rest, soft, lse);
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) dot = fmaf(q[i], c[i], dot);
            dot = token_sum<LPT>(dot);
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                float d = q[i] * (c[i] - dot);
                if constexpr (SIGMOID) d *= rest[i];
                if (want_z) d = fmaf(unit_z * lse, soft[i], d);
                if (l[i] == -INFINITY) d = 0.0f;
                if (routed) g[i] += d;
            }
        }
        if (live) store_token<LPT, VPL, BF16>(g, p.dlogits, tok * p.dstride, at, p.E, p.dvec_ok != 0);
        __syncwarp();
    }
}

size_t aligned(size_t n) { return (n + 15) & ~(size_t)15; }

template <int LPT, int VPL, bool BF16>
cudaError_t loss_width(const BalanceParams& p, bool sigmoid, unsigned grid, cudaStream_t st)
{
    const size_t smem = (size_t)kWarps * 32 * VPL * sizeof(float);
    return sigmoid ? launch_pdl(balance_kernel<LPT, VPL, BF16, true>, grid, kWarps * 32, smem, st, p)
                   : launch_pdl(balance_kernel<LPT, VPL, BF16, false>, grid, kWarps * 32, smem, st, p);
}
template <int LPT, int VPL, bool BF16>
cudaError_t grad_width(const BalanceGradParams& p, bool sigmoid, unsigned grid, cudaStream_t st)
{
    return sigmoid ? launch_pdl(balance_grad_kernel<LPT, VPL, BF16, true>, grid, kWarps * 32, 0, st, p)
                   : launch_pdl(balance_grad_kernel<LPT, VPL, BF16, false>, grid, kWarps * 32, 0, st, p);
}

}  // namespace

size_t balance_scratch_bytes(const strata_moe_shape& s, const strata_balance_params& b, int n_sm)
{
    const BalanceGeom g = balance_geom(s, b, n_sm * loss_blocks(width_of(s.E)), kLossTokens);
    const size_t blocks = (size_t)g.groups * g.slices;
    return 2 * aligned(blocks * s.E * 4) + 2 * aligned(blocks * 4) + aligned((size_t)g.groups * g.col_blocks * 4);
}

#define STRATA_BY_WIDTH(f, ...)                                                                                    \
    switch (s.E <= 256 ? lanes_of(s.E) : width_of(s.E) * 4) {                                                      \
        case 4: return bf ? f<4, 8, true>(__VA_ARGS__) : f<4, 8, false>(__VA_ARGS__);                              \
        case 8: return bf ? f<8, 8, true>(__VA_ARGS__) : f<8, 8, false>(__VA_ARGS__);                              \
        case 16: return bf ? f<16, 8, true>(__VA_ARGS__) : f<16, 8, false>(__VA_ARGS__);                           \
        case 32: return bf ? f<32, 8, true>(__VA_ARGS__) : f<32, 8, false>(__VA_ARGS__);                           \
        case 64: return bf ? f<32, 16, true>(__VA_ARGS__) : f<32, 16, false>(__VA_ARGS__);                         \
        default: return bf ? f<32, 32, true>(__VA_ARGS__) : f<32, 32, false>(__VA_ARGS__);                         \
    }

namespace {
cudaError_t first_pass(const strata_moe_shape& s, const BalanceParams& p, bool bf, bool sigmoid, unsigned grid, cudaStream_t st)
{
    STRATA_BY_WIDTH(loss_width, p, sigmoid, grid, st)
}
}  // namespace

cudaError_t launch_balance_loss(const strata_moe_shape& s, const strata_balance_params& b, const void* logits, int type,
                                long long stride, const int32_t* ids, float* loss, const strata_balance_stats& stats,
                                void* scratch, int* status, unsigned* ticket, int n_sm, cudaStream_t st, int* n_launches)
{
    const BalanceGeom g = balance_geom(s, b, n_sm * loss_blocks(width_of(s.E)), kLossTokens);
    const size_t blocks = (size_t)g.groups * g.slices;
    BalanceParams p{};
    p.logits = logits;
    p.stride = stride;
    p.group_tokens = g.group_tokens;
    p.ids = ids;
    char* at = static_cast<char*>(scratch);
    p.part_p = reinterpret_cast<float*>(at);
    at += aligned(blocks * s.E * 4);
    p.part_c = reinterpret_cast<int32_t*>(at);
    at += aligned(blocks * s.E * 4);
    p.part_n = reinterpret_cast<int32_t*>(at);
    at += aligned(blocks * 4);
    p.part_z = reinterpret_cast<float*>(at);
    at += aligned(blocks * 4);
    p.part_loss = reinterpret_cast<float*>(at);
    p.count = stats.count;
    p.tokens = stats.tokens;
    p.prob = stats.prob;
    p.loss = loss;
    p.status = status;
    p.ticket = ticket;
    p.E = s.E;
    p.K = s.K;
    p.groups = g.groups;
    p.slices = g.slices;
    p.vec_ok = rows_on_16(logits, stride, type);
    p.weight = b.weight;
    p.z_weight = b.z_weight;
    // A second launch costs 0.5 to 1 us on the GPU and 2 us on the host.  Without it a thread of the last block adds all slices of its
    // expert up: us with two launches and with one, softmax, fp32, at 1, 8, 16, 32, 64 and 256 slices: 256 x 8 9.6, 8.8; 2048 x 8 9.7,
    // 9.3; 4096 x 8 10.1, 9.5; 8192 x 8 10.0, 10.6; 16,384 x 8 10.7, 12.1; 65,536 x 8 13.7, 21.7; where a thread has several experts,
    // at 8, 16 and 32: 8 groups of 2048 x 8 9.8, 9.9; 16 groups of 4096 x 16 12.6, 14.6; 8 groups of 8192 x 8 10.4, 15.5.
    p.finish = g.slices <= 8 && blocks * s.E <= 4096;
    *n_launches = 1;
    const cudaError_t err = first_pass(s, p, type == STRATA_T_BF16, b.score == STRATA_SCORE_SIGMOID, (unsigned)blocks, st);
    if (err != cudaSuccess || p.finish) return err;
    *n_launches = 2;
    return launch_pdl(balance_sum_kernel, (unsigned)(g.groups * g.col_blocks), kSumCols * 32, 0, st, p, g.col_blocks);
}

cudaError_t launch_balance_grad(const strata_moe_shape& s, const strata_balance_params& b, const void* logits, int type,
                                long long stride, const int32_t* ids, const strata_balance_stats& stats, const float* dloss,
                                const void* add, long long add_stride, void* dlogits, long long dstride, int n_sm,
                                cudaStream_t st)
{
    const BalanceGeom g = balance_geom(s, b, n_sm * grad_blocks(width_of(s.E)), kGradTokens);
    BalanceGradParams p{};
    p.logits = logits;
    p.add = add;
    p.dlogits = dlogits;
    p.stride = stride;
    p.add_stride = add_stride;
    p.dstride = dstride;
    p.group_tokens = g.group_tokens;
    p.ids = ids;
    p.count = stats.count;
    p.tokens = stats.tokens;
    p.dloss = dloss;
    p.E = s.E;
    p.K = s.K;
    p.groups = g.groups;
    p.slices = g.slices;
    p.vec_ok = rows_on_16(logits, stride, type);
    p.add_vec_ok = add && rows_on_16(add, add_stride, type);
    p.dvec_ok = rows_on_16(dlogits, dstride, type);
    p.weight = b.weight;
    p.z_weight = b.z_weight;
    const bool bf = type == STRATA_T_BF16, sigmoid = b.score == STRATA_SCORE_SIGMOID;
    const unsigned grid = (unsigned)(g.groups * g.slices);
    STRATA_BY_WIDTH(grad_width, p, sigmoid, grid, st)
}

}  // namespace strata
