// Router: logits -> top-k expert ids and gate weights, and the gradient of the logits (strata_layer.h has the
// formulas).  One warp owns one token; lane q holds the logits of experts q*VPL .. q*VPL + VPL-1 in registers, so the
// order (lane, register) is the order of expert indexes and "ties to the lower index" needs no index in the key.
#include "layer.cuh"

namespace strata {

namespace {

constexpr int kRouteWarps = 8;
constexpr unsigned kFull = 0xffffffffu;

struct RouteParams {
    const void* logits;
    long long stride;
    const float* bias;
    int32_t* ids;
    float* w;
    int n_tok, E, K;
    int n_group, topk_group, group_size;
    int renormalise, top2;
    int vec_ok;            // rows start on 16 bytes
    float scale;
};

// Order-preserving map of a float to an unsigned key; 0 is below every number and means "not to be chosen".
__device__ __forceinline__ uint32_t key_of(float c)
{
    if (!(c > -INFINITY)) return 0u;                              // -inf and NaN
    const uint32_t u = __float_as_uint(c + 0.0f);                 // -0 and +0 are equal
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k)
{
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

// The sum is pinned to its own rounding: a contraction into the exponential's last multiply would move scores by an
// ulp, and with them the order of near-ties.
__device__ __forceinline__ float sigmoid_f(float l) { return __frcp_rn(__fadd_rn(1.0f, expf(-l))); }
// exp(l - m) for l <= m; infinities at the maximum count as equal to it
__device__ __forceinline__ float softmax_term(float l, float m) { return l == m ? 1.0f : expf(l - m); }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// VPL logits of experts e0 .. e0+VPL-1; experts beyond E, and NaN logits, read as -inf.
template <int VPL, bool BF16>
__device__ __forceinline__ void load_logits(float (&l)[VPL], const void* base, long long row_off, int e0, int E, bool vec_ok)
{
    constexpr int VW = BF16 ? 8 : 4;                              // logits in 16 bytes
    if constexpr (VPL >= VW) {
#pragma unroll
        for (int j = 0; j < VPL; j += VW) {
            if (vec_ok && e0 + j + VW <= E) {
                if constexpr (BF16) {
                    const uint4 v = ld_stream16(static_cast<const uint16_t*>(base) + row_off + e0 + j);
                    unpack_bf16x8(v, &l[j]);
                } else {
                    const uint4 v = ld_stream16(static_cast<const float*>(base) + row_off + e0 + j);
                    l[j] = __uint_as_float(v.x);
                    l[j + 1] = __uint_as_float(v.y);
                    l[j + 2] = __uint_as_float(v.z);
                    l[j + 3] = __uint_as_float(v.w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < VW; ++i)
                    l[j + i] = e0 + j + i < E ? load_as_float<BF16>(base, row_off + e0 + j + i) : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i) l[i] = e0 + i < E ? load_as_float<BF16>(base, row_off + e0 + i) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;
}

// Choice of the K largest of 32*VPL keys.  A direct selection (K rounds of: lane maxima, a warp-wide maximum, removal
// of the winner from one lane's registers) issues about 40 instructions a round at VPL = 8.  Instead the K-th largest of
// the 32 lane maxima is found first: it is a lower bound of the K-th largest key, and only about K + 2 keys
// reach it; those are compacted in index order, one per lane, and each counts the keys that come before it.  Where more
// than 32 reach it (many equal keys, K near 32), the direct selection runs.  At 65,536 tokens x 256 experts, sigmoid
// scores in 4 of 8 groups, with the group choice below: see the measurements at the launcher.
template <int VPL, bool BF16, bool SIGMOID, bool BY_SCORE>
__global__ void __launch_bounds__(kRouteWarps * 32) route_kernel(const RouteParams p)
{
    extern __shared__ uint32_t dyn_keys[];                        // [warps][E], only for groups that split a lane's run
    __shared__ uint32_t s_key[kRouteWarps][32], s_two[kRouteWarps][32];
    __shared__ float s_l[kRouteWarps][32];
    __shared__ int s_id[kRouteWarps][32];
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int tok = (int)blockIdx.x * kRouteWarps + warp;
    griddep_wait();
    griddep_launch_dependents();
    if (tok >= p.n_tok) return;
    const int e0 = lane * VPL;

    float l[VPL];
    load_logits<VPL, BF16>(l, p.logits, (long long)tok * p.stride, e0, p.E, p.vec_ok != 0);

    float m = 0.0f, inv_or_sum = 1.0f;
    if constexpr (!SIGMOID) {
        m = l[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) m = fmaxf(m, l[i]);
        m = warp_max(m);
    }
    uint32_t key[VPL];
    if (!SIGMOID && (BY_SCORE || !p.renormalise)) {               // the full sum of the softmax is needed
        float s = 0.0f, t[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            t[i] = l[i] == -INFINITY ? 0.0f : softmax_term(l[i], m);
            s += t[i];
        }
        inv_or_sum = warp_sum(s);
        if constexpr (BY_SCORE) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                const float c = __fadd_rn(__fdiv_rn(t[i], inv_or_sum), p.bias && e0 + i < p.E ? p.bias[e0 + i] : 0.0f);
                key[i] = l[i] == -INFINITY ? 0u : key_of(c);
            }
        }
    }
    if constexpr (SIGMOID && BY_SCORE) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const float b = p.bias && e0 + i < p.E ? p.bias[e0 + i] : 0.0f;
            key[i] = l[i] == -INFINITY ? 0u : key_of(__fadd_rn(sigmoid_f(l[i]), b));
        }
    }
    if constexpr (!BY_SCORE) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) key[i] = key_of(l[i]);
    }

    if (p.n_group > 1) {
        const int gs = p.group_size;
        uint32_t k1 = 0u, k2 = 0u;                                // lane g < n_group: the two largest keys of group g
        if (gs % VPL == 0) {                                      // a group is a run of whole lanes
            uint32_t a1 = 0u, a2 = 0u;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                a2 = max(a2, min(a1, key[i]));
                a1 = max(a1, key[i]);
            }
            s_key[warp][lane] = a1;
            s_two[warp][lane] = a2;
            __syncwarp();
            const int lpg = gs / VPL;
            if (lane < p.n_group)
                for (int q = lane * lpg; q < (lane + 1) * lpg; ++q) {
                    const uint32_t b1 = s_key[warp][q];
                    k2 = max(max(k2, min(k1, b1)), s_two[warp][q]);
                    k1 = max(k1, b1);
                }
        } else {
            uint32_t* all = dyn_keys + (size_t)warp * p.E;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (e0 + i < p.E) all[e0 + i] = key[i];
            __syncwarp();
            if (lane < p.n_group)
                for (int e = lane * gs; e < (lane + 1) * gs; ++e) {
                    k2 = max(k2, min(k1, all[e]));
                    k1 = max(k1, all[e]);
                }
        }
        __syncwarp();
        uint32_t gkey = k1;
        if (p.top2 && k2 != 0u) gkey = max(1u, key_of(__fadd_rn(value_of(k1), value_of(k2))));
        uint32_t kept = 0u;
        for (int r = 0; r < p.topk_group; ++r) {
            const uint32_t best = __reduce_max_sync(kFull, gkey);
            if (best == 0u) break;
            const int g = __ffs(__ballot_sync(kFull, gkey == best)) - 1;
            kept |= 1u << g;
            if (lane == g) gkey = 0u;
        }
        int g = e0 / gs, left = gs - (e0 - g * gs);               // experts of group g from e0 on
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            if (g >= p.n_group || !((kept >> g) & 1u)) key[i] = 0u;
            if (--left == 0) {
                ++g;
                left = gs;
            }
        }
    }

    // the bound: the K-th largest lane maximum, 0 where fewer than K lanes hold anything
    uint32_t lane_max = key[0];
#pragma unroll
    for (int i = 1; i < VPL; ++i) lane_max = max(lane_max, key[i]);
    uint32_t bound = 0u, rest = lane_max;
    for (int r = 0; r < p.K; ++r) {
        bound = __reduce_max_sync(kFull, rest);
        if (bound == 0u) break;
        if (lane == __ffs(__ballot_sync(kFull, rest == bound)) - 1) rest = 0u;
    }
    bound = max(bound, 1u);
    int mine = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) mine += key[i] >= bound ? 1 : 0;
    int at = mine;                                                // inclusive prefix over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, at, o);
        if (lane >= o) at += v;
    }
    const int total = __shfl_sync(kFull, at, 31);
    at -= mine;

    int rank = p.K, id = -1, found;
    float lk = 0.0f;
    if (total <= 32) {
        found = min(total, p.K);
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (key[i] >= bound) {
                s_key[warp][at] = key[i];
                s_id[warp][at] = e0 + i;
                s_l[warp][at] = l[i];
                ++at;
            }
        __syncwarp();
        if (lane < total) {
            const uint32_t k = s_key[warp][lane];
            id = s_id[warp][lane];
            lk = s_l[warp][lane];
            rank = 0;
            for (int j = 0; j < total; ++j) {
                const uint32_t o = s_key[warp][j];
                rank += (o > k || (o == k && j < lane)) ? 1 : 0;
            }
        }
    } else {
        found = 0;
        for (int r = 0; r < p.K; ++r) {
            lane_max = key[0];
#pragma unroll
            for (int i = 1; i < VPL; ++i) lane_max = max(lane_max, key[i]);
            const uint32_t best = __reduce_max_sync(kFull, lane_max);
            if (best == 0u) break;
            const int win = __ffs(__ballot_sync(kFull, lane_max == best)) - 1;
            int ri = 0;
            float rl = 0.0f;
            bool taken = lane != win;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (!taken && key[i] == best) {
                    taken = true;
                    ri = e0 + i;
                    rl = l[i];
                    key[i] = 0u;
                }
            ri = __shfl_sync(kFull, ri, win);
            rl = __shfl_sync(kFull, rl, win);
            if (lane == r) {
                rank = r;
                id = ri;
                lk = rl;
            }
            ++found;
        }
    }
    const bool sel = rank < p.K;
    float s = 0.0f;
    if (sel) {
        if constexpr (SIGMOID) s = sigmoid_f(lk);
        else s = p.renormalise ? softmax_term(lk, m) : __fdiv_rn(softmax_term(lk, m), inv_or_sum);
    }
    if (p.renormalise) {
        const float d = warp_sum(s);
        s = d > 0.0f ? __fdiv_rn(s, d) : 0.0f;
    }
    int32_t* ids = p.ids + (long long)tok * p.K;
    float* w = p.w + (long long)tok * p.K;
    if (sel) {
        ids[rank] = id;
        w[rank] = s * p.scale;
    }
    if (lane >= found && lane < p.K) {
        ids[lane] = -1;
        w[lane] = 0.0f;
    }
}

struct RouteGradParams {
    const void* logits;
    long long stride;
    const int32_t* ids;
    const float* dw;
    void* dlogits;
    long long dstride;
    int* status;
    int n_tok, E, K;
    int renormalise;
    int vec_ok, dvec_ok;
    float scale;
};

// Lane k < K owns slot k.  Only a softmax that is not renormalised needs the whole row of logits: a sigmoid's
// gradient is zero outside the chosen experts, and so is that of renormalised softmax weights, which depend on the
// chosen logits alone (w_k = scale * t_k, t = softmax over the chosen: dl_k = scale * t_k * (dw_k - sum_j dw_j t_j)).
// The per-expert values meet in a row of shared memory; a repeated id adds its slots up in slot order.
enum GradMode { kGradSigmoid, kGradSoftmax, kGradSoftmaxChosen };
template <int VPL, bool BF16, GradMode MODE>
__global__ void __launch_bounds__(kRouteWarps * 32) route_grad_kernel(const RouteGradParams p)
{
    extern __shared__ float s_rows[];                             // [warps][32 * VPL]
    constexpr bool kFullRow = MODE == kGradSoftmax;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int tok = (int)blockIdx.x * kRouteWarps + warp;
    griddep_wait();
    griddep_launch_dependents();
    if (tok >= p.n_tok) return;
    const int e0 = lane * VPL;
    float* row = s_rows + warp * 32 * VPL;
#pragma unroll
    for (int i = 0; i < VPL; ++i) row[i * 32 + lane] = 0.0f;

    const long long base = (long long)tok * p.stride;
    int id = lane < p.K ? p.ids[(long long)tok * p.K + lane] : -1;
    float dw = lane < p.K ? p.dw[(long long)tok * p.K + lane] : 0.0f;
    if (id < -1 || id >= p.E) {
        report_status(p.status, STRATA_ERR_BAD_EXPERT_ID);
        id = -1;
    }
    float lk = id >= 0 ? load_as_float<BF16>(p.logits, base + id) : -INFINITY;
    if (!(lk > -INFINITY)) lk = -INFINITY;                        // NaN
    const bool live = lk > -INFINITY;
    if (!live) dw = 0.0f;

    float l[VPL], m = 0.0f, sum = 1.0f, mean = 0.0f, d;
    if constexpr (kFullRow) {
        load_logits<VPL, BF16>(l, p.logits, base, e0, p.E, p.vec_ok != 0);
        m = l[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) m = fmaxf(m, l[i]);
        m = warp_max(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            l[i] = l[i] == -INFINITY ? 0.0f : softmax_term(l[i], m);
            s += l[i];
        }
        sum = warp_sum(s);
        d = p.scale * dw;
        mean = warp_sum(live ? d * __fdiv_rn(softmax_term(lk, m), sum) : 0.0f);
    } else if constexpr (MODE == kGradSigmoid) {
        const float s = live ? sigmoid_f(lk) : 0.0f;
        const float slope = live ? s * sigmoid_f(-lk) : 0.0f;     // s * (1 - s) without the cancellation
        d = p.scale * dw;
        if (p.renormalise) {
            const float total = warp_sum(s);
            const float w = total > 0.0f ? __fdiv_rn(s, total) : 0.0f;
            const float dot = warp_sum(dw * w);
            d = total > 0.0f ? __fdiv_rn(p.scale * (dw - dot), total) : 0.0f;
        }
        d = live ? d * slope : 0.0f;
    } else {
        m = warp_max(lk);
        float t = live ? softmax_term(lk, m) : 0.0f;
        const float total = warp_sum(t);
        t = total > 0.0f ? __fdiv_rn(t, total) : 0.0f;
        const float dot = warp_sum(dw * t);
        d = live ? p.scale * t * (dw - dot) : 0.0f;
    }
    if (!live) d = 0.0f;
    float add = 0.0f;
    for (int k = 0; k < p.K; ++k) {
        const int ik = __shfl_sync(kFull, id, k);
        const float dk = __shfl_sync(kFull, d, k);
        if (ik == id) add += dk;
    }
    __syncwarp();
    if (id >= 0) row[(id % VPL) * 32 + id / VPL] = add;           // register i of lane q, without bank conflicts
    __syncwarp();

    float g[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        g[i] = row[i * 32 + lane];
        if constexpr (kFullRow) g[i] = sum > 0.0f ? __fdiv_rn(l[i], sum) * (g[i] - mean) : 0.0f;
    }
    store_row<VPL, BF16>(g, p.dlogits, (long long)tok * p.dstride, e0, p.E, p.dvec_ok != 0);
}

int lanes_width(int E)
{
    int v = 1;
    while (32 * v < E) v *= 2;
    return v;
}

template <int VPL, bool BF16>
cudaError_t route_vpl(const RouteParams& p, const strata_route_params& r, cudaStream_t st)
{
    const bool by_score = p.bias != nullptr || p.top2;
    const unsigned grid = (unsigned)((p.n_tok + kRouteWarps - 1) / kRouteWarps);
    const size_t smem = p.n_group > 1 && p.group_size % VPL != 0 ? (size_t)kRouteWarps * p.E * sizeof(uint32_t) : 0;
    if (r.score == STRATA_SCORE_SIGMOID)
        return by_score ? launch_pdl(route_kernel<VPL, BF16, true, true>, grid, kRouteWarps * 32, smem, st, p)
                        : launch_pdl(route_kernel<VPL, BF16, true, false>, grid, kRouteWarps * 32, smem, st, p);
    return by_score ? launch_pdl(route_kernel<VPL, BF16, false, true>, grid, kRouteWarps * 32, smem, st, p)
                    : launch_pdl(route_kernel<VPL, BF16, false, false>, grid, kRouteWarps * 32, smem, st, p);
}

template <int VPL, bool BF16>
cudaError_t route_grad_vpl(const RouteGradParams& p, const strata_route_params& r, cudaStream_t st)
{
    const unsigned grid = (unsigned)((p.n_tok + kRouteWarps - 1) / kRouteWarps);
    const size_t smem = (size_t)kRouteWarps * 32 * VPL * sizeof(float);
    if (r.score == STRATA_SCORE_SIGMOID)
        return launch_pdl(route_grad_kernel<VPL, BF16, kGradSigmoid>, grid, kRouteWarps * 32, smem, st, p);
    return r.renormalise ? launch_pdl(route_grad_kernel<VPL, BF16, kGradSoftmaxChosen>, grid, kRouteWarps * 32, smem, st, p)
                         : launch_pdl(route_grad_kernel<VPL, BF16, kGradSoftmax>, grid, kRouteWarps * 32, smem, st, p);
}

bool rows_on_16(const void* base, long long stride, int type)
{
    const int size = type == STRATA_T_F32 ? 4 : 2;
    return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && stride * size % 16 == 0;
}

}  // namespace

cudaError_t launch_route(const strata_moe_shape& s, const strata_route_params& r, const void* logits, int type,
                         long long stride, const float* bias, int32_t* ids, float* w, cudaStream_t st)
{
    RouteParams p{};
    p.logits = logits;
    p.stride = stride;
    p.bias = bias;
    p.ids = ids;
    p.w = w;
    p.n_tok = s.R * s.T;
    p.E = s.E;
    p.K = s.K;
    p.n_group = r.n_group;
    p.topk_group = r.topk_group;
    p.group_size = s.E / r.n_group;
    p.renormalise = r.renormalise;
    p.top2 = r.n_group > 1 && r.group_score == STRATA_GROUP_TOP2;
    p.vec_ok = rows_on_16(logits, stride, type);
    p.scale = r.scale;
    const bool bf = type == STRATA_T_BF16;
    switch (lanes_width(s.E)) {
        case 1: return bf ? route_vpl<1, true>(p, r, st) : route_vpl<1, false>(p, r, st);
        case 2: return bf ? route_vpl<2, true>(p, r, st) : route_vpl<2, false>(p, r, st);
        case 4: return bf ? route_vpl<4, true>(p, r, st) : route_vpl<4, false>(p, r, st);
        case 8: return bf ? route_vpl<8, true>(p, r, st) : route_vpl<8, false>(p, r, st);
        case 16: return bf ? route_vpl<16, true>(p, r, st) : route_vpl<16, false>(p, r, st);
        default: return bf ? route_vpl<32, true>(p, r, st) : route_vpl<32, false>(p, r, st);
    }
}

cudaError_t launch_route_grad(const strata_moe_shape& s, const strata_route_params& r, const void* logits, int type,
                              long long stride, const int32_t* ids, const float* dw, void* dlogits, long long dstride,
                              int* status, cudaStream_t st)
{
    RouteGradParams p{};
    p.logits = logits;
    p.stride = stride;
    p.ids = ids;
    p.dw = dw;
    p.dlogits = dlogits;
    p.dstride = dstride;
    p.status = status;
    p.n_tok = s.R * s.T;
    p.E = s.E;
    p.K = s.K;
    p.vec_ok = rows_on_16(logits, stride, type);
    p.renormalise = r.renormalise;
    p.dvec_ok = rows_on_16(dlogits, dstride, type);
    p.scale = r.scale;
    const bool bf = type == STRATA_T_BF16;
    switch (lanes_width(s.E)) {
        case 1: return bf ? route_grad_vpl<1, true>(p, r, st) : route_grad_vpl<1, false>(p, r, st);
        case 2: return bf ? route_grad_vpl<2, true>(p, r, st) : route_grad_vpl<2, false>(p, r, st);
        case 4: return bf ? route_grad_vpl<4, true>(p, r, st) : route_grad_vpl<4, false>(p, r, st);
        case 8: return bf ? route_grad_vpl<8, true>(p, r, st) : route_grad_vpl<8, false>(p, r, st);
        case 16: return bf ? route_grad_vpl<16, true>(p, r, st) : route_grad_vpl<16, false>(p, r, st);
        default: return bf ? route_grad_vpl<32, true>(p, r, st) : route_grad_vpl<32, false>(p, r, st);
    }
}

}  // namespace strata
