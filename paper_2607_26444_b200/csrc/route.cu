// Router: logits -> top-k expert ids and gate weights, and the gradient of the logits (strata_layer.h has the
// formulas).  One warp owns one token; a lane holds up to VPL logits of neighbouring experts in registers, lanes in the order of
// the experts, so the order (lane, register) is the order of expert indexes and "ties to the lower index" needs no
// index in the key.
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
    unsigned n_tok;        // below 2^31; tokens are counted unsigned, since a warp's stride takes the count past the end
    int E, K;
    int n_group, topk_group, group_size;
    int renormalise, top2;
    int fast, fast_vec;    // fast = 0: every token takes the exact path
    int lanes_per_group, run;
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

// The same for gradients.  A bf16 gradient takes the hardware's power of two, whose argument is rounded: within 2 + 1.2 |l - m| ulp
// (CUDA's bound for __expf), 2^-16 where the term is still a normal number, against 2^-9 of the result's own rounding.
template <bool BF16>
__device__ __forceinline__ float softmax_grad_term(float l, float m)
{
    return l == m ? 1.0f : BF16 ? __expf(l - m) : expf(l - m);
}

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

// VPL logits of experts e0 .. e0+VPL-1.  RAW: experts beyond E read as zero and NaN stays; otherwise both read as -inf.
template <int VPL, bool BF16, bool RAW = false>
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
                    l[j + i] = e0 + j + i < E ? load_as_float<BF16>(base, row_off + e0 + j + i) : RAW ? 0.0f : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            l[i] = e0 + i < E ? load_as_float<BF16>(base, row_off + e0 + i) : RAW ? 0.0f : -INFINITY;
    }
    if constexpr (!RAW) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;
    }
}

struct __align__(16) RouteSmem {          // of one warp
    uint32_t one[32], two[32];
    float l[32];
    int id[32];
};

// The whole choice of one token in exact arithmetic.  route_kernel below sends here what its shorter way does not decide:
// masked or NaN logits, softmax scores compared as such, near-ties of groups, and more than CAP candidates.  Scores become ordered integer keys; the K-th largest of the 32 lane maxima bounds the K-th largest
// key from below; the keys that reach it are compacted in index order and ranked; if more than 32 do, K
// rounds of a warp-wide maximum take the winners one by one.  1,138 instructions per token at 256 experts in 4 of
// 8 groups.
template <int VPL, bool BF16, bool SIGMOID, bool BY_SCORE>
__device__ __noinline__ void route_exact(const RouteParams& p, unsigned tok, RouteSmem& sm, uint32_t* all)
{
    const int lane = (int)threadIdx.x & 31;
    const int e0 = lane * VPL;
    __syncwarp();

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
            sm.one[lane] = a1;
            sm.two[lane] = a2;
            __syncwarp();
            const int lpg = gs / VPL;
            if (lane < p.n_group)
                for (int q = lane * lpg; q < (lane + 1) * lpg; ++q) {
                    const uint32_t b1 = sm.one[q];
                    k2 = max(max(k2, min(k1, b1)), sm.two[q]);
                    k1 = max(k1, b1);
                }
        } else {
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
                sm.one[at] = key[i];
                sm.id[at] = e0 + i;
                sm.l[at] = l[i];
                ++at;
            }
        __syncwarp();
        if (lane < total) {
            const uint32_t k = sm.one[lane];
            id = sm.id[lane];
            lk = sm.l[lane];
            rank = 0;
            for (int j = 0; j < total; ++j) {
                const uint32_t o = sm.one[j];
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
    if constexpr (!SIGMOID)
        if (p.renormalise) m = warp_max(sel ? lk : -INFINITY);    // weights among the chosen only; a bias or sums may leave the largest out
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

// redux.sync on floats: the largest over the warp, NaN never wins
__device__ __forceinline__ float warp_redux_max(float v)
{
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b)         // NaN if either is
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 1 / (1 + exp(-l)) within 2^-22: the exponential is good to 2^-22 relative (its argument's rounding included, since
// the slope t / (1 + t)^2 falls faster than |l| grows) and the slope is at most 1/4; reciprocal and sum add 2^-23;
// results below 2^-126 flush to zero.
__device__ __forceinline__ float sigmoid_approx(float l)
{
    float t, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(l * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + t));
    return s;
}

template <int N>
struct TopTwo {                           // the two largest of N values
    static __device__ __forceinline__ float2 of(const float* c)
    {
        const float2 a = TopTwo<N / 2>::of(c), b = TopTwo<N / 2>::of(c + N / 2);
        return make_float2(fmaxf(a.x, b.x), fmaxf(fminf(a.x, b.x), fmaxf(a.y, b.y)));
    }
};
template <>
struct TopTwo<2> {
    static __device__ __forceinline__ float2 of(const float* c) { return make_float2(fmaxf(c[0], c[1]), fminf(c[0], c[1])); }
};
template <>
struct TopTwo<1> {
    static __device__ __forceinline__ float2 of(const float* c) { return make_float2(c[0], -INFINITY); }
};

// The router is bound by instruction issue (in exact arithmetic throughout: 1,138 instructions per token at 256 experts,
// 3.5 issued per cycle and SM, 75 us for 65,536 tokens, where reading the logits takes 11 us).  So the bulk of the work is
// done on approximate choice values with a known error, and only the candidates, one per lane, are evaluated exactly:
//  1. c ~ sigmoid + bias within err = 2^-21 + 2^-22 (1 + max|bias|), the roundings of the sum on both sides included
//     (without a bias the logits themselves are compared, err = 0);
//  2. groups: two largest per lane, merged over the lanes of a group; the topk_group best by warp-wide maxima.  If the
//     last kept and the first dropped lie closer than their errors, or equal scores leave too many, the exact path decides;
//  3. the K-th largest lane maximum, less twice the error, is a bound that every expert of the true choice reaches;
//  4. the experts that reach it (about K + 2) are compacted; each lane evaluates one of them exactly, and its rank
//     is the number of candidates with a larger choice value, or an equal one and a lower index.
// A warp keeps its biases in registers from token to token and fetches the next token's logits ahead.  Step 4 takes CAP
// lanes: with CAP = 16 (at most eight slots) the candidates of two tokens are evaluated together.
constexpr int route_blocks_per_sm(int vpl) { return vpl <= 8 ? 4 : vpl == 16 ? 2 : 1; }
template <int VPL, bool BF16, bool SIGMOID, bool BY_SCORE, int CAP>
__global__ void __launch_bounds__(kRouteWarps * 32, route_blocks_per_sm(VPL)) route_kernel(const RouteParams p)
{
    extern __shared__ uint32_t dyn_keys[];                        // [warps][E], only for groups that split a lane's run
    __shared__ RouteSmem s_route[kRouteWarps];
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const unsigned step = gridDim.x * kRouteWarps;
    unsigned tok = blockIdx.x * kRouteWarps + warp;
    RouteSmem& sm = s_route[warp];
    griddep_wait();
    if (tok >= p.n_tok) return;
    if (!p.fast) {
        for (; tok < p.n_tok; tok += step)
            route_exact<VPL, BF16, SIGMOID, BY_SCORE>(p, tok, sm, dyn_keys + (size_t)warp * p.E);
        return;
    }
    // A group owns a power of two of lanes; a lane holds `run` (or fewer) experts of its group from e0 on.
    const int lpg = p.lanes_per_group, in_group = (lane & (lpg - 1)) * p.run;
    const int left = lane / lpg < p.n_group ? max(0, min(p.run, p.group_size - in_group)) : 0;
    const int e0 = left > 0 ? lane / lpg * p.group_size + in_group : 0, end = e0 + left;
    float bias[BY_SCORE ? VPL : 1], err = 0.0f;
    if constexpr (BY_SCORE) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            bias[i] = i >= left ? -INFINITY : p.bias ? p.bias[e0 + i] : 0.0f;
            if (bias[i] != bias[i]) bias[i] = -INFINITY;
            if (bias[i] > -INFINITY) err = fmaxf(err, fabsf(bias[i]));
        }
        err = 0x1p-21f + 0x1p-22f * (1.0f + warp_redux_max(err));
    }
    const bool padded = p.E != 32 * VPL;

    float l[VPL];
    load_logits<VPL, BF16, true>(l, p.logits, (long long)tok * p.stride, e0, end, p.fast_vec != 0);
    constexpr int kBatch = 32 / CAP;                              // tokens whose candidates share the warp
    const int sub = lane & (CAP - 1), mine_b = lane / CAP;        // place among the candidates of token mine_b of the batch
    for (; tok < p.n_tok; tok += kBatch * step) {
        int total = 0;                                            // of token mine_b: candidates, and its softmax statistics
        float m_sel = 0.0f, sum_sel = 1.0f;
        unsigned redo = 0;                                        // tokens of the batch that the exact path decides
        __syncwarp();                                             // the last batch's candidates have been read
#pragma unroll 1
        for (int b = 0; b < kBatch; ++b) {
            const unsigned t = tok + b * step;
            if (t >= p.n_tok) {
                if (mine_b == b) total = -1;
                break;
            }
            float c[VPL], least = l[0];
#pragma unroll
            for (int i = 1; i < VPL; ++i) least = min_nan(least, l[i]);
            bool exact = __any_sync(kFull, !(least > -INFINITY));
#pragma unroll
            for (int i = 0; i < VPL; ++i) c[i] = BY_SCORE ? sigmoid_approx(l[i]) + bias[i] : l[i];
            if (!BY_SCORE && padded) {
#pragma unroll
                for (int i = 0; i < VPL; ++i)
                    if (i >= left) c[i] = -INFINITY;
            }
            float m = 0.0f, sum = 1.0f;
            if constexpr (!SIGMOID) {                                 // logits are compared (BY_SCORE softmax is never fast)
                m = c[0];
#pragma unroll
                for (int i = 1; i < VPL; ++i) m = fmaxf(m, c[i]);
                m = warp_redux_max(m);
                if (!p.renormalise) {
                    float s = 0.0f;
#pragma unroll
                    for (int i = 0; i < VPL; ++i) s += softmax_term(c[i], m);
                    sum = warp_sum(s);
                }
            }
            // the next token's logits travel while this one is decided
            if (t + step < p.n_tok) load_logits<VPL, BF16, true>(l, p.logits, (long long)(t + step) * p.stride, e0, end, p.fast_vec != 0);

            float2 two = TopTwo<VPL>::of(c);
            float lane_max = two.x;
            bool kept = true;
            if (p.n_group > 1) {
                for (int o = 1; o < lpg; o <<= 1) {
                    const float bx = __shfl_xor_sync(kFull, two.x, o), by = __shfl_xor_sync(kFull, two.y, o);
                    two = make_float2(fmaxf(two.x, bx), fmaxf(fminf(two.x, bx), fmaxf(two.y, by)));
                }
                float g = p.top2 && two.y > -INFINITY ? two.x + two.y : two.x;
                float last = 0.0f;
                kept = false;
#pragma unroll 4
                for (int r = 0; r < p.topk_group; ++r) {
                    last = warp_redux_max(g);
                    if (g == last) {
                        kept = g > -INFINITY;
                        g = -INFINITY;
                    }
                }
                const float first_out = warp_redux_max(g);
                const int n_kept = __popc(__ballot_sync(kFull, kept));
                // no more groups than asked for may be kept; fewer only if no other has a member left
                exact |= n_kept > p.topk_group * lpg || first_out >= last - 8.0f * err ||
                         (n_kept < p.topk_group * lpg && first_out > -INFINITY);
                lane_max = kept ? lane_max : -INFINITY;
            }
            float bound = -INFINITY;
#pragma unroll 4
            for (int r = 0; r < p.K; ++r) {
                bound = warp_redux_max(lane_max);
                if (lane_max == bound) lane_max = -INFINITY;
            }
            if constexpr (BY_SCORE) bound -= 4.0f * err;
            bound = bound >= -3.402823466e38f ? bound : -3.402823466e38f;     // -inf (and the NaN of its margin): all finite ones
            if (!kept) bound = INFINITY;
            uint32_t flags = 0;
#pragma unroll
            for (int i = 0; i < VPL; ++i) flags |= c[i] >= bound ? 1u << i : 0u;
            int at = __popc(flags);
            const int mine = at;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(kFull, at, o);
                if (lane >= o) at += v;
            }
            const int found = __shfl_sync(kFull, at, 31);
            at -= mine;
            exact |= found > CAP;
            if (found <= CAP)
                for (at += b * CAP; flags; flags &= flags - 1) sm.id[at++] = e0 + __ffs(flags) - 1;
            if (exact) redo |= 1u << b;
            if (mine_b == b) {
                total = exact ? -1 : found;
                m_sel = m;
                sum_sel = sum;
            }
        }
        __syncwarp();
        const unsigned my_tok = tok + mine_b * step;
        int id = -1, rank = p.K;
        float lk = 0.0f, s = 0.0f;
        uint32_t key = 0;
        if (sub < total) {
            id = sm.id[lane];
            lk = load_as_float<BF16>(p.logits, (long long)my_tok * p.stride + id);
            float ck = lk;
            if constexpr (SIGMOID) s = sigmoid_f(lk);
            if constexpr (BY_SCORE) ck = __fadd_rn(s, p.bias ? p.bias[id] : 0.0f);
            key = key_of(ck);
        }
        sm.one[lane] = key;
        __syncwarp();
        const uint32_t* keys = sm.one + mine_b * CAP;
        if (sub < total) {
            rank = 0;
            for (int j = 0; j < total; j += 4) {                  // slots beyond the candidates hold the lowest key
                const uint4 o = *reinterpret_cast<const uint4*>(keys + j);
                rank += (o.x > key ? 1 : 0) + (o.y > key ? 1 : 0) + (o.z > key ? 1 : 0) + (o.w > key ? 1 : 0);
            }
        }
        // equal keys share a rank; candidates lie in index order, so those in front go first
        const uint32_t here = __ballot_sync(kFull, sub < total);
        if (__reduce_or_sync(kFull, sub < total ? 1u << (rank + mine_b * CAP) : 0u) != here && sub < total)
            for (int j = 0; j < sub; ++j) rank += keys[j] == key ? 1 : 0;
        const bool sel = rank < p.K;
        if constexpr (!SIGMOID) s = sel ? softmax_term(lk, m_sel) : 0.0f;
        // s / d before the caller's scale enters: scale / d overflows where a few tiny scores make up d.  Both are lifted by 2^32, which is
        // exact, because 1 / d alone overflows at the smallest score there is (2^-128).  (A division for it: 1.3 us more at 65,536 tokens.)
        float over = 1.0f;
        if (p.renormalise) {
            float d = sel ? s : 0.0f;
#pragma unroll
            for (int o = CAP / 2; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
            over = d > 0.0f ? __frcp_rn(0x1p32f * d) : 0.0f;
            s *= 0x1p32f;
        } else if (!SIGMOID) {
            over = __frcp_rn(sum_sel);
        }
        const long long at0 = (long long)my_tok * p.K;
        if (sel) {
            p.ids[at0 + rank] = id;
            p.w[at0 + rank] = s * over * p.scale;
        }
        if (total >= 0 && sub >= total && sub < p.K) {
            p.ids[at0 + sub] = -1;
            p.w[at0 + sub] = 0.0f;
        }
        if (redo) {
            for (int b = 0; b < kBatch; ++b)
                if ((redo >> b) & 1u)
                    route_exact<VPL, BF16, SIGMOID, BY_SCORE>(p, tok + b * step, sm, dyn_keys + (size_t)warp * p.E);
        }
    }
    griddep_launch_dependents();
}

struct RouteGradParams {
    const void* logits;
    long long stride;
    const int32_t* ids;
    const float* dw;
    void* dlogits;
    long long dstride;
    int* status;
    unsigned n_tok;
    int E, K;
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
    const unsigned tok = blockIdx.x * kRouteWarps + warp;
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

    float l[VPL], m = 0.0f, inv = 0.0f, mean = 0.0f, d;
    if constexpr (kFullRow) {
        load_logits<VPL, BF16>(l, p.logits, base, e0, p.E, p.vec_ok != 0);
        m = l[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) m = fmaxf(m, l[i]);
        m = warp_max(m);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            l[i] = l[i] == -INFINITY ? 0.0f : softmax_grad_term<BF16>(l[i], m);
            s += l[i];
        }
        s = warp_sum(s);
        inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
        d = p.scale * dw;
        mean = warp_sum(live ? d * softmax_grad_term<BF16>(lk, m) * inv : 0.0f);
    } else if constexpr (MODE == kGradSigmoid) {
        const float s = live ? sigmoid_f(lk) : 0.0f;
        const float rest = live ? sigmoid_f(-lk) : 0.0f;          // 1 - s without the cancellation
        d = p.scale * dw * s;
        if (p.renormalise) {
            // (scale / D) * (dw - dot) * s through the weight s / D: 1 / D overflows where a few tiny scores make up D
            const float total = warp_sum(s);
            const float w = total > 0.0f ? __fdiv_rn(s, total) : 0.0f;
            const float dot = warp_sum(dw * w);
            d = p.scale * (dw - dot) * w;
        }
        d *= rest;
    } else {
        m = warp_max(lk);
        float t = live ? softmax_term(lk, m) : 0.0f;
        const float total = warp_sum(t);
        t = total > 0.0f ? __fdiv_rn(t, total) : 0.0f;
        const float dot = warp_sum(dw * t);
        d = live ? p.scale * t * (dw - dot) : 0.0f;
    }
    if (!live) d = 0.0f;
    __syncwarp();
    float* slot = row + (id % VPL) * 32 + id / VPL;               // register i of lane q, without bank conflicts
    if (id >= 0) *slot = __int_as_float(lane);
    __syncwarp();
    // an expert that stands twice in a token: its slots add up, in slot order
    if (__any_sync(kFull, id >= 0 && __float_as_int(*slot) != lane)) {
        float add = 0.0f;
        for (int k = 0; k < p.K; ++k) {
            const int ik = __shfl_sync(kFull, id, k);
            const float dk = __shfl_sync(kFull, d, k);
            if (ik == id) add += dk;
        }
        d = add;
    }
    __syncwarp();
    if (id >= 0) *slot = d;
    __syncwarp();

    float g[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        g[i] = row[i * 32 + lane];
        if constexpr (kFullRow) g[i] = l[i] * inv * (g[i] - mean);
    }
    store_row<VPL, BF16>(g, p.dlogits, (long long)tok * p.dstride, e0, p.E, p.dvec_ok != 0);
}

// registers per lane for runs of `lanes` lanes over `n` experts
int lanes_width(int n, int lanes = 32)
{
    int v = 1;
    while (lanes * v < n) v *= 2;
    return v;
}

template <int VPL, bool BF16>
cudaError_t route_vpl(RouteParams& p, const strata_route_params& r, int n_sm, cudaStream_t st)
{
    const bool by_score = p.bias != nullptr || p.top2;
    constexpr int kVec = BF16 ? 8 : 4;                            // logits in 16 bytes
    // The shorter way needs every group inside its lanes.  Where the group count is no power of two, lanes stay without a
    // group, and above 560 experts the others may have more than 32 each: those shapes take the exact path, whose runs cover
    // all 1,024 whatever the groups.
    p.fast = !(by_score && r.score == STRATA_SCORE_SOFTMAX) && p.group_size <= p.lanes_per_group * VPL;
    p.run = (p.group_size + p.lanes_per_group - 1) / p.lanes_per_group;
    if (VPL >= kVec) p.run = (p.run + kVec - 1) / kVec * kVec;
    p.fast_vec = p.vec_ok && p.run % kVec == 0 && p.group_size % kVec == 0;
    const unsigned grid = min((p.n_tok + kRouteWarps - 1) / kRouteWarps, (unsigned)(n_sm * route_blocks_per_sm(VPL)));
    const size_t smem = p.n_group > 1 && p.group_size % VPL != 0 ? (size_t)kRouteWarps * p.E * sizeof(uint32_t) : 0;
    // two tokens per batch where their candidates (about K + 2) fit 16 lanes, and where a warp has two tokens at all
    const bool pairs = VPL <= 8 && p.K <= 8 && p.n_tok > grid * kRouteWarps;
    constexpr int kPairCap = VPL <= 8 ? 16 : 32;
#define STRATA_ROUTE(SIG, BY)                                                                                            \
    (pairs ? launch_pdl(route_kernel<VPL, BF16, SIG, BY, kPairCap>, grid, kRouteWarps * 32, smem, st, p)                 \
           : launch_pdl(route_kernel<VPL, BF16, SIG, BY, 32>, grid, kRouteWarps * 32, smem, st, p))
    if (r.score == STRATA_SCORE_SIGMOID) return by_score ? STRATA_ROUTE(true, true) : STRATA_ROUTE(true, false);
    return by_score ? STRATA_ROUTE(false, true) : STRATA_ROUTE(false, false);
#undef STRATA_ROUTE
}

template <int VPL, bool BF16>
cudaError_t route_grad_vpl(const RouteGradParams& p, const strata_route_params& r, cudaStream_t st)
{
    const unsigned grid = (p.n_tok + kRouteWarps - 1) / kRouteWarps;
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
                         long long stride, const float* bias, int32_t* ids, float* w, int n_sm, cudaStream_t st)
{
    RouteParams p{};
    p.logits = logits;
    p.stride = stride;
    p.bias = bias;
    p.ids = ids;
    p.w = w;
    p.n_tok = (unsigned)s.R * (unsigned)s.T;
    p.E = s.E;
    p.K = s.K;
    p.n_group = r.n_group;
    p.topk_group = r.topk_group;
    p.group_size = s.E / r.n_group;
    p.lanes_per_group = 32;
    while (p.lanes_per_group * r.n_group > 32) p.lanes_per_group /= 2;
    p.renormalise = r.renormalise;
    p.top2 = r.n_group > 1 && r.group_score == STRATA_GROUP_TOP2;
    p.vec_ok = rows_on_16(logits, stride, type);
    p.scale = r.scale;
    const bool bf = type == STRATA_T_BF16;
    switch (lanes_width(p.group_size, p.lanes_per_group)) {
        case 1: return bf ? route_vpl<1, true>(p, r, n_sm, st) : route_vpl<1, false>(p, r, n_sm, st);
        case 2: return bf ? route_vpl<2, true>(p, r, n_sm, st) : route_vpl<2, false>(p, r, n_sm, st);
        case 4: return bf ? route_vpl<4, true>(p, r, n_sm, st) : route_vpl<4, false>(p, r, n_sm, st);
        case 8: return bf ? route_vpl<8, true>(p, r, n_sm, st) : route_vpl<8, false>(p, r, n_sm, st);
        case 16: return bf ? route_vpl<16, true>(p, r, n_sm, st) : route_vpl<16, false>(p, r, n_sm, st);
        // 32, and what only the exact path holds (see p.fast)
        default: return bf ? route_vpl<32, true>(p, r, n_sm, st) : route_vpl<32, false>(p, r, n_sm, st);
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
    p.n_tok = (unsigned)s.R * (unsigned)s.T;
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
