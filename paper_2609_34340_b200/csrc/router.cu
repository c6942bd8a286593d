// Routing of tokens to experts (the indices vp_demand_from_routing and vp_pack take, and the weights vp_combine takes) and
// its gradient.
//
// Of the logits z of a token: scores s = softmax(z) or 1 / (1 + exp(-z)), keys = s + bias; with groups, the topk_group groups
// with the largest sum of their best group_top keys; of what is left the topk largest keys, the lower index among equals.
// Weights are the scores without the bias, divided by their sum if wanted, times a factor.
//
// Which of two experts is chosen hangs on the last bit of a key, so keys in 32 bits, whose error depends on the exponential's
// code, are not enough to make the choice reproducible.  Without a bias there is nothing to round: scores rise with logits, so
// logits are compared.  With one, 32-bit keys are computed with a bound on their error; where two keys that matter are nearer
// than twice that bound and do not come from equal logits and biases, those are compared in 64 bits (one token in some 400).
//
// Bound by instructions: about 760 a token of 256 experts, of which a quarter are the scores.  16,384 tokens x 256 fp32 logits, sigmoid, bias, best
// 8 of 4 of 8 groups: 16 to 18 us from one run to another (41 with all keys of an unclear token in 64 bits and one expert chosen per round), where
// reading the logits takes 2.7; 128 tokens 2.9 us, a launch and one warp's chain.  Equal logits leave more than 32 candidates, chosen one by one in
// 64 bits: the same tokens 78 us then, and 33 without groups and bias.
#include <cmath>
#include <type_traits>

#include "elements.cuh"
#include "route_bound.h"

namespace {

constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxTop = 32;                  // a lane per chosen expert
constexpr int kRouteMaxGroups = 32;
constexpr int kRouteWarps = 4;

struct RouteArgs {
    const void* logits;
    long long ld;
    int T, E, topk;
    const float* bias;
    bool sigmoid, renormalise, wide, wide_bias;   // wide: rows can be loaded by vectors
    int n_group, topk_group, group_top, per;      // per: experts of a group
    int lanes_per_group, group_shift;             // 2^group_shift when groups are that many whole lanes', else 0
    float scale;
    int32_t* idx;
    float* weights;
};

// A logit or a bias as it counts: -inf for NaN (the maximum of a NaN and a number is the number), the largest number for inf.
__device__ __forceinline__ float logit_of(float x) { return fminf(fmaxf(x, -CUDART_INF_F), CUDART_MAX_NORMAL_F); }

// Logits of experts lane * VPL .. of one row; -inf for those that cannot be chosen (NaN, -inf, none there).
template <typename T, int VPL>
__device__ __forceinline__ void load_logits(const T* row, int E, bool wide, float (&z)[VPL]) {
    constexpr int most = 16 / (int)sizeof(T);
    constexpr int V = VPL % 8 == 0 && most >= 8 ? 8 : (VPL % 4 == 0 && most >= 4 ? 4 : (VPL % 2 == 0 ? 2 : 1));
    const int first = (int)(threadIdx.x & 31) * VPL;
    T raw[VPL];
#pragma unroll
    for (int v = 0; v < VPL; v += V) {
        if (wide && first + v + V <= E) {
            const Pack<T, V> p = *(const Pack<T, V>*)(row + first + v);
#pragma unroll
            for (int u = 0; u < V; u++) raw[v + u] = p.v[u];
        } else {
#pragma unroll
            for (int u = 0; u < V; u++) raw[v + u] = first + v + u < E ? row[first + v + u] : rounded<T>(-CUDART_INF_F);
        }
    }
#pragma unroll
    for (int v = 0; v < VPL; v++) z[v] = logit_of(value_of(raw[v]));
}

// Biases of experts lane * VPL .. as they are, 0 without one.
template <int VPL>
__device__ __forceinline__ void load_bias(const float* bias, int E, bool wide, float (&b)[VPL]) {
    constexpr int V = VPL % 4 == 0 ? 4 : (VPL % 2 == 0 ? 2 : 1);
    const int first = (int)(threadIdx.x & 31) * VPL;
#pragma unroll
    for (int v = 0; v < VPL; v += V) {
        if (wide && first + v + V <= E) {
            const Pack<float, V> p = *(const Pack<float, V>*)(bias + first + v);
#pragma unroll
            for (int u = 0; u < V; u++) b[v + u] = p.v[u];
        } else {
#pragma unroll
            for (int u = 0; u < V; u++) b[v + u] = bias && first + v + u < E ? bias[first + v + u] : 0.f;
        }
    }
}

__device__ __forceinline__ float reciprocal(float x) {           // within a unit in the last place; of infinity 0
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float fast_exp(float x) {             // 2^(x log2 e), the product rounded: |x| 2^-24 + 2^-22, relative
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}

// Largest and second largest: of a pair and a third value, and of two pairs.
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }
template <typename K>
__device__ __forceinline__ void insert(K& hi, K& lo, K x) {
    lo = larger(lo, smaller(hi, x));
    hi = larger(hi, x);
}
template <typename K>
__device__ __forceinline__ void merge(K& hi, K& lo, K hi2, K lo2) {
    lo = larger(larger(lo, lo2), smaller(hi, hi2));
    hi = larger(hi, hi2);
}
// What a group is judged by; -inf only where it has nothing to choose.  Two keys of the lowest value, an expert's bias where it is kept out that
// way, add up to less than 32 bits hold: held there, such groups are equal, and compared in 64 bits.
__device__ __forceinline__ float within(float x) { return fminf(fmaxf(x, -CUDART_MAX_NORMAL_F), CUDART_MAX_NORMAL_F); }
__device__ __forceinline__ double within(double x) { return x; }
template <typename K>
__device__ __forceinline__ K sum_of_two(K a, K b, int top) {
    return top > 1 && b > -(K)CUDART_INF_F ? within(a + b) : a;
}

// What a softmax score in 64 bits is taken from: the largest logit and the sum of the exponentials below it.
struct Total { double most, sum; };
template <int VPL>
__device__ __forceinline__ Total exact_total(const float* zs, bool sigmoid) {
    if (sigmoid) return Total{0, 1};
    double most = -(double)CUDART_INF_F, sum = 0;
    for (int v = 0; v < VPL; v++) most = fmax(most, (double)zs[v]);
    for (int o = 16; o; o >>= 1) most = fmax(most, __shfl_xor_sync(kAll, most, o));
    for (int v = 0; v < VPL; v++) sum += zs[v] > -CUDART_INF_F ? exp((double)zs[v] - most) : 0.0;
    return Total{most, warp_sum(sum)};
}
__device__ __forceinline__ double exact_score(float z, bool sigmoid, const Total& t) {
    return sigmoid ? 1 / (1 + exp(-(double)z)) : exp((double)z - t.most) / t.sum;
}

// Groups that a token may use, from scores in 64 bits.
template <int VPL>
__device__ __noinline__ unsigned open_groups_exactly(const float* zs, const RouteArgs& a) {
    const int lane = threadIdx.x & 31, first = lane * VPL;
    const double none = -(double)CUDART_INF_F;
    const Total total = exact_total<VPL>(zs, a.sigmoid);
    double by[VPL];
#pragma unroll
    for (int v = 0; v < VPL; v++) {
        const float b = a.bias && first + v < a.E ? logit_of(a.bias[first + v]) : 0.f;
        const bool there = zs[v] > -CUDART_INF_F && b > -CUDART_INF_F;
        by[v] = there ? exact_score(zs[v], a.sigmoid, total) + (double)b : none;
    }
    double mine = none;                           // lane g: the score of group g
    if (a.lanes_per_group) {
        double hi = none, lo = none;
#pragma unroll
        for (int v = 0; v < VPL; v++) insert(hi, lo, by[v]);
        for (int o = 1; o < a.lanes_per_group; o *= 2) merge(hi, lo, __shfl_xor_sync(kAll, hi, o), __shfl_xor_sync(kAll, lo, o));
        mine = __shfl_sync(kAll, sum_of_two(hi, lo, a.group_top), lane * a.lanes_per_group & 31);
    } else {
        for (int g = 0; g < a.n_group; g++) {
            double hi = none, lo = none;
#pragma unroll
            for (int v = 0; v < VPL; v++)
                if (first + v < a.E && (first + v) / a.per == g) insert(hi, lo, by[v]);
            for (int o = 16; o; o >>= 1) merge(hi, lo, __shfl_xor_sync(kAll, hi, o), __shfl_xor_sync(kAll, lo, o));
            if (lane == g) mine = sum_of_two(hi, lo, a.group_top);
        }
    }
    int rank = 0;
    for (int g = 0; g < a.n_group; g++) {
        const double other = __shfl_sync(kAll, mine, g);
        rank += other > mine || (other == mine && g < lane);
    }
    return __ballot_sync(kAll, lane < a.n_group && rank < a.topk_group);
}

// The choice among the experts `can` marks, one per round, in 64 bits: for tokens with more than 32 candidates (many experts to a
// lane and most of them shut).  Lane r returns the r-th chosen expert or -1.
template <int VPL>
__device__ __noinline__ int choose_by_rounds(const float* zs, unsigned can, const RouteArgs& a) {
    const int lane = threadIdx.x & 31, first = lane * VPL;
    const double none = -(double)CUDART_INF_F;
    const Total total = a.bias ? exact_total<VPL>(zs, a.sigmoid) : Total{0, 1};
    double key[VPL];
    for (int v = 0; v < VPL; v++) {
        const float b = a.bias && first + v < a.E ? a.bias[first + v] : 0.f;
        key[v] = can >> v & 1 ? (a.bias ? exact_score(zs[v], a.sigmoid, total) + (double)logit_of(b) : (double)zs[v]) : none;
    }
    int chosen = -1;
    for (int r = 0; r < a.topk; r++) {
        double best = none;
        int at = kRouteMaxExperts;
        for (int v = 0; v < VPL; v++)
            if (key[v] > best) { best = key[v]; at = first + v; }
        for (int o = 16; o; o >>= 1) {
            const double other = __shfl_xor_sync(kAll, best, o);
            const int from = __shfl_xor_sync(kAll, at, o);
            if (other > best || (other == best && from < at)) { best = other; at = from; }
        }
        if (!(best > none)) break;                // (the same in every lane)
        if (lane == r) chosen = at;
        for (int v = 0; v < VPL; v++)
            if (first + v == at) key[v] = none;
    }
    return chosen;
}

// Rank of the lanes' keys among the first n, the lower index first among equals; 32 from lane n on.
template <typename K>
__device__ __forceinline__ int rank_of(K k, int at, int n) {
    int rank = (int)(threadIdx.x & 31) < n ? 0 : 32;
    for (int c = 0; c < n; c++) {
        const K other = __shfl_sync(kAll, k, c);
        const int from = __shfl_sync(kAll, at, c);
        rank += other > k || (other == k && from < at);
    }
    return rank;
}

// Scores of the chosen (lane r has the r-th, `here` if there is one) up to a factor common to the token, which is 1 unless the
// weights are divided by their sum: that factor keeps small scores from vanishing in 32 bits.
__device__ __forceinline__ float chosen_score(bool sigmoid, bool renormalise, float z, float most, float total) {
    if (!sigmoid) return renormalise ? fast_exp(z - most) : fast_exp(z - most) * reciprocal(total);
    const float under = renormalise ? fminf(most, 0.f) : 0.f;          // (a factor of e^-under for every score)
    return z >= 0 ? reciprocal(1 + fast_exp(-z)) : fast_exp(z - under) * reciprocal(1 + fast_exp(z));
}

// A warp per token; lane l holds experts l * VPL .. l * VPL + VPL - 1.  The topk-th largest of the lanes' maxima is a lower bound of
// the topk-th key, so the few keys above it (about 10 of 256 for the best 8) are put side by side, a lane each, and ranked by counting.
template <typename T, int VPL>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_kernel(const __grid_constant__ RouteArgs a) {
    extern __shared__ float s_keys[];             // [warps][E], groups that are not whole lanes' only
    __shared__ alignas(16) float s_key[kRouteWarps][32];
    __shared__ int s_at[kRouteWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = lane * VPL;
    grid_wait();
    const int t = (int)(blockIdx.x * kRouteWarps) + warp;
    if ((unsigned)t >= (unsigned)a.T) return;     // (the last CTA's warps may pass 2^31)
    const T* const row = (const T*)a.logits + t * a.ld;
    float z[VPL], key[VPL];
    load_logits<T, VPL>(row, a.E, a.wide, z);
    float most = -CUDART_INF_F, total = 1;
    if (!a.sigmoid) {                             // softmax: its largest logit and the sum below it
#pragma unroll
        for (int v = 0; v < VPL; v++) most = fmaxf(most, z[v]);
        most = warp_max(most);
        const float top = most > -CUDART_INF_F ? most : 0.f;
        total = 0;
#pragma unroll
        for (int v = 0; v < VPL; v++) total += fast_exp(z[v] - top);
        total = warp_sum(total);
    }
    // keys, and what groups are judged by where that is something else
    const bool rounded_keys = a.bias != nullptr, rounded_groups = rounded_keys || a.group_top > 1;
    float tol = 0;
    float by[VPL];
#pragma unroll
    for (int v = 0; v < VPL; v++) key[v] = by[v] = z[v];
    if (rounded_keys || (a.n_group > 1 && rounded_groups)) {
        float largest = 0;
        const float over = a.sigmoid ? 1.f : reciprocal(total);
        float b[VPL];
        load_bias<VPL>(a.bias, a.E, a.wide_bias, b);
#pragma unroll
        for (int v = 0; v < VPL; v++) {
            const float k = (a.sigmoid ? reciprocal(1 + fast_exp(-z[v])) : fast_exp(z[v] - most) * over) + b[v];
            largest = fmaxf(largest, fabsf(k));
            by[v] = z[v] > -CUDART_INF_F ? fmaxf(k, -CUDART_INF_F) : -CUDART_INF_F;      // (NaN of the bias: -inf)
            if (rounded_keys) key[v] = by[v];
        }
        largest = warp_max(largest);
        if (!(largest < CUDART_INF_F)) {          // a bias of -inf, or of inf, which counts as the largest number, or no logit
            largest = 0;
#pragma unroll
            for (int v = 0; v < VPL; v++) {
                by[v] = fminf(by[v], CUDART_MAX_NORMAL_F);
                if (rounded_keys) key[v] = by[v];
                if (by[v] > -CUDART_INF_F) largest = fmaxf(largest, fabsf(by[v]));
            }
            largest = warp_max(largest);
        }
        tol = over * twice_score_error(a.sigmoid, VPL) + 2.5e-7f * largest;       // (the sum with the bias: half a unit of the key)
    }
    if (a.n_group > 1) {
        float mine = -CUDART_INF_F;
        if (a.lanes_per_group) {                  // every lane of a group gets its score
            float hi = -CUDART_INF_F, lo = -CUDART_INF_F;
#pragma unroll
            for (int v = 0; v < VPL; v++) insert(hi, lo, by[v]);
            for (int o = 1; o < a.lanes_per_group; o *= 2) merge(hi, lo, __shfl_xor_sync(kAll, hi, o), __shfl_xor_sync(kAll, lo, o));
            mine = __shfl_sync(kAll, sum_of_two(hi, lo, a.group_top), lane * a.lanes_per_group & 31);
        } else {
            float* const k = s_keys + warp * a.E;
#pragma unroll
            for (int v = 0; v < VPL; v++)
                if (first + v < a.E) k[first + v] = by[v];
            __syncwarp();
            if (lane < a.n_group) {
                float hi = -CUDART_INF_F, lo = -CUDART_INF_F;
                for (int e = lane * a.per; e < (lane + 1) * a.per; e++) insert(hi, lo, k[e]);
                mine = sum_of_two(hi, lo, a.group_top);
            }
        }
        // topk_group times the best that is left, the lowest index among equals (groups without an expert that can be chosen need no choice).
        if (lane >= a.n_group) mine = -CUDART_INF_F;
        unsigned open = 0;
        float worst_in = CUDART_INF_F;
        for (int r = 0; r < a.topk_group; r++) {
            worst_in = warp_max(mine);
            const unsigned best = __ballot_sync(kAll, mine == worst_in);
            open |= best & (0u - best);
            if (open >> lane & 1) mine = -CUDART_INF_F;
        }
        if (rounded_groups) {                     // is the last group in clear of the first one out?
            const float best_out = warp_max(mine);
            if (best_out > -CUDART_INF_F && !(worst_in - best_out > 2 * tol)) {
                float copy[VPL];                  // (z itself stays in registers)
#pragma unroll
                for (int v = 0; v < VPL; v++) copy[v] = z[v];
                open = open_groups_exactly<VPL>(copy, a);
            }
        }
        if (a.lanes_per_group) {
            const bool shut = !(open >> (lane >> a.group_shift) & 1);
#pragma unroll
            for (int v = 0; v < VPL; v++)
                if (shut) key[v] = -CUDART_INF_F;
        } else {
#pragma unroll
            for (int v = 0; v < VPL; v++)
                if (first + v < a.E && !(open >> ((first + v) / a.per) & 1)) key[v] = -CUDART_INF_F;
        }
    }
    const float near = rounded_keys ? tol : 0.f;
    float x = -CUDART_INF_F, bound = -CUDART_INF_F;
#pragma unroll
    for (int v = 0; v < VPL; v++) x = fmaxf(x, key[v]);
    for (int r = 0; r < a.topk; r++) {            // (equal maxima leave together: the bound is lower then, and still one)
        bound = warp_max(x);
        if (x == bound) x = -CUDART_INF_F;
    }
    bound = fmaxf(bound - near, -CUDART_MAX_NORMAL_F);
    // Candidates side by side, in the order of their indices: places by a scan over the lanes' counts.
    unsigned mine = 0;
#pragma unroll
    for (int v = 0; v < VPL; v++) mine |= (unsigned)(key[v] >= bound) << v;
    int n = __popc(mine);
    const int own = n;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int other = __shfl_up_sync(kAll, n, o);
        if (lane >= o) n += other;
    }
    int place = n - own;
    n = __shfl_sync(kAll, n, 31);
    int chosen;
    if (n <= 32) {
        s_key[warp][lane] = -CUDART_INF_F;
        __syncwarp();
#pragma unroll
        for (int v = 0; v < VPL; v++)
            if (mine >> v & 1) {
                s_key[warp][place] = key[v];
                s_at[warp][place] = first + v;
                place++;
            }
        __syncwarp();
        const float k = s_key[warp][lane];
        const int at = lane < n ? s_at[warp][lane] : kRouteMaxExperts;
        int rank = 0;
#pragma unroll 1
        for (int c = 0; c < n; c += 4) {          // (places behind the n-th hold -inf)
            const float4 q = *(const float4*)&s_key[warp][c];
            rank += (q.x > k || (q.x == k && c < lane)) + (q.y > k || (q.y == k && c + 1 < lane)) +
                    (q.z > k || (q.z == k && c + 2 < lane)) + (q.w > k || (q.w == k && c + 3 < lane));
        }
        if (lane >= n) rank = lane;
        if (near > 0) {
            // Keys in descending order: is one that is not clearly below the topk-th near the one behind it, and not from the same
            // logit and bias?  (Of equal ones the lower index goes first, which is right.)
            __syncwarp();
            s_key[warp][rank] = k;
            __syncwarp();
            const float here = s_key[warp][lane], last = s_key[warp][min(a.topk, n) - 1 & 31];
            const float behind = lane < 31 ? s_key[warp][lane + 1] : -CUDART_INF_F;
            const bool close = lane + 1 < n && here - behind <= near && here >= last - near;
            if (__any_sync(kAll, close)) {
                const float my_z = lane < n ? logit_of(value_of(row[at])) : 0.f, my_b = lane < n ? logit_of(a.bias[at]) : 0.f;
                const unsigned where = __ballot_sync(kAll, close);
                bool differ = false;
                for (int r = 0; r < 31; r++)
                    if (where >> r & 1) {         // (the same in every lane)
                        const int up = __ffs(__ballot_sync(kAll, rank == r)) - 1, down = __ffs(__ballot_sync(kAll, rank == r + 1)) - 1;
                        differ |= __shfl_sync(kAll, my_z, up) != __shfl_sync(kAll, my_z, down) ||
                                  __shfl_sync(kAll, my_b, up) != __shfl_sync(kAll, my_b, down);
                    }
                if (differ) {
                    float copy[VPL];
#pragma unroll
                    for (int v = 0; v < VPL; v++) copy[v] = z[v];
                    const Total all = exact_total<VPL>(copy, a.sigmoid);
                    rank = rank_of(lane < n ? exact_score(my_z, a.sigmoid, all) + (double)my_b : -(double)CUDART_INF_F, at, n);
                }
            }
        }
        __syncwarp();
        s_at[warp][lane] = -1;
        __syncwarp();
        if (lane < n && rank < a.topk) s_at[warp][rank] = at;
        __syncwarp();
        chosen = s_at[warp][lane];
    } else {
        float copy[VPL];
        unsigned can = 0;                         // bit v: expert first + v can be chosen
#pragma unroll
        for (int v = 0; v < VPL; v++) {
            copy[v] = z[v];
            can |= (unsigned)(key[v] > -CUDART_INF_F) << v;
        }
        chosen = choose_by_rounds<VPL>(copy, can, a);
    }
    const bool here = chosen >= 0;
    const float zc = here ? logit_of(value_of(row[chosen])) : -CUDART_INF_F;
    const float top = a.renormalise ? warp_max(zc) : most;
    float w = here ? chosen_score(a.sigmoid, a.renormalise, zc, top, total) : 0.f;
    if (a.renormalise) {
        const float sum = warp_sum(w);
        w = sum > 0 ? w * reciprocal(sum) : 0.f;
    }
    if (lane < a.topk) {
        const int at = t * a.topk + lane;         // (below 2^31 in all)
        a.idx[at] = chosen;
        a.weights[at] = w * a.scale;
    }
}

struct RouteGradArgs {
    const void* logits;
    long long ld;
    int T, E, topk;
    bool sigmoid, renormalise, wide;
    float scale;
    const int32_t* idx;
    const float* grad;
    void* out;
    long long out_ld;
    bool out_wide;
};

// Gradient of the weights with respect to the logits, the choice held fixed.  With w the weights (scores s, divided by their sum
// S if they are renormalised) and g the gradient of the weights times the factor:
//   softmax               dz_i = s_i (g_i - sum_k g_k s_k)            every expert of the row
//   softmax, renormalised dz_j = w_j (g_j - sum_k g_k w_k)            the chosen, 0 elsewhere
//   sigmoid               dz_j = g_j s_j (1 - s_j)                    the chosen
//   sigmoid, renormalised dz_j = w_j (1 - s_j) (g_j - sum_k g_k w_k)  the chosen
// A warp per token; the row is put together in shared memory and leaves by vectors.  16,384 tokens x 128 bf16 logits, softmax as it is: 6.3 us (its
// bytes 1.5), bound by instructions and three trips to memory: indices, the logits at them, the row.
template <typename T, int VPL>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_backward_kernel(const __grid_constant__ RouteGradArgs a) {
    extern __shared__ float s_rows[];             // [warps][E]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = lane * VPL;
    grid_wait();
    const long long t = (long long)blockIdx.x * kRouteWarps + warp;
    if (t >= a.T) return;
    const T* const row = (const T*)a.logits + t * a.ld;
    float* const out = s_rows + warp * (32 * VPL);
    const bool every = !a.sigmoid && !a.renormalise;
    int at = lane < a.topk ? a.idx[t * a.topk + lane] : -1;
    float g = lane < a.topk ? a.grad[t * a.topk + lane] * a.scale : 0.f;
    float z = -CUDART_INF_F;
    if (at >= 0 && at < a.E) z = logit_of(value_of(row[at]));
    const bool here = z > -CUDART_INF_F;
    if (!here) { at = -1; g = 0; }
    float p[VPL];
    float most = -CUDART_INF_F, total = 1;
    if (every) {
        load_logits<T, VPL>(row, a.E, a.wide, p);
#pragma unroll
        for (int v = 0; v < VPL; v++) most = fmaxf(most, p[v]);
        most = warp_max(most);
        const float top = most > -CUDART_INF_F ? most : 0.f;
        total = 0;
#pragma unroll
        for (int v = 0; v < VPL; v++) total += p[v] = fast_exp(p[v] - top);
        total = warp_sum(total);
    }
    const float top = a.renormalise ? warp_max(z) : most;
    float w = here ? chosen_score(a.sigmoid, a.renormalise, z, top, total) : 0.f;
    if (a.renormalise) {
        const float sum = warp_sum(w);
        w = sum > 0 ? w * reciprocal(sum) : 0.f;
    }
    const bool centred = a.renormalise || !a.sigmoid;
    const float mean = centred ? warp_sum(g * w) : 0.f;
    float d = every ? g * w : (a.sigmoid ? w / (1 + expf(z)) * (a.renormalise ? g - mean : g) : w * (g - mean));
    if (!here) d = 0;
    const float over = every && total > 0 ? mean / total : 0.f;
#pragma unroll
    for (int v = 0; v < VPL; v++) out[first + v] = every ? -p[v] * over : 0.f;
    __syncwarp();
    const unsigned same = __match_any_sync(kAll, at);             // an index that stands there twice collects both
    float sum = 0;
    if (at >= 0 && __popc(same) > 1) {
        for (int l = 0; l < 32; l++)
            if (same >> l & 1) sum += __shfl_sync(same, d, l);
    } else {
        sum = d;
    }
    if (at >= 0 && (same & ((1u << lane) - 1)) == 0) out[at] += sum;
    __syncwarp();
    T* const to = (T*)a.out + t * a.out_ld;
    constexpr int V = 16 / (int)sizeof(T);
    if (a.out_wide) {
        for (int e = lane * V; e < a.E; e += 32 * V) {
            Pack<T, V> q;
#pragma unroll
            for (int u = 0; u < V; u++) q.v[u] = rounded<T>(out[e + u]);
            *(Pack<T, V>*)(to + e) = q;
        }
    } else {
        for (int e = lane; e < a.E; e += 32) to[e] = rounded<T>(out[e]);
    }
}

// Calls fn with the number of experts per lane as a constant.
template <typename F>
void with_vpl(int E, F fn) {
    const int n = (E + 31) / 32;
#define VPL(k) if (n <= k) return fn(std::integral_constant<int, k>{});
    VPL(1) VPL(2) VPL(3) VPL(4) VPL(5) VPL(6) VPL(8) VPL(12) VPL(16) VPL(24) VPL(32)
#undef VPL
}

int check_route(const vp_route_params* p) {
    if (!p || p->experts <= 0 || p->topk <= 0 || p->topk > p->experts) return VP_E_BAD_ARG;
    if (p->scoring != VP_SCORE_SOFTMAX && p->scoring != VP_SCORE_SIGMOID) return VP_E_BAD_ARG;
    if (p->n_group <= 0 || p->experts % p->n_group || p->topk_group <= 0 || p->topk_group > p->n_group) return VP_E_BAD_ARG;
    if (p->group_top != 1 && p->group_top != 2) return VP_E_BAD_ARG;
    if (p->topk > p->topk_group * (p->experts / p->n_group)) return VP_E_BAD_ARG;
    if (!std::isfinite(p->scale)) return VP_E_BAD_ARG;
    if (p->experts > kRouteMaxExperts || p->topk > kRouteMaxTop || p->n_group > kRouteMaxGroups) return VP_E_UNSUPPORTED;
    return VP_OK;
}

// Whether rows of `ld` elements from `p` on can be moved by vectors of `bytes`.
bool rows_aligned(const void* p, long long ld, int size, int bytes) {
    return (uintptr_t)p % bytes == 0 && (unsigned long long)ld * size % bytes == 0;
}

// CTAs of kRouteWarps tokens at every size (a warp per CTA instead: 128 tokens 3.1 us against 2.9, 592 3.95 against 4.1, 2,000 4.5 against 4.6).
int route_ctas(int T) { return (int)(((long long)T + kRouteWarps - 1) / kRouteWarps); }

}  // namespace

extern "C" int vp_route(const vp_route_params* p, const void* logits, int dtype, int64_t ld, int T, const float* bias,
                        int32_t* expert_idx, float* weights, void* cuda_stream) {
    const int rc = check_route(p);
    if (rc) return rc;
    if (!is_type(dtype) || T < 0 || ld < p->experts) return VP_E_BAD_ARG;
    if ((long long)T * p->topk >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    if (T == 0) return VP_OK;
    if (!logits || !expert_idx || !weights) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)logits % size || ((uintptr_t)expert_idx | (uintptr_t)weights | (uintptr_t)bias) % 4) return VP_E_BAD_ARG;
    RouteArgs a;
    a.logits = logits; a.ld = ld; a.T = T; a.E = p->experts; a.topk = p->topk; a.bias = bias;
    a.sigmoid = p->scoring == VP_SCORE_SIGMOID; a.renormalise = p->renormalise != 0; a.wide = rows_aligned(logits, ld, size, 16);
    a.wide_bias = bias && (uintptr_t)bias % 16 == 0;
    a.n_group = p->n_group; a.topk_group = p->topk_group; a.group_top = p->group_top; a.per = p->experts / p->n_group;
    a.scale = p->scale; a.idx = expert_idx; a.weights = weights;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        with_vpl(a.E, [&](auto vpl) {
            constexpr int n = decltype(vpl)::value;
            const int lanes = a.per % n ? 0 : a.per / n;
            a.lanes_per_group = lanes > 0 && (lanes & (lanes - 1)) == 0 && a.n_group * lanes <= 32 ? lanes : 0;
            a.group_shift = 0;
            while (1 << a.group_shift < a.lanes_per_group) a.group_shift++;
            const size_t smem = a.n_group > 1 && !a.lanes_per_group ? (size_t)kRouteWarps * a.E * 4 : 0;
            e = launch_after(route_kernel<X, n>, route_ctas(T), kRouteWarps * 32, smem, (cudaStream_t)cuda_stream, a);
        });
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}

extern "C" int vp_route_backward(const vp_route_params* p, const void* logits, int dtype, int64_t ld, int T, const int32_t* expert_idx,
                                 const float* grad_weights, void* grad_logits, int64_t grad_ld, void* cuda_stream) {
    const int rc = check_route(p);
    if (rc) return rc;
    if (!is_type(dtype) || T < 0 || ld < p->experts || grad_ld < p->experts) return VP_E_BAD_ARG;
    if ((long long)T * p->topk >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    if (T == 0) return VP_OK;
    if (!logits || !expert_idx || !grad_weights || !grad_logits) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)logits % size || (uintptr_t)grad_logits % size || ((uintptr_t)expert_idx | (uintptr_t)grad_weights) % 4) return VP_E_BAD_ARG;
    RouteGradArgs a;
    a.logits = logits; a.ld = ld; a.T = T; a.E = p->experts; a.topk = p->topk;
    a.sigmoid = p->scoring == VP_SCORE_SIGMOID; a.renormalise = p->renormalise != 0; a.wide = rows_aligned(logits, ld, size, 16);
    a.scale = p->scale; a.idx = expert_idx; a.grad = grad_weights; a.out = grad_logits; a.out_ld = grad_ld;
    a.out_wide = rows_aligned(grad_logits, grad_ld, size, 16) && a.E * size % 16 == 0;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        with_vpl(a.E, [&](auto vpl) {
            constexpr int n = decltype(vpl)::value;
            e = launch_after(route_backward_kernel<X, n>, route_ctas(T), kRouteWarps * 32, (size_t)kRouteWarps * 32 * n * 4, (cudaStream_t)cuda_stream, a);
        });
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
