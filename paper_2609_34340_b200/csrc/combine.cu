// The end of a mixture-of-experts layer: the returned rows in the token layout (what vp_unpack_tokens writes) summed with the
// router's weights, and the gradients of that sum.
//
//   out[t] = base[t] + sum over slots s with expert_idx[t][s] >= 0 of weights[t][s] * rows[t * topk + s]
//   grad_rows[t * topk + s] = weights[t][s] * grad[t]        grad_weights[t][s] = <grad[t], rows[t * topk + s]>
//
// Both are bound by HBM: every row is read once (and its gradient written once), in 16-byte vectors, all slots of a vector in
// flight at once.  Sums are in 32 bits, slots in ascending order; a dropped copy's row is not read (its memory may hold anything).
#include <type_traits>

#include "elements.cuh"

namespace {

constexpr int kCombineThreads = 256;
constexpr int kSlots = 8;                         // slots whose rows are in flight together
constexpr int kCombineMaxTop = 4096;              // (8 bytes of shared memory per slot)

// A vector of a row that is there, zeros for one that is not (its memory may hold anything): loads under a predicate, no branch
// between them, so that all slots' are in flight together.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_if(const T* at, bool here) {
    Pack<T, V> r;
    if constexpr (sizeof(T) * V == 16) {
        uint4 q;
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n mov.u32 %0, 0;\n mov.u32 %1, 0;\n mov.u32 %2, 0;\n mov.u32 %3, 0;\n"
                     " @p ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}\n"
                     : "=&r"(q.x), "=&r"(q.y), "=&r"(q.z), "=&r"(q.w) : "l"(at), "r"((unsigned)here));
        r = *(Pack<T, V>*)&q;
    } else {
#pragma unroll
        for (int u = 0; u < V; u++) r.v[u] = here ? at[u] : rounded<T>(0.f);
    }
    return r;
}

struct CombineArgs {
    const void *rows, *base;
    const int32_t* idx;
    const float* weights;
    void* out;
    long long T, H;
    int topk, tokens, pieces;                     // tokens per CTA, CTAs per that many tokens
};

// A CTA takes a piece of `tokens` tokens side by side: their indices and weights are fetched once, which otherwise stands in front of
// every load of a row.  16,384 tokens x 8 of 7,168 bf16: one token per CTA 417 us.
template <typename T, int V>
__global__ void __launch_bounds__(kCombineThreads, 4)
combine_kernel(const __grid_constant__ CombineArgs a) {
    extern __shared__ int2 s_slot[];              // per slot: whether it counts, its weight
    grid_wait();
    const long long t0 = (long long)(blockIdx.x / a.pieces) * a.tokens;
    const int tokens = (int)min((long long)a.tokens, a.T - t0);
    for (int i = threadIdx.x; i < tokens * a.topk; i += blockDim.x) {
        const int here = a.idx[t0 * a.topk + i] >= 0;
        s_slot[i] = make_int2(here, here ? __float_as_int(a.weights[t0 * a.topk + i]) : 0);
    }
    __syncthreads();
    const long long n = a.H / V, all = n * tokens, piece = blockIdx.x % a.pieces;
    const long long lo = all * piece / a.pieces, hi = all * (piece + 1) / a.pieces;
    for (long long i = lo + threadIdx.x; i < hi; i += blockDim.x) {
        const long long k = tokens > 1 ? i / n : 0, c = (i - k * n) * V, t = t0 + k;
        const T* const rows = (const T*)a.rows + t * a.topk * a.H + c;
        float sum[V];
#pragma unroll
        for (int u = 0; u < V; u++) sum[u] = 0;
        if (a.base) {
            const Pack<T, V> x = *(const Pack<T, V>*)((const T*)a.base + t * a.H + c);
#pragma unroll
            for (int u = 0; u < V; u++) sum[u] = value_of(x.v[u]);
        }
        for (int s0 = 0; s0 < a.topk; s0 += kSlots) {
            Pack<T, V> x[kSlots];
            float w[kSlots];
#pragma unroll
            for (int s = 0; s < kSlots; s++) {
                const int slot = min(s0 + s, a.topk - 1);
                const int2 q = s_slot[(int)k * a.topk + slot];
                const bool here = q.x && s0 + s < a.topk;
                w[s] = here ? __int_as_float(q.y) : 0.f;
                x[s] = load_if<T, V>(rows + slot * a.H, here);
            }
#pragma unroll
            for (int s = 0; s < kSlots; s++)
#pragma unroll
                for (int u = 0; u < V; u++) sum[u] = fmaf(w[s], value_of(x[s].v[u]), sum[u]);
        }
        Pack<T, V> y;
#pragma unroll
        for (int u = 0; u < V; u++) y.v[u] = rounded<T>(sum[u]);
        *(Pack<T, V>*)((T*)a.out + t * a.H + c) = y;
    }
}

struct CombineGradArgs {
    const void *grad, *rows;
    const int32_t* idx;
    const float* weights;
    void* grad_rows;
    float* grad_weights;
    long long T, H;
    int topk, warps;                              // warps that share a token (a power of two)
};

// `warps` warps per token and kSlots slots, so that a thread has a few vectors; every thread keeps its part of the slots' inner products,
// which meet in a fixed order.
template <typename T, int V>
__global__ void __launch_bounds__(kCombineThreads)
combine_backward_kernel(const __grid_constant__ CombineGradArgs a) {
    __shared__ float s_part[kCombineThreads / 32][kSlots];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per_cta = kCombineThreads / 32 / a.warps;
    grid_wait();
    const int batches = (a.topk + kSlots - 1) / kSlots;
    const long long item = (long long)blockIdx.x * per_cta + warp / a.warps, t = item / batches;
    const bool in = t < a.T;
    const int s0 = (int)(item % batches) * kSlots, slots = in ? min(kSlots, a.topk - s0) : 0;
    const long long first = t * a.topk + s0, n = in ? a.H / V : 0;
    const T *const grad = (const T*)a.grad + t * a.H, *const rows = (const T*)a.rows + first * a.H;
    T* const grad_rows = (T*)a.grad_rows + first * a.H;
    bool here[kSlots];
    float w[kSlots], dot[kSlots];
#pragma unroll
    for (int s = 0; s < kSlots; s++) {
        here[s] = s < slots && a.idx[first + s] >= 0;
        w[s] = here[s] ? a.weights[first + s] : 0.f;
        dot[s] = 0;
    }
    for (long long i = (warp % a.warps) * 32 + lane; i < n; i += a.warps * 32) {
        const Pack<T, V> g = *(const Pack<T, V>*)(grad + i * V);
        Pack<T, V> x[kSlots];
        if (a.grad_weights)
#pragma unroll
            for (int s = 0; s < kSlots; s++) x[s] = load_if<T, V>(rows + (here[s] ? s : 0) * a.H + i * V, here[s]);
        if (a.grad_rows)
#pragma unroll
            for (int s = 0; s < kSlots; s++)
                if (s < slots) {
                    Pack<T, V> y;
#pragma unroll
                    for (int u = 0; u < V; u++) y.v[u] = rounded<T>(here[s] ? w[s] * value_of(g.v[u]) : 0.f);
                    *(Pack<T, V>*)(grad_rows + s * a.H + i * V) = y;
                }
        if (a.grad_weights)
#pragma unroll
            for (int s = 0; s < kSlots; s++)
#pragma unroll
                for (int u = 0; u < V; u++) dot[s] = fmaf(value_of(g.v[u]), value_of(x[s].v[u]), dot[s]);
    }
    if (!a.grad_weights) return;
    float mine = 0;
#pragma unroll
    for (int s = 0; s < kSlots; s++) {
        const float d = warp_sum(dot[s]);
        if (lane == s) mine = d;
    }
    if (a.warps > 1) {
        if (lane < kSlots) s_part[warp][lane] = mine;
        __syncthreads();
        mine = 0;
        if (warp % a.warps == 0 && lane < kSlots)
            for (int k = 0; k < a.warps; k++) mine += s_part[warp + k][lane];
    }
    if (warp % a.warps == 0 && lane < slots) a.grad_weights[first + lane] = mine;
}

// Vectors of 16 bytes where rows begin on such borders, single values elsewhere.
bool vectors(int size, int64_t H, std::initializer_list<const void*> at) {
    if (H * size % 16) return false;
    for (const void* p : at)
        if ((uintptr_t)p % 16) return false;
    return true;
}

}  // namespace

extern "C" int vp_combine(const void* rows, int dtype, const int32_t* expert_idx, const float* weights, int T, int topk, int64_t H,
                          const void* base, void* out, void* cuda_stream) {
    if (!is_type(dtype) || T < 0 || topk <= 0 || H <= 0 || H >= VP_ENTRY_LIMIT) return VP_E_BAD_ARG;
    if ((long long)T * topk >= ((long long)1 << 31) || topk > kCombineMaxTop) return VP_E_UNSUPPORTED;
    if (T == 0) return VP_OK;
    if (!rows || !expert_idx || !weights || !out) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)rows % size || (uintptr_t)base % size || (uintptr_t)out % size) return VP_E_BAD_ARG;
    const int sms = sm_count_of_device();
    if (!sms) return VP_E_CUDA;
    CombineArgs a{rows, base, expert_idx, weights, out, T, H, topk, 1, 1};
    const bool wide = vectors(size, H, {rows, base, out});
    const long long n = wide ? H * size / 16 : H;
    // Tokens side by side as long as every SM keeps four CTAs; then pieces of one vector a thread.
    while (a.tokens < 4 && a.tokens * 2 * topk <= kCombineMaxTop && (long long)T * ((n + kCombineThreads - 1) / kCombineThreads) >= (long long)a.tokens * 2 * 8 * sms)
        a.tokens *= 2;
    const long long groups = ((long long)T + a.tokens - 1) / a.tokens, most = (((long long)1 << 31) - 1) / groups;
    long long pieces = (n + kCombineThreads - 1) / kCombineThreads;
    if (pieces > most) pieces = most;
    a.pieces = (int)pieces;
    const long long per = (n * a.tokens + pieces - 1) / pieces;
    const int threads = per >= kCombineThreads ? kCombineThreads : (int)((per + 31) / 32 * 32);
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(wide ? combine_kernel<X, 16 / (int)sizeof(X)> : combine_kernel<X, 1>, (int)(groups * pieces), threads, (size_t)a.tokens * topk * 8,
                         (cudaStream_t)cuda_stream, a);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}

extern "C" int vp_combine_backward(const void* grad, const void* rows, int dtype, const int32_t* expert_idx, const float* weights, int T,
                                   int topk, int64_t H, void* grad_rows, float* grad_weights, void* cuda_stream) {
    if (!is_type(dtype) || T < 0 || topk <= 0 || H <= 0 || H >= VP_ENTRY_LIMIT) return VP_E_BAD_ARG;
    if ((long long)T * topk >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    if (T == 0) return VP_OK;
    if (!grad || !expert_idx || !weights || (!grad_rows && !grad_weights) || (grad_weights && !rows)) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)grad % size || (uintptr_t)rows % size || (uintptr_t)grad_rows % size) return VP_E_BAD_ARG;
    CombineGradArgs a{grad, rows, expert_idx, weights, grad_rows, grad_weights, T, H, topk, 1};
    const bool wide = vectors(size, H, {grad, rows, grad_rows});
    const long long n = wide ? H * size / 16 : H;
    while (a.warps < kCombineThreads / 32 && n > 4 * 32 * a.warps) a.warps *= 2;        // about four vectors a thread
    const int per_cta = kCombineThreads / 32 / a.warps;
    const long long items = (long long)T * ((topk + kSlots - 1) / kSlots), grid = (items + per_cta - 1) / per_cta;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(wide ? combine_backward_kernel<X, 16 / (int)sizeof(X)> : combine_backward_kernel<X, 1>, (int)grid, kCombineThreads, 0,
                         (cudaStream_t)cuda_stream, a);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
