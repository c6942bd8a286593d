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

struct CombineArgs {
    const void *rows, *base;
    const int32_t* idx;
    const float* weights;
    void* out;
    long long T, H;
    int topk, pieces;                             // CTAs per token
};

// A CTA takes one piece of one token's row: `pieces` CTAs of about kCombineThreads vectors.
template <typename T, int V>
__global__ void __launch_bounds__(kCombineThreads)
combine_kernel(const __grid_constant__ CombineArgs a) {
    grid_wait();
    const long long t = blockIdx.x / a.pieces;
    const int piece = (int)(blockIdx.x % a.pieces);
    const long long n = a.H / V, lo = n * piece / a.pieces, hi = n * (piece + 1) / a.pieces;
    const T* const rows = (const T*)a.rows + t * a.topk * a.H;
    for (long long i = lo + threadIdx.x; i < hi; i += blockDim.x) {
        float sum[V];
#pragma unroll
        for (int u = 0; u < V; u++) sum[u] = 0;
        if (a.base) {
            const Pack<T, V> x = *(const Pack<T, V>*)((const T*)a.base + t * a.H + i * V);
#pragma unroll
            for (int u = 0; u < V; u++) sum[u] = value_of(x.v[u]);
        }
        for (int s0 = 0; s0 < a.topk; s0 += kSlots) {
            Pack<T, V> x[kSlots];
            float w[kSlots];
            bool here[kSlots];
#pragma unroll
            for (int s = 0; s < kSlots; s++) {
                here[s] = s0 + s < a.topk && a.idx[t * a.topk + s0 + s] >= 0;
                if (here[s]) {
                    w[s] = a.weights[t * a.topk + s0 + s];
                    x[s] = *(const Pack<T, V>*)(rows + (s0 + s) * a.H + i * V);
                }
            }
#pragma unroll
            for (int s = 0; s < kSlots; s++)
                if (here[s])
#pragma unroll
                    for (int u = 0; u < V; u++) sum[u] = fmaf(w[s], value_of(x[s].v[u]), sum[u]);
        }
        Pack<T, V> y;
#pragma unroll
        for (int u = 0; u < V; u++) y.v[u] = rounded<T>(sum[u]);
        *(Pack<T, V>*)((T*)a.out + t * a.H + i * V) = y;
    }
}

struct CombineGradArgs {
    const void *grad, *rows;
    const int32_t* idx;
    const float* weights;
    void* grad_rows;
    float* grad_weights;
    long long T, H;
    int topk;
};

// A CTA per token and kSlots slots; every thread keeps its part of the slots' inner products, which meet in a fixed order.
template <typename T, int V>
__global__ void __launch_bounds__(kCombineThreads)
combine_backward_kernel(const __grid_constant__ CombineGradArgs a) {
    __shared__ float s_part[kCombineThreads / 32][kSlots];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_wait();
    const int batches = (a.topk + kSlots - 1) / kSlots;
    const long long t = blockIdx.x / batches;
    const int s0 = (int)(blockIdx.x % batches) * kSlots, slots = min(kSlots, a.topk - s0);
    const long long first = t * a.topk + s0, n = a.H / V;
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
    for (long long i = threadIdx.x; i < n; i += blockDim.x) {
        const Pack<T, V> g = *(const Pack<T, V>*)(grad + i * V);
        Pack<T, V> x[kSlots];
        if (a.grad_weights)
#pragma unroll
            for (int s = 0; s < kSlots; s++)
                if (here[s]) x[s] = *(const Pack<T, V>*)(rows + s * a.H + i * V);
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
                if (here[s])
#pragma unroll
                    for (int u = 0; u < V; u++) dot[s] = fmaf(value_of(g.v[u]), value_of(x[s].v[u]), dot[s]);
    }
    if (!a.grad_weights) return;
#pragma unroll
    for (int s = 0; s < kSlots; s++) {
        const float d = warp_sum(dot[s]);
        if (lane == 0) s_part[warp][s] = d;
    }
    __syncthreads();
    if (threadIdx.x < slots) {
        float d = 0;
        for (int k = 0; k < (int)(blockDim.x >> 5); k++) d += s_part[k][threadIdx.x];
        a.grad_weights[first + threadIdx.x] = d;
    }
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
    if ((long long)T * topk >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    if (T == 0) return VP_OK;
    if (!rows || !expert_idx || !weights || !out) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)rows % size || (uintptr_t)base % size || (uintptr_t)out % size) return VP_E_BAD_ARG;
    CombineArgs a{rows, base, expert_idx, weights, out, T, H, topk, 1};
    const bool wide = vectors(size, H, {rows, base, out});
    const long long n = wide ? H * size / 16 : H;
    // one vector a thread: pieces of at most kCombineThreads vectors, of equal size (7,168 bf16: four CTAs of 224 threads)
    long long pieces = (n + kCombineThreads - 1) / kCombineThreads;
    const long long most = (((long long)1 << 31) - 1) / T;
    if (pieces > most) pieces = most;
    a.pieces = (int)pieces;
    const long long per = (n + pieces - 1) / pieces;
    const int threads = per >= kCombineThreads ? kCombineThreads : (int)((per + 31) / 32 * 32);
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(wide ? combine_kernel<X, 16 / (int)sizeof(X)> : combine_kernel<X, 1>, (int)(T * pieces), threads, 0,
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
    const CombineGradArgs a{grad, rows, expert_idx, weights, grad_rows, grad_weights, T, H, topk};
    const bool wide = vectors(size, H, {grad, rows, grad_rows});
    const long long n = wide ? H * size / 16 : H;
    const int threads = n >= kCombineThreads ? kCombineThreads : (int)((n + 31) / 32 * 32);
    const long long grid = (long long)T * ((topk + kSlots - 1) / kSlots);
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(wide ? combine_backward_kernel<X, 16 / (int)sizeof(X)> : combine_backward_kernel<X, 1>, (int)grid, threads, 0,
                         (cudaStream_t)cuda_stream, a);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
