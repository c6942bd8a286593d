// The end of a mixture-of-experts layer: the returned rows in the token layout (what vp_unpack_tokens writes) summed with the
// router's weights, and the gradients of that sum.
//
//   out[t] = base[t] + sum over slots s with expert_idx[t][s] >= 0 of weights[t][s] * rows[t * topk + s]
//   grad_rows[t * topk + s] = weights[t][s] * grad[t]        grad_weights[t][s] = <grad[t], rows[t * topk + s]>
//
// Both are bound by HBM: every row is read once (and its gradient written once), in 16-byte vectors, all slots of a vector in
// flight at once.  Sums are in 32 bits, slots in ascending order; a dropped copy's row is not read (its memory may hold anything).
// The sum of 16,384 tokens x 8 rows of 7,168 bf16: 324 us, 6.5 TB/s.
#include <type_traits>

#include "elements.cuh"

namespace {

constexpr int kCombineThreads = 256;
constexpr int kSlots = 8;                         // slots whose rows are in flight together, at most
constexpr int kGradThreads = 64, kGradAhead = 5;   // (three to six stages, two or four warps: within 3 %)
constexpr int kGradShared = 256;
constexpr int kGradLong = 2 * kGradShared;        // vectors of a row
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
template <typename T, int V, int S>
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
        for (int s0 = 0; s0 < a.topk; s0 += S) {
            Pack<T, V> x[S];
            float w[S];
#pragma unroll
            for (int s = 0; s < S; s++) {
                const int slot = min(s0 + s, a.topk - 1);
                const int2 q = s_slot[(int)k * a.topk + slot];
                const bool here = q.x && s0 + s < a.topk;
                w[s] = here ? __int_as_float(q.y) : 0.f;
                x[s] = load_if<T, V>(rows + slot * a.H, here);
            }
#pragma unroll
            for (int s = 0; s < S; s++)
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
    int topk;
};

// 16 bytes to shared memory while the thread goes on; zeros where there is nothing to copy (nothing is read then).
__device__ __forceinline__ void copy_16(unsigned to, const void* from, bool here) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(here ? 16 : 0) : "memory");
}

// A warp per token and S slots.  Every lane copies the vectors that it will work on itself, kGradAhead - 1 steps of 32 vectors ahead, so
// that nothing waits for another thread and the loads in flight cost no registers: with loads into registers, one step at a time or two,
// reads and writes together reached 4.9 to 6.1 TB/s (8,192 tokens x 8 of 4,096 bf16 186 to 235 us); so 168 us, 6.8 TB/s.
// SHARED: the CTA's warps share a token and S slots (with few tokens a call would wait for one warp's steps one after another: a token of
// 7,168 values, 28 steps, 16.7 us, so 4.6).
// The order of the additions depends on the row's length alone, not on which form a call of so many tokens takes.  Rows of kGradLong vectors
// and more (LONG) are always SHARED: a thread adds up vectors 256 apart.  Below, vectors are summed by themselves and then added up 32 apart,
// which a SHARED CTA, with every vector's sum in some thread, does through shared memory.
template <typename T, int S, bool SHARED, bool LONG>
__global__ void __launch_bounds__(SHARED ? kGradShared : kGradThreads)
combine_backward_kernel(const __grid_constant__ CombineGradArgs a) {
    constexpr int V = 16 / (int)sizeof(T), kGradStages = SHARED ? 2 : kGradAhead;
    extern __shared__ uint4 s_stage[];            // [warps][stages][S + 1][32]
    __shared__ float s_part[SHARED ? kGradShared / 32 : 1][S];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_wait();
    const int batches = (a.topk + S - 1) / S;
    const long long item = SHARED ? blockIdx.x : (long long)blockIdx.x * (kGradThreads / 32) + warp, t = item / batches;
    if (!SHARED && t >= a.T) return;
    const int s0 = (int)(item % batches) * S, slots = min(S, a.topk - s0);
    const long long first = t * a.topk + s0, n = a.H / V;
    const int at = lane < slots ? a.idx[first + lane] : -1;
    const float own = at >= 0 ? a.weights[first + lane] : 0.f;
    const unsigned here = __ballot_sync(kAll, at >= 0), read = a.grad_weights ? here : 0;
    const uint4 *const grad = (const uint4*)a.grad + t * n, *const rows = (const uint4*)a.rows + first * n;
    uint4* const grad_rows = (uint4*)a.grad_rows + first * n;
    uint4* const stage = s_stage + warp * kGradStages * (S + 1) * 32 + lane;
    const unsigned stage_at = (unsigned)__cvta_generic_to_shared(stage);
    const int first_vector = SHARED ? (int)threadIdx.x : lane;
    const auto issue = [&](long long i, int k) {
        const unsigned to = stage_at + k * (S + 1) * 512;
        copy_16(to, grad + i, i < n);
#pragma unroll
        for (int s = 0; s < S; s++) copy_16(to + (s + 1) * 512, rows + s * n + i, i < n && (read >> s & 1));
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float w[S], dot[S], first_dot[S];                // first_dot: a SHARED thread's first vector
#pragma unroll
    for (int s = 0; s < S; s++) {
        w[s] = __shfl_sync(kAll, own, s);
        dot[s] = first_dot[s] = 0;
    }
    constexpr int step = SHARED ? kGradShared : 32;
#pragma unroll
    for (int k = 0; k < kGradStages - 1; k++) issue(first_vector + step * k, k);
    int k = 0;
    for (long long i = first_vector; __any_sync(kAll, i < n); i += step) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kGradStages - 2) : "memory");
        const uint4* const from = stage + k * (S + 1) * 32;
        const Pack<T, V> g = *(const Pack<T, V>*)from;
        float f[V];
#pragma unroll
        for (int u = 0; u < V; u++) f[u] = value_of(g.v[u]);
#pragma unroll
        for (int s = 0; s < S; s++) {
            const Pack<T, V> x = *(const Pack<T, V>*)(from + (s + 1) * 32);
            float sum = LONG ? dot[s] : 0;
#pragma unroll
            for (int u = 0; u < V; u++) sum = fmaf(f[u], value_of(x.v[u]), sum);
            if (LONG) dot[s] = sum;
            else if (SHARED && i == first_vector) first_dot[s] = sum;
            else dot[s] += sum;
        }
        const int last = k == 0 ? kGradStages - 1 : k - 1;
        issue(i + step * (kGradStages - 1), last);
        if (a.grad_rows && i < n)
#pragma unroll
            for (int s = 0; s < S; s++) {
                const bool is = here >> s & 1;    // (0 times an infinity is not 0)
                Pack<T, V> y;
#pragma unroll
                for (int u = 0; u < V; u++) y.v[u] = rounded<T>(is ? w[s] * f[u] : 0.f);
                if (s < slots) *(Pack<T, V>*)(grad_rows + s * n + i) = y;
            }
        if (++k == kGradStages) k = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.grad_weights) return;
    if (SHARED && !LONG) {                        // at most two vectors a thread: their sums side by side, a warp for a slot's
        float* const sums = (float*)s_stage;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < S; s++) {
            sums[s * kGradLong + threadIdx.x] = first_dot[s];
            sums[s * kGradLong + kGradShared + threadIdx.x] = dot[s];
        }
        __syncthreads();
        if (warp >= slots) return;
        float part[kGradLong / 32], d = 0;        // (0 behind the row's end)
#pragma unroll
        for (int i = 0; i < kGradLong / 32; i++) part[i] = sums[warp * kGradLong + 32 * i + lane];
#pragma unroll
        for (int i = 0; i < kGradLong / 32; i++) d += part[i];
        d = warp_sum(d);
        if (lane == 0) a.grad_weights[first + warp] = here >> warp & 1 ? d : 0.f;
        return;
    }
    float mine = 0;
#pragma unroll
    for (int s = 0; s < S; s++) {
        const float d = warp_sum(dot[s]);
        if (lane == s) mine = d;
    }
    if (SHARED) {
        if (lane < S) s_part[warp][lane] = mine;
        __syncthreads();
        mine = 0;
        if (warp > 0) return;
        for (int k = 0; k < kGradShared / 32 && lane < S; k++) mine += s_part[k][lane];
    }
    if (lane < slots) a.grad_weights[first + lane] = at >= 0 ? mine : 0.f;      // (a dropped copy's zeros times an infinity are not 0)
}

// The same value by value, for rows that do not begin on 16-byte borders.
template <typename T>
__global__ void __launch_bounds__(kGradThreads)
combine_backward_plain_kernel(const __grid_constant__ CombineGradArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_wait();
    const long long item = (long long)blockIdx.x * (kGradThreads / 32) + warp, t = item / a.topk;
    if (t >= a.T) return;
    const bool here = a.idx[item] >= 0;
    const float w = here ? a.weights[item] : 0.f;
    const T *const grad = (const T*)a.grad + t * a.H, *const row = (const T*)a.rows + item * a.H;
    float dot = 0;
    for (long long i = lane; i < a.H; i += 32) {
        const float f = value_of(grad[i]);
        if (here && a.grad_weights) dot = fmaf(f, value_of(row[i]), dot);
        if (a.grad_rows) ((T*)a.grad_rows)[item * a.H + i] = rounded<T>(here ? w * f : 0.f);
    }
    dot = warp_sum(dot);
    if (lane == 0 && a.grad_weights) a.grad_weights[item] = dot;
}

// Calls fn with the slots that are in flight together as a constant, next to their number: 4,000 tokens of 4,096 bf16, us, so | eight at once: the sum
// of 1 23.6 | 35.8, of 2 26.6 | 36.2, of 3 29.9 | 36.9, of 5 35.0 | 37.9; gradients of 1 19.1 | 40.9, of 2 28.7 | 45.2, of 3 37.8 | 49.8, of 5 61.1 | 61.8.
template <typename F>
void with_slots(int topk, F fn) {
    if (topk > 6) return fn(std::integral_constant<int, kSlots>{});
    if (topk > 4) return fn(std::integral_constant<int, 6>{});
    if (topk > 2) return fn(std::integral_constant<int, 4>{});
    return topk > 1 ? fn(std::integral_constant<int, 2>{}) : fn(std::integral_constant<int, 1>{});
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
    if ((uintptr_t)rows % size || (uintptr_t)base % size || (uintptr_t)out % size || ((uintptr_t)expert_idx | (uintptr_t)weights) % 4) return VP_E_BAD_ARG;
    const int sms = sm_count_of_device();
    if (!sms) return VP_E_CUDA;
    CombineArgs a{rows, base, expert_idx, weights, out, T, H, topk, 1, 1};
    const bool wide = vectors(size, H, {rows, base, out});
    const long long n = wide ? H * size / 16 : H;
    // Tokens side by side as long as every SM keeps four CTAs; then pieces of one vector a thread.  One | two | four tokens, us, 8 rows each of 7,168
    // bf16: 128 tokens 4.6 | 5.5 | 7.4, 1,200 29.2 | 28.1 | 29.7, 2,500 61.4 | 56.1 | 55.7, 16,384 404 | 354 | 337; of 512, 20,000 tokens 33.0 | 33.8 | 34.4.
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
        with_slots(wide ? topk : kSlots, [&](auto slots) {
            constexpr int s = decltype(slots)::value;
            e = launch_after(wide ? combine_kernel<X, 16 / (int)sizeof(X), s> : combine_kernel<X, 1, kSlots>, (int)(groups * pieces), threads,
                             (size_t)a.tokens * topk * 8, (cudaStream_t)cuda_stream, a);
        });
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
    if ((uintptr_t)grad % size || (uintptr_t)rows % size || (uintptr_t)grad_rows % size ||
        ((uintptr_t)expert_idx | (uintptr_t)weights | (uintptr_t)grad_weights) % 4)
        return VP_E_BAD_ARG;
    const CombineGradArgs a{grad, rows, expert_idx, weights, grad_rows, grad_weights, T, H, topk};
    const bool wide = vectors(size, H, {grad, rows, grad_rows});
    const long long n = H * size / 16;
    const int sms = sm_count_of_device();
    if (!sms) return VP_E_CUDA;
    const auto ctas = [&](long long items) { return (int)((items + kGradThreads / 32 - 1) / (kGradThreads / 32)); };
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        if (!wide) {
            e = launch_after(combine_backward_plain_kernel<X>, ctas((long long)T * topk), kGradThreads, 0, (cudaStream_t)cuda_stream, a);
            return;
        }
        with_slots(topk, [&](auto slots) {
            constexpr int s = decltype(slots)::value;
            const long long items = (long long)T * ((topk + s - 1) / s);
            const auto go = [&](auto fn, int grid, int threads, int stages) {
                const size_t smem = (size_t)(threads / 32) * stages * (s + 1) * 512;
                e = smem > 48 * 1024 ? cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) : cudaSuccess;
                if (e == cudaSuccess) e = launch_after(fn, grid, threads, smem, (cudaStream_t)cuda_stream, a);
            };
            // Warps share a token where rows are long or tokens few: 4,096 x 8 of 7,168 bf16 150 against 160 us; 128 x 8 of 1,024 2.6 against
            // 4.1, 300 x 8 of 2,048 5.4 against 7.0; but 592 x 8 of 2,048 10.7 against 9.8, 1,531 x 6 16.8 against 16.1.
            if (n >= kGradLong) go(combine_backward_kernel<X, s, true, true>, (int)items, kGradShared, 2);
            else if (items <= 4 * sms && n > 64) go(combine_backward_kernel<X, s, true, false>, (int)items, kGradShared, 2);
            else go(combine_backward_kernel<X, s, false, false>, ctas(items), kGradThreads, kGradAhead);
        });
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
