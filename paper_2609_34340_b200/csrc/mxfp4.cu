// Rows in 4-bit microscaled floating point (MXFP4 of the OCP Microscaling Formats specification 1.0): 32 values share a scale, a
// power of two in 8 bits (E8M0, exponent + 127, 255 = NaN); a value is 4 bits, E2M1: +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.  The lower half
// of a byte holds the value with the lower index.
//
//   scale = 2^(floor(log2(largest magnitude of the 32)) - 2), at least 2^-127;   code = value / scale, nearest, ties to even, at most 6
//
// Dividing by a power of two is exact, so the only rounding is that to 4 bits.  A block that holds an infinity or a NaN gets the
// scale NaN.  Bound by HBM: a value is read once in its own type and written as 4.25 bits, or the other way round.
#include <cuda_fp4.h>
#include <type_traits>

#include "elements.cuh"

namespace {

constexpr int kMxThreads = 256;
constexpr int kMxPer = 8;                         // values of a thread's piece: four threads share a scale
constexpr int kMxPieces = 4;                      // pieces of a thread, all loaded before the first is worked on

struct MxArgs {
    const void* x;
    long long ld;
    uint8_t *codes, *scales;
    long long codes_ld, scales_ld;
    const int32_t* n_rows;                        // rows in use, on the device; null: all
    long long R, K;
    int groups;                                   // of kMxPer values per row
    SmallDiv by_groups;
    bool wide, wide_codes;
};

__device__ __forceinline__ long long rows_in_use(const int32_t* n_rows, long long R) {
    if (!n_rows) return R;
    const long long n = *n_rows;
    return n < 0 ? 0 : (n < R ? n : R);
}

// Eight values in 32 bits, from kMxPer places of a row.
template <typename T>
__device__ __forceinline__ void load_eight(const T* at, bool wide, float (&x)[kMxPer]) {
    constexpr int V = 16 / (int)sizeof(T);
    alignas(16) T raw[kMxPer];
    if (wide) {
#pragma unroll
        for (int v = 0; v < kMxPer; v += V) *(Pack<T, V>*)(raw + v) = *(const Pack<T, V>*)(at + v);
    } else {
#pragma unroll
        for (int v = 0; v < kMxPer; v++) raw[v] = at[v];
    }
#pragma unroll
    for (int v = 0; v < kMxPer; v++) x[v] = value_of(raw[v]);
}

// Two values to a byte: nearest, ties to even, magnitudes above 6 to 6.
__device__ __forceinline__ unsigned codes_of(float lo, float hi) {
    unsigned r;
    asm("{\n .reg .b8 b;\n cvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n cvt.u32.u8 %0, b;\n}\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// 2^e, -127 <= e <= 127.
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 1 << 22); }

// Row and piece of a row of the CTA's u-th piece of this thread; false behind the last row in use.  A CTA's pieces are consecutive.
struct Piece { long long r; int c; };
__device__ __forceinline__ bool piece_of(const MxArgs& a, long long r0, int c0, long long rows, int u, Piece& p) {
    const int i = c0 + u * kMxThreads + (int)threadIdx.x, down = a.by_groups.div(i);
    p.r = r0 + down;
    p.c = i - down * a.groups;
    return p.r < rows;
}

// GATED: rows are 2 K wide, the value is silu(x[k]) * x[K + k], in 32 bits.
template <typename T, bool GATED>
__global__ void __launch_bounds__(kMxThreads)
mxfp4_quantize_kernel(const __grid_constant__ MxArgs a) {
    grid_wait();
    const long long rows = rows_in_use(a.n_rows, a.R), i0 = (long long)blockIdx.x * (kMxThreads * kMxPieces), r0 = i0 / a.groups;
    if (r0 >= rows) return;
    const int c0 = (int)(i0 - r0 * a.groups);
    Piece p[kMxPieces];
    bool in[kMxPieces];
    float x[kMxPieces][kMxPer], up[GATED ? kMxPieces : 1][kMxPer];
#pragma unroll
    for (int u = 0; u < kMxPieces; u++) {
        in[u] = piece_of(a, r0, c0, rows, u, p[u]);
        const T* const at = (const T*)a.x + (in[u] ? p[u].r * a.ld + p[u].c * kMxPer : 0);      // (the first is in use)
        load_eight<T>(at, a.wide, x[u]);
        if (GATED) load_eight<T>(at + a.K, a.wide, up[u]);
    }
#pragma unroll
    for (int u = 0; u < kMxPieces; u++) {
        if (GATED)
#pragma unroll
            for (int v = 0; v < kMxPer; v++) x[u][v] = x[u][v] / (1 + expf(-x[u][v])) * up[u][v];
        unsigned most = 0;                        // of magnitudes as bits: their order is that of the values, NaN above all
#pragma unroll
        for (int v = 0; v < kMxPer; v++) most = max(most, __float_as_uint(x[u][v]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(kAll, most, 1));        // (groups is a multiple of four: a block's threads are neighbours)
        most = max(most, __shfl_xor_sync(kAll, most, 2));
        const bool finite = most < 0x7f800000u;
        const int e = max((int)(most >> 23) - 129, -127);        // (magnitudes below 2^-125, zero among them: 2^-127)
        const float inverse = power_of_two(-e);
        unsigned word = 0;
#pragma unroll
        for (int v = 0; v < kMxPer; v += 2) word |= codes_of(x[u][v] * inverse, x[u][v + 1] * inverse) << (4 * v);
        if (!finite) word = 0;
        if (in[u]) {
            uint8_t* const to = a.codes + p[u].r * a.codes_ld + p[u].c * (kMxPer / 2);
            if (a.wide_codes) *(unsigned*)to = word;
            else
#pragma unroll
                for (int b = 0; b < 4; b++) to[b] = (uint8_t)(word >> (8 * b));
            if ((p[u].c & 3) == 0) a.scales[p[u].r * a.scales_ld + p[u].c / 4] = finite ? (uint8_t)(e + 127) : 255;
        }
    }
}

// To the values that codes and scales stand for, rounded once to T (exact in bf16 and fp32).
template <typename T>
__global__ void __launch_bounds__(kMxThreads)
mxfp4_dequantize_kernel(const __grid_constant__ MxArgs a) {
    grid_wait();
    const long long rows = rows_in_use(a.n_rows, a.R), i0 = (long long)blockIdx.x * (kMxThreads * kMxPieces), r0 = i0 / a.groups;
    if (r0 >= rows) return;
    const int c0 = (int)(i0 - r0 * a.groups);
    Piece p[kMxPieces];
    bool in[kMxPieces];
    unsigned word[kMxPieces];
    int s[kMxPieces];
#pragma unroll
    for (int u = 0; u < kMxPieces; u++) {
        in[u] = piece_of(a, r0, c0, rows, u, p[u]);
        if (!in[u]) p[u] = Piece{r0, 0};
        const uint8_t* const from = a.codes + p[u].r * a.codes_ld + p[u].c * (kMxPer / 2);
        if (a.wide_codes) word[u] = *(const unsigned*)from;
        else word[u] = (unsigned)from[0] | (unsigned)from[1] << 8 | (unsigned)from[2] << 16 | (unsigned)from[3] << 24;
        s[u] = a.scales[p[u].r * a.scales_ld + p[u].c / 4];
    }
#pragma unroll
    for (int u = 0; u < kMxPieces; u++) {
        const float scale = s[u] == 255 ? CUDART_NAN_F : power_of_two(s[u] - 127);
        alignas(16) T y[kMxPer];
#pragma unroll
        for (int v = 0; v < kMxPer; v += 2) {
            const __half2 h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(word[u] >> (4 * v)), __NV_E2M1);
            y[v] = rounded<T>(__low2float(h) * scale);
            y[v + 1] = rounded<T>(__high2float(h) * scale);
        }
        T* const to = (T*)a.x + p[u].r * a.ld + p[u].c * kMxPer;
        constexpr int V = 16 / (int)sizeof(T);
        if (!in[u]) continue;
        if (a.wide) {
#pragma unroll
            for (int v = 0; v < kMxPer; v += V) *(Pack<T, V>*)(to + v) = *(const Pack<T, V>*)(y + v);
        } else {
#pragma unroll
            for (int v = 0; v < kMxPer; v++) to[v] = y[v];
        }
    }
}

int fill(MxArgs& a, const void* x, int dtype, int64_t ld, int64_t width, int64_t R, int64_t K, const uint8_t* codes, int64_t codes_ld,
         const uint8_t* scales, int64_t scales_ld, const int32_t* n_rows) {
    if (!is_type(dtype) || R < 0 || K <= 0 || K % VP_MXFP4_BLOCK || ld < width || codes_ld < K / 2 || scales_ld < K / VP_MXFP4_BLOCK)
        return VP_E_BAD_ARG;
    if (R >= ((int64_t)1 << 31) || K >= ((int64_t)1 << 31)) return VP_E_UNSUPPORTED;
    if (R == 0) return VP_OK;
    if (!x || !codes || !scales) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)x % size) return VP_E_BAD_ARG;
    a = MxArgs{x, ld, (uint8_t*)codes, (uint8_t*)scales, codes_ld, scales_ld, n_rows, R, K, (int)(K / kMxPer), small_div((int)(K / kMxPer)),
               (uintptr_t)x % 16 == 0 && ld * size % 16 == 0, (uintptr_t)codes % 4 == 0 && codes_ld % 4 == 0};
    return VP_OK;
}

long long mx_grid(const MxArgs& a) { return (a.R * a.groups + kMxThreads * kMxPieces - 1) / (kMxThreads * kMxPieces); }

}  // namespace

extern "C" int vp_mxfp4_quantize(const void* x, int dtype, int64_t ld, int64_t rows, int64_t cols, int gated, const int32_t* n_rows,
                                 uint8_t* codes, int64_t codes_ld, uint8_t* scales, int64_t scales_ld, void* cuda_stream) {
    MxArgs a;
    const int rc = fill(a, x, dtype, ld, gated ? 2 * cols : cols, rows, cols, codes, codes_ld, scales, scales_ld, n_rows);
    if (rc || rows == 0) return rc;
    const long long grid = mx_grid(a);
    if (grid >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(gated ? mxfp4_quantize_kernel<X, true> : mxfp4_quantize_kernel<X, false>, (int)grid, kMxThreads, 0,
                         (cudaStream_t)cuda_stream, a);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}

extern "C" int vp_mxfp4_dequantize(const uint8_t* codes, int64_t codes_ld, const uint8_t* scales, int64_t scales_ld, int64_t rows,
                                   int64_t cols, const int32_t* n_rows, void* out, int dtype, int64_t ld, void* cuda_stream) {
    MxArgs a;
    const int rc = fill(a, out, dtype, ld, cols, rows, cols, codes, codes_ld, scales, scales_ld, n_rows);
    if (rc || rows == 0) return rc;
    const long long grid = mx_grid(a);
    if (grid >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = launch_after(mxfp4_dequantize_kernel<X>, (int)grid, kMxThreads, 0, (cudaStream_t)cuda_stream, a);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
