// Rows in 4-bit microscaled floating point (MXFP4 of the OCP Microscaling Formats specification 1.0): 32 values share a scale, a
// power of two in 8 bits (E8M0, exponent + 127, 255 = NaN); a value is 4 bits, E2M1: +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.  The lower half
// of a byte holds the value with the lower index.
//
//   scale = 2^(floor(log2(largest magnitude of the 32)) - 2), at least 2^-127;   code = value / scale, nearest, ties to even, at most 6
//
// Dividing by a power of two is exact, so the only rounding is that to 4 bits.  A block that holds an infinity or a NaN gets the
// scale NaN.  Bound by HBM: a value is read once in its own type and written as 4.25 bits, or the other way round: 16,384 rows of 7,168
// bf16 there and back 95 us, 6.25 TB/s (fp32 166 us, 6.4).  Next to that bound: instructions, about 75 a thread for 16 values; with eight
// values a thread, 64-bit row arithmetic and a maximum value by value it was 139 us.
#include <cuda_fp4.h>
#include <type_traits>

#include "elements.cuh"
#include "row_pieces.h"

namespace {

constexpr int kMxThreads = 256;
constexpr int kMxPer = 16;                        // values of a thread's piece: two threads share a scale

struct MxArgs {
    const void* x;
    uint8_t *codes, *scales;
    const int32_t* n_rows;                        // rows in use, on the device; null: all
    uint32_t x_step, codes_step, scales_step;     // bytes from a row to the next
    int R, groups;                                // groups of kMxPer values per row
    long long up;                                 // bytes from a value to what its activation is multiplied with
    SmallDiv by_groups;
    bool wide, wide_codes;
};

__device__ __forceinline__ int rows_in_use(const int32_t* n_rows, int R) { return n_rows ? min(max(*n_rows, 0), R) : R; }

// Sixteen values as they lie in memory, moved 32 bytes at a time: with 16-byte accesses at that distance a warp's touch every sector
// twice, which cost a tenth of the time.
template <typename T>
struct alignas(32) Raw { T v[kMxPer]; };
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* at, bool wide) {
    Raw<T> r;
    if (wide) {
        unsigned* const w = (unsigned*)r.v;
#pragma unroll
        for (int i = 0; i < (int)sizeof(r) / 4; i += 8)
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
                         : "l"((const unsigned*)at + i) : "memory");
    } else {
#pragma unroll
        for (int v = 0; v < kMxPer; v++) r.v[v] = at[v];
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_raw(T* at, const Raw<T>& r, bool wide) {
    if (wide) {
        const unsigned* const w = (const unsigned*)r.v;
#pragma unroll
        for (int i = 0; i < (int)sizeof(r) / 4; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"((unsigned*)at + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]),
                         "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
    } else {
#pragma unroll
        for (int v = 0; v < kMxPer; v++) at[v] = r.v[v];
    }
}

// The largest magnitude of a block of 32 as the bits of a float (their order is that of the values, NaN above all); 16-bit types
// two at a time.
__device__ __forceinline__ unsigned with_neighbour(unsigned most) { return max(most, __shfl_xor_sync(kAll, most, 1)); }
__device__ __forceinline__ unsigned block_most(const Raw<float>& r) {
    unsigned most = 0;
#pragma unroll
    for (int v = 0; v < kMxPer; v++) most = max(most, __float_as_uint(r.v[v]) & 0x7fffffffu);
    return with_neighbour(most);
}
template <typename T>
__device__ __forceinline__ unsigned block_most(const Raw<T>& r) {
    const unsigned* const w = (const unsigned*)r.v;
    unsigned most = 0;
#pragma unroll
    for (int v = 0; v < kMxPer / 2; v++) most = __vmaxu2(most, w[v] & 0x7fff7fffu);
    most = with_neighbour(max(most >> 16, most & 0xffffu));
    return __float_as_uint(value_of(*(const T*)&most));
}

// Eight values to four bytes: nearest, ties to even, magnitudes above 6 to 6.
__device__ __forceinline__ unsigned codes_of(const float (&x)[8]) {
    unsigned r;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}\n"
        : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}

// x / (1 + e^-x) over all of x: off by five units in the last place at most (a result below the normal numbers: by half of their smallest
// step as well).
//   e^-x = 2^n 2^f with n an integer next to -x log2 e (found by adding 1.5 * 2^23, which leaves no bits behind the point) and f the rest, in
//   two steps with log2 e split into its 32-bit value and what that lacks (the reduction of Cody and Waite).
//   1 / (1 + 2^n 2^f) = 2^-n / (2^-n + 2^f): nothing leaves the normal numbers before the result does.
//   n is held within -30 (the sum is 1 from there on) and 126 by a product that saturates; f takes what is beyond, up to an infinity, whose
//   reciprocal is 0.
constexpr double kLog2e = 1.4426950408889634;
constexpr float kLog2eHigh = (float)kLog2e, kLog2eRest = (float)(kLog2e - (double)kLog2eHigh);
__device__ __forceinline__ float silu(float x) {
    constexpr float whole = 12582912, least = -30, range = 156;
    float held;
    asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(held) : "f"(x), "f"((float)(-kLog2e / range)), "f"(-least / range));
    const float m = fmaf(held, range, whole + least);
    const float f = fmaf(x, -kLog2eRest, fmaf(x, -kLog2eHigh, whole - m));
    const float down = __uint_as_float(__float_as_uint(m) * (0u - (1u << 23)) + (127u << 23));      // 2^-n (the bits of m end in those of n)
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(down + e));
    return x * r * down;
}

// 2^e, -127 <= e <= 127.
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 1 << 22); }

// Row and piece of a row of the CTA's u-th piece of this thread; false behind the last row in use (the row is that one then).  A CTA's
// pieces are consecutive.
struct Piece { int r, c; };
__device__ __forceinline__ bool piece_of(const MxArgs& a, int r0, int c0, int rows, int u, Piece& p) {
    const int i = c0 + u * kMxThreads + (int)threadIdx.x, down = a.by_groups.div(i);
    p.c = i - down * a.groups;
    return row_below(r0, down, rows, p.r);
}

// N pieces a thread, all loaded before the first is worked on.  GATED: rows are 2 K wide, the value is silu(x[k]) * x[K + k], in 32
// bits.
template <typename T, int N, bool GATED>
__global__ void __launch_bounds__(kMxThreads)
mxfp4_quantize_kernel(const __grid_constant__ MxArgs a) {
    grid_wait();
    const int rows = rows_in_use(a.n_rows, a.R);
    const long long i0 = (long long)blockIdx.x * (kMxThreads * N), first = i0 / a.groups;
    if (first >= rows) return;
    const int r0 = (int)first, c0 = (int)(i0 - first * a.groups);
    Piece p[N];
    bool in[N];
    Raw<T> raw[N], up[GATED ? N : 1];
#pragma unroll
    for (int u = 0; u < N; u++) {
        in[u] = piece_of(a, r0, c0, rows, u, p[u]);
        const char* const at = (const char*)a.x + (uint64_t)p[u].r * a.x_step + p[u].c * (kMxPer * (int)sizeof(T));
        raw[u] = load_raw((const T*)at, a.wide);
        if (GATED) up[u] = load_raw((const T*)(at + a.up), a.wide);
    }
#pragma unroll
    for (int u = 0; u < N; u++) {
        unsigned most;                            // (groups is even: a block's two threads are neighbours)
        Raw<float> x;
#pragma unroll
        for (int v = 0; v < kMxPer; v++) x.v[v] = value_of(raw[u].v[v]);
        if (GATED) {
#pragma unroll
            for (int v = 0; v < kMxPer; v++) x.v[v] = silu(x.v[v]) * value_of(up[u].v[v]);
            most = block_most(x);
        } else {
            most = block_most(raw[u]);
        }
        const bool finite = most < 0x7f800000u;
        const int e = max((int)(most >> 23) - 129, -127);        // (magnitudes below 2^-125, zero among them: 2^-127)
        const float inverse = power_of_two(-e);
        unsigned word[2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float y[8];
#pragma unroll
            for (int v = 0; v < 8; v++) y[v] = x.v[8 * h + v] * inverse;
            word[h] = finite ? codes_of(y) : 0;
        }
        if (in[u]) {
            uint8_t* const to = a.codes + (uint64_t)p[u].r * a.codes_step + p[u].c * (kMxPer / 2);
            if (a.wide_codes) *(uint2*)to = make_uint2(word[0], word[1]);
            else
#pragma unroll
                for (int b = 0; b < 8; b++) to[b] = (uint8_t)(word[b / 4] >> (8 * (b % 4)));
            if ((p[u].c & 1) == 0) a.scales[(uint64_t)p[u].r * a.scales_step + p[u].c / 2] = finite ? (uint8_t)(e + 127) : 255;
        }
    }
}

// To the values that codes and scales stand for, rounded once to T (exact in bf16 and fp32).
template <typename T, int N>
__global__ void __launch_bounds__(kMxThreads)
mxfp4_dequantize_kernel(const __grid_constant__ MxArgs a) {
    grid_wait();
    const int rows = rows_in_use(a.n_rows, a.R);
    const long long i0 = (long long)blockIdx.x * (kMxThreads * N), first = i0 / a.groups;
    if (first >= rows) return;
    const int r0 = (int)first, c0 = (int)(i0 - first * a.groups);
    Piece p[N];
    bool in[N];
    uint2 word[N];
    int s[N];
#pragma unroll
    for (int u = 0; u < N; u++) {
        in[u] = piece_of(a, r0, c0, rows, u, p[u]);
        const uint8_t* const from = a.codes + (uint64_t)p[u].r * a.codes_step + p[u].c * (kMxPer / 2);
        if (a.wide_codes) word[u] = *(const uint2*)from;
        else {
            word[u].x = (unsigned)from[0] | (unsigned)from[1] << 8 | (unsigned)from[2] << 16 | (unsigned)from[3] << 24;
            word[u].y = (unsigned)from[4] | (unsigned)from[5] << 8 | (unsigned)from[6] << 16 | (unsigned)from[7] << 24;
        }
        s[u] = a.scales[(uint64_t)p[u].r * a.scales_step + p[u].c / 2];
    }
#pragma unroll
    for (int u = 0; u < N; u++) {
        const float scale = s[u] == 255 ? CUDART_NAN_F : power_of_two(s[u] - 127);
        Raw<T> y;
#pragma unroll
        for (int v = 0; v < kMxPer; v += 2) {
            const unsigned w = v < 8 ? word[u].x >> (4 * v) : word[u].y >> (4 * (v - 8));
            const float2 f = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)w, __NV_E2M1)));
            y.v[v] = rounded<T>(f.x * scale);
            y.v[v + 1] = rounded<T>(f.y * scale);
        }
        if (in[u]) store_raw((T*)((char*)a.x + (uint64_t)p[u].r * a.x_step + p[u].c * (kMxPer * (int)sizeof(T))), y, a.wide);
    }
}

int fill(MxArgs& a, const void* x, int dtype, int64_t ld, int64_t width, int64_t R, int64_t K, const uint8_t* codes, int64_t codes_ld,
         const uint8_t* scales, int64_t scales_ld, const int32_t* n_rows) {
    if (!is_type(dtype) || R < 0 || K <= 0 || K % VP_MXFP4_BLOCK || ld < width || codes_ld < K / 2 || scales_ld < K / VP_MXFP4_BLOCK)
        return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    const int64_t most = (int64_t)1 << 31;        // rows, bytes of a row
    if (R >= most || ld >= most / size || codes_ld >= most || scales_ld >= most) return VP_E_UNSUPPORTED;
    if (R == 0) return VP_OK;
    if (!x || !codes || !scales) return VP_E_BAD_ARG;
    if ((uintptr_t)x % size || (uintptr_t)n_rows % 4) return VP_E_BAD_ARG;
    const int groups = (int)(K / kMxPer);
    a = MxArgs{x, (uint8_t*)codes, (uint8_t*)scales, n_rows, (uint32_t)(ld * size), (uint32_t)codes_ld, (uint32_t)scales_ld, (int)R, groups,
               K * size, small_div(groups), (uintptr_t)x % 32 == 0 && ld * size % 32 == 0, (uintptr_t)codes % 8 == 0 && codes_ld % 8 == 0};
    return VP_OK;
}

// Pieces a thread: one until the GPU is full of threads, then two, so that more is on its way.  One | two, us, rows of 7,168 bf16: 128 to codes
// 1.74 | 1.73, 500 2.9 | 2.4, 676 3.1 | 3.6, 3,000 10.5 | 10.3, 16,384 48.9 | 45.9; back 500 3.1 | 2.6, 676 3.4 | 3.1, 16,384 51.5 | 45.4; gated rows of
// 2,048: 300 2.2 | 2.6, 2,000 7.0 | 7.2, 16,384 36.7 | 34.2.
template <typename F>
int launch_pieces(const MxArgs& a, F fn) {
    const int sms = sm_count_of_device();
    if (!sms) return VP_E_CUDA;
    const long long pieces = (long long)a.R * a.groups;
    const int n = pieces <= (long long)sms * 2048 ? 1 : 2;
    const long long grid = (pieces + kMxThreads * n - 1) / (kMxThreads * n);
    if (grid >= ((long long)1 << 31)) return VP_E_UNSUPPORTED;
    return fn(n, (int)grid) == cudaSuccess ? VP_OK : VP_E_CUDA;
}

}  // namespace

extern "C" int vp_mxfp4_quantize(const void* x, int dtype, int64_t ld, int64_t rows, int64_t cols, int gated, const int32_t* n_rows,
                                 uint8_t* codes, int64_t codes_ld, uint8_t* scales, int64_t scales_ld, void* cuda_stream) {
    MxArgs a;
    const int rc = fill(a, x, dtype, ld, gated ? 2 * cols : cols, rows, cols, codes, codes_ld, scales, scales_ld, n_rows);
    if (rc || rows == 0) return rc;
    int done = VP_E_BAD_ARG;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
            done = launch_pieces(a, [&](int n, int grid) {
            const auto go = [&](auto kernel) { return launch_after(kernel, grid, kMxThreads, 0, (cudaStream_t)cuda_stream, a); };
            if (gated) return n == 1 ? go(mxfp4_quantize_kernel<X, 1, true>) : go(mxfp4_quantize_kernel<X, 2, true>);
            return n == 1 ? go(mxfp4_quantize_kernel<X, 1, false>) : go(mxfp4_quantize_kernel<X, 2, false>);
        });
    });
    return done;
}

extern "C" int vp_mxfp4_dequantize(const uint8_t* codes, int64_t codes_ld, const uint8_t* scales, int64_t scales_ld, int64_t rows,
                                   int64_t cols, const int32_t* n_rows, void* out, int dtype, int64_t ld, void* cuda_stream) {
    MxArgs a;
    const int rc = fill(a, out, dtype, ld, cols, rows, cols, codes, codes_ld, scales, scales_ld, n_rows);
    if (rc || rows == 0) return rc;
    int done = VP_E_BAD_ARG;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        done = launch_pieces(a, [&](int n, int grid) {
            return launch_after(n == 1 ? mxfp4_dequantize_kernel<X, 1> : mxfp4_dequantize_kernel<X, 2>, grid, kMxThreads, 0,
                                (cudaStream_t)cuda_stream, a);
        });
    });
    return done;
}
