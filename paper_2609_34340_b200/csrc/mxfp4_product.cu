// The experts' products in 4-bit microscaled floating point: expert-major rows (what vp_unpack writes, quantised) times the
// transposed matrix of their expert,
//
//   out[r][f] = sum_k value(x[r][k]) * value(w[e][f][k]),   expert_off[e] <= r < expert_off[e + 1],
//
// on the block-scaled tensor-core path (tcgen05.mma, E2M1 operands, an E8M0 scale per 32 values): products are exact, sums are
// in 32 bits in tensor memory, rounded once to the output's type.
//
// One persistent CTA per SM takes output tiles of 128 rows x NT features in turn.  Per 256 values of k a stage of shared memory holds
// both operands (TMA, 128-byte swizzle) and their scales; warp 0 loads operands, warps 2 and 3 load scales and lay them out as the
// tensor core reads them, warp 1 issues the copies of scales into tensor memory and the products, warps 4 to 7 bring finished
// tiles from tensor memory to the output while the next tile is summed.
#include <cuda.h>
#include <type_traits>

#include "bulk_copy.cuh"
#include "elements.cuh"

namespace {

constexpr int kPrMaxExperts = 1024;
constexpr int kPrMaxK = 1 << 20, kPrMaxF = 1 << 20;      // (a matrix is below 2^40 bytes, a tile's sum below a millisecond)
constexpr int kPrM = 128;                         // rows of a tile: lanes of tensor memory
constexpr int kPrK = 256;                         // values of k per stage: one swizzle atom of 128 bytes
constexpr int kPrBox = 32;                        // rows per TMA box of the rows' operand
constexpr int kPrThreads = 256;
constexpr unsigned kPrPolls = 1u << 22;

template <int NT>
struct Shape {
    static constexpr int stages = NT == 256 ? 4 : 6;
    static constexpr int a_bytes = kPrM * (kPrK / 2), b_bytes = NT * (kPrK / 2);
    static constexpr int sa_bytes = kPrM * (kPrK / 32), sb_bytes = NT * (kPrK / 32);
    static constexpr int stage = a_bytes + b_bytes + sa_bytes + sb_bytes;
    // Tensor memory, 512 columns.  Scales have a place per stage, so a stage's scales are overwritten only after the products that
    // read them.  Two tiles of 256 columns and the scales do not fit side by side: the second tile then shares columns with the
    // first, and a tile is begun as soon as the shared columns of the one before it have been read.
    static constexpr int scale_cols = 8 + NT / 32 * 2;
    static constexpr int scales_at = 512 - stages * scale_cols;
    static constexpr int second_at = NT == 256 ? scales_at - NT : NT;
    static constexpr bool shared_cols = second_at < NT;
    static constexpr int lag = shared_cols ? 1 : 2;
    static constexpr int first_chunks = shared_cols ? (NT - second_at) / 32 : NT / 32;     // of 32 columns: read before the next tile
    static_assert(scales_at >= second_at + NT && (NT - second_at) % 32 == 0, "columns of tensor memory");
};

struct ProductArgs {
    const uint8_t *xs, *ws;                       // scales: rows of xs_ld bytes, contiguous [E][F][K / 32]
    long long xs_ld;
    const int32_t* off;
    int E, R, F, K;
    void* out;
    long long out_ld;
    bool out_wide;                                // rows of the output begin at 16-byte borders
    int32_t* status;
};

__device__ __forceinline__ void mbar_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory operand descriptors: 128-byte swizzle, rows of 128 bytes in groups of eight; and plain rows of 16 bytes for scales.
__device__ __forceinline__ uint64_t operand_desc(unsigned at) {
    return (uint64_t)(at >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t scale_desc(unsigned at) {
    return (uint64_t)(at >> 4) | (uint64_t)(128 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
__device__ __forceinline__ void copy_scales(unsigned tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_mxf4(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned sa, unsigned sb, bool add) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void mma_commit(unsigned bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 32 columns of the warp's 32 lanes.
__device__ __forceinline__ void load_columns(unsigned tmem, unsigned (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(tmem) : "memory");
}

// The experts that have rows, in order: id, first row, rows, and the row tiles in front of them.
struct Experts {
    int *id, *first, *rows, *tiles;               // tiles: one entry more
    int n;
};

struct Tile {
    int e, first, rows, n0;                       // expert, first row, rows (at most kPrM), first feature
};

__device__ __forceinline__ Tile tile_of(const Experts& x, long long tile, int n_tiles, int nt) {
    // tiles of an expert: its row tiles next to one another, feature tile by feature tile
    int lo = 0, hi = x.n - 1;
    while (lo < hi) {                             // the last expert whose first tile is not behind `tile`
        const int mid = (lo + hi + 1) / 2;
        if ((long long)x.tiles[mid] * n_tiles <= tile) lo = mid; else hi = mid - 1;
    }
    const int m_tiles = x.tiles[lo + 1] - x.tiles[lo];
    const int q = (int)(tile - (long long)x.tiles[lo] * n_tiles), m = q % m_tiles;
    return Tile{x.id[lo], x.first[lo] + m * kPrM, min(kPrM, x.rows[lo] - m * kPrM), q / m_tiles * nt};
}

// 16 bytes of scales from byte k of a row of `bytes`; 1 behind its end and in rows that are not there.
__device__ __forceinline__ uint4 load_scales(const uint8_t* row, int k, int bytes, bool there) {
    uint4 v = make_uint4(0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f, 0x7f7f7f7f);
    if (!there || k >= bytes) return v;
    const uint8_t* const p = row + k;
    if (k + 16 <= bytes && ((uintptr_t)p & 15) == 0) return *(const uint4*)p;
    unsigned* const w = (unsigned*)&v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (k + 4 * i + 4 <= bytes && ((uintptr_t)p & 3) == 0) w[i] = *(const unsigned*)(p + 4 * i);
        else
#pragma unroll
            for (int b = 0; b < 4; b++)
                if (k + 4 * i + b < bytes) w[i] = (w[i] & ~(255u << (8 * b))) | (unsigned)p[4 * i + b] << (8 * b);
    }
    return v;
}

template <int NT, typename T>
__global__ void __launch_bounds__(kPrThreads, 1)
mxfp4_product_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map,
                     const __grid_constant__ ProductArgs a) {
    using S = Shape<NT>;
    extern __shared__ unsigned char s_raw[];
    __shared__ uint64_t s_bar[2 * S::stages + 5];
    __shared__ unsigned s_tmem;
    __shared__ int s_n;
    __shared__ volatile int s_stop;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned base = (smem_u32(s_raw) + 1023) & ~1023u;
    int* const lists = (int*)(s_raw + (base - smem_u32(s_raw)) + S::stages * S::stage);
    Experts ex{lists, lists + a.E, lists + 2 * a.E, lists + 3 * a.E, 0};
    const unsigned bars = smem_u32(s_bar);
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto empty = [&](int s) { return bars + 8 * (S::stages + s); };
    const auto done = [&](int b) { return bars + 8 * (2 * S::stages + b); };            // a tile is summed
    const auto free_ = [&](int b) { return bars + 8 * (2 * S::stages + 2 + b); };       // its columns may be used again
    const unsigned drained = bars + 8 * (2 * S::stages + 4);
    if (tid == 0) {
        for (int s = 0; s < S::stages; s++) {
            mbar_init(full(s), 3);                // the operands' loader and two warps of scales
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(done(b), 1);
            mbar_init(free_(b), 4);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_stop = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    grid_wait();
    if (warp == 0) {                              // experts with rows; offsets are held inside the buffer whatever they are
        int n = 0, tiles = 0;
        bool bad = false;
        for (int e0 = 0; e0 < a.E; e0 += 32) {
            const int e = e0 + lane;
            int first = 0, rows = 0;
            if (e < a.E) {
                const int lo = a.off[e], hi = a.off[e + 1];
                bad |= lo < 0 || hi < lo || hi > a.R;
                first = min(max(lo, 0), a.R);
                rows = max(min(max(hi, 0), a.R) - first, 0);
            }
            int sum = (rows + kPrM - 1) / kPrM;
            const int own = sum;
            for (int o = 1; o < 32; o *= 2) {
                const int other = __shfl_up_sync(kAll, sum, o);
                if (lane >= o) sum += other;
            }
            const unsigned who = __ballot_sync(kAll, rows > 0);
            if (rows > 0) {
                const int at = n + __popc(who & ((1u << lane) - 1));
                ex.id[at] = e;
                ex.first[at] = first;
                ex.rows[at] = rows;
                ex.tiles[at] = tiles + sum - own;
            }
            n += __popc(who);
            tiles += __shfl_sync(kAll, sum, 31);
        }
        if (lane == 0) {
            ex.tiles[n] = tiles;
            s_n = n;
        }
        if (bad && blockIdx.x == 0) atomicOr(a.status, VP_ST_PACK_MISMATCH);
    }
    fence_before();
    __syncthreads();
    fence_after();
    ex.n = s_n;
    const unsigned tmem = s_tmem;
    const int n_tiles = (a.F + NT - 1) / NT, k_tiles = (a.K + kPrK - 1) / kPrK;
    const long long tiles = (long long)ex.tiles[ex.n] * n_tiles;
    // Every wait is bounded: the one that gives up sets the flag, which ends the others'.
    const auto wait = [&](unsigned bar, unsigned parity) {
        for (unsigned i = 0; i < kPrPolls; i++) {
            if (mbar_try_wait(bar, parity)) return true;
            if (s_stop) return false;
        }
        s_stop = 1;
        atomicOr(a.status, VP_ST_INTERNAL_TIMEOUT);
        return false;
    };
    int s = 0;
    unsigned phase = 0;
    const auto next_stage = [&] { if (++s == S::stages) { s = 0; phase ^= 1; } };
    const auto a_at = [&](int st) { return base + st * S::stage; };

    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
                const Tile tile = tile_of(ex, t, n_tiles, NT);
                const int boxes = (tile.rows + kPrBox - 1) / kPrBox;
                for (int k = 0; k < k_tiles; k++) {
                    if (!(ok = wait(empty(s), phase ^ 1))) break;
                    const unsigned at = a_at(s);
                    mbar_expect_tx(full(s), boxes * kPrBox * (kPrK / 2) + S::b_bytes);
                    for (int b = 0; b < boxes; b++)
                        tma_2d(at + b * kPrBox * (kPrK / 2), &x_map, k * (kPrK / 2), tile.first + b * kPrBox, full(s));
                    tma_3d(at + S::a_bytes, &w_map, k * (kPrK / 2), tile.n0, tile.e, full(s));
                    next_stage();
                }
            }
            if (!ok)                              // copies that are still on their way (bounded as well)
                for (int i = 0; i < S::stages; i++) mbar_wait_bounded(full(i), i < s ? phase : phase ^ 1, 1u << 16);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr unsigned idesc = 1u << 7 | 1u << 10 | (unsigned)(NT >> 3) << 17 | 1u << 23 | (unsigned)(kPrM >> 7) << 27;
            bool ok = true;
            int j = 0;
            for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x, j++) {
                if (j >= S::lag && !(ok = wait(free_((j - S::lag) & 1), ((j - S::lag) >> 1) & 1))) break;
                fence_after();
                const unsigned d = tmem + (j & 1 ? S::second_at : 0);
                for (int k = 0; k < k_tiles; k++) {
                    if (!(ok = wait(full(s), phase))) break;
                    fence_after();
                    const unsigned at = a_at(s), sa = at + S::a_bytes + S::b_bytes, sb = sa + S::sa_bytes;
                    const unsigned ta = tmem + S::scales_at + s * S::scale_cols, tb = ta + 8;
#pragma unroll
                    for (int c = 0; c < 2; c++) copy_scales(ta + 4 * c, scale_desc(sa + 512 * c));
#pragma unroll
                    for (int c = 0; c < NT / 64; c++) copy_scales(tb + 4 * c, scale_desc(sb + 512 * c));
#pragma unroll
                    for (int u = 0; u < 4; u++) {       // 64 values of k each; two of a word's four scales
                        const unsigned half = (u & 1) * 2;
                        mma_mxf4(d, operand_desc(at + 32 * u), operand_desc(at + S::a_bytes + 32 * u), idesc | half << 29 | half << 4,
                                 ta + 4 * (u / 2), tb + NT / 32 * (u / 2), k > 0 || u > 0);
                    }
                    mma_commit(empty(s));
                    next_stage();
                }
                if (ok) mma_commit(done(j & 1));
            }
            if (!ok) {                            // products that are still running
                mma_commit(drained);
                mbar_wait_bounded(drained, 0, 1u << 16);
            }
        }
    } else if (warp < 4) {
        // Scales: row lane + 32 j of the tile is word j of lane's 16 bytes; per 128 values of k and 128 rows 512 bytes.
        const bool is_b = warp == 3;
        constexpr int kMost = NT / 32 > 4 ? NT / 32 : 4;
        const int count = is_b ? NT / 32 : 4, bytes = a.K / 32;
        const auto load = [&](const Tile& tile, int chunk, uint4 (&v)[kMost][2]) {
#pragma unroll
            for (int j = 0; j < kMost; j++) {
                if (j >= count) break;
                const int r = lane + 32 * j;
                const bool there = is_b ? tile.n0 + r < a.F : r < tile.rows;
                const uint8_t* const row = is_b ? a.ws + ((long long)tile.e * a.F + tile.n0 + r) * bytes
                                                : a.xs + (long long)(tile.first + r) * a.xs_ld;
                v[j][0] = load_scales(row, chunk * 32, bytes, there);
                v[j][1] = load_scales(row, chunk * 32 + 16, bytes, there);
            }
        };
        const int chunks = (k_tiles + 3) / 4;     // of four stages: 32 scales of a row, the next ones on their way
        uint4 next[kMost][2], now[kMost][2];
        long long t = blockIdx.x;
        Tile tile{};
        if (t < tiles) {
            tile = tile_of(ex, t, n_tiles, NT);
            load(tile, 0, next);
        }
        bool ok = true;
        for (int chunk = 0; ok && t < tiles;) {
#pragma unroll
            for (int j = 0; j < kMost; j++) { now[j][0] = next[j][0]; now[j][1] = next[j][1]; }
            const int k0 = chunk * 4;
            if (++chunk == chunks) {
                chunk = 0;
                t += gridDim.x;
                if (t < tiles) tile = tile_of(ex, t, n_tiles, NT);
            }
            if (t < tiles) load(tile, chunk, next);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (k0 + k >= k_tiles) break;
                if (!(ok = __all_sync(kAll, wait(empty(s), phase ^ 1)))) break;
                const unsigned at = a_at(s) + S::a_bytes + S::b_bytes + (is_b ? S::sa_bytes : 0) + lane * 16;
                const int blocks = count / 4;
#pragma unroll
                for (int c = 0; c < kMost / 4; c++) {
                    if (c >= blocks) break;
#pragma unroll
                    for (int w = 0; w < 2; w++) {       // words 2 k + w of the rows' 32 bytes
                        const int i = 2 * k + w;
                        const auto word = [&](int j) {
                            const uint4& q = now[4 * c + j][i / 4];
                            return i % 4 == 0 ? q.x : (i % 4 == 1 ? q.y : (i % 4 == 2 ? q.z : q.w));
                        };
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 512 * (w * blocks + c)), "r"(word(0)), "r"(word(1)),
                                     "r"(word(2)), "r"(word(3)) : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(full(s));
                next_stage();
            }
        }
    } else {
        const int quarter = warp - 4;             // lanes 32 * quarter .. of tensor memory: rows of the tile
        bool ok = true;
        int j = 0;
        for (long long t = blockIdx.x; ok && t < tiles; t += gridDim.x, j++) {
            const Tile tile = tile_of(ex, t, n_tiles, NT);
            const int r = quarter * 32 + lane;
            T* const row = (T*)a.out + (long long)(tile.first + r) * a.out_ld + tile.n0;
            const bool there = r < tile.rows;
            if (!(ok = __all_sync(kAll, wait(done(j & 1), (j >> 1) & 1)))) break;
            fence_after();
            const unsigned from = tmem + ((unsigned)(quarter * 32) << 16) + (j & 1 ? S::second_at : 0);
            const auto store = [&](const unsigned (&v)[32], int c) {
                if (!there) return;
                constexpr int V = 16 / (int)sizeof(T);
                if (a.out_wide && tile.n0 + c * 32 + 32 <= a.F) {
#pragma unroll
                    for (int i = 0; i < 32; i += V) {
                        Pack<T, V> p;
#pragma unroll
                        for (int u = 0; u < V; u++) p.v[u] = rounded<T>(__uint_as_float(v[i + u]));
                        *(Pack<T, V>*)(row + c * 32 + i) = p;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i++)
                        if (tile.n0 + c * 32 + i < a.F) row[c * 32 + i] = rounded<T>(__uint_as_float(v[i]));
                }
            };
            // the columns that the next tile waits for first
            const int c0 = S::shared_cols && (j & 1) == 0 ? S::second_at / 32 : 0;
            unsigned v[S::first_chunks][32];
#pragma unroll
            for (int c = 0; c < S::first_chunks; c++) load_columns(from + 32 * (c0 + c), v[c]);
            wait_loads();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(free_(j & 1));
#pragma unroll
            for (int c = 0; c < S::first_chunks; c++) store(v[c], c0 + c);
#pragma unroll 1
            for (int c = S::first_chunks; c < NT / 32; c++) {
                const int at = (c0 + c) % (NT / 32);
                load_columns(from + 32 * at, v[0]);
                wait_loads();
                store(v[0], at);
            }
        }
        fence_before();
    }
    __syncwarp();
    __syncthreads();
    if (warp == 1) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static EncodeTiled s_fn = nullptr;
    EncodeTiled fn = __atomic_load_n(&s_fn, __ATOMIC_ACQUIRE);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        fn = (EncodeTiled)p;
        __atomic_store_n(&s_fn, fn, __ATOMIC_RELEASE);
    }
    return fn;
}

// Bytes of codes, 128 of a row and `box_rows` rows at a time, 128-byte swizzle; zeros behind the ends.
bool make_map(CUtensorMap* map, int rank, const void* p, const cuuint64_t* dims, const cuuint64_t* strides, unsigned box_rows) {
    const EncodeTiled fn = encode_tiled();
    const cuuint32_t box[3] = {kPrK / 2, box_rows, 1}, one[3] = {1, 1, 1};
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, (void*)p, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT>
size_t product_smem(int E) { return (size_t)Shape<NT>::stages * Shape<NT>::stage + 1024 + (size_t)(4 * E + 1) * 4; }

}  // namespace

extern "C" int vp_mxfp4_product(const uint8_t* x_codes, int64_t x_codes_ld, const uint8_t* x_scales, int64_t x_scales_ld,
                                int64_t capacity_rows, const uint8_t* w_codes, const uint8_t* w_scales, int E, int64_t F, int64_t K,
                                const int32_t* expert_off, void* out, int dtype, int64_t out_ld, int32_t* status, void* cuda_stream) {
    if (!is_type(dtype) || capacity_rows < 0 || E <= 0 || F <= 0 || K <= 0 || K % VP_MXFP4_BLOCK || out_ld < F || x_codes_ld < K / 2 ||
        x_scales_ld < K / VP_MXFP4_BLOCK || x_codes_ld % 16)
        return VP_E_BAD_ARG;
    if (E > kPrMaxExperts || K > kPrMaxK || F > kPrMaxF || capacity_rows >= ((int64_t)1 << 31) - 256)
        return VP_E_UNSUPPORTED;
    if (capacity_rows == 0) return VP_OK;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !expert_off || !out || !status) return VP_E_BAD_ARG;
    const int size = size_of_type(dtype);
    if ((uintptr_t)x_codes % 16 || (uintptr_t)w_codes % 16 || (uintptr_t)out % size || (uintptr_t)expert_off % 4 || (uintptr_t)status % 4)
        return VP_E_BAD_ARG;
    const int sms = sm_count_of_device();
    if (!sms) return VP_E_CUDA;
    const ProductArgs a{x_scales, w_scales, x_scales_ld, expert_off, E, (int)capacity_rows, (int)F, (int)K, out, out_ld,
                        (uintptr_t)out % 16 == 0 && out_ld * size % 16 == 0, status};
    // Row tiles there can be at most: a part of one per expert more than the rows fill.
    const long long most = (capacity_rows + kPrM - 1) / kPrM + (E < capacity_rows ? E : capacity_rows);
    const bool large = most * ((F + 255) / 256) >= 2 * sms;
    const long long tiles = most * ((F + (large ? 255 : 127)) / (large ? 256 : 128));
    const int grid = (int)(tiles < sms ? tiles : sms);
    CUtensorMap x_map, w_map;
    const cuuint64_t x_dims[2] = {(cuuint64_t)(K / 2), (cuuint64_t)capacity_rows}, x_strides[1] = {(cuuint64_t)x_codes_ld};
    const cuuint64_t w_dims[3] = {(cuuint64_t)(K / 2), (cuuint64_t)F, (cuuint64_t)E};
    const cuuint64_t w_strides[2] = {(cuuint64_t)(K / 2), (cuuint64_t)(K / 2) * (cuuint64_t)F};
    if (!make_map(&x_map, 2, x_codes, x_dims, x_strides, kPrBox) || !make_map(&w_map, 3, w_codes, w_dims, w_strides, large ? 256 : 128))
        return VP_E_CUDA;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        const auto go = [&](auto fn, size_t smem) {
            e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 1024);
            if (e == cudaSuccess) e = launch_after(fn, grid, kPrThreads, smem, (cudaStream_t)cuda_stream, x_map, w_map, a);
        };
        if (large) go(mxfp4_product_kernel<256, X>, product_smem<256>(E));
        else go(mxfp4_product_kernel<128, X>, product_smem<128>(E));
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
