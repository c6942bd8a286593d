// The experts' products in 4-bit microscaled floating point: expert-major rows (what vp_unpack writes, quantised) times the
// transposed matrix of their expert,
//
//   out[r][f] = sum_k value(x[r][k]) * value(w[e][f][k]),   expert_off[e] <= r < expert_off[e + 1],
//
// on the block-scaled tensor-core path (tcgen05.mma, E2M1 operands, an E8M0 scale per 32 values): products are exact, sums are
// in 32 bits in tensor memory, rounded once to the output's type.
//
// Persistent CTAs take output tiles in turn: one CTA 128 rows x 128 features, or, where there are tiles enough, a pair of CTAs 256 x 256,
// each holding its own 128 rows and half of the features (cta_group::2), which halves what the features' operand costs in L2
// traffic.  Per 256 values of k a stage of shared memory holds both operands (TMA, 128-byte swizzle) and their scales; warp 0 loads
// operands, warps 2, 3 and 8 load scales and lay them out as the tensor core reads them, warp 1 (of the first CTA of a pair) issues the
// copies of scales into tensor memory and the products, warps 4 to 7 bring finished tiles from tensor memory to the output while the next
// tile is summed.
//
// What bounds it: with few rows per expert HBM, by which the matrices come (16 experts x 4,096 x 7,168, 128 rows: 48 us back to back, 5.2 TB/s, 53 with
// other inputs from call to call; without the loads of scales 43, so a seventh is their latency); with many the operands' way from L2 to the SMs, 11 TB/s here (16,384 rows, 8 experts, 7,168 x 4,096: 175 us,
// 5.5 PFLOP/s, 181 under the power cap; the loads alone 176, the products alone 122); a single row is a chain of a third of a microsecond per
// 256 values of k (7,168 x 4,096: 11 us).  Tried: scales through asynchronous copies to shared memory, or two to four chunks ahead in registers (1.1 to 1.5 times the
// time), scales in tensor memory a stage ahead with barriers of their own (1.4 times), one CTA on 128 x 256 (274 us).
#include <cuda.h>
#include <type_traits>

#include "bulk_copy.cuh"
#include "elements.cuh"
#include "odd_words.h"
#include "ring_drain.h"

namespace {

constexpr int kPrMaxExperts = 1024;
constexpr int kPrMaxK = 1 << 20, kPrMaxF = 1 << 20;      // (a matrix is below 2^40 bytes, a tile's sum below a millisecond)
constexpr int kPrM = 128;                         // rows of a tile: lanes of tensor memory
constexpr int kPrK = 256;                         // values of k per stage: one swizzle atom of 128 bytes
constexpr int kPrBox = 32;                        // the least rows of a stage
constexpr int kPrThreads = 320;
constexpr int kPrLine = 64;                       // bytes of an output row that leave together
constexpr unsigned kPrPolls = 1u << 22, kPrDrainPolls = 1u << 16;

// CG: CTAs that share a tile.
template <int CG>
struct Shape {
    static constexpr int NT = 128 * CG;           // features of a tile
    static constexpr int a_bytes = kPrM * (kPrK / 2), b_bytes = 128 * (kPrK / 2);           // operands of a stage, per CTA (of rows at most)
    static constexpr int sa_bytes = kPrM * (kPrK / 32), s_bytes = sa_bytes + NT * (kPrK / 32);        // scales (every CTA holds all features')
    static constexpr int stages = CG == 1 ? 6 : 5, most_stages = CG == 1 ? 16 : 5;
    static constexpr int out_begin = stages * (a_bytes + b_bytes + s_bytes);
    static constexpr int out_bytes = 4 * 32 * kPrLine, lists_begin = out_begin + out_bytes; // a line of every row of the four warps
    // Tensor memory, 512 columns.  Scales have a place per stage, so a stage's are copied over those of products that are done.  Two tiles
    // of 256 columns and the scales do not fit side by side: the second tile then shares columns with the first, and a tile is begun
    // as soon as the shared columns of the one before it have been read.
    static constexpr int scale_cols = 8 + NT / 32 * 2;
    static constexpr int scales_at = 512 - most_stages * scale_cols;
    static constexpr int second_at = 128;
    static constexpr bool shared_cols = second_at < NT;
    static constexpr int lag = shared_cols ? 1 : 2;
    static constexpr int first_chunks = shared_cols ? (NT - second_at) / 32 : NT / 32;      // of 32 columns: read before the next tile
    static_assert(scales_at >= second_at + NT && first_chunks == 4, "columns of tensor memory");
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
    unsigned polls;                               // of a wait, at most
};

// An address of this CTA's shared memory in the CTA of that rank of the cluster.
__device__ __forceinline__ unsigned in_cta(unsigned at, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
// Arrivals at the other CTA's barriers carry order only, no data: what a stage holds is read by the SM that holds it, after a proxy fence in
// that SM, and tensor memory is ordered by the tcgen05 fences.  With release and acquire of the cluster's scope, in every arrival and poll,
// the product of 16,384 rows, 7,168 x 4,096, took 439 us instead of 252.
__device__ __forceinline__ void cluster_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_expect_tx(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}
// Stores to an address of the cluster's shared memory.
__device__ __forceinline__ void cluster_store(unsigned at, unsigned x) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(x) : "memory"); }
__device__ __forceinline__ void cluster_store(unsigned at, unsigned long long x) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(x) : "memory"); }
// Boxes of a tensor map into this CTA's shared memory (no multicast); the barrier may be the pair's first CTA's.
template <int CG>
__device__ __forceinline__ void tma_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory operand descriptors: 128-byte swizzle, rows of 128 bytes in groups of eight; and plain rows of 16 bytes for scales.
constexpr uint64_t kOperandDesc = (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
constexpr uint64_t kScaleDesc = (uint64_t)(128 >> 4) << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
__device__ __forceinline__ uint64_t desc_of(uint64_t kind, unsigned at16) { return kind | at16; }     // at16: the address over 16
__device__ __forceinline__ bool elect_one() {
    unsigned r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r != 0;
}
// Per CTA of the pair: its own shared memory to its own tensor memory.
template <int CG>
__device__ __forceinline__ void copy_scales(unsigned tmem, uint64_t desc) {
    if constexpr (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_mxf4(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned sa, unsigned sb, bool add) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add) : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned)add) : "memory");
}
// One arrival at the barrier (of both CTAs of a pair) when everything issued so far is done.
template <int CG>
__device__ __forceinline__ void mma_commit(unsigned bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
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

// The experts that have rows, in order: id, first row, and the row tiles in front of them.  No row has two experts, whatever the offsets
// are, so there are at most a tile per expert more than the rows fill, and their numbers stay within 32 bits.
struct Experts {
    int* tiles;                                   // one entry more
    int* first;
    uint16_t* id;
    int n;
};

// An offset, held inside the buffer whatever it is.
__device__ __forceinline__ int offset_of(const ProductArgs& a, int e) { return min(max(a.off[e], 0), a.R); }

struct Tile {
    int e, first, rows, n0;                       // expert, first row, rows (at most mt), first feature
};

__device__ __forceinline__ Tile tile_of(const ProductArgs& a, const Experts& x, long long tile, int n_tiles, int mt, int nt) {
    // tiles of an expert: its row tiles next to one another, feature tile by feature tile
    int lo = 0, hi = x.n - 1;
    while (lo < hi) {                             // the last expert whose first tile is not behind `tile`
        const int mid = (lo + hi + 1) / 2;
        if ((long long)x.tiles[mid] * n_tiles <= tile) lo = mid; else hi = mid - 1;
    }
    const int e = x.id[lo], m_tiles = x.tiles[lo + 1] - x.tiles[lo];
    const int q = (int)(tile - (long long)x.tiles[lo] * n_tiles), m = q % m_tiles, first = x.first[lo] + m * mt;
    return Tile{e, first, min(mt, offset_of(a, e + 1) - first), q / m_tiles * nt};
}

// 32 scales of a row.
struct Scales { unsigned w[8]; };
// n[j] scales from p[j], any alignment, and 1 behind them.  All loads before the first use; out of line: inside the loop of every loader it
// cost instruction cache.
__device__ __noinline__ void load_odd_scales(const uint8_t* const (&p)[4], const int (&n)[4], Scales (&v)[4]) {
    unsigned w[4][9];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int off = (int)((uintptr_t)p[j] & 3);
#pragma unroll
        for (int i = 0; i < 9; i++) w[j][i] = odd_word_holds(i, off, n[j]) ? *(const unsigned*)(p[j] - off + 4 * i) : 0;
    }
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int i = 0; i < 8; i++) v[j].w[i] = odd_word(w[j][i], w[j][i + 1], i, (int)((uintptr_t)p[j] & 3), n[j], 0x7f7f7f7fu);
}
// 32 scales of four rows from byte k of rows of `bytes`; 1 behind their ends and in rows that are not there.
__device__ __forceinline__ void load_scales(const uint8_t* const (&row)[4], const bool (&there)[4], int k, int bytes, int aligned, Scales (&v)[4]) {
    if (k + 32 <= bytes && aligned >= 16) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint8_t* const p = row[j] + k;
            if (there[j] && aligned == 32) {      // a sector at once: every part of it is a request to L2 of its own
                asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(v[j].w[0]), "=r"(v[j].w[1]), "=r"(v[j].w[2]), "=r"(v[j].w[3]), "=r"(v[j].w[4]), "=r"(v[j].w[5]),
                               "=r"(v[j].w[6]), "=r"(v[j].w[7]) : "l"(p));
            } else if (there[j]) {
                const uint4 a = *(const uint4*)p, b = *(const uint4*)(p + 16);
                v[j] = Scales{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[j].w[i] = 0x7f7f7f7f;
            }
        }
        return;
    }
    const uint8_t* p[4];
    int n[4];
    Scales odd[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        p[j] = row[j] + k;
        n[j] = there[j] ? min(bytes - k, 32) : 0;
    }
    load_odd_scales(p, n, odd);
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = odd[j];
}

// A wait has run out: its CTA's flag, and the other's of a pair.  Out of line, as what stands in none of the loops.
template <int CG>
__device__ __noinline__ void give_up(unsigned stop, int32_t* status) {
    for (int i = 0; i < CG; i++) cluster_store(in_cta(stop, i), 1u);
    atomicOr(status, VP_ST_INTERNAL_TIMEOUT);
}
// The end of a call that was given up.  Copies that are still on their way are counted on the first CTA's barriers, whichever CTA asked for
// them; products that are still running are waited for by the lane that issued them.
template <int CG>
__device__ __noinline__ void finish_stopped(const unsigned long long* made, int stages, unsigned full, unsigned drained, int rank, bool issues) {
    if (threadIdx.x == 0 && rank == 0)
        drain_ring(made, 2 * CG, CG, stages, [&](int i) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full + 8 * i) : "memory"); },
                   [&](int i, unsigned parity) { mbar_wait_bounded(full + 8 * i, parity, kPrDrainPolls); });
    if (issues) {
        if (rank == 0) mma_commit<CG>(drained);
        mbar_wait_bounded(drained, 0, kPrDrainPolls);
    }
}

template <int CG, typename T>
__global__ void __launch_bounds__(kPrThreads, 1)
mxfp4_product_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap x_64_map,
                     const __grid_constant__ CUtensorMap x_32_map, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ ProductArgs a) {
    using S = Shape<CG>;
    constexpr int NT = S::NT, MT = kPrM * CG;
    extern __shared__ unsigned char s_raw[];
    __shared__ uint64_t s_bar[3 * S::most_stages + 5];
    __shared__ unsigned s_tmem;
    __shared__ int s_n, s_most;
    __shared__ volatile int s_stop;
    __shared__ unsigned long long s_made[2 * CG]; // of the first CTA: stages that each CTA's operands were asked for, whose scales it passed on
    static_assert(3 * S::most_stages + 5 <= 64, "a thread per barrier");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = CG == 1 ? 0 : (int)(blockIdx.x % CG);          // of the pair
    const unsigned base = (smem_u32(s_raw) + 1023) & ~1023u;
    int* const lists = (int*)(s_raw + (base - smem_u32(s_raw)) + S::lists_begin);
    Experts ex{lists, lists + a.E + 1, (uint16_t*)(lists + 2 * a.E + 1), 0};
    const unsigned bars = smem_u32(s_bar);
    const auto first_cta = [&](unsigned bar) { return CG == 1 ? bar : in_cta(bar, 0); };
    const auto full = [&](int s) { return bars + 8 * s; };                                  // of the first CTA: what a stage needs is there
    const auto empty = [&](int s) { return bars + 8 * (S::most_stages + s); };              // of each: a stage has been read
    const auto written = [&](int s) { return bars + 8 * (2 * S::most_stages + s); };        // of each: a stage's scales are written
    const unsigned bars3 = bars + 24 * S::most_stages;
    const auto done = [&](int b) { return bars3 + 8 * b; };                                 // of each: a tile is summed
    const auto free_ = [&](int b) { return bars3 + 8 * (2 + b); };                          // of the first: its columns may be used again
    const unsigned drained = bars3 + 32;
    if (tid < 3 * S::most_stages + 5) {           // a barrier each
        const int i = tid / S::most_stages, last = tid - 3 * S::most_stages;
        // (full: per CTA the operands' loader, and warp 9 for the scales)
        const int arrivals = last >= 0 ? (last == 2 || last == 3 ? 4 * CG : 1) : (i == 0 ? 2 * CG : (i == 1 ? 1 : 1 + CG));
        mbar_init(bars + 8 * tid, arrivals);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (tid >= 64 && tid < 68) {
        const CUtensorMap* const maps[4] = {&x_map, &x_64_map, &x_32_map, &w_map};
        asm volatile("prefetch.tensormap [%0];" ::"l"(maps[tid - 64]) : "memory");
    } else if (tid == 96) {
        s_stop = 0;
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
    }
    grid_wait();
    if (warp == 0) {                              // experts with rows
        int n = 0, tiles = 0, most = 0, end = 0;                   // end: the largest offset so far
        bool bad = false;
        for (int e0 = 0; e0 < a.E; e0 += 32) {
            const int e = e0 + lane;
            int first = 0, next = 0;
            if (e < a.E) {
                first = offset_of(a, e);
                next = offset_of(a, e + 1);
                bad |= a.off[e] != first || a.off[e + 1] != next || next < first;
            }
            bad = __any_sync(kAll, bad);
            if (bad) {                            // a row belongs to the first expert that reaches it
                first = max(first, end);
                for (int o = 1; o < 32; o *= 2) first = max(first, __shfl_up_sync(kAll, first, o));
            }
            end = max(end, __reduce_max_sync(kAll, max(first, next)));
            const int rows = max(next - first, 0);
            most = max(most, rows);
            int sum = (rows + MT - 1) / MT;
            const int own = sum;
            for (int o = 1; o < 32; o *= 2) {
                const int other = __shfl_up_sync(kAll, sum, o);
                if (lane >= o) sum += other;
            }
            const unsigned who = __ballot_sync(kAll, rows > 0);
            if (rows > 0) {
                const int at = n + __popc(who & ((1u << lane) - 1));
                ex.id[at] = (uint16_t)e;
                ex.first[at] = first;
                ex.tiles[at] = tiles + sum - own;
            }
            n += __popc(who);
            tiles += __shfl_sync(kAll, sum, 31);
        }
        most = __reduce_max_sync(kAll, most);
        if (lane == 0) {
            ex.tiles[n] = tiles;
            s_n = n;
            s_most = most;
        }
        if (bad && lane == 0 && blockIdx.x == 0) atomicOr(a.status, VP_ST_PACK_MISMATCH);
    }
    fence_before();
    __syncthreads();
    if constexpr (CG > 1) cluster_sync();         // (the other CTA's barriers are there)
    fence_after();
    ex.n = s_n;
    const unsigned tmem = s_tmem;
    const int n_tiles = (a.F + NT - 1) / NT, k_tiles = (a.K + kPrK - 1) / kPrK;
    const long long tiles = (long long)ex.tiles[ex.n] * n_tiles, t0 = blockIdx.x / CG, step = gridDim.x / CG;
    // Every wait is bounded: the one that gives up sets the flag, which ends the others', in both CTAs.  (The count is looked at behind a poll: in
    // front of it, one row of 7,168 x 4,096 took 11.6 us instead of 11.0.)
    const auto wait = [&](unsigned bar, unsigned parity) {
        unsigned i = 0;
        do {
            if (mbar_try_wait(bar, parity)) return true;
            if (s_stop) return false;
        } while (++i < a.polls);
        give_up<CG>(smem_u32((const void*)&s_stop), a.status);
        return false;
    };
    const auto made = [&](int i, unsigned long long stages) { cluster_store(first_cta(smem_u32(&s_made[i])), stages); };
    // One CTA: where no expert has more than 32 or 64 rows, a stage holds that many, and there are more stages (the products read 128 rows
    // all the same: what lies behind, any bits being numbers, makes rows that nobody stores).  They come as one box, whosever they are:
    // four boxes of 32 cost as much time as their bytes (16,384 rows, 7,168 x 4,096: 212 us against 175), which is also why tiles do not
    // get narrower where CTAs are idle (one row of one expert 14.7 us with 32 features a tile, 12.7 with 128).
    const int a_rows = CG > 1 || s_most > 2 * kPrBox ? kPrM : (s_most > kPrBox ? 2 * kPrBox : kPrBox), a_bytes = a_rows * (kPrK / 2);
    const int stages = CG == 1 ? min(S::out_begin / (a_bytes + S::b_bytes + S::s_bytes), S::most_stages) : S::stages;
    struct Ring {                                 // a place of a ring of barriers, and the parity of its turn
        int at;
        unsigned phase;
        __device__ __forceinline__ void next(int n) { if (++at == n) { at = 0; phase ^= 1; } }
    };
    Ring s{0, 0};
    const auto stage_at = [&](int st) { return base + st * (a_bytes + S::b_bytes + S::s_bytes); };
    const auto scales_at = [&](int st) { return stage_at(st) + a_bytes + S::b_bytes; };

    bool one = false;                             // the lane of warp 1 that issues
    if (warp == 0) {
        if (lane == 0) {
            bool ok = true;
            unsigned long long asked = 0;
            for (long long t = t0; ok && t < tiles; t += step) {
                const Tile tile = tile_of(a, ex, t, n_tiles, MT, NT);
                const CUtensorMap* const map = a_rows == kPrM ? &x_map : (a_rows == kPrBox ? &x_32_map : &x_64_map);
                const int bytes = a_bytes + S::b_bytes;
                for (int k = 0; k < k_tiles; k++) {
                    if (!(ok = wait(empty(s.at), s.phase ^ 1))) break;
                    const unsigned at = stage_at(s.at), bar = first_cta(full(s.at));
                    if (CG == 1) mbar_expect_tx(bar, bytes);
                    else cluster_expect_tx(bar, bytes);
                    tma_3d<CG>(at + a_bytes, &w_map, k * (kPrK / 2), tile.n0 + rank * 128, tile.e, bar);
                    tma_2d<CG>(at, map, k * (kPrK / 2), tile.first + rank * kPrM, bar);
                    s.next(stages);
                    asked++;
                }
            }
            // The pair's first CTA arrives at this one's barriers until the last stage has been read.
            for (int i = 0; CG > 1 && ok && i < stages; i++) {
                ok = wait(empty(s.at), s.phase ^ 1);
                s.next(stages);
            }
            made(rank, asked);
        }
    } else if (warp == 1) {
        one = elect_one();
        // The whole warp goes along, so that what the instructions take is the same in all lanes and known to be; one lane issues them.
        if (rank == 0) {
            const unsigned tm = __reduce_max_sync(kAll, tmem), rows_bytes = __reduce_max_sync(kAll, (unsigned)a_bytes),
                           b16 = __reduce_max_sync(kAll, base) >> 4, n_stages = __reduce_max_sync(kAll, (unsigned)stages),
                           stage16 = (rows_bytes + S::b_bytes + S::s_bytes) >> 4;
            constexpr unsigned idesc = 1u << 7 | 1u << 10 | (unsigned)(NT >> 3) << 17 | 1u << 23 | (unsigned)(MT >> 7) << 27;
            const int my_tiles = __reduce_max_sync(kAll, t0 < tiles ? (int)((tiles - 1 - t0) / step) + 1 : 0);
            bool ok = true;
            unsigned st = 0, parity = 0;
            for (int j = 0; ok && j < my_tiles; j++) {
                if (j >= S::lag && !(ok = __all_sync(kAll, wait(free_((j - S::lag) & 1), ((j - S::lag) >> 1) & 1)))) break;
                fence_after();
                const unsigned d = tm + (j & 1 ? S::second_at : 0);
                for (int k = 0; k < k_tiles; k++) {
                    if (!(ok = __all_sync(kAll, wait(full(st), parity)))) break;
                    fence_after();
                    const unsigned at16 = b16 + st * stage16, sa16 = at16 + ((rows_bytes + S::b_bytes) >> 4);
                    const unsigned ta = tm + S::scales_at + st * S::scale_cols, tb = ta + 8;
                    if (one) {
#pragma unroll
                        for (int c = 0; c < 2; c++) copy_scales<CG>(ta + 4 * c, desc_of(kScaleDesc, sa16 + 32 * c));
#pragma unroll
                        for (int c = 0; c < NT / 64; c++) copy_scales<CG>(tb + 4 * c, desc_of(kScaleDesc, sa16 + S::sa_bytes / 16 + 32 * c));
#pragma unroll
                        for (int u = 0; u < 4; u++) {         // 64 values of k each; two of a word's four scales
                            const unsigned half = (u & 1) * 2;
                            mma_mxf4<CG>(d, desc_of(kOperandDesc, at16 + 2 * u), desc_of(kOperandDesc, at16 + (rows_bytes >> 4) + 2 * u),
                                         idesc | half << 29 | half << 4, ta + 4 * (u / 2), tb + NT / 32 * (u / 2), k > 0 || u > 0);
                        }
                        mma_commit<CG>(empty(st));
                    }
                    __syncwarp();
                    if (++st == n_stages) { st = 0; parity ^= 1; }
                }
                if (ok && one) mma_commit<CG>(done(j & 1));
                __syncwarp();
            }
        }
    } else if (warp < 4 || (warp == 8 && CG == 2)) {
        // Scales of 128 rows or features: row lane + 32 j is word j of lane's 16 bytes, 512 bytes per 128 values of k.  Stages go by
        // chunks of four (32 scales of a row); the next chunk is on its way while one is handed out.
        const bool is_b = warp != 2;
        const int half = warp == 8 ? 1 : 0, bytes = a.K / 32, chunks = (k_tiles + 3) / 4;
        const unsigned to = (is_b ? S::sa_bytes + 512 * half : 0) + lane * 16, word_step = is_b ? 512 * CG : 512;
        const unsigned long long border = is_b ? (uintptr_t)a.ws | (unsigned long long)bytes : (uintptr_t)a.xs | (unsigned long long)a.xs_ld;
        const int aligned = border % 32 == 0 ? 32 : (border % 16 == 0 ? 16 : 1);
        Tile tile{};
        const auto load = [&](long long t, int chunk, Scales (&v)[4]) {
            if (t >= tiles) return;
            if (chunk == 0) tile = tile_of(a, ex, t, n_tiles, MT, NT);
            const uint8_t* row[4];
            bool there[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int r = lane + 32 * j + (is_b ? 128 * half : kPrM * rank);
                there[j] = is_b ? tile.n0 + r < a.F : r < tile.rows;
                row[j] = is_b ? a.ws + ((long long)tile.e * a.F + tile.n0 + r) * bytes : a.xs + (long long)(tile.first + r) * a.xs_ld;
            }
            load_scales(row, there, chunk * 32, bytes, aligned, v);
        };
        Scales next[4], v[4];
        load(t0, 0, next);
        bool ok = true;
        long long t = t0;
        for (int chunk = 0; ok && t < tiles;) {
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = next[j];
            const int k0 = chunk * 4;
            if (++chunk == chunks) { chunk = 0; t += step; }
            load(t, chunk, next);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (k0 + k >= k_tiles) break;
                if (!(ok = __all_sync(kAll, wait(empty(s.at), s.phase ^ 1)))) break;
                const unsigned at = scales_at(s.at) + to;
#pragma unroll
                for (int w = 0; w < 2; w++)               // words 2 k + w of the rows' 32 bytes
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + word_step * w), "r"(v[0].w[2 * k + w]),
                                 "r"(v[1].w[2 * k + w]), "r"(v[2].w[2 * k + w]), "r"(v[3].w[2 * k + w]) : "memory");
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(written(s.at)) : "memory");
                s.next(stages);
            }
        }
    } else if (warp == 9) {
        // Makes scales that are written visible to the tensor core's copies: by a warp that has no loads on their way, for which the fence would
        // wait in the warps that load.  (What it fences has been seen by its wait; the arrival behind it is what the copies wait for.)
        if (lane == 0) {
            bool ok = true;
            unsigned long long passed = 0;
            for (long long t = t0; ok && t < tiles; t += step)
                for (int k = 0; k < k_tiles; k++) {
                    if (!(ok = wait(written(s.at), s.phase))) break;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    if (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full(s.at)) : "memory");
                    else cluster_arrive(first_cta(full(s.at)));
                    s.next(stages);
                    passed++;
                }
            made(CG + rank, passed);
        }
    } else if (warp < 8) {
        const int quarter = warp - 4;             // lanes 32 * quarter .. of tensor memory: rows of the tile
        constexpr int V = 16 / (int)sizeof(T), cols = kPrLine / (int)sizeof(T), per = 32 / cols;        // columns of a line, lines of 32 columns
        const long long row_bytes = a.out_ld * (long long)sizeof(T);
        const unsigned stage = base + S::out_begin + quarter * 32 * kPrLine;
        bool ok = true;
        int j = 0;
        for (long long t = t0; ok && t < tiles; t += step, j++) {
            const Tile tile = tile_of(a, ex, t, n_tiles, MT, NT);
            const int rows = tile.rows - rank * kPrM - quarter * 32;        // of this warp (or fewer than none)
            T* const out = (T*)a.out + (long long)(tile.first + rank * kPrM + quarter * 32) * a.out_ld;
            if (!(ok = __all_sync(kAll, wait(done(j & 1), (j >> 1) & 1)))) break;
            fence_after();
            const unsigned from = tmem + ((unsigned)(quarter * 32) << 16) + (j & 1 ? S::second_at : 0);
            // A line of each of the warp's rows: 16-byte pieces to shared memory (piece p of row r at p ^ r / 2 % 4: no bank twice), then
            // eight rows at a time to the output.
            const auto store = [&](const unsigned (*v)[32], int line) {
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    Pack<T, V> q;
#pragma unroll
                    for (int u = 0; u < V; u++) q.v[u] = rounded<T>(__uint_as_float(v[0][(line * cols + p * V + u) % 32]));
                    const uint4 w = *(const uint4*)&q;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * kPrLine + ((p ^ (lane >> 1 & 3)) << 4)), "r"(w.x),
                                 "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
                }
                __syncwarp();
                const int c = tile.n0 + line * cols + (lane & 3) * V, r0 = lane >> 2;
                uint4 w[4];
#pragma unroll
                for (int i = 0; i < 4; i++)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                                 : "r"(stage + (8 * i + r0) * kPrLine + (((lane & 3) ^ (r0 >> 1 & 3)) << 4)) : "memory");
                char* to = (char*)(out + c) + r0 * row_bytes;
                if (a.out_wide && c + V <= a.F) {
#pragma unroll
                    for (int i = 0; i < 4; i++, to += 8 * row_bytes)
                        if (8 * i + r0 < rows) *(uint4*)to = w[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++, to += 8 * row_bytes) {
                        const Pack<T, V> q = *(const Pack<T, V>*)&w[i];
#pragma unroll
                        for (int u = 0; u < V; u++)
                            if (8 * i + r0 < rows && c + u < a.F) ((T*)to)[u] = q.v[u];
                    }
                }
                __syncwarp();
            };
            // the columns that the next tile waits for first
            const int c0 = S::shared_cols && (j & 1) == 0 ? S::second_at / 32 : 0;
            unsigned v[4][32];
#pragma unroll
            for (int c = 0; c < 4; c++) load_columns(from + 32 * (c0 + c), v[c]);
            wait_loads();
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(free_(j & 1)) : "memory");
                else cluster_arrive(first_cta(free_(j & 1)));
            }
            if (rows > 0)
#pragma unroll
                for (int c = 0; c < 4 * per; c++)
                    if (tile.n0 + (c0 * per + c) * cols < a.F) store(&v[c / per], c0 * per + c);
            if (CG > 1) {
                const int c1 = c0 ^ 4;
#pragma unroll
                for (int c = 0; c < 4; c++) load_columns(from + 32 * (c1 + c), v[c]);
                wait_loads();
                if (rows > 0)
#pragma unroll
                    for (int c = 0; c < 4 * per; c++)
                        if (tile.n0 + (c1 * per + c) * cols < a.F) store(&v[c / per], c1 * per + c);
            }
        }
        fence_before();
    }
    __syncwarp();
    __syncthreads();
    if constexpr (CG > 1) cluster_sync();         // (nobody leaves while its memory is read or its barriers are arrived at)
    if (s_stop) {                                 // (in both CTAs or in none, and nobody begins anything any more)
        finish_stopped<CG>(s_made, stages, full(0), drained, rank, one);
        __syncthreads();
        if constexpr (CG > 1) cluster_sync();
    }
    if (warp == 1) {
        fence_after();
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
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

template <int CG>
size_t product_smem(int E) { return (size_t)Shape<CG>::lists_begin + 1024 + (size_t)E * 10 + 4; }

template <int CG, typename T>
cudaError_t launch_product(const CUtensorMap (&x_maps)[3], const CUtensorMap& w_map, const ProductArgs& a, int grid,
                           cudaStream_t stream) {
    const auto fn = mxfp4_product_kernel<CG, T>;
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)product_smem<CG>(kPrMaxExperts));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kPrThreads);
    cfg.dynamicSmemBytes = product_smem<CG>(a.E);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CG > 1 ? 2 : 1;
    g_vp_launches++;
    return cudaLaunchKernelEx(&cfg, fn, x_maps[0], x_maps[1], x_maps[2], w_map, a);
}

}  // namespace

extern "C" int vp_mxfp4_product(const uint8_t* x_codes, int64_t x_codes_ld, const uint8_t* x_scales, int64_t x_scales_ld,
                                int64_t capacity_rows, const uint8_t* w_codes, const uint8_t* w_scales, int E, int64_t F, int64_t K,
                                const int32_t* expert_off, void* out, int dtype, int64_t out_ld, int32_t* status, void* cuda_stream) {
    return vp_mxfp4_product_polls(x_codes, x_codes_ld, x_scales, x_scales_ld, capacity_rows, w_codes, w_scales, E, F, K, expert_off, out, dtype, out_ld,
                                  status, cuda_stream, kPrPolls);
}

extern "C" int vp_mxfp4_product_polls(const uint8_t* x_codes, int64_t x_codes_ld, const uint8_t* x_scales, int64_t x_scales_ld,
                                      int64_t capacity_rows, const uint8_t* w_codes, const uint8_t* w_scales, int E, int64_t F, int64_t K,
                                      const int32_t* expert_off, void* out, int dtype, int64_t out_ld, int32_t* status, void* cuda_stream,
                                      unsigned polls) {
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
                        (uintptr_t)out % 16 == 0 && out_ld * size % 16 == 0, status, polls};
    // Row tiles there can be at most: a part of one per expert more than the rows fill.
    const auto most_tiles = [&](int mt, int nt) { return ((capacity_rows + mt - 1) / mt + (E < capacity_rows ? E : capacity_rows)) * ((F + nt - 1) / nt); };
    // A pair where experts may have rows for 256 and there are tiles for more than a quarter of the GPU.  Pairs | one CTA each, us, 4,096 features of
    // 7,168: 16 x 128 rows 62 | 52 (half of a pair's rows empty), 8 x 128 40 | 33, 8 x 192 41 | 52, 16 x 200 64 | 77, 8 x 386 57 | 75; one expert's 512 rows
    // 21.6 | 17.2, 1,024 19.7 | 24.3, 2,048 34.7 | 46.8, and 2,048 on 1,024 features 19.6 | 16.5, on 2,048 21.9 | 26.6.  The rows themselves are known on the
    // device only: 16 x 8 rows take 48 us in a buffer for 128, where this choice is right, 58 in one for 3,200 (49 with one CTA each) and
    // 68 in one for 16,384 (56).
    const bool pairs = capacity_rows >= (int64_t)192 * E && capacity_rows / 256 * ((F + 255) / 256) * 15 >= 4 * sms;
    const long long tiles = pairs ? 2 * most_tiles(256, 256) : most_tiles(128, 128);
    const int grid = (int)(tiles < sms ? tiles : sms) / (pairs ? 2 : 1) * (pairs ? 2 : 1);
    CUtensorMap x_maps[3], w_map;             // of 128, 64 and 32 rows
    const cuuint64_t x_dims[2] = {(cuuint64_t)(K / 2), (cuuint64_t)capacity_rows}, x_strides[1] = {(cuuint64_t)x_codes_ld};
    const cuuint64_t w_dims[3] = {(cuuint64_t)(K / 2), (cuuint64_t)F, (cuuint64_t)E};
    const cuuint64_t w_strides[2] = {(cuuint64_t)(K / 2), (cuuint64_t)(K / 2) * (cuuint64_t)F};
    if (!make_map(&w_map, 3, w_codes, w_dims, w_strides, 128)) return VP_E_CUDA;
    for (int i = 0; i < 3; i++)
        if (!make_map(&x_maps[i], 2, x_codes, x_dims, x_strides, i == 0 ? kPrM : 2 * kPrBox / i)) return VP_E_CUDA;
    cudaError_t e = cudaErrorInvalidValue;
    with_type(dtype, [&](auto* type) {
        using X = std::remove_pointer_t<decltype(type)>;
        e = pairs ? launch_product<2, X>(x_maps, w_map, a, grid, (cudaStream_t)cuda_stream)
                  : launch_product<1, X>(x_maps, w_map, a, grid, (cudaStream_t)cuda_stream);
    });
    return e == cudaSuccess ? VP_OK : VP_E_CUDA;
}
