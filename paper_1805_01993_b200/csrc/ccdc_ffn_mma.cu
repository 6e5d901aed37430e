// The matrix products of the feed-forward block on tcgen05 tensor cores.
//
// A product is C[m][n] = sum_k A(m, k) B(n, k) in 16-bit operands and binary32 sums.  One persistent block per SM
// walks output tiles; two SMs of a cluster share a 256 x 512 or 256 x 256 tile (cta_group::2: each holds 128 rows of A
// and half of the columns of B, the tensor cores read both) or one SM computes a 128 x 128 tile.  What bounds the
// products is the way into an SM: its TMA path was measured at 35 to 41 bytes a cycle, whatever the tile order, the
// number of stages or of SMs in use, and the full rate of the tensor cores needs 64 bytes a cycle and SM for the
// 256 x 256 tile and 48 for 256 x 512.  Hence the largest tile that tensor memory holds, where there are enough tiles.
// Warps have roles:
//   0      fetches: 128 x 64 blocks of A and B by TMA into a ring of 32 KiB (256 x 512: 48 KiB) stages
//   1      issues tcgen05.mma, one thread, four K = 16 steps a stage, accumulating in tensor memory
//   2..9   epilogue: accumulators from tensor memory, 32 rows a warp, the elementwise work, and the results through
//          a small shared-memory ring and TMA to global memory
// Two accumulators alternate where both fit, so that a tile's epilogue runs under the next tile's products; 256 x 512
// fills tensor memory, and its epilogue (a few thousand cycles to the products' 16 K) is waited for.
//
// Either side may lie along k (a 16 KiB box of 128 rows of 64 k) or across it (two 8 KiB boxes of 64 rows of 64
// indices), both with the 128-byte swizzle: only the descriptor's strides and the instruction's transpose bits differ, so
// the backward pass needs no transposed copies.  Several products (the backward pass has four) share one launch, and a
// product with few tiles and a long k is cut along k.
//
// Binary32 blocks: an operand is three bf16 planes, and a product the six plane products that reach 2^-24.  The tensor
// cores add to an accumulator with truncation, a bias of about 2^-24 of the running sum for every K = 16 step: 10^-5 at
// K = 4096, harmless under the rounding of 16-bit results but not here.  So a stage holds all planes of 64 k (each is
// fetched once for its products), and after every stage the accumulator of hi hi (one of three) is added to registers
// with rounding.  The five small products have an accumulator of their own: 2^-8 of the size, they bear 32 stages of
// truncation, and where an operand is infinite they mean nothing (infinity times a plane of a finite value, which may be
// zero or of the other sign) and are left out: hi hi alone has the result of IEEE arithmetic there.  (All six in one
// accumulator of four took 3 % less time and was off by 6 % more.)  Tile 256 x 128 by a pair: the registers' share of it
// fits.
//
// Measured: 2048 rows, 4096 x 8192, bf16: forward 0.33 ms, 1.26 PFLOP/s; 8192 rows, 4096 x 16384 forward and backward
// 8.0 ms, 1.24 PFLOP/s (256 x 256 tiles alone: 10.1 ms).  Between epilogues a step of 64 k on the large tile takes about
// 1056 cycles, 1024 at the tensor cores' rate; the gate's epilogue costs 16 %, its backward pass's 25 % of their launches.
// 1024 rows, 1024 x 4096 in binary32, forward and backward: 0.58 ms.
//
// All waits are bounded: one that runs out sets g_wait_failed, and its warp issues nothing more and waits for the block's
// end, which comes once the other warps' waits have run out too and copies and products in flight had time to land.
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "ccdc_ffn.h"
#include "ccdc_ffn_mma.h"

namespace {

constexpr int MAX_PRODUCTS = 4;
constexpr int BLOCK_BYTES = 16384, BOX_BYTES = 8192;    // 128 x 64 of an operand; half of it
constexpr int FETCH_BYTES = 12 * BLOCK_BYTES;           // ring of fetched blocks
constexpr int BLOCK_K = 64;
constexpr int EPI_WARPS = 8, THREADS = 64 + 32 * EPI_WARPS;
constexpr int SMALL_STEPS = 32;                         // steps of 64 k between drains of the small plane products
constexpr int RING_SLOT = 2048, RING_SLOTS = 2;         // 32 rows of 64 bytes
constexpr int SMEM_BYTES = FETCH_BYTES + EPI_WARPS * RING_SLOT * RING_SLOTS + 1024 + 256;
#ifndef CCDC_FFN_WAIT_LIMIT
#define CCDC_FFN_WAIT_LIMIT (1 << 20)       // polls of a barrier (each may sleep) before a wait has failed
#endif

__device__ int g_wait_failed;

struct alignas(64) Problem {
    CUtensorMap a[2], b[2], c[2];
    void *cp;                   // STORE without TMA
    long long ldc, split_stride;
    float *h, *u;
    int M, N, tiles_m, tiles_n, splits, first, kblocks, terms;
    int a_across, b_across, c_f32, c_tma, act, groups;
    uint32_t idesc;
};
struct Work {
    Problem p[MAX_PRODUCTS];
    int count, items, f16;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// the same address in the cluster's first block
__device__ __forceinline__ uint32_t in_first(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < CCDC_FFN_WAIT_LIMIT; ++i) {
        uint32_t ok;
        if constexpr (CG == 2)
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                         "selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        else
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
                         "selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    atomicExch(&g_wait_failed, 1);
    return false;
}
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2"
                     " [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
                     " [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, int z, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
// KEEP: 0 the block of A is read for this product alone; 1 it stays in the tensor core for the next one; 2 it is there
template <int CG, int KEEP = 0>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
#define CCDC_MMA(GROUP, COLLECT)                                                                                   \
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::" GROUP ".kind::f16" COLLECT         \
                 " [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory")
    if constexpr (CG == 1)
        CCDC_MMA("1", "");
    else if constexpr (KEEP == 0)
        CCDC_MMA("2", "");
    else if constexpr (KEEP == 1)
        CCDC_MMA("2", ".collector::a::fill");
    else
        CCDC_MMA("2", ".collector::a::lastuse");
#undef CCDC_MMA
}
// arrives at the barrier (of both blocks of a pair) when the products issued so far are done
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this thread's row
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&f)[32]) {
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]);
}
// Waits for this thread's loads.  Their registers go through it: otherwise the compiler could move plain arithmetic on them
// ahead of the wait, which it does not know to write them.
__device__ __forceinline__ void arrived(float (&f)[32]) {
    asm volatile("" : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]),
                   "+f"(f[8]), "+f"(f[9]), "+f"(f[10]), "+f"(f[11]), "+f"(f[12]), "+f"(f[13]), "+f"(f[14]), "+f"(f[15]),
                   "+f"(f[16]), "+f"(f[17]), "+f"(f[18]), "+f"(f[19]), "+f"(f[20]), "+f"(f[21]), "+f"(f[22]), "+f"(f[23]),
                   "+f"(f[24]), "+f"(f[25]), "+f"(f[26]), "+f"(f[27]), "+f"(f[28]), "+f"(f[29]), "+f"(f[30]), "+f"(f[31]));
}
template <class... F>
__device__ __forceinline__ void tmem_wait(F &...f) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    (arrived(f), ...);
}

// Shared-memory descriptor of a 128-byte-swizzled operand.  Along k: rows of 128 bytes, eight to a 1 KiB group
// (stride 1 KiB between groups).  Across k: a row of 128 bytes is 64 indices at one k; eight k to a 1 KiB group, and
// the next 64 indices start one box further.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int across) {
    const uint64_t lead = across ? BOX_BYTES >> 4 : 1;
    return (uint64_t)((addr & 0x3FFFF) >> 4) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

struct Tile {
    int problem, m, n, split, it0, it1;
};
__device__ __forceinline__ Tile tile_of(const Work &w, int item) {
    Tile t;
    t.problem = 0;
    while (t.problem + 1 < w.count && item >= w.p[t.problem + 1].first) ++t.problem;
    const Problem &p = w.p[t.problem];
    int i = item - p.first;
    const int tiles = p.tiles_m * p.tiles_n;
    t.split = i / tiles;
    i -= t.split * tiles;
    // bands of eight tile rows, walked column by column: neighbours in time share A and B tiles in L2
    const int band = i / (8 * p.tiles_n), rows = min(8, p.tiles_m - 8 * band);
    i -= band * 8 * p.tiles_n;
    t.n = i / rows;
    t.m = band * 8 + i - t.n * rows;
    const long long its = (long long)p.kblocks * p.terms;
    t.it0 = (int)(its * t.split / p.splits);
    t.it1 = (int)(its * (t.split + 1) / p.splits);
    return t;
}

// What the epilogue needs of a problem, copied into registers once a tile: left in the kernel's parameters, every field
// is loaded again after every barrier (1 to 3 % of the small and middle sizes).
struct Output {
    const CUtensorMap *c0, *c1;
    void *cp;
    long long ldc, split_stride;
    float *h, *u;
    int M, N, c_f32, c_tma, act, groups;
    __device__ __forceinline__ explicit Output(const Problem &p)
        : c0(&p.c[0]), c1(&p.c[1]), cp(p.cp), ldc(p.ldc), split_stride(p.split_stride), h(p.h), u(p.u), M(p.M), N(p.N),
          c_f32(p.c_f32), c_tma(p.c_tma), act(p.act), groups(p.groups) {}
};

// The epilogue warps' way out: 32 rows of 64 bytes a slot, swizzled so that the row writes meet no bank conflict.  Every use
// of a slot ends with a group of bulk stores (or an empty one): all but the last group read out means this slot is free.
struct Ring {
    char *base;
    int slot;
    __device__ __forceinline__ char *next(int lane) {
        slot ^= 1;
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(RING_SLOTS - 1) : "memory");
        __syncwarp();
        return base + slot * RING_SLOT;
    }
};
__device__ __forceinline__ void out_by_tma(const CUtensorMap *map, int x, int y, int z, const char *slot, int lane) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        tma_store(map, x, y, z, smem_u32(slot));
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
__device__ __forceinline__ char *slot_at(char *slot, int row, int chunk) {      // 16 bytes of a row of 64
    return slot + row * 64 + ((chunk ^ (row >> 1 & 3)) << 4);
}
template <class T>
__device__ __forceinline__ void put16(char *slot, int row, const float (&f)[32]) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint4 *>(slot_at(slot, row, c)) =
            make_uint4(pack2<T>(f[8 * c], f[8 * c + 1]), pack2<T>(f[8 * c + 2], f[8 * c + 3]),
                       pack2<T>(f[8 * c + 4], f[8 * c + 5]), pack2<T>(f[8 * c + 6], f[8 * c + 7]));
}
// 32 columns as 16-bit words, or as the planes of binary32 words
template <bool PLANES>
__device__ __forceinline__ void emit(const CUtensorMap *map, int f16, float (&f)[32], int col, int row0, int lane, Ring &ring) {
    if constexpr (!PLANES) {
        char *slot = ring.next(lane);
        if (f16)
            put16<fp16>(slot, lane, f);
        else
            put16<bf16>(slot, lane, f);
        out_by_tma(map, col, row0, 0, slot, lane);
    } else {
        auto plane = [&](int z, auto next) {
            char *slot = ring.next(lane);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = next(f[8 * c + 2 * i], f[8 * c + 2 * i + 1]);
                *reinterpret_cast<uint4 *>(slot_at(slot, lane, c)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            out_by_tma(map, col, row0, z, slot, lane);
        };
        bool plain = true;
#pragma unroll
        for (int i = 0; i < 32; ++i) plain = plain && fabsf(f[i]) < FIRST_MOST;
        int z = 0;
        if (!__all_sync(~0u, plain)) plane(z++, first_plane_of_any);
#pragma unroll 1
        for (; z < 3; ++z) plane(z, next_plane);
    }
}

// The values of a tile that leave as they are: 32 columns from `col` on.
__device__ __forceinline__ void store_columns(const Output &p, int f16, const float (&f)[32], int col, int row0, int split,
                                              int lane, Ring &ring) {
    const int width = p.c_f32 ? 16 : 32;            // columns of a slot
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half && !p.c_f32) break;
        const int at = col + 16 * half;
        if (at >= p.N) break;
        char *slot = ring.next(lane);
        if (p.c_f32) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(slot_at(slot, lane, i)) = make_float4(
                    f[16 * half + 4 * i], f[16 * half + 4 * i + 1], f[16 * half + 4 * i + 2], f[16 * half + 4 * i + 3]);
        } else if (f16) {
            put16<fp16>(slot, lane, f);
        } else {
            put16<bf16>(slot, lane, f);
        }
        if (p.c_tma) {
            out_by_tma(p.c0, at, row0, split, slot, lane);
            continue;
        }
        // rows that TMA cannot address: a row (binary32: two) at a time, neighbouring threads neighbouring words
        __syncwarp();
        const int c = lane & (width - 1), step = 32 / width;
        const int end = min(32, p.M - row0);
        if (at + c < p.N)
            for (int r = lane / width; r < end; r += step) {
                const long long to = split * p.split_stride + (row0 + r) * p.ldc + at + c;
                if (p.c_f32)
                    static_cast<float *>(p.cp)[to] = *reinterpret_cast<float *>(slot_at(slot, r, c >> 2) + (c & 3) * 4);
                else
                    static_cast<uint16_t *>(p.cp)[to] = *reinterpret_cast<uint16_t *>(slot_at(slot, r, c >> 3) + (c & 7) * 2);
            }
        __syncwarp();
        // an empty group: next() counts groups, and one of an earlier product may still be read from the other slot
        if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// h and u of 32 columns of this thread's row
__device__ __forceinline__ void load_saved(const Output &p, long long block, int col, int lane, float4 (&h)[8], float4 (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = u[i] = make_float4(0, 0, 0, 0);
        if ((col >> 2) + i < p.groups) {
            const long long at = (block + (col >> 2) + i) * 32 + lane;
            h[i] = reinterpret_cast<const float4 *>(p.h)[at];
            u[i] = reinterpret_cast<const float4 *>(p.u)[at];
        }
    }
}
template <bool EXACT>
__device__ __forceinline__ void gate_columns(const Output &p, int f16, float (&h)[32], float (&u)[32], long long block, int col,
                                             int row0, int lane, Ring &ring) {
    if (p.h) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((col >> 2) + i < p.groups) {
                const long long at = (block + (col >> 2) + i) * 32 + lane;
                reinterpret_cast<float4 *>(p.h)[at] = make_float4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                reinterpret_cast<float4 *>(p.u)[at] = make_float4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
            }
    }
    act_apply<EXACT>(p.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float slope;
            u[i] *= act(h[i], &slope);
        }
    });
    emit<EXACT>(p.c0, f16, u, col, row0, lane, ring);
}
// d (da on entry) becomes dh, du the other
template <bool EXACT>
__device__ __forceinline__ void gate_back_columns(const Output &p, float (&d)[32], float (&du)[32], const float4 (&h)[8],
                                                  const float4 (&u)[8]) {
    act_apply<EXACT>(p.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float4 hv = h[i >> 2], uv = u[i >> 2];
            const float x = (i & 3) == 0 ? hv.x : (i & 3) == 1 ? hv.y : (i & 3) == 2 ? hv.z : hv.w;
            const float y = (i & 3) == 0 ? uv.x : (i & 3) == 1 ? uv.y : (i & 3) == 2 ? uv.z : uv.w;
            float slope;
            du[i] = d[i] * act(x, &slope);
            d[i] *= y * slope;
        }
    });
}
// CG SMs to a tile of 128 CG rows and 128 CG NB columns.  PLANES: binary32 blocks, see above; 256 rows, 128 columns.
template <int CG, int NB, int EPI, bool PLANES>
__global__ void __launch_bounds__(THREADS, 1) k_ffn_mma(const __grid_constant__ Work w) {
    extern __shared__ char smem_raw[];
    constexpr int HALF_N = PLANES ? 128 : 128 * CG, TILE_M = 128 * CG, TILE_N = HALF_N * NB;
    constexpr int STAGE_BYTES = PLANES ? 3 * (BLOCK_BYTES + BOX_BYTES) : (1 + NB) * BLOCK_BYTES;
    constexpr int B_AT = PLANES ? 3 * BLOCK_BYTES : BLOCK_BYTES;    // A's blocks come first
    constexpr int STAGES = FETCH_BYTES / STAGE_BYTES;
    constexpr int ACCS = PLANES ? 3 : 512 / TILE_N < 2 ? 1 : 2;     // accumulators in tensor memory
    constexpr int SMALL_AT = ACCS * TILE_N;                         // PLANES: the small products' accumulator
    constexpr uint32_t TMEM_COLUMNS = (ACCS + PLANES) * TILE_N;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    char *ring_base = smem + FETCH_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(ring_base + EPI_WARPS * RING_SLOT * RING_SLOTS);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 8);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_full = empty + 8 * STAGES, acc_empty = acc_full + 32;
    const uint32_t small_empty = acc_empty + 8 * ACCS;

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (int i = 0; i < ACCS; ++i) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, EPI_WARPS * CG);
        if constexpr (PLANES) bar_init(small_empty, EPI_WARPS * CG);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLUMNS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLUMNS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    bool ok = true;             // no wait of this thread has run out
    if (warp == 0) {
        if (lane == 0) {
            const uint32_t ring = smem_u32(smem), first_full = CG == 2 ? in_first(full) : full;
            uint32_t stage = 0, phase = 0;
            for (int item = cluster; ok && item < w.items; item += clusters) {
                const Tile t = tile_of(w, item);
                const Problem &p = w.p[t.problem];
                const int am = t.m * TILE_M + 128 * (int)rank;
                // The tile's B: halves of HALF_N columns, each half's 128 CG rows shared out over the blocks.  GATE: the
                // first half of the columns is h's, the second u's; with one half, its blocks (or boxes) are.
                const bool a_across = p.a_across, b_across = p.b_across;
                for (int it = t.it0; ok && it < t.it1;) {
                    const int term = it / p.kblocks, end = min(t.it1, (term + 1) * p.kblocks);
                    const CUtensorMap *ma = &p.a[term];
                    const CUtensorMap *mb = &p.b[EPI != MMA_GATE ? term : NB == 1 && CG == 2 ? (int)rank : 0];
                    const int bn = EPI != MMA_GATE ? t.n * TILE_N + HALF_N / CG * (int)rank
                                                   : t.n * (TILE_N / 2) + (NB == 2 ? 128 * (int)rank : 0);
                    for (int k = (it - term * p.kblocks) * BLOCK_K; it < end; ++it, k += BLOCK_K) {
                        if (ok = bar_wait<CG>(empty + 8 * stage, phase ^ 1); !ok) break;
                        const uint32_t bar = first_full + 8 * stage, dst = ring + stage * STAGE_BYTES;
                        if (rank == 0) bar_expect(full + 8 * stage, CG * STAGE_BYTES);
#pragma unroll
                        for (int z = 0; z < (PLANES ? 3 : 1); ++z) {
                            const uint32_t to = dst + z * BLOCK_BYTES;
                            if (!a_across) {
                                tma_load<CG>(to, ma, k, am, z, bar);
                            } else {
                                tma_load<CG>(to, ma, am, k, z, bar);
                                tma_load<CG>(to + BOX_BYTES, ma, am + 64, k, z, bar);
                            }
                        }
                        if constexpr (PLANES) {
#pragma unroll
                            for (int z = 0; z < 3; ++z)
                                tma_load<CG>(dst + B_AT + z * BOX_BYTES, mb, b_across ? bn : k, b_across ? k : bn, z, bar);
                        } else if constexpr (EPI == MMA_GATE && CG == 1 && NB == 1) {
                            tma_load<CG>(dst + B_AT, mb, k, bn, 0, bar);
                            tma_load<CG>(dst + B_AT + BOX_BYTES, mb + 1, k, bn, 0, bar);
                        } else {
#pragma unroll
                            for (int j = 0; j < NB; ++j) {
                                const CUtensorMap *m = EPI == MMA_GATE ? mb + j : mb;
                                const int n = EPI == MMA_GATE ? bn : bn + HALF_N * j;
                                const uint32_t to = dst + B_AT + j * BLOCK_BYTES;
                                if (!b_across) {
                                    tma_load<CG>(to, m, k, n, 0, bar);
                                } else {
                                    tma_load<CG>(to, m, n, k, 0, bar);
                                    tma_load<CG>(to + BOX_BYTES, m, n + 64, k, 0, bar);
                                }
                            }
                        }
                        if (++stage == STAGES) stage = 0, phase ^= 1;
                    }
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0, small_phase = 0;
            for (int item = cluster; ok && item < w.items; item += clusters) {
                const Tile t = tile_of(w, item);
                const Problem &p = w.p[t.problem];
                const uint32_t idesc = p.idesc;
                const uint64_t a0 = operand_desc(smem_u32(smem), p.a_across);
                const uint64_t b0 = operand_desc(smem_u32(smem) + B_AT, p.b_across);
                const uint32_t a_step = p.a_across ? 2048 >> 4 : 32 >> 4, b_step = p.b_across ? 2048 >> 4 : 32 >> 4;
                for (int it = t.it0; ok && it < t.it1;) {
                    const int end = PLANES ? it + 1 : t.it1;
                    const uint32_t d = tmem + acc * TILE_N;
                    if (ok = bar_wait<CG>(acc_empty + 8 * acc, acc_phase ^ 1); !ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    bool add = false;
                    for (; it < end; ++it) {
                        if (ok = bar_wait<CG>(full + 8 * stage, phase); !ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = a0 + stage * (STAGE_BYTES >> 4), b = b0 + stage * (STAGE_BYTES >> 4);
                        if constexpr (PLANES) {
                            const bool first = (it - t.it0) % SMALL_STEPS == 0;
                            if (first) {
                                if (ok = bar_wait<CG>(small_empty, small_phase ^ 1); !ok) break;
                                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                                small_phase ^= 1;
                            }
                            // lo hi, hi lo, mid mid, mid hi, hi mid, and apart from them hi hi
                            constexpr int order[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
#pragma unroll
                            for (int i = 0; i < 6; ++i)
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    mma<CG>(i < 5 ? tmem + SMALL_AT : d, a + order[i][0] * (BLOCK_BYTES >> 4) + k * a_step,
                                            b + order[i][1] * (BOX_BYTES >> 4) + k * b_step, idesc,
                                            i < 5 ? !first || i + k > 0 : k > 0);
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                mma<CG, NB == 2 ? 1 : 0>(d, a + k * a_step, b + k * b_step, idesc, add);
                                if constexpr (NB == 2)
                                    mma<CG, 2>(d + HALF_N, a + k * a_step, b + (BLOCK_BYTES >> 4) + k * b_step, idesc, add);
                                add = true;
                            }
                        }
                        mma_commit<CG>(empty + 8 * stage);
                        if (++stage == STAGES) stage = 0, phase ^= 1;
                    }
                    if (!ok) break;
                    mma_commit<CG>(acc_full + 8 * acc);
                    if (++acc == ACCS) acc = 0, acc_phase ^= 1;
                }
            }
        }
    } else {
        const int quarter = warp & 3;               // the tensor-memory lanes a warp may read
        const int part = (warp - 2) >> 2;           // two warps a quarter: each takes half of the columns
        const int f16 = w.f16;
        Ring ring = {ring_base + (warp - 2) * RING_SLOT * RING_SLOTS, 0};
        uint32_t acc = 0, acc_phase = 0;
        auto release = [&](uint32_t bar) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2)
                    bar_arrive_cluster(in_first(bar));
                else
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
            }
        };
        constexpr int COLS = EPI == MMA_GATE ? TILE_N / 2 : TILE_N;     // output columns of a tile
        for (int item = cluster; ok && item < w.items; item += clusters) {
            const Tile t = tile_of(w, item);
            const Output p(w.p[t.problem]);
            const int row0 = t.m * TILE_M + 128 * (int)rank + 32 * quarter;
            const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
            const bool rows = row0 < p.M;
            const int col0 = t.n * COLS + part * (COLS / 2), col1 = min(p.N, col0 + COLS / 2);
            const long long block = (long long)(row0 >> 5) * p.groups;
            if constexpr (!PLANES) {
                const uint32_t from = tmem + acc * TILE_N + part * (COLS / 2) + lanes;
                float4 h[8], u[8];
                if (EPI == MMA_GATE_BACK && rows && col0 < col1) load_saved(p, block, col0, lane, h, u);
                if (ok = __all_sync(~0u, bar_wait<CG>(acc_full + 8 * acc, acc_phase)); !ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int c = 0; rows && col0 + c < col1; c += 32) {
                    float f[32];
                    tmem_load(from + c, f);
                    if constexpr (EPI == MMA_STORE) {
                        tmem_wait(f);
                        store_columns(p, f16, f, col0 + c, row0, t.split, lane, ring);
                    } else if constexpr (EPI == MMA_GATE) {
                        float g[32];
                        tmem_load(from + COLS + c, g);
                        tmem_wait(f, g);
                        gate_columns<false>(p, f16, f, g, block, col0 + c, row0, lane, ring);
                    } else {
                        tmem_wait(f);
                        float g[32];
                        gate_back_columns<false>(p, f, g, h, u);
                        if (col0 + c + 32 < col1) load_saved(p, block, col0 + c + 32, lane, h, u);     // on their way during the stores
                        emit<false>(p.c0, f16, f, col0 + c, row0, lane, ring);
                        emit<false>(p.c1, f16, g, col0 + c, row0, lane, ring);
                    }
                }
                release(acc_empty + 8 * acc);
                if (++acc == ACCS) acc = 0, acc_phase ^= 1;
            } else {
                // this warp's 64 columns: GATE 32 of h and the 32 of u that belong to them
                constexpr int SECOND = EPI == MMA_GATE ? TILE_N / 2 : 32;
                float f[2][32] = {};
                const uint32_t columns = tmem + part * (COLS / 2) + lanes;
                for (int it = t.it0; it < t.it1; ++it) {
                    if (ok = __all_sync(~0u, bar_wait<CG>(acc_full + 8 * acc, acc_phase)); !ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    float v[2][32];
                    tmem_load(columns + acc * TILE_N, v[0]);
                    tmem_load(columns + acc * TILE_N + SECOND, v[1]);
                    tmem_wait(v[0], v[1]);
                    release(acc_empty + 8 * acc);
                    if (++acc == ACCS) acc = 0, acc_phase ^= 1;
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[0][i] += v[0][i], f[1][i] += v[1][i];
                    if ((it - t.it0) % SMALL_STEPS != SMALL_STEPS - 1 && it + 1 < t.it1) continue;
                    tmem_load(columns + SMALL_AT, v[0]);
                    tmem_load(columns + SMALL_AT + SECOND, v[1]);
                    tmem_wait(v[0], v[1]);
                    release(small_empty);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[j][i] = isfinite(f[j][i]) ? f[j][i] + v[j][i] : f[j][i];
                }
                if (ok && rows && col0 < col1) {
                    if constexpr (EPI == MMA_GATE) {
                        gate_columns<true>(p, f16, f[0], f[1], block, col0, row0, lane, ring);
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (col0 + 32 * j >= col1) break;
                            if constexpr (EPI == MMA_STORE) {
                                store_columns(p, f16, f[j], col0 + 32 * j, row0, t.split, lane, ring);
                            } else {
                                float4 h[8], u[8];
                                load_saved(p, block, col0 + 32 * j, lane, h, u);
                                float g[32];
                                gate_back_columns<true>(p, f[j], g, h, u);
                                emit<true>(p.c0, f16, f[j], col0 + 32 * j, row0, lane, ring);
                                emit<true>(p.c1, f16, g, col0 + 32 * j, row0, lane, ring);
                            }
                        }
                    }
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (!ok) {          // let copies that are still in flight land before the block ends
        const long long until = clock64() + 2000000;
        while (clock64() < until) {}
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLUMNS));
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLUMNS));
    }
}

// ------------------------------------------------------------------ host
using encode_fn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                               const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
encode_fn encoder() {
    static encode_fn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<encode_fn>(p);
    }();
    return fn;
}

bool encode(CUtensorMap *map, int type, const void *p, long long cols, long long rows, long long ld, long long planes,
            int box_cols, int box_rows) {
    const int size = type_bytes(type);
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(rows * ld * size)};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    const CUtensorMapDataType t = type == CCDC_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : type == CCDC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                      : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const CUtensorMapSwizzle swizzle = box_cols * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    return encoder()(map, t, 3, const_cast<void *>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, int NB, int EPI, bool PLANES>
int launch(const Work &w, int sms, cudaStream_t s) {
    auto *kernel = k_ffn_mma<CG, NB, EPI, PLANES>;
    static std::atomic<unsigned long long> done;
    const int rc = block_allow_smem(reinterpret_cast<const void *>(kernel), SMEM_BYTES, &done);
    if (rc != CCDC_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(w.items, std::max(1, sms / CG)) * CG));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, w);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}
template <int EPI>
int launch_tile(const Work &w, MmaTile tile, int sms, cudaStream_t s) {
    return tile == MMA_PLANES ? launch<2, 1, EPI, true>(w, sms, s)
           : tile == MMA_WIDE ? launch<2, 2, EPI, false>(w, sms, s)
           : tile == MMA_PAIR ? launch<2, 1, EPI, false>(w, sms, s) : launch<1, 1, EPI, false>(w, sms, s);
}

}  // namespace

int mma_launch(const MmaProduct *products, int count, MmaEpilogue epilogue, int type, MmaTile shape, int sms, cudaStream_t s) {
    if (count < 1) return CCDC_OK;
    if (!encoder()) return CCDC_ECUDA;
    static thread_local Work w;
    w.count = count, w.items = 0, w.f16 = type == CCDC_F16;
    const bool halves = shape == MMA_PLANES || (epilogue == MMA_GATE && shape == MMA_SINGLE);      // boxes of 64 B rows
    const int tile = mma_tile_rows(shape), tile_n = mma_tile_columns(shape) / (epilogue == MMA_GATE ? 2 : 1);
    for (int i = 0; i < count; ++i) {
        const MmaProduct &q = products[i];
        Problem &p = w.p[i];
        p.M = (int)q.M, p.N = (int)q.N;
        p.tiles_m = (int)((q.M + tile - 1) / tile), p.tiles_n = (int)((q.N + tile_n - 1) / tile_n);
        p.splits = epilogue == MMA_STORE ? std::max(1, q.splits) : 1;
        p.kblocks = (int)((q.K + BLOCK_K - 1) / BLOCK_K);
        p.first = w.items;
        w.items += p.tiles_m * p.tiles_n * p.splits;
        p.a_across = q.a[0].transposed, p.b_across = q.b[0].transposed;
        p.act = q.act, p.h = q.h, p.u = q.u, p.groups = (int)ffn_saved_groups(q.N);
        const uint32_t f = type == CCDC_BF16 ? 1 : 0;
        p.idesc = 1u << 4 | f << 7 | f << 10 | (uint32_t)p.a_across << 15 | (uint32_t)p.b_across << 16 |
                  (uint32_t)((shape == MMA_PLANES ? 128 : tile) >> 3) << 17 | (uint32_t)(tile >> 4) << 24;
        p.terms = q.terms;
        const int nb = epilogue == MMA_GATE ? 2 : q.terms;
        bool ok = true;
        auto side = [&](CUtensorMap *map, const MmaSide &d, bool half) {
            ok = ok && encode(map, type, d.m.p, d.m.cols, d.m.rows, d.m.ld, d.m.planes, 64, half ? 64 : 128);
        };
        for (int t = 0; t < q.terms; ++t) side(&p.a[t], q.a[t], q.a[t].transposed);
        for (int t = 0; t < nb; ++t) side(&p.b[t], q.b[t], q.b[t].transposed || halves);
        if (epilogue == MMA_STORE) {
            p.cp = q.c, p.ldc = q.ldc, p.split_stride = q.M * q.ldc, p.c_f32 = q.c_type == CCDC_F32;
            p.c_tma = aligned_to(q.c, 16) && q.ldc * type_bytes(q.c_type) % 16 == 0;
            if (p.c_tma) ok = ok && encode(&p.c[0], q.c_type, q.c, q.N, q.M, q.ldc, p.splits, p.c_f32 ? 16 : 32, 32);
        } else {
            for (int t = 0; t < (epilogue == MMA_GATE ? 1 : 2); ++t)
                ok = ok && encode(&p.c[t], type, q.out[t].p, q.out[t].cols, q.out[t].rows, q.out[t].ld, q.out[t].planes, 32, 32);
        }
        if (!ok) return CCDC_ECUDA;
    }
    return epilogue == MMA_STORE  ? launch_tile<MMA_STORE>(w, shape, sms, s)
           : epilogue == MMA_GATE ? launch_tile<MMA_GATE>(w, shape, sms, s)
                                  : launch_tile<MMA_GATE_BACK>(w, shape, sms, s);
}

int mma_status(int *failed) {
    const cudaError_t e = cudaMemcpyFromSymbol(failed, g_wait_failed, sizeof(int));
    return e != cudaSuccess ? ccdc_internal_cuda_fail((int)e) : CCDC_OK;
}
