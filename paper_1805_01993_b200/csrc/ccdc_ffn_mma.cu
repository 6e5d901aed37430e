// The matrix products of the feed-forward block on tcgen05 tensor cores.
//
// A product is C[m][n] = sum_k A(m, k) B(n, k) in 16-bit operands and binary32 sums.  One persistent block per SM
// walks output tiles; two SMs of a cluster share a 256 x 256 tile (cta_group::2: each holds 128 rows of A and 128
// columns of B, the tensor cores read both) or one SM computes a 128 x 128 tile.  Warps have roles:
//   0      fetches: 128 x 64 blocks of A and B by TMA into a ring of 32 KiB stages (four 8 KiB boxes a stage)
//   1      issues tcgen05.mma, one thread, four K = 16 steps a stage, accumulating in tensor memory
//   2..5   epilogue: accumulators from tensor memory, 32 rows a warp, the elementwise work, and the results through
//          a small shared-memory ring and TMA to global memory
// Two accumulators alternate, so that a tile's epilogue runs under the next tile's products.
//
// Either side may lie along k (rows of 64 k) or across it (rows of 64 indices): both are 8 KiB boxes with the
// 128-byte swizzle, only the descriptor's strides and the instruction's transpose bits differ, so the backward pass
// needs no transposed copies.  Several products (the backward pass has four) share one launch, and a product with
// few tiles and a long k is cut along k.
//
// All waits are bounded: one that runs out sets g_wait_failed and the thread goes on without waiting.
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "ccdc_ffn.h"
#include "ccdc_ffn_mma.h"

namespace {

constexpr int MAX_PRODUCTS = 4, MAX_SEGMENTS = 12;
constexpr int STAGES = 6, STAGE_BYTES = 32768, BOX_BYTES = 8192;
constexpr int BLOCK_K = 64;
constexpr int THREADS = 192, EPI_WARPS = 4;
constexpr int RING_SLOT = 4096, RING_SLOTS = 2;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + EPI_WARPS * RING_SLOT * RING_SLOTS + 1024 + 256;
constexpr int WAIT_LIMIT = 1 << 20;

__device__ int g_wait_failed;

struct Segment {
    uint8_t a, b, za, zb;       // which maps and planes
};
struct alignas(64) Problem {
    CUtensorMap a[2], b[2], c[2];
    Segment seg[MAX_SEGMENTS];
    void *cp;                   // STORE without TMA
    long long ldc, split_stride;
    float *h, *u;
    int M, N, tiles_m, tiles_n, splits, first, kblocks, segments;
    int a_across, b_across, c_f32, c_tma, planes, act, groups;
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
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, int &limit) {
    for (int i = 0; i < limit; ++i) {
        uint32_t ok;
        if constexpr (CG == 2)
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                         "selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        else
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
                         "selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return;
    }
    atomicExch(&g_wait_failed, 1);
    limit = 4;
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
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if constexpr (CG == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
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
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

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
    const long long its = (long long)p.kblocks * p.segments;
    t.it0 = (int)(its * t.split / p.splits);
    t.it1 = (int)(its * (t.split + 1) / p.splits);
    return t;
}

// The epilogue warps' way out: 32 rows x 32 columns a slot, swizzled so that the row writes meet no bank conflict.
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
__device__ __forceinline__ char *slot16(char *slot, int row, int chunk) {       // 64-byte rows
    return slot + row * 64 + ((chunk ^ (row >> 1 & 3)) << 4);
}
__device__ __forceinline__ char *slot32(char *slot, int row, int chunk) {       // 128-byte rows
    return slot + row * 128 + ((chunk ^ (row & 7)) << 4);
}
template <class T>
__device__ __forceinline__ void put16(char *slot, int row, const float (&f)[32]) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint4 *>(slot16(slot, row, c)) =
            make_uint4(pack2<T>(f[8 * c], f[8 * c + 1]), pack2<T>(f[8 * c + 2], f[8 * c + 3]),
                       pack2<T>(f[8 * c + 4], f[8 * c + 5]), pack2<T>(f[8 * c + 6], f[8 * c + 7]));
}
// 32 columns as 16-bit words, or as the planes of binary32 words
__device__ __forceinline__ void emit(const Problem &p, const CUtensorMap *map, int f16, float (&f)[32], int col, int row0,
                                     int lane, Ring &ring) {
    for (int z = 0; z < p.planes; ++z) {
        char *slot = ring.next(lane);
        if (f16)
            put16<fp16>(slot, lane, f);
        else
            put16<bf16>(slot, lane, f);
        out_by_tma(map, col, row0, z, slot, lane);
        if (z + 1 < p.planes) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {     // infinities and NaN stay in the first plane
                const float hi = to_f32<bf16>(from_f32<bf16>(f[i]));
                f[i] = isfinite(hi) ? f[i] - hi : 0.0f;
            }
        }
    }
}

template <int CG, int EPI>
__global__ void __launch_bounds__(THREADS, 1) k_ffn_mma(const __grid_constant__ Work w) {
    extern __shared__ char smem_raw[];
    constexpr int TILE_M = 128 * CG, TILE_N = 128 * CG;
    constexpr uint32_t TMEM_COLUMNS = 2 * TILE_N;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    char *ring_base = smem + STAGES * STAGE_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(ring_base + EPI_WARPS * RING_SLOT * RING_SLOTS);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_full = empty + 8 * STAGES, acc_empty = acc_full + 16;

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (int i = 0; i < 2; ++i) bar_init(acc_full + 8 * i, 1), bar_init(acc_empty + 8 * i, EPI_WARPS * CG);
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

    int limit = WAIT_LIMIT;
    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = 0;
            for (int item = cluster; item < w.items; item += clusters) {
                const Tile t = tile_of(w, item);
                const Problem &p = w.p[t.problem];
                const int am = t.m * TILE_M + 128 * (int)rank;
                int seg = t.it0 / p.kblocks, kb = t.it0 - seg * p.kblocks;
                for (int it = t.it0; it < t.it1; ++it, ++n) {
                    const uint32_t s = n % STAGES, turn = n / STAGES;
                    bar_wait<CG>(empty + 8 * s, (turn & 1) ^ 1, limit);
                    const uint32_t bar = CG == 2 ? in_first(full + 8 * s) : full + 8 * s;
                    if (rank == 0) bar_expect(full + 8 * s, CG * STAGE_BYTES);
                    const uint32_t dst = smem_u32(smem + s * STAGE_BYTES);
                    const Segment g = p.seg[seg];
                    const int k = kb * BLOCK_K;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r = am + 64 * i;
                        tma_load<CG>(dst + i * BOX_BYTES, &p.a[g.a], p.a_across ? r : k, p.a_across ? k : r, g.za, bar);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // GATE: the tile's first half of columns is h's, the second u's
                        const int which = EPI != MMA_GATE ? g.b : CG == 2 ? (int)rank : i;
                        const int r = EPI != MMA_GATE ? t.n * TILE_N + 128 * (int)rank + 64 * i
                                                      : t.n * (TILE_N / 2) + (CG == 2 ? 64 * i : 0);
                        tma_load<CG>(dst + (2 + i) * BOX_BYTES, &p.b[which], p.b_across ? r : k, p.b_across ? k : r, g.zb, bar);
                    }
                    if (++kb == p.kblocks) kb = 0, ++seg;
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t n = 0, tiles = 0;
            for (int item = cluster; item < w.items; item += clusters, ++tiles) {
                const Tile t = tile_of(w, item);
                const Problem &p = w.p[t.problem];
                const uint32_t acc = tiles & 1, d = tmem + acc * TILE_N;
                bar_wait<CG>(acc_empty + 8 * acc, (tiles >> 1 & 1) ^ 1, limit);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const int a_step = p.a_across ? 2048 >> 4 : 32 >> 4, b_step = p.b_across ? 2048 >> 4 : 32 >> 4;
                for (int it = t.it0; it < t.it1; ++it, ++n) {
                    const uint32_t s = n % STAGES;
                    bar_wait<CG>(full + 8 * s, n / STAGES & 1, limit);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem_u32(smem + s * STAGE_BYTES);
                    const uint64_t a = operand_desc(at, p.a_across), b = operand_desc(at + 2 * BOX_BYTES, p.b_across);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma<CG>(d, a + k * a_step, b + k * b_step, p.idesc, it > t.it0 || k > 0);
                    mma_commit<CG>(empty + 8 * s);
                }
                mma_commit<CG>(acc_full + 8 * acc);
            }
        }
    } else {
        const int quarter = warp & 3;       // the tensor-memory lanes a warp may read
        Ring ring = {ring_base + (warp - 2) * RING_SLOT * RING_SLOTS, 0};
        uint32_t tiles = 0;
        for (int item = cluster; item < w.items; item += clusters, ++tiles) {
            const Tile t = tile_of(w, item);
            const Problem &p = w.p[t.problem];
            const uint32_t acc = tiles & 1;
            const int row0 = t.m * TILE_M + 128 * (int)rank + 32 * quarter;
            const uint32_t from = tmem + acc * TILE_N + ((uint32_t)(32 * quarter) << 16);
            const bool rows = row0 < p.M;
            const int col0 = t.n * (EPI == MMA_GATE ? TILE_N / 2 : TILE_N);
            const long long block = (long long)(row0 >> 5) * p.groups;
            bar_wait<CG>(acc_full + 8 * acc, tiles >> 1 & 1, limit);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if constexpr (EPI == MMA_STORE) {
                for (int c = 0; c < TILE_N; c += 32) {
                    const int col = col0 + c;
                    if (!rows || col >= p.N) break;
                    float f[32];
                    tmem_load(from + c, f);
                    tmem_wait();
                    char *slot = ring.next(lane);
                    if (p.c_f32) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<float4 *>(slot32(slot, lane, i)) =
                                make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    } else if (w.f16) {
                        put16<fp16>(slot, lane, f);
                    } else {
                        put16<bf16>(slot, lane, f);
                    }
                    if (p.c_tma) {
                        out_by_tma(&p.c[0], col, row0, t.split, slot, lane);
                    } else {        // rows that TMA cannot address: a row at a time, neighbouring threads neighbouring words
                        __syncwarp();
                        if (col + lane < p.N) {
                            const long long at = t.split * p.split_stride + (long long)row0 * p.ldc + col + lane;
                            const int end = min(32, p.M - row0);
                            for (int r = 0; r < end; ++r) {
                                if (p.c_f32)
                                    static_cast<float *>(p.cp)[at + r * p.ldc] =
                                        *reinterpret_cast<float *>(slot32(slot, r, lane >> 2) + (lane & 3) * 4);
                                else
                                    static_cast<uint16_t *>(p.cp)[at + r * p.ldc] =
                                        *reinterpret_cast<uint16_t *>(slot16(slot, r, lane >> 3) + (lane & 7) * 2);
                            }
                        }
                        __syncwarp();
                    }
                }
            } else if constexpr (EPI == MMA_GATE) {
                for (int c = 0; c < TILE_N / 2; c += 32) {
                    const int col = col0 + c;
                    if (!rows || col >= p.N) break;
                    float h[32], u[32];
                    tmem_load(from + c, h);
                    tmem_load(from + TILE_N / 2 + c, u);
                    tmem_wait();
                    if (p.h) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if ((col >> 2) + i < p.groups) {
                                const long long at = (block + (col >> 2) + i) * 32 + lane;
                                reinterpret_cast<float4 *>(p.h)[at] = make_float4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                                reinterpret_cast<float4 *>(p.u)[at] = make_float4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
                            }
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float slope;
                        u[i] *= act_value(p.act, h[i], &slope);
                    }
                    emit(p, &p.c[0], w.f16, u, col, row0, lane, ring);
                }
            } else {
                for (int c = 0; c < TILE_N; c += 32) {
                    const int col = col0 + c;
                    if (!rows || col >= p.N) break;
                    float d[32], h[32], u[32];
                    tmem_load(from + c, d);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float4 a = make_float4(0, 0, 0, 0), b = a;
                        if ((col >> 2) + i < p.groups) {
                            const long long at = (block + (col >> 2) + i) * 32 + lane;
                            a = reinterpret_cast<const float4 *>(p.h)[at];
                            b = reinterpret_cast<const float4 *>(p.u)[at];
                        }
                        h[4 * i] = a.x, h[4 * i + 1] = a.y, h[4 * i + 2] = a.z, h[4 * i + 3] = a.w;
                        u[4 * i] = b.x, u[4 * i + 1] = b.y, u[4 * i + 2] = b.z, u[4 * i + 3] = b.w;
                    }
                    tmem_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float slope;
                        const float v = act_value(p.act, h[i], &slope);
                        h[i] = d[i] * u[i] * slope;
                        u[i] = d[i] * v;
                    }
                    emit(p, &p.c[0], w.f16, h, col, row0, lane, ring);
                    emit(p, &p.c[1], w.f16, u, col, row0, lane, ring);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2)
                    bar_arrive_cluster(in_first(acc_empty + 8 * acc));
                else
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(acc_empty + 8 * acc) : "memory");
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (limit != WAIT_LIMIT) {          // a wait ran out: let copies that are still in flight land before the block ends
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

template <int CG, int EPI>
int launch(const Work &w, int sms, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(k_ffn_mma<CG, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
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
    e = cudaLaunchKernelEx(&cfg, k_ffn_mma<CG, EPI>, w);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}

}  // namespace

int mma_launch(const MmaProduct *products, int count, MmaEpilogue epilogue, int type, bool pair, int sms, cudaStream_t s) {
    if (count < 1) return CCDC_OK;
    if (!encoder()) return CCDC_ECUDA;
    static thread_local Work w;
    w.count = count, w.items = 0, w.f16 = type == CCDC_F16;
    const int tile = pair ? 256 : 128, tile_n = epilogue == MMA_GATE ? tile / 2 : tile;
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
                  (uint32_t)(tile >> 3) << 17 | (uint32_t)(tile >> 4) << 24;
        // terms, and within a term of three planes the six products that reach 2^-24, the small ones first
        static const uint8_t order[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
        const int planes = q.a[0].m.planes;
        p.segments = 0;
        for (int k = planes == 1 ? 5 : 0; k < 6; ++k)
            for (int t = 0; t < q.terms; ++t) p.seg[p.segments++] = {(uint8_t)t, (uint8_t)t, order[k][0], order[k][1]};
        const int nb = epilogue == MMA_GATE ? 2 : q.terms;
        bool ok = true;
        auto side = [&](CUtensorMap *map, const MmaSide &d) {
            ok = ok && encode(map, type, d.m.p, d.m.cols, d.m.rows, d.m.ld, d.m.planes, 64, 64);
        };
        for (int t = 0; t < q.terms; ++t) side(&p.a[t], q.a[t]);
        for (int t = 0; t < nb; ++t) side(&p.b[t], q.b[t]);
        if (epilogue == MMA_STORE) {
            p.cp = q.c, p.ldc = q.ldc, p.split_stride = q.M * q.ldc, p.c_f32 = q.c_type == CCDC_F32, p.planes = 1;
            p.c_tma = aligned_to(q.c, 16) && q.ldc * type_bytes(q.c_type) % 16 == 0;
            if (p.c_tma) ok = ok && encode(&p.c[0], q.c_type, q.c, q.N, q.M, q.ldc, p.splits, 32, 32);
        } else {
            p.planes = q.out[0].planes;
            for (int t = 0; t < (epilogue == MMA_GATE ? 1 : 2); ++t)
                ok = ok && encode(&p.c[t], type, q.out[t].p, q.out[t].cols, q.out[t].rows, q.out[t].ld, p.planes, 32, 32);
        }
        if (!ok) return CCDC_ECUDA;
    }
    if (pair)
        return epilogue == MMA_STORE ? launch<2, MMA_STORE>(w, sms, s)
               : epilogue == MMA_GATE ? launch<2, MMA_GATE>(w, sms, s) : launch<2, MMA_GATE_BACK>(w, sms, s);
    return epilogue == MMA_STORE ? launch<1, MMA_STORE>(w, sms, s)
           : epilogue == MMA_GATE ? launch<1, MMA_GATE>(w, sms, s) : launch<1, MMA_GATE_BACK>(w, sms, s);
}

extern "C" int ccdc_block_status(void) {
    int failed = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(&failed, g_wait_failed, sizeof(int));
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    return failed ? CCDC_ESTATE : CCDC_OK;
}
