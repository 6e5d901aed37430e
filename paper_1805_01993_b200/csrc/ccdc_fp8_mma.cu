// The 8-bit product y[m][n] = sum_b xs[m][b] ws[n / 128][b] sum_{k in b} x[m][k] w[n][k] on tcgen05 tensor cores.
//
// Few tokens: weights lie along the tensor core's rows and tokens along its columns.  A tile has 128 rows of a weight and NT
// tokens, so that few tokens cost few columns, and a warp's stores are 32 neighbouring outputs of a token.  More tokens lie along
// the rows, 128 to an SM or 256 to a pair, and 256 rows of the weight along the columns: a thread's scales are then one number
// a block (its token's times the weight's), where a scale for each column costs a shared-memory read for every four products
// (670 cycles a block of 128 x 128).  A block's 128 products are summed in tensor memory, read out, and added to
// registers with the product of scales, because the scales change from block to block; accumulators alternate, so that the
// tensor core works on the next blocks meanwhile.  Warps have roles, as in the feed-forward products:
//   0      fetches 128 bytes of each of the tile's rows of w and x (a pair: half of them each) by TMA into a ring of stages
//   1      issues tcgen05.mma (kind::f8f6f4), one thread, four K = 32 steps a stage
//   4..11  add blocks: 32 rows and half of the columns a warp.  256 columns need 128 registers for their sums alone, which
//          the other four warps give up.
// One persistent block per SM walks the tiles.  With offsets, each expert's rows are cut into tiles by themselves; the list of
// tiles comes from the offsets in every block's shared memory, so that nothing waits for the host.  With few tiles, k is cut
// over the blocks of a cluster, whose sums meet in shared memory in the order of k.
//
// Measured (one B200, calls in a stream on changing inputs, without the quantisation of x): 8192^3 545 us, 2.0 PFLOP/s; 2048 rows
// of 4096 x 4096 44 us; 200 rows over 64 weights of 2048 x 4096 72 us; one row of 16384 x 4096 16.4 us.  What bounds them:
//   large   the turn of the two accumulators.  A block of the pair's tile takes about 930 cycles: 512 of products, 425 of reading and
//           adding, and between them the ways of commit and arrival.  8192^3 takes 330 us without loads and turns, 390 without turns,
//           455 without reading, 495 with reading but without adding.  Tried and not kept: halves of 128 columns, each with its
//           barriers and its issuing thread (591: they read shared memory half as often again), two issuing threads in turn (554),
//           products issued by a warp that goes together (557), 16 adding warps (625), scales through shared memory (551), one
//           polling thread a warp (560).  Waits and arrivals that order memory across the cluster took 1176 us.
//   few     a block's weights by TMA (128 x 128 bytes a stage) at 5 to 7 TB/s once it runs; start, join and end take 7 us.  The
//           first weights on their way to L2 before the kernel before has ended: 0.6 us less for one row, 0.8 more for 512.
//
// All waits are bounded: one that runs out sets g_wait_failed, and its warp issues nothing more and waits for the block's end.
#include <cuda.h>

#include <algorithm>

#include "ccdc_block.h"
#include "ccdc_fp8.h"

namespace {

constexpr int EPI_WARPS = 8, FIRST_EPI = 4, THREADS = 32 * (FIRST_EPI + EPI_WARPS);
constexpr int RING_BYTES = 192 * 1024;
constexpr int JOIN_PAD = 4;                 // words between tokens that wait to be joined, so that writes meet no conflicts
constexpr int MAX_SPLIT = 8;                // a power of two, as all splits
#ifndef CCDC_FP8_WAIT_LIMIT
#define CCDC_FP8_WAIT_LIMIT (1 << 20)       // polls of a barrier (each may sleep) before a wait has failed
#endif

__device__ int g_wait_failed;

struct alignas(64) Args {
    CUtensorMap x, w;
    const float *xs, *ws;
    long long xs_row, xs_col, ldy;
    const int *offsets;
    void *y;
    int M, N, kb, nb, experts, y_type, splits, tiles_n;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// the same address in the cluster's block `rank`
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// No barrier here guards memory that threads write: copies and tensor-core products order what they touch themselves.  So the
// waits and arrivals ask for no order across the cluster, which would cost them an invalidation of the L1 cache each.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < CCDC_FP8_WAIT_LIMIT; ++i) {
        uint32_t ok;
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
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if constexpr (CG == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// arrives at the barrier (of both blocks of a pair) when the products this thread has issued are done: a stage may be filled again,
// and its products may be added
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 8, 16 or 32 columns of this thread's row
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}
// Waits for this thread's loads.  Their registers go through the wait, so that no arithmetic on them moves ahead of it.
template <int W>
__device__ __forceinline__ void arrived(uint32_t (&r)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]),
                     "+r"(r[i + 7]));
}
template <class... R>
__device__ __forceinline__ void tmem_wait(R &...r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    (arrived(r), ...);
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// shared-memory descriptor of rows of 128 bytes with the 128-byte swizzle, eight to a 1 KiB group
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

struct Tile {
    int expert, n, row0, rows;          // expert == experts: rows behind the last, to be set to zero
};
// Where tile `item` lies.  ends[e] = end of expert e's rows, first[e] = its first tile; `e` only moves forward.  An expert's
// tiles go in bands of eight weight tiles, token tile by token tile: neighbours in time share both in L2.
template <int NT>
__device__ __forceinline__ Tile tile_of(const Args &a, const int *ends, const int *first, int item, int &e) {
    while (item >= first[e + 1]) ++e;
    const int start = e ? ends[e - 1] : 0, rows = ends[e] - start, tokens = (rows + NT - 1) / NT;
    int i = item - first[e];
    const int band = i / (8 * tokens), width = min(8, a.tiles_n - 8 * band);
    i -= band * 8 * tokens;
    const int t = i / width;
    return {e, 8 * band + i - t * width, start + t * NT, min(NT, rows - t * NT)};
}
__device__ __forceinline__ void put(const Args &a, int token, int n, float v) {
    const long long at = token * a.ldy + n;
    if (a.y_type == CCDC_F32)
        static_cast<float *>(a.y)[at] = v;
    else if (a.y_type == CCDC_BF16)
        static_cast<bf16 *>(a.y)[at] = from_f32<bf16>(v);
    else
        static_cast<fp16 *>(a.y)[at] = from_f32<fp16>(v);
}

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
        "fma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// COLS neighbouring outputs of each of a warp's 32 tokens, one token a thread.  Rows that start at whole sectors of 32 bytes are
// written sector by sector; others go through shared memory (`stage`), 64 bytes of a row at a time, so that neighbouring threads
// write neighbouring elements.  `left`: tokens of the warp's that are there.
constexpr int STAGE_ROW = 64 + 4, STAGE_WARP = 32 * STAGE_ROW;
template <class T, int COLS>
__device__ __forceinline__ void put_rows_as(const Args &a, long long token0, int left, int n0, const float2 (&sum)[COLS / 2], int lane, char *stage) {
    constexpr int N = 64 / sizeof(T);           // columns of a step
    T *y = static_cast<T *>(a.y) + token0 * a.ldy + n0;
    if ((reinterpret_cast<uintptr_t>(a.y) | (uintptr_t)(a.ldy * sizeof(T))) % 32 == 0 && n0 + COLS <= a.N) {
        T *row = y + lane * a.ldy;
        if (lane < left)
#pragma unroll
            for (int c = 0; c < COLS; c += N / 2) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if constexpr (sizeof(T) == 4)
                        w[i] = __float_as_uint(i & 1 ? sum[(c + i) / 2].y : sum[(c + i) / 2].x);
                    else
                        w[i] = pack2<T>(sum[c / 2 + i].x, sum[c / 2 + i].y);
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + c), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                             "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
            }
        return;
    }
#pragma unroll
    for (int c = 0; c < COLS; c += N) {
        if (n0 + c >= a.N) break;
        uint32_t *mine = reinterpret_cast<uint32_t *>(stage + lane * STAGE_ROW);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if constexpr (sizeof(T) == 4)
                mine[i] = __float_as_uint(i & 1 ? sum[(c + i) / 2].y : sum[(c + i) / 2].x);
            else
                mine[i] = pack2<T>(sum[c / 2 + i].x, sum[c / 2 + i].y);
        __syncwarp();
        const int column = lane % N, row = lane / N;
        if (n0 + c + column < a.N) {
            T *to = y + row * a.ldy + c + column;
            const char *from = stage + row * STAGE_ROW + column * (int)sizeof(T);
            const long long step = 32 / N * a.ldy;
            if (left == 32) {
#pragma unroll 16
                for (int r = 0; r < N; ++r, to += step) *to = *reinterpret_cast<const T *>(from + r * (32 / N * STAGE_ROW));
            } else {
                for (int r = row; r < left; r += 32 / N, to += step, from += 32 / N * STAGE_ROW) *to = *reinterpret_cast<const T *>(from);
            }
        }
        __syncwarp();
    }
}
template <int COLS>
__device__ __forceinline__ void put_rows(const Args &a, long long token0, int left, int n0, const float2 (&sum)[COLS / 2], int lane, char *stage) {
    if (a.y_type == CCDC_F32)
        put_rows_as<float, COLS>(a, token0, left, n0, sum, lane, stage);
    else if (a.y_type == CCDC_BF16)
        put_rows_as<bf16, COLS>(a, token0, left, n0, sum, lane, stage);
    else
        put_rows_as<fp16, COLS>(a, token0, left, n0, sum, lane, stage);
}

// CG SMs to a tile of NT tokens and NW weight rows
template <int CG, int NT, int NW>
struct Shape {
    static constexpr bool ROWS = NT >= 128;                 // tokens lie along the rows
    static constexpr int N = ROWS ? NW : NT;                // columns
    static_assert((ROWS ? NT : NW) == 128 * CG, "rows of the tensor core");
    static constexpr int STAGE_BYTES = 128 * 128 + N / CG * 128;
    // Two blocks an SM where their sums' registers allow it: one adds and writes while the other fetches (200 rows over 64
    // weights of 2048 x 4096: 99 us with one, 77 with two).
    static constexpr int PER_SM = ROWS ? 1 : 2;
    static constexpr int STAGES = RING_BYTES / PER_SM / STAGE_BYTES;
    static constexpr int COLS = N / 2;                      // columns of an adding warp
    static constexpr int ACCS = N <= 128 ? 4 : 2;
    static constexpr bool WIDE = COLS == 128;               // registers move to the adding warps
    // of each adding warp: the scales of two blocks, or outputs on their way
    static constexpr int WARP_BYTES = ROWS ? STAGE_WARP : 2 * COLS * 4;
    static constexpr int FIXED = STAGES * STAGE_BYTES + EPI_WARPS * WARP_BYTES + 256 + 1024;
    static constexpr int smem(int experts) { return FIXED + 2 * 4 * (experts + 3); }
};

// four neighbouring outputs of a token
__device__ __forceinline__ void put4(const Args &a, int token, int n, const float (&v)[4]) {
    const long long at = token * a.ldy + n;
    const int size = a.y_type == CCDC_F32 ? 4 : 2;
    if (n + 4 <= a.N && (reinterpret_cast<uintptr_t>(a.y) + at * size) % (4 * size) == 0) {
        if (a.y_type == CCDC_F32)
            *reinterpret_cast<float4 *>(static_cast<float *>(a.y) + at) = make_float4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<uint2 *>(static_cast<bf16 *>(a.y) + at) =
                a.y_type == CCDC_BF16 ? make_uint2(pack2<bf16>(v[0], v[1]), pack2<bf16>(v[2], v[3]))
                                      : make_uint2(pack2<fp16>(v[0], v[1]), pack2<fp16>(v[2], v[3]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < a.N) put(a, token, n + i, v[i]);
}
// This block's share of the tokens, each output added over the blocks in the order of k.  A warp to 128 outputs of a token, and
// to as many tokens at a time as keep the loads of eight sums under way.
template <int NT, int NW, int SPLITS>
__device__ __forceinline__ void join(const Args &a, const Tile &t, uint32_t smem, int rank, int warp, int lane) {
    constexpr int SHARE = NT / SPLITS, UNITS = SHARE * (NW / 128), AT_ONCE = MAX_SPLIT / SPLITS;
#pragma unroll 1
    for (int u0 = warp; u0 < UNITS; u0 += EPI_WARPS * AT_ONCE) {
        float v[AT_ONCE][SPLITS][4];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int u = min(u0 + j * EPI_WARPS, UNITS - 1), token = SHARE * rank + u / (NW / 128), n = 128 * (u % (NW / 128)) + 4 * lane;
#pragma unroll
            for (int r = 0; r < SPLITS; ++r)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(v[j][r][0]), "=f"(v[j][r][1]), "=f"(v[j][r][2]), "=f"(v[j][r][3])
                             : "r"(in_block(smem + 4 * (token * (NW + JOIN_PAD) + n), r)) : "memory");
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int u = u0 + j * EPI_WARPS, token = SHARE * rank + u / (NW / 128);
#pragma unroll
            for (int r = 1; r < SPLITS; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][0][i] += v[j][r][i];
            if (u < UNITS && token < t.rows) put4(a, t.row0 + token, NW * t.n + 128 * (u % (NW / 128)) + 4 * lane, v[j][0]);
        }
    }
}

template <int CG, int NT, int NW>
__global__ void __launch_bounds__(THREADS, Shape<CG, NT, NW>::PER_SM) k_fp8(const __grid_constant__ Args a) {
    using S = Shape<CG, NT, NW>;
    constexpr int W = S::COLS == 32 ? 16 : S::COLS < 32 ? S::COLS : 32;     // columns of one load from tensor memory
    constexpr int JOIN_ROW = NW + JOIN_PAD;
    constexpr uint32_t TMEM_COLUMNS = S::ACCS * S::N;
    extern __shared__ char smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int splits = CG == 2 ? 1 : a.splits, per = CG == 2 ? 2 : splits;
    const int cluster = blockIdx.x / per, clusters = gridDim.x / per;
    char *smem = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    char *warp_base = smem + S::STAGES * S::STAGE_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(warp_base + EPI_WARPS * S::WARP_BYTES);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 31);
    int *ends = reinterpret_cast<int *>(bars + 32), *first = ends + a.experts + 1;      // [experts + 1], [experts + 2]
    const uint32_t full = smem_u32(bars), empty = full + 8 * S::STAGES, acc_empty = empty + 8 * S::STAGES;
    static_assert(2 * S::STAGES + S::ACCS <= 31, "barriers");
    static_assert(S::ACCS <= S::STAGES, "a stage's products are added before its next ones end");

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::STAGES; ++i) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (int i = 0; i < S::ACCS; ++i) bar_init(acc_empty + 8 * i, EPI_WARPS * CG);
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
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&a.x) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&a.w) : "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // the list of tiles: running maximum of the offsets, then running sums of tiles
    const auto list_tiles = [&] {
        int end = 0, tiles = 0;
        for (int e0 = 0; e0 <= a.experts; e0 += 32) {
            const int e = e0 + lane;
            int v = e < a.experts && a.offsets ? a.offsets[e + 1] : a.M;
            v = max(0, min(v, a.M));
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int u = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v = max(v, u);
            }
            v = max(v, end);
            const int before = __shfl_up_sync(~0u, v, 1);
            int sum = (v - (lane ? before : end) + NT - 1) / NT * a.tiles_n;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int u = __shfl_up_sync(~0u, sum, d);
                if (lane >= d) sum += u;
            }
            if (e <= a.experts) ends[e] = v, first[e + 1] = tiles + sum;
            end = __shfl_sync(~0u, v, 31);
            tiles += __shfl_sync(~0u, sum, 31);
        }
        if (lane == 0) first[0] = 0;
    };
    // all that needs nothing of the kernel before runs under its end
    if (warp == 2 && !a.offsets) list_tiles();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (per > 1) cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.offsets) {
        if (warp == 2) list_tiles();
        __syncthreads();
    }
    const uint32_t tmem = *tmem_slot;
    const int items = first[a.experts + 1];
    // this block's part of k
    const int b0 = CG == 2 ? 0 : (int)((long long)a.kb * rank / splits), b1 = CG == 2 ? a.kb : (int)((long long)a.kb * (rank + 1) / splits);

    bool ok = true;             // no wait of this thread has run out
    int expert = 0;
    if constexpr (S::WIDE) {
        // 128 x 56 + 256 x 224 registers: what 384 threads were launched with at 168
        if (warp < FIRST_EPI) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    }
    if (warp == 0) {
        if (lane == 0) {
            const uint32_t ring = smem_u32(smem), first_full = CG == 2 ? in_block(full, 0) : full;
            uint32_t stage = 0, phase = 0;
            for (int item = cluster; ok && item < items; item += clusters) {
                const Tile t = tile_of<NT>(a, ends, first, item, expert);
                if (t.expert == a.experts) break;           // what follows is set to zero
                const int own = CG == 2 ? 128 * (int)rank : 0, n = NW * t.n + own, row = t.row0 + own;
                constexpr int W_AT = S::ROWS ? 128 * 128 : 0, X_AT = S::ROWS ? 0 : 128 * 128;
                for (int b = b0; b < b1; ++b) {
                    if (ok = bar_wait(empty + 8 * stage, phase ^ 1); !ok) break;
                    const uint32_t bar = first_full + 8 * stage, dst = ring + stage * S::STAGE_BYTES;
                    if (CG == 1 || rank == 0) bar_expect(full + 8 * stage, CG * S::STAGE_BYTES);
                    tma_load<CG>(dst + W_AT, &a.w, 128 * b, n, t.expert, bar);
                    tma_load<CG>(dst + X_AT, &a.x, 128 * b, row, 0, bar);
                    if (++stage == S::STAGES) stage = 0, phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && (CG == 1 || rank == 0)) {
            // D binary32, A and B e4m3, both along k
            constexpr uint32_t idesc = 1u << 4 | (uint32_t)(S::N >> 3) << 17 | (uint32_t)(128 * CG >> 4) << 24;
            const uint64_t rows0 = operand_desc(smem_u32(smem)), columns0 = operand_desc(smem_u32(smem) + 128 * 128);
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
            for (int item = cluster; ok && item < items; item += clusters) {
                if (tile_of<NT>(a, ends, first, item, expert).expert == a.experts) break;
                for (int b = b0; b < b1; ++b) {
                    if (ok = bar_wait(acc_empty + 8 * acc, acc_phase ^ 1); !ok) break;
                    if (ok = bar_wait(full + 8 * stage, phase); !ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t rows = rows0 + stage * (S::STAGE_BYTES >> 4), columns = columns0 + stage * (S::STAGE_BYTES >> 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma<CG>(tmem + acc * S::N, rows + 2 * k, columns + 2 * k, idesc, k > 0);
                    mma_commit<CG>(empty + 8 * stage);
                    if (++stage == S::STAGES) stage = 0, phase ^= 1;
                    if (++acc == S::ACCS) acc = 0, acc_phase ^= 1;
                }
            }
        }
    } else if (warp >= FIRST_EPI) {
        if constexpr (S::WIDE) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int quarter = warp & 3;               // the tensor-memory lanes a warp may read
        const int part = (warp - FIRST_EPI) >> 2;   // two warps a quarter: each takes half of the columns
        char *own_bytes = warp_base + (warp - FIRST_EPI) * S::WARP_BYTES;
        uint32_t acc = 0, stage = 0, phase = 0, buffer = 0;
        for (int item = cluster; ok && item < items; item += clusters) {
            const Tile t = tile_of<NT>(a, ends, first, item, expert);
            const int row = 32 * quarter + lane, column0 = part * S::COLS;      // this thread's row of the SM's, its first column
            const int nb = NW / 128 * t.n + column0 / 128 * S::ROWS;            // the weight's block of 128 rows
            const int own_row = (CG == 2 ? 128 * (int)rank : 0) + row;
            float2 sum[S::COLS / 2] = {};
            if (t.expert < a.experts) {
                const float *ws = a.ws + ((long long)t.expert * a.nb + nb) * a.kb;
                constexpr int PER = S::ROWS ? 1 : (S::COLS + 31) / 32;          // tokens' scales that a lane fetches
                float xs[3][PER], sw[3];                                        // of this block and the next two
                const auto fetch = [&](int b, int to) {
                    sw[to] = b < b1 && nb < a.nb ? ws[b] : 0.0f;
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const int token = t.row0 + (S::ROWS ? own_row : column0 + 32 * i + lane);
                        xs[to][i] = b < b1 && token < a.M ? a.xs[token * a.xs_row + b * a.xs_col] : 0.0f;
                    }
                };
                fetch(b0, 1);
                fetch(b0 + 1, 2);
                // Two blocks to a turn where registers allow, so that the scales need not be moved on, which waits for them (200 rows
                // over 64 weights: 77 and 72 us).
#pragma unroll(NT <= 32 ? 2 : 1)
                for (int b = b0; b < b1; ++b) {
                    float *s = reinterpret_cast<float *>(own_bytes) + buffer * S::COLS;
                    buffer ^= 1;
                    sw[0] = sw[1], sw[1] = sw[2];
#pragma unroll
                    for (int i = 0; i < PER; ++i) xs[0][i] = xs[1][i], xs[1][i] = xs[2][i];
                    const float2 own = make_float2(sw[0] * xs[0][0], sw[0] * xs[0][0]);
                    if constexpr (!S::ROWS) {
#pragma unroll
                        for (int i = 0; i < PER; ++i)
                            if (32 * i + lane < S::COLS) s[32 * i + lane] = sw[0] * xs[0][i];
                    }
                    fetch(b + 2, 2);                        // on its way during this block and the next
                    __syncwarp();
                    if (ok = __all_sync(~0u, bar_wait(empty + 8 * stage, phase)); !ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t from = tmem + acc * S::N + column0 + ((uint32_t)(32 * quarter) << 16);
                    const auto give_back = [&] {            // read out: the tensor core may have it back
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            if constexpr (CG == 2)
                                asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_block(acc_empty + 8 * acc, 0)) : "memory");
                            else
                                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(acc_empty + 8 * acc) : "memory");
                        }
                    };
                    const auto add = [&](const uint32_t (&r)[W], int c) {
#pragma unroll
                        for (int i = 0; i < W; i += 4) {
                            float4 v = make_float4(own.x, own.y, own.x, own.y);
                            if constexpr (!S::ROWS) v = *reinterpret_cast<const float4 *>(s + c + i);
                            float2 &lo = sum[(c + i) / 2], &hi = sum[(c + i) / 2 + 1];
                            lo = fma2(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), make_float2(v.x, v.y), lo);
                            hi = fma2(make_float2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), make_float2(v.z, v.w), hi);
                        }
                    };
                    if constexpr (S::PER_SM == 2) {
#pragma unroll
                        for (int c = 0; c < S::COLS; c += W) {
                            uint32_t r[W];
                            tmem_load(from + c, r);
                            tmem_wait(r);
                            if (c + W == S::COLS) give_back();
                            add(r, c);
                        }
                    } else {                                // two loads under way at a time
                        uint32_t r[2][W];
                        tmem_load(from, r[0]);
                        tmem_load(from + W, r[1]);
#pragma unroll
                        for (int c = 0; c < S::COLS; c += 2 * W) {
                            tmem_wait(r[0], r[1]);
                            if (c + 2 * W == S::COLS) give_back();
                            add(r[0], c);
                            if (c + 2 * W < S::COLS) tmem_load(from + c + 2 * W, r[0]);
                            add(r[1], c + W);
                            if (c + 2 * W < S::COLS) tmem_load(from + c + 3 * W, r[1]);
                        }
                    }
                    if (++acc == S::ACCS) acc = 0;
                    if (++stage == S::STAGES) stage = 0, phase ^= 1;
                }
            }
            if (CG == 1 && splits > 1) {        // to be joined below, token by token; the ring is not needed any more
                float *mine = reinterpret_cast<float *>(smem);
#pragma unroll
                for (int i = 0; i < S::COLS; i += 4) {
                    const float4 v = make_float4(sum[i / 2].x, sum[i / 2].y, sum[i / 2 + 1].x, sum[i / 2 + 1].y);
                    if constexpr (S::ROWS) {
                        *reinterpret_cast<float4 *>(mine + row * JOIN_ROW + column0 + i) = v;
                    } else {
                        mine += i ? 4 * JOIN_ROW : column0 * JOIN_ROW + row;
                        mine[0] = v.x, mine[JOIN_ROW] = v.y, mine[2 * JOIN_ROW] = v.z, mine[3 * JOIN_ROW] = v.w;
                    }
                }
            } else if constexpr (S::ROWS) {
                const int token = own_row - lane, n0 = NW * t.n + column0;
                if (ok && token < t.rows && n0 < a.N) put_rows<S::COLS>(a, t.row0 + token, min(32, t.rows - token), n0, sum, lane, own_bytes);
            } else if (ok && 128 * t.n + row < a.N) {
#pragma unroll
                for (int i = 0; i < S::COLS; ++i)
                    if (column0 + i < t.rows) put(a, t.row0 + column0 + i, 128 * t.n + row, i & 1 ? sum[i / 2].y : sum[i / 2].x);
            }
        }
    }
    if (!ok) {          // let copies that are still in flight land before the block ends
        const long long until = clock64() + 2000000;
        while (clock64() < until) {}
    }
    __syncwarp();
    if (CG == 1 && splits > 1) {
        // one tile a cluster at most: each block adds its share of the tokens over the blocks, in the order of k
        cluster_sync();
        if (cluster < items && warp >= FIRST_EPI) {
            int e = 0;
            const Tile t = tile_of<NT>(a, ends, first, cluster, e);
            if (splits == 2) join<NT, NW, 2>(a, t, smem_u32(smem), (int)rank, warp - FIRST_EPI, lane);
            if (splits == 4) join<NT, NW, 4>(a, t, smem_u32(smem), (int)rank, warp - FIRST_EPI, lane);
            if (splits == 8) join<NT, NW, 8>(a, t, smem_u32(smem), (int)rank, warp - FIRST_EPI, lane);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (per > 1) cluster_sync();
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
// bytes [planes][rows][cols], read in boxes of box_rows x 128; what lies outside reads as zero
bool encode(CUtensorMap *map, const uint8_t *p, long long cols, long long rows, long long ld, long long planes, long long plane, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)(planes > 1 ? plane : ld)};
    const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<uint8_t *>(p), dims, strides, box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, int NT, int NW>
int launch(const Fp8Product &p, int splits, long long most_tiles, int sms, cudaStream_t s) {
    using S = Shape<CG, NT, NW>;
    static std::atomic<unsigned long long> done;
    const void *kernel = reinterpret_cast<const void *>(k_fp8<CG, NT, NW>);
    const int rc = block_allow_smem(kernel, S::smem(1024), &done);
    if (rc != CCDC_OK) return rc;
    Args a;
    if (!encode(&a.x, p.x, p.K, p.M, p.ldx, 1, 0, NT / CG) ||
        !encode(&a.w, p.w, p.K, p.N, p.ldw, p.experts, p.w_expert, NW / CG)) return CCDC_ECUDA;
    a.xs = p.xs, a.ws = p.ws, a.xs_row = p.xs_row, a.xs_col = p.xs_col, a.ldy = p.ldy, a.offsets = p.offsets, a.y = p.y;
    a.M = (int)p.M, a.N = (int)p.N, a.kb = (int)((p.K + 127) / 128), a.nb = (int)((p.N + 127) / 128), a.experts = p.experts;
    a.y_type = p.y_type, a.splits = splits, a.tiles_n = (int)((p.N + NW - 1) / NW);
    const int per = CG == 2 ? 2 : splits;
    cudaLaunchConfig_t cfg = {};
    // a cluster that cuts k takes one tile
    cfg.gridDim = dim3((unsigned)((per == 1 || CG == 2 ? std::min<long long>(most_tiles, std::max(1, S::PER_SM * sms / per)) : most_tiles) * per));
    cfg.blockDim = dim3(THREADS), cfg.dynamicSmemBytes = S::smem(p.experts), cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = per, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_fp8<CG, NT, NW>, a);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}

}  // namespace

int fp8_mma_launch(const Fp8Product &p, int sms, cudaStream_t s) {
    if (!encoder()) return CCDC_ECUDA;
    const long long nb = (p.N + 127) / 128, kb = (p.K + 127) / 128, each = (p.M + p.experts - 1) / p.experts;
    // no more tiles than these, the ones of rows behind the last expert's among them
    const auto most = [&](long long nt, long long rows_n) {
        return (p.offsets ? p.M / nt + std::min<long long>(p.experts + 1, p.M) : (p.M + nt - 1) / nt) * rows_n;
    };
    if (most(16, nb) > 0x7FFFFFFF) return CCDC_ESIZE;
    // k is cut as long as the blocks that run at once are not all taken
    const auto cuts = [&](long long tiles, int blocks) {
        int splits = 1;
        while (splits < MAX_SPLIT && tiles * splits * 2 <= blocks && 2 * splits <= kb) splits *= 2;
        return splits;
    };
    if (each > 64) {
        // A pair's tile does twice the work of a single SM's in the time of a block (0.6 us: the way into an SM, and the turn of
        // the accumulators), but there have to be enough of them.  Rounds of tiles in units of that time; a tile's start and
        // end cost about five.  (256 rows, 8192 x 8192: 41 us by pairs, 27 by single SMs with k cut in two; 8192 rows:
        // 540 by pairs.)
        const long long wide = (nb + 1) / 2, single = most(128, wide);
        const int splits = cuts(single, sms);
        const auto rounds = [&](long long nt, int at_once) {
            const long long tiles = (p.offsets ? p.M / nt + (p.experts + 1) / 2 : (p.M + nt - 1) / nt) * wide;
            return (std::max(tiles, 1LL) + at_once - 1) / at_once;
        };
        if (each > 128 && rounds(256, std::max(1, sms / 2)) * (kb + 5) <= rounds(128, std::max(1, sms / splits)) * (kb / splits + 5) + (splits > 1 ? 5 : 0))
            return launch<2, 256, 256>(p, 1, most(256, wide), sms, s);
        return launch<1, 128, 256>(p, splits, single, sms, s);
    }
    const int nt = each <= 8 ? 16 : each <= 16 ? 32 : 64;      // room for experts with twice their share
    const long long tiles = most(nt, nb);
    const int splits = cuts(tiles, 2 * sms);
    return nt == 16   ? launch<1, 16, 128>(p, splits, tiles, sms, s)
           : nt == 32 ? launch<1, 32, 128>(p, splits, tiles, sms, s) : launch<1, 64, 128>(p, splits, tiles, sms, s);
}

int fp8_mma_status(int *failed) {
    const cudaError_t e = cudaMemcpyFromSymbol(failed, g_wait_failed, sizeof(int));
    return e != cudaSuccess ? ccdc_internal_cuda_fail((int)e) : CCDC_OK;
}
