// The feed-forward products for few rows (a running answer's one token, a small batch).
//
// Every weight is read once and meets all rows; at 8 rows that is 16 operations a byte, far below what the tensor cores
// need, so the kernel is built to keep loads in flight: a block owns 16 rows of the weights (of both matrices for the
// gated product), its eight warps take the steps along k in turn, two batches of loads alternate in a thread's
// registers, and the warps' sums meet in shared memory at the end.
//   16-bit types: mma.sync m16n8k16 with the weights as the 16-row side and the rows of x as the other.  A thread
//     loads 16 bytes (8 k) of two weight rows and of its row of x and uses them as the fragments of two
//     multiplications: the order of k inside a step is free as long as both sides agree, so no shuffles are needed.
//   binary32 (up to 32 rows): plain multiply-adds, two or four weight rows a warp, the lanes along k.
// Measured at 4096 x 16384, bf16: one row 70 us, eight 74 us for 403 MB of weights, 5.7 TB/s.
// (Bulk copies of row slices into shared memory were slower: about 33 cycles a copy and SM, whatever its size.)
// Where there are too few blocks of 16 rows to keep the memory busy, a cluster of up to eight blocks shares the k
// range and the first block adds their sums, in order, through distributed shared memory.
#include <cooperative_groups.h>

#include <algorithm>

#include "ccdc_ffn.h"
#include "ccdc_ffn_mma.h"
#include "ccdc_ffn_rows.h"

namespace cg = cooperative_groups;

namespace {

constexpr int ROWS = 16, WARPS = 8, THREADS = WARPS * 32;

__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, bf16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};" : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, fp16) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};" : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes of a row from element k on, zeros past its end; STREAM: weights, which are not read again
template <class T, bool ALIGNED, bool STREAM>
__device__ __forceinline__ uint4 load16(const T *row, long long k, long long K, bool valid) {
    constexpr int N = 16 / sizeof(T);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (!valid || k >= K) return v;
    if constexpr (ALIGNED) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + k);
        if constexpr (STREAM)
            asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
        else
            v = *p;
    } else {
        T e[N];
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = k + i < K ? row[k + i] : from_f32<T>(0.0f);
        memcpy(&v, e, 16);
    }
    return v;
}

// MATS: 1 or 2 matrices; TOKENS: rows of x (8; binary32 also 32); ALIGNED: rows of 16-byte multiples
template <class T, int MATS, int TOKENS, bool ALIGNED>
__global__ void __launch_bounds__(THREADS, TOKENS == 8 ? 2 : 1) k_ffn_rows(const RowsProduct p) {
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr int STEP = WIDE ? 128 : 32;               // k of a step
    constexpr int UNROLL = (WIDE ? 2 : 4) / MATS;       // steps of a batch
    constexpr int PER = !WIDE ? 2 : TOKENS == 8 ? 4 : 4 / MATS;         // weight rows of a thread
    constexpr int SHARES = WIDE ? PER * WARPS / ROWS : WARPS;           // warps (binary32: groups of them) that take steps in turn
    constexpr int BATCHES = WIDE ? 1 : 2;
    __shared__ float part[SHARES][MATS][ROWS][TOKENS + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int cluster = (int)cg::this_cluster().num_blocks(), rank = (int)cg::this_cluster().block_rank();
    const long long n0 = (long long)(blockIdx.x / cluster) * ROWS;
    const long long steps = (p.K + STEP - 1) / STEP;
    const long long s0 = steps * rank / cluster, s1 = steps * (rank + 1) / cluster;
    const int r0 = WIDE ? warp % (ROWS / PER) * PER : g, dr = WIDE ? 1 : 8, share = WIDE ? warp / (ROWS / PER) : warp;
    const T *w[MATS][PER], *x = static_cast<const T *>(p.x);
    bool in[PER];
#pragma unroll
    for (int r = 0; r < PER; ++r) {
        const long long n = n0 + r0 + dr * r;
        in[r] = n < p.N;
        w[0][r] = static_cast<const T *>(p.w) + n * p.ldw;
        if constexpr (MATS == 2) w[1][r] = static_cast<const T *>(p.w2) + n * p.ldw;
    }

    if (!p.weights_early) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int k_lane = WIDE ? 4 * lane : 8 * t;
    uint4 q[BATCHES][UNROLL][MATS][PER], b[BATCHES][UNROLL];
    float acc[MATS][WIDE ? PER : 1][WIDE ? TOKENS : 4] = {};
    auto fetch_w = [&](int z, long long s) {
#pragma unroll
        for (int i = 0; i < UNROLL; ++i)
#pragma unroll
            for (int m = 0; m < MATS; ++m)
#pragma unroll
                for (int r = 0; r < PER; ++r) {
                    const long long at = s + i * SHARES;
                    q[z][i][m][r] = load16<T, ALIGNED, true>(w[m][r], at * STEP + k_lane, p.K, in[r] && at < s1);
                }
    };
    auto fetch_x = [&](int z, long long s) {
        if constexpr (!WIDE) {
#pragma unroll
            for (int i = 0; i < UNROLL; ++i) {
                const long long at = s + i * SHARES;
                b[z][i] = load16<T, ALIGNED, false>(x + g * p.ldx, at * STEP + k_lane, p.K, g < p.M && at < s1);
            }
        }
    };
    auto use = [&](int z, long long s) {
#pragma unroll
        for (int i = 0; i < UNROLL; ++i) {
            if constexpr (!WIDE) {
#pragma unroll
                for (int m = 0; m < MATS; ++m) {
                    const uint4 &u = q[z][i][m][0], &v = q[z][i][m][1];
                    multiply(acc[m][0], u.x, v.x, u.y, v.y, b[z][i].x, b[z][i].y, T());
                    multiply(acc[m][0], u.z, v.z, u.w, v.w, b[z][i].z, b[z][i].w, T());
                }
            } else {
                const long long at = s + i * SHARES;
                if (at >= s1) break;
#pragma unroll
                for (int m0 = 0; m0 < TOKENS; m0 += 8) {
                    if (m0 >= p.M) break;
                    uint4 xv[8];        // eight rows of x asked for together
#pragma unroll
                    for (int m = 0; m < 8; ++m)
                        xv[m] = load16<T, ALIGNED, false>(x + (m0 + m) * p.ldx, at * STEP + k_lane, p.K, m0 + m < p.M);
#pragma unroll
                    for (int m = 0; m < 8; ++m) {
                        const float4 c = *reinterpret_cast<const float4 *>(&xv[m]);
#pragma unroll
                        for (int k = 0; k < MATS; ++k)
#pragma unroll
                            for (int r = 0; r < PER; ++r) {
                                const float4 a = *reinterpret_cast<const float4 *>(&q[z][i][k][r]);
                                float &sum = acc[k][r][m0 + m];
                                sum = fmaf(a.x, c.x, fmaf(a.y, c.y, fmaf(a.z, c.z, fmaf(a.w, c.w, sum))));
                            }
                    }
                }
            }
        }
    };
    constexpr int HOP = UNROLL * SHARES;
    long long s = s0 + share;
    fetch_w(0, s);
    if (p.weights_early) asm volatile("griddepcontrol.wait;" ::: "memory");     // x may be the last launch's
    fetch_x(0, s);
    while (s < s1) {
        if constexpr (BATCHES == 2) {
            fetch_w(1, s + HOP), fetch_x(1, s + HOP);
            use(0, s);
            fetch_w(0, s + 2 * HOP), fetch_x(0, s + 2 * HOP);
            use(1, s + HOP);
            s += 2 * HOP;
        } else {
            use(0, s);
            s += HOP;
            fetch_w(0, s);
        }
    }
    if constexpr (!WIDE) {
#pragma unroll
        for (int k = 0; k < MATS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][k][g + 8 * (i >> 1)][2 * t + (i & 1)] = acc[k][0][i];
    } else {
#pragma unroll
        for (int k = 0; k < MATS; ++k)
#pragma unroll
            for (int r = 0; r < PER; ++r)
#pragma unroll
                for (int m = 0; m < TOKENS; ++m) {
                    float v = acc[k][r][m];
#pragma unroll
                    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
                    if (lane == 0) part[share][k][r0 + r][m] = v;
                }
    }
    __syncthreads();
    // the block's sums, into the first share's place
    for (int i = threadIdx.x; i < MATS * ROWS * TOKENS; i += THREADS) {
        const int k = i / (ROWS * TOKENS), r = i / TOKENS % ROWS, m = i % TOKENS;
        float v = part[0][k][r][m];
#pragma unroll
        for (int o = 1; o < SHARES; ++o) v += part[o][k][r][m];
        part[0][k][r][m] = v;
    }
    if (cluster > 1)
        cg::this_cluster().sync();
    else
        __syncthreads();
    if (rank == 0)
        for (int i = threadIdx.x; i < ROWS * TOKENS; i += THREADS) {
            const int r = i % ROWS, m = i / ROWS;
            const long long n = n0 + r;
            if (m >= p.M || n >= p.N) continue;
            float v[MATS];
#pragma unroll
            for (int k = 0; k < MATS; ++k) {
                v[k] = part[0][k][r][m];
                for (int o = 1; o < cluster; ++o) v[k] += *cg::this_cluster().map_shared_rank(&part[0][k][r][m], o);
            }
            float f = v[0];
            if constexpr (MATS == 2) {
                if (p.h) {
                    const long long at = ffn_saved_index(m, n, ffn_saved_groups(p.N));
                    p.h[at] = v[0], p.u[at] = v[1];
                }
                act_apply<WIDE>(p.act, [&](auto act) {
                    float slope;
                    f = act(v[0], &slope) * v[1];
                });
            }
            static_cast<T *>(p.out)[m * p.ldo + n] = from_f32<T>(f);
        }
    if (cluster > 1) cg::this_cluster().sync();     // the others' shared memory is read until here
}

template <class T, int MATS, int TOKENS, bool ALIGNED>
int launch(const RowsProduct &p, int sms, cudaStream_t s) {
    // a block for every SM, as long as a warp keeps four steps (clusters start slower: with one for every SM and more, 4 rows of
    // 4096 x 4096 took 27 us instead of 21)
    const long long blocks = (p.N + ROWS - 1) / ROWS, step = sizeof(T) == 4 ? 128 * 2 : 32 * WARPS;
    int cluster = 1;
    while (cluster < 8 && blocks * cluster < sms && p.K >= 8 * cluster * step) cluster *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_ffn_rows<T, MATS, TOKENS, ALIGNED>, p);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}
template <class T, int MATS, int TOKENS>
int launch_aligned(const RowsProduct &p, int sms, cudaStream_t s) {
    auto rows = [&](const void *q, long long ld, long long n) {
        return !q || (aligned_to(q, 16) && (n < 2 || ld * sizeof(T) % 16 == 0));
    };
    const bool aligned = p.K * sizeof(T) % 16 == 0 && rows(p.x, p.ldx, p.M) && rows(p.w, p.ldw, p.N) && rows(p.w2, p.ldw, p.N);
    return aligned ? launch<T, MATS, TOKENS, true>(p, sms, s) : launch<T, MATS, TOKENS, false>(p, sms, s);
}

}  // namespace

int rows_launch(const RowsProduct &p, int sms, cudaStream_t s) {
    if (p.dtype == CCDC_F32 && p.M > 8) return p.w2 ? launch_aligned<float, 2, 32>(p, sms, s) : launch_aligned<float, 1, 32>(p, sms, s);
    if (p.dtype == CCDC_F32) return p.w2 ? launch_aligned<float, 2, 8>(p, sms, s) : launch_aligned<float, 1, 8>(p, sms, s);
    if (p.dtype == CCDC_BF16) return p.w2 ? launch_aligned<bf16, 2, 8>(p, sms, s) : launch_aligned<bf16, 1, 8>(p, sms, s);
    return p.w2 ? launch_aligned<fp16, 2, 8>(p, sms, s) : launch_aligned<fp16, 1, 8>(p, sms, s);
}
