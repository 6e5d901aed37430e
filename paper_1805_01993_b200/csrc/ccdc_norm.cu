// Norms before and after a block, fused with its gate, dropout and residual scale, and the dropout itself.
//
//   n   = unit(y) * w_post                 unit(v) = (v - mean v) / sqrt(var v + eps)   (layer)
//   out = alpha x + drop(gate * n)                 = v / sqrt(mean v^2 + eps)           (rms)
//   z   = unit(out) * w_pre
//
// and backward, with t the whole gradient that reaches `out`:
//   t   = dout + unit'(out)(dz * w_pre),   unit'(v)(e) = r (e - mean e - unit(v) mean(e unit(v)))
//   dx  = alpha t,  dq = drop(t),  dgate += dq n,  dy = unit'(y)(dq gate w_post)
// (no mean term for rms; r = the rstd of the row, kept by the forward).
//
// One block (or a team of warps) owns a row: its columns stay in registers between the passes over them, so every tensor is read
// once and written once.  The sums over rows (w_post, w_pre, gate) are held per column in registers while a
// block walks a contiguous range of rows, and meet through the workspace in block order: no atomics, so that
// a file's gradients have the same bits at every node that maps it.
#include <algorithm>

#include "ccdc_block.h"

namespace {

constexpr long long MAX_D = 32768;      // the most columns of a row: 32 for each thread of the largest block

struct NormArgs {
    long long M, D;
    const void *x, *y, *w_post, *w_pre, *gate;
    long long ldx, ldy, per;            // per: rows that share a gate row, at most M (its multiples stay within 64 bits)
    float alpha, eps;
    int layer;
    Dropout drop;
    // forward
    void *out, *z;
    long long ldo, ldz;
    float4 *stats;                      // per row: mean and rstd of y, mean and rstd of out
    // backward
    const void *dout, *dz;
    long long lddout, lddz;
    void *dx, *dy;
    long long lddx, lddy;
    void *dgate;
    int grad_f32;
    float *partial;                     // [blocks] w_post, [blocks] w_pre, [shares] first and [shares] last piece of a
                                        // split gate row, each [D]
};

// first row of block b's share
__host__ __device__ __forceinline__ long long share(long long M, int blocks, int b) { return M * b / blocks; }

// ------------------------------------------------------------------ rows by blocks
// The form for any alignment and up to MAX_D columns: a block owns a row and loads it straight into registers, all of it
// before the first barrier.  Measured with gate and dropout at 16384 x 1001, binary32: forward 64 us, 4.1 TB/s; backward
// 134 us, 2.9 TB/s (the loads spread between the barriers: 2.5 times that).  16-bit rows that vectors cannot address go by
// 2-byte accesses: at 1001 and 4095 columns forward 2.0 TB/s, backward 1.0 to 1.1.
// A thread's columns fit its registers up to 4096 (forward 8192); the backward pass spills 0.3 to 0.5 KB a thread up to 8192
// and 3.6 to 4.5 KB beyond (forward 0.3 to 2 KB), at 16384 columns some 35 GB through L1 and L2 for 0.8 GB of tensors:
// 4096 x 16384 bf16 forward 0.35 ms, backward 3.6 ms (0.23 TB/s), binary32 0.45 and 4.3 ms.

// sums of two values over the block; one barrier, buffers used in turn
template <int THREADS>
__device__ __forceinline__ float2 block_sum(float a, float b, float2 (*buf)[THREADS / 32], int &turn) {
#pragma unroll
    for (int i = 16; i; i >>= 1) {
        a += __shfl_xor_sync(~0u, a, i);
        b += __shfl_xor_sync(~0u, b, i);
    }
    if constexpr (THREADS > 32) {
        float2 *s = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        const float2 v = s[threadIdx.x & (THREADS / 32 - 1)];
        a = v.x, b = v.y;
#pragma unroll
        for (int i = THREADS / 64; i; i >>= 1) {
            a += __shfl_xor_sync(~0u, a, i);
            b += __shfl_xor_sync(~0u, b, i);
        }
    }
    return make_float2(a, b);
}

// a thread's columns of a row: ITEMS runs of VEC
template <class T, int VEC, int ITEMS, int THREADS>
struct Row {
    static __device__ __forceinline__ int col(int i) { return (i * THREADS + (int)threadIdx.x) * VEC; }
    static __device__ __forceinline__ void load(const T *p, int D, float (&f)[ITEMS][VEC]) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = col(i);
            if constexpr (VEC == 8) {
                if (c < D) {
                    unpack8<T>(load8(p + c), f[i]);
                } else {
#pragma unroll
                    for (int v = 0; v < 8; ++v) f[i][v] = 0.0f;
                }
            } else {
                f[i][0] = c < D ? to_f32<T>(p[c]) : 0.0f;
            }
        }
    }
    static __device__ __forceinline__ void store(T *p, int D, const float (&f)[ITEMS][VEC]) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = col(i);
            if (c >= D) continue;
            if constexpr (VEC == 8)
                store8(p + c, pack8<T>(f[i]));
            else
                p[c] = from_f32<T>(f[i][0]);
        }
    }
};

// The row's dropout factors as bits (bit v of word i: column v of run i is kept).  Rows that start on a
// multiple of eight elements take theirs straight from the generator; others share the bytes of the row's
// generator calls through shared memory, so that no call is made twice.
template <int VEC, int ITEMS, int THREADS>
__device__ __forceinline__ void row_keep(const NormArgs &a, long long m, uint32_t (&keep)[ITEMS], uint8_t *bytes) {
    const unsigned long long e0 = a.drop.offset + (unsigned long long)(m * a.D);
    const int D = (int)a.D;
    if (VEC == 8 && (e0 & 7) == 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * THREADS + (int)threadIdx.x) * VEC;
            keep[i] = c < D ? keep_bits(a.drop, (e0 + c) >> 3) : 0;
        }
        return;
    }
    const int shift = (int)(e0 & 7), n = (shift + D + 7) >> 3;
    for (int j = threadIdx.x; j < n; j += THREADS) bytes[j] = (uint8_t)keep_bits(a.drop, ((e0 >> 3) + j) & COUNTERS);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * THREADS + (int)threadIdx.x) * VEC + shift;
        uint32_t w = 0;
        if (c - shift < D) {
            if constexpr (VEC == 8)
                w = ((bytes[c >> 3] | ((uint32_t)bytes[(c >> 3) + 1] << 8)) >> (c & 7)) & 0xFFu;
            else
                w = (bytes[c >> 3] >> (c & 7)) & 1u;
        }
        keep[i] = w;
    }
}

template <class T, int VEC, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS) k_residual_norm(const NormArgs a) {
    using R = Row<T, VEC, ITEMS, THREADS>;
    __shared__ float2 buf[2][THREADS / 32];
    __shared__ uint8_t bytes[2][VEC * ITEMS * THREADS / 8 + 2];
    const int D = (int)a.D;
    const float inv = 1.0f / (float)D;
    int turn = 0, parity = 0;
    for (long long m = blockIdx.x; m < a.M; m += gridDim.x, parity ^= 1) {
        float o[ITEMS][VEC], q[ITEMS][VEC];
        R::load(static_cast<const T *>(a.x) + m * a.ldx, D, o);
        float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) o[i][v] *= a.alpha;
        // mean and rstd of a row held in registers; columns past D hold zeros and are left out
        auto unit = [&](const float(&f)[ITEMS][VEC], float &mean, float &rstd) {
            float s = 0.0f;
            mean = 0.0f;
            if (a.layer) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) s += f[i][v];
                mean = block_sum<THREADS>(s, 0.0f, buf, turn).x * inv;
                s = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (R::col(i) < D) {
#pragma unroll
                    for (int v = 0; v < VEC; ++v) s += (f[i][v] - mean) * (f[i][v] - mean);
                }
            rstd = rsqrtf(block_sum<THREADS>(s, 0.0f, buf, turn).x * inv + a.eps);
        };
        if (a.y) {
            R::load(static_cast<const T *>(a.y) + m * a.ldy, D, q);
            uint32_t keep[ITEMS];
            if (a.drop.cut) row_keep<VEC, ITEMS, THREADS>(a, m, keep, bytes[parity]);
            if (a.w_post) {
                unit(q, st.x, st.y);
                float w[ITEMS][VEC];
                R::load(static_cast<const T *>(a.w_post), D, w);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) q[i][v] = (q[i][v] - st.x) * st.y * w[i][v];
            }
            if (a.gate) {
                float g[ITEMS][VEC];
                R::load(static_cast<const T *>(a.gate) + m / a.per * a.D, D, g);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) q[i][v] *= g[i][v];
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    const float d = !a.drop.cut ? q[i][v] : (keep[i] >> v & 1) ? q[i][v] * a.drop.scale : 0.0f;
                    o[i][v] += R::col(i) < D ? d : 0.0f;
                }
        }
        if (a.out) R::store(static_cast<T *>(a.out) + m * a.ldo, D, o);
        if (a.w_pre) {
            unit(o, st.z, st.w);
            float w[ITEMS][VEC];
            R::load(static_cast<const T *>(a.w_pre), D, w);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) o[i][v] = (o[i][v] - st.z) * st.w * w[i][v];
            R::store(static_cast<T *>(a.z) + m * a.ldz, D, o);
        }
        if (a.stats && threadIdx.x == 0) a.stats[m] = st;
    }
}

template <class T, int VEC, int ITEMS, int THREADS>
__global__ void __launch_bounds__(THREADS) k_residual_norm_back(const NormArgs a) {
    using R = Row<T, VEC, ITEMS, THREADS>;
    __shared__ float2 buf[2][THREADS / 32];
    __shared__ uint8_t bytes[2][VEC * ITEMS * THREADS / 8 + 2];
    const int D = (int)a.D;
    const float inv = 1.0f / (float)D;
    int turn = 0, parity = 0;
    float sum_post[ITEMS][VEC] = {}, sum_pre[ITEMS][VEC] = {}, sum_gate[ITEMS][VEC] = {};
    const long long first = share(a.M, gridDim.x, blockIdx.x), last = share(a.M, gridDim.x, blockIdx.x + 1);
    const long long first_group = first / a.per;
    for (long long m = first; m < last; ++m, parity ^= 1) {
        // everything the row needs is asked for before the first barrier
        const float4 st = a.stats[m];
        float oh[ITEMS][VEC], yh[ITEMS][VEC], cg[ITEMS][VEC], t[ITEMS][VEC], e[ITEMS][VEC], w_post[ITEMS][VEC], gate[ITEMS][VEC];
        R::load(static_cast<const T *>(a.x) + m * a.ldx, D, oh);
        if (a.y) R::load(static_cast<const T *>(a.y) + m * a.ldy, D, yh);
        if (a.w_pre) R::load(static_cast<const T *>(a.dz) + m * a.lddz, D, e);
        if (a.dout) R::load(static_cast<const T *>(a.dout) + m * a.lddout, D, t);
        if (a.w_post) R::load(static_cast<const T *>(a.w_post), D, w_post);
        if (a.gate) R::load(static_cast<const T *>(a.gate) + m / a.per * a.D, D, gate);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                oh[i][v] *= a.alpha, cg[i][v] = 1.0f;
                if (!a.y) yh[i][v] = 0.0f;
                if (!a.dout) t[i][v] = 0.0f;
            }
        if (a.y) {
            if (a.drop.cut) {
                uint32_t keep[ITEMS];
                row_keep<VEC, ITEMS, THREADS>(a, m, keep, bytes[parity]);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) cg[i][v] = (keep[i] >> v & 1) ? a.drop.scale : 0.0f;
            }
        }
        float s1 = 0.0f, s0 = 0.0f;
        // out again from the forward's inputs: exact, where the stored `out` is rounded
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                if (a.w_post) yh[i][v] = (yh[i][v] - st.x) * st.y;
                float n = yh[i][v];
                if (a.w_post) n *= w_post[i][v];
                if (a.gate) n *= gate[i][v];
                n = cg[i][v] == 0.0f ? 0.0f : n * cg[i][v];
                if (a.y) oh[i][v] += n;
            }
        if (a.w_pre) {
            float w[ITEMS][VEC];
            R::load(static_cast<const T *>(a.w_pre), D, w);
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    oh[i][v] = (oh[i][v] - st.z) * st.w;
                    sum_pre[i][v] += e[i][v] * oh[i][v];
                    e[i][v] *= w[i][v];
                    s1 += e[i][v] * oh[i][v];
                    s0 += e[i][v];
                }
            const float2 s = block_sum<THREADS>(s1, s0, buf, turn);
            s1 = s.x * inv, s0 = a.layer ? s.y * inv : 0.0f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) t[i][v] += st.w * (e[i][v] - s0 - oh[i][v] * s1);
        }
        if (a.dx) {
            float d[ITEMS][VEC];
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) d[i][v] = a.alpha * t[i][v];
            R::store(static_cast<T *>(a.dx) + m * a.lddx, D, d);
        }
        if (!a.y) continue;
        s1 = s0 = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                float d = cg[i][v] == 0.0f ? 0.0f : t[i][v] * cg[i][v];
                if (a.gate) {
                    sum_gate[i][v] += cg[i][v] == 0.0f ? 0.0f : d * yh[i][v] * (a.w_post ? w_post[i][v] : 1.0f);
                    d *= gate[i][v];
                }
                if (a.w_post) {
                    sum_post[i][v] += d * yh[i][v];
                    d *= w_post[i][v];
                    if (R::col(i) < D) s1 += d * yh[i][v], s0 += d;
                }
                t[i][v] = d;
            }
        if (a.w_post) {
            const float2 s = block_sum<THREADS>(s1, s0, buf, turn);
            s1 = s.x * inv, s0 = a.layer ? s.y * inv : 0.0f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) t[i][v] = st.y * (t[i][v] - s0 - yh[i][v] * s1);
        }
        if (a.dy) R::store(static_cast<T *>(a.dy) + m * a.lddy, D, t);
        if (a.gate && a.dgate && (m + 1 == last || (m + 1) % a.per == 0)) {    // the last row of this gate row here
            const long long g = m / a.per;
            const long long begin = g * a.per, end = min(begin + a.per, a.M);
            if (begin >= first && end <= last) {            // all its rows are this block's
                if (a.grad_f32)
                    Row<float, VEC, ITEMS, THREADS>::store(static_cast<float *>(a.dgate) + g * a.D, D, sum_gate);
                else
                    R::store(static_cast<T *>(a.dgate) + g * a.D, D, sum_gate);
            } else {
                float *to = a.partial + ((g == first_group ? 2LL : 3LL) * gridDim.x + blockIdx.x) * a.D;
                Row<float, VEC, ITEMS, THREADS>::store(to, D, sum_gate);
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) sum_gate[i][v] = 0.0f;
        }
    }
    if (a.w_post) Row<float, VEC, ITEMS, THREADS>::store(a.partial + (long long)blockIdx.x * a.D, D, sum_post);
    if (a.w_pre) Row<float, VEC, ITEMS, THREADS>::store(a.partial + ((long long)gridDim.x + blockIdx.x) * a.D, D, sum_pre);
}

// ------------------------------------------------------------------ rows by teams
// The form for rows of 16-byte multiples and up to 8192 columns.  A team of W warps owns a row, a thread ITEMS runs of
// eight of its columns, so that small rows need few threads to meet for their sums (one warp's row no barrier at all),
// and teams of a block are independent.  Every thread copies its own columns of the rows to come into its own
// shared-memory slots (cp.async, STAGES rows ahead): it waits for its own copies alone, and memory stays busy while a
// row's sums are formed.
// Rows asked for ahead: two; three take the L1 share that w_pre and the factors are read through (16384 x 4096 bf16,
// backward: 224 us with two, 249 with three).
// Measured at 16384 x 4096, bf16, rms, with dropout: forward 108 us, 5.0 TB/s; backward 217 us, 3.7 TB/s.  Neither issue
// slots (52 to 55 % used; 34 and 61 instructions an element, of which the generator takes about 6) nor DRAM (42 to 45 %)
// are at their limit: 16 warps an SM at 112 to 128 registers do not hide the latency of a row's two meetings.
constexpr int STAGES = 2;

template <int W>
struct Team {
    float2 (*buf)[W];
    int turn, bar;
    __device__ __forceinline__ float2 sum(float a, float b) {
#pragma unroll
        for (int i = 16; i; i >>= 1) {
            a += __shfl_xor_sync(~0u, a, i);
            b += __shfl_xor_sync(~0u, b, i);
        }
        if constexpr (W > 1) {
            const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & (W - 1);
            if (lane == 0) buf[turn][warp] = make_float2(a, b);
            asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(32 * W) : "memory");
            const float2 v = buf[turn][lane & (W - 1)];
            a = v.x, b = v.y;
            turn ^= 1;
#pragma unroll
            for (int i = W / 2; i; i >>= 1) {
                a += __shfl_xor_sync(~0u, a, i);
                b += __shfl_xor_sync(~0u, b, i);
            }
        }
        return make_float2(a, b);
    }
    __device__ __forceinline__ float sum1(float a) {
#pragma unroll
        for (int i = 16; i; i >>= 1) a += __shfl_xor_sync(~0u, a, i);
        if constexpr (W > 1) {
            const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & (W - 1);
            if (lane == 0) buf[turn][warp].x = a;
            asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(32 * W) : "memory");
            a = buf[turn][lane & (W - 1)].x;
            turn ^= 1;
#pragma unroll
            for (int i = W / 2; i; i >>= 1) a += __shfl_xor_sync(~0u, a, i);
        }
        return a;
    }
};

template <class T, int ITEMS, int W, int THREADS, int ARRAYS, int DEPTH>
struct RowStream {
    static constexpr int PIECES = ITEMS * (int)sizeof(T) / 2;          // 16-byte pieces of a thread's columns
    static constexpr int SMEM = DEPTH * ARRAYS * PIECES * THREADS * 16;
    const T *from[ARRAYS];
    long long ld[ARRAYS];
    int D, tid;
    uint4 *slots;
    __device__ __forceinline__ int col(int i) const { return (i * 32 * W + tid) * 8; }
    // columns past D are never fetched: they read as zeros
    __device__ __forceinline__ void clear() {
        if (col(ITEMS - 1) < D) return;
#pragma unroll
        for (int i = 0; i < DEPTH * ARRAYS * PIECES; ++i) slots[i * THREADS] = make_uint4(0, 0, 0, 0);
    }
    // the copies of one row; past the last row an empty group keeps the count
    __device__ __forceinline__ void fetch(long long m, bool valid, int stage) {
        if (valid) {
#pragma unroll
            for (int k = 0; k < ARRAYS; ++k) {
                if (!from[k]) continue;
                const T *row = from[k] + m * ld[k];
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    if (col(i) >= D) continue;
#pragma unroll
                    for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
                        const uint32_t to = (uint32_t)__cvta_generic_to_shared(
                            slots + ((stage * ARRAYS + k) * PIECES + i * (int)sizeof(T) / 2 + q) * THREADS);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                                     ::"r"(to), "l"(row + col(i) + q * (16 / (int)sizeof(T))) : "memory");
                    }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory"); }
    __device__ __forceinline__ void get(int stage, int k, int i, float (&f)[8]) const {
        Eight<T> r;
#pragma unroll
        for (int q = 0; q < (int)sizeof(T) / 2; ++q)
            r.v[q] = slots[((stage * ARRAYS + k) * PIECES + i * (int)sizeof(T) / 2 + q) * THREADS];
        unpack8<T>(r, f);
    }
};

// The generator's words for the thread's run at column c of row m; all ones where nothing is dropped
__device__ __forceinline__ uint4 team_words(const NormArgs &a, long long m, int c) {
    if (!a.drop.cut) return make_uint4(~0u, ~0u, ~0u, ~0u);
    return drop_words(a.drop, (a.drop.offset + (unsigned long long)(m * a.D) + c) >> 3);
}
// gate * w_post * the dropout's factor for the thread's columns: the same for all rows that share a gate row.  A gate of
// its own for every row comes through the stream, as array `streamed` of the stage (-1: it does not).
template <class T, int ITEMS, class Stream>
__device__ __forceinline__ void team_factor(const NormArgs &a, const Stream &in, long long group, float (&f)[ITEMS][8],
                                            int streamed = -1, int stage = 0) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = in.col(i);
#pragma unroll
        for (int v = 0; v < 8; ++v) f[i][v] = a.drop.cut ? a.drop.scale : 1.0f;
        if (c >= in.D) continue;
        float w[8];
        if (a.w_post) {
            unpack8<T>(load8(static_cast<const T *>(a.w_post) + c), w);
#pragma unroll
            for (int v = 0; v < 8; ++v) f[i][v] *= w[v];
        }
        if (a.gate) {
            if (streamed >= 0)
                in.get(stage, streamed, i, w);
            else
                unpack8<T>(load8(static_cast<const T *>(a.gate) + group * a.D + c), w);
#pragma unroll
            for (int v = 0; v < 8; ++v) f[i][v] *= w[v];
        }
    }
}

template <class T, int ITEMS, int W, int TEAMS>
__global__ void __launch_bounds__(32 * W * TEAMS, 512 / (32 * W * TEAMS)) k_norm_rows(const NormArgs a) {
    constexpr int THREADS = 32 * W * TEAMS;
    using Stream = RowStream<T, ITEMS, W, THREADS, 3, STAGES>;
    extern __shared__ uint4 slots[];
    __shared__ float2 buf[TEAMS][2][W];
    const int team = threadIdx.x / (32 * W), tid = threadIdx.x % (32 * W), D = (int)a.D;
    Team<W> sums = {buf[team], 0, 1 + team};
    const bool row_gate = a.gate && a.per == 1;
    Stream in = {{static_cast<const T *>(a.x), static_cast<const T *>(a.y), row_gate ? static_cast<const T *>(a.gate) : nullptr},
                 {a.ldx, a.ldy, a.D}, D, tid, slots + threadIdx.x};
    const float inv = 1.0f / (float)D;
    const int shares = gridDim.x * TEAMS, mine = blockIdx.x * TEAMS + team;
    const long long first = share(a.M, shares, mine), last = share(a.M, shares, mine + 1);
    long long group = first / a.per, group_end = (group + 1) * a.per;
    float factor[ITEMS][8];
    if (!row_gate && first < last) team_factor<T>(a, in, group, factor);
    in.clear();
#pragma unroll
    for (int i = 0; i < STAGES; ++i) in.fetch(first + i, first + i < last, i);
    int stage = 0;
    for (long long m = first; m < last; ++m) {
        if (m == group_end) {
            ++group, group_end += a.per;
            if (!row_gate) team_factor<T>(a, in, group, factor);
        }
        in.arrived();
        if (row_gate) team_factor<T>(a, in, group, factor, 2, stage);
        float o[ITEMS][8], q[ITEMS][8];
        float4 st = make_float4(0.0f, 1.0f, 0.0f, 1.0f);
        // mean and rstd of a row in registers; columns past D hold zeros
        auto unit = [&](const float(&f)[ITEMS][8], float &mean, float &rstd) {
            float s = 0.0f;
            if (a.layer) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < 8; ++v) s += f[i][v];
                mean = sums.sum1(s) * inv;
                s = 0.0f;
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    float e = 0.0f;
#pragma unroll
                    for (int v = 0; v < 8; ++v) e += (f[i][v] - mean) * (f[i][v] - mean);
                    s += in.col(i) < D ? e : 0.0f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < 8; ++v) s += f[i][v] * f[i][v];
            }
            rstd = rsqrtf(sums.sum1(s) * inv + a.eps);
        };
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            in.get(stage, 0, i, o[i]);
            if (a.y) in.get(stage, 1, i, q[i]);
        }
        in.fetch(m + STAGES, m + STAGES < last, stage);         // this thread's slots are read
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (a.y) {
            if (a.w_post) unit(q, st.x, st.y);
            const float shift = -st.x * st.y;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const uint4 w = team_words(a, m, in.col(i));
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    o[i][v] = fmaf(o[i][v], a.alpha, kept(w, v, a.drop.below, fmaf(q[i][v], st.y, shift) * factor[i][v]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < 8; ++v) o[i][v] *= a.alpha;
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (in.col(i) < D) {
                if (a.out) store8(static_cast<T *>(a.out) + m * a.ldo + in.col(i), pack8<T>(o[i]));
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v) o[i][v] = 0.0f;
            }
        }
        if (a.w_pre) {
            unit(o, st.z, st.w);
            const float shift = -st.z * st.w;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = in.col(i);
                if (c >= D) continue;
                float w[8];
                unpack8<T>(load8(static_cast<const T *>(a.w_pre) + c), w);
#pragma unroll
                for (int v = 0; v < 8; ++v) w[v] *= fmaf(o[i][v], st.w, shift);
                store8(static_cast<T *>(a.z) + m * a.ldz + c, pack8<T>(w));
            }
        }
        if (a.stats && tid == 0) a.stats[m] = st;
    }
}

// Backward.  The sums over rows use that gate and w_post are the same for all rows of a gate row: with
// S = sum of drop(t) unit(y) over those rows, dgate = w_post S and w_post's gradient is the sum of gate S, so the rows
// feed one accumulator; w_post's own sum is added to (in shared memory) when a gate row ends.
template <class T, int ITEMS, int W, int TEAMS>
__global__ void __launch_bounds__(32 * W * TEAMS, 512 / (32 * W * TEAMS)) k_norm_rows_back(const NormArgs a) {
    constexpr int THREADS = 32 * W * TEAMS;
    using Stream = RowStream<T, ITEMS, W, THREADS, 5, STAGES>;
    extern __shared__ uint4 slots[];
    __shared__ float2 buf[TEAMS][2][W];
    const int team = threadIdx.x / (32 * W), tid = threadIdx.x % (32 * W), D = (int)a.D;
    Team<W> sums = {buf[team], 0, 1 + team};
    const bool row_gate = a.gate && a.per == 1;
    Stream in = {{static_cast<const T *>(a.x), static_cast<const T *>(a.y), static_cast<const T *>(a.dout),
                  static_cast<const T *>(a.dz), row_gate ? static_cast<const T *>(a.gate) : nullptr},
                 {a.ldx, a.ldy, a.lddout, a.lddz, a.D}, D, tid, slots + threadIdx.x};
    float4 *post = reinterpret_cast<float4 *>(slots + Stream::SMEM / 16) + threadIdx.x;     // [ITEMS * 2][THREADS]
    const float inv = 1.0f / (float)D;
    const int shares = gridDim.x * TEAMS, mine = blockIdx.x * TEAMS + team;
    const long long first = share(a.M, shares, mine), last = share(a.M, shares, mine + 1);
    const long long first_group = first / a.per;
    long long group = first_group, group_end = (group + 1) * a.per;
    float sum_pre[ITEMS][8] = {}, sum_y[ITEMS][8] = {}, factor[ITEMS][8];
    if (!row_gate && first < last) team_factor<T>(a, in, group, factor);
    in.clear();
#pragma unroll
    for (int i = 0; i < STAGES; ++i) in.fetch(first + i, first + i < last, i);
#pragma unroll
    for (int i = 0; i < 2 * ITEMS; ++i) post[i * THREADS] = make_float4(0, 0, 0, 0);
    int stage = 0;
    for (long long m = first; m < last; ++m) {
        const float4 st = a.stats[m];
        uint4 words[ITEMS];
        if (a.y) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) words[i] = team_words(a, m, in.col(i));
        }
        in.arrived();
        if (row_gate) team_factor<T>(a, in, group, factor, 4, stage);
        float oh[ITEMS][8], yh[ITEMS][8], e[ITEMS][8];
        float s1 = 0.0f, s0 = 0.0f;
        const float shift_y = -st.x * st.y, shift_o = -st.z * st.w;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            in.get(stage, 0, i, oh[i]);
            // out again from the forward's inputs: exact, where the stored `out` is rounded
            if (a.y) {
                in.get(stage, 1, i, yh[i]);
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    yh[i][v] = fmaf(yh[i][v], st.y, shift_y);
                    oh[i][v] = fmaf(oh[i][v], a.alpha, kept(words[i], v, a.drop.below, yh[i][v] * factor[i][v]));
                }
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v) oh[i][v] *= a.alpha;
            }
            if (a.w_pre) {
                const int c = in.col(i);
                float w[8];
                in.get(stage, 3, i, e[i]);
                unpack8<T>(load8(static_cast<const T *>(a.w_pre) + (c < D ? c : 0)), w);
                if (c >= D) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) w[v] = oh[i][v] = e[i][v] = 0.0f;
                }
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    oh[i][v] = fmaf(oh[i][v], st.w, shift_o);
                    sum_pre[i][v] = fmaf(e[i][v], oh[i][v], sum_pre[i][v]);
                    e[i][v] *= w[v];
                    s1 = fmaf(e[i][v], oh[i][v], s1);
                }
                if (a.layer) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) s0 += e[i][v];
                }
            }
        }
        if (a.w_pre) {
            if (a.layer) {
                const float2 s = sums.sum(s1, s0);
                s1 = s.x * inv, s0 = s.y * inv;
            } else {
                s1 = sums.sum1(s1) * inv;
            }
        }
        float r1 = 0.0f, r0 = 0.0f;
        const float c1 = -s1 * st.w, c0 = -s0 * st.w;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = in.col(i);
            float t[8];
            if (a.dout) {
                in.get(stage, 2, i, t);
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v) t[v] = 0.0f;
            }
            if (a.w_pre) {
#pragma unroll
                for (int v = 0; v < 8; ++v) t[v] = fmaf(oh[i][v], c1, fmaf(e[i][v], st.w, t[v]));
                if (a.layer) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) t[v] += c0;
                }
            }
            if (a.dx && c < D) {
                float d[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) d[v] = a.alpha * t[v];
                store8(static_cast<T *>(a.dx) + m * a.lddx + c, pack8<T>(d));
            }
            if (a.y) {
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    t[v] = kept(words[i], v, a.drop.below, t[v]);
                    sum_y[i][v] = fmaf(t[v], kept(words[i], v, a.drop.below, yh[i][v]), sum_y[i][v]);
                    e[i][v] = t[v] * factor[i][v];
                }
                if (a.w_post && c < D) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) r1 = fmaf(e[i][v], yh[i][v], r1);
                    if (a.layer) {
#pragma unroll
                        for (int v = 0; v < 8; ++v) r0 += e[i][v];
                    }
                }
            }
        }
        const int here = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (!row_gate) in.fetch(m + STAGES, m + STAGES < last, here);      // this thread's slots are read
        if (!a.y) continue;
        if (a.w_post) {
            if (a.layer) {
                const float2 s = sums.sum(r1, r0);
                r1 = s.x * inv, r0 = s.y * inv;
            } else {
                r1 = sums.sum1(r1) * inv;
            }
            const float d1 = -r1 * st.y, d0 = -r0 * st.y;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < 8; ++v) e[i][v] = fmaf(yh[i][v], d1, fmaf(e[i][v], st.y, d0));
        }
        if (a.dy) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (in.col(i) < D) store8(static_cast<T *>(a.dy) + m * a.lddy + in.col(i), pack8<T>(e[i]));
        }
        if (m + 1 == last || m + 1 == group_end) {          // the last row of this gate row here
            const long long begin = group * a.per, end = min(group_end, a.M);
            const float scale = a.drop.cut ? a.drop.scale : 1.0f;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = in.col(i);
                if (c >= D) continue;
                float w[8], g[8];
                if (a.gate && a.dgate) {
                    if (a.w_post) {
                        unpack8<T>(load8(static_cast<const T *>(a.w_post) + c), w);
                    } else {
#pragma unroll
                        for (int v = 0; v < 8; ++v) w[v] = 1.0f;
                    }
#pragma unroll
                    for (int v = 0; v < 8; ++v) w[v] *= sum_y[i][v] * scale;
                    if (begin >= first && end <= last) {    // all its rows are this team's
                        if (a.grad_f32)
                            store8(static_cast<float *>(a.dgate) + group * a.D + c, pack8<float>(w));
                        else
                            store8(static_cast<T *>(a.dgate) + group * a.D + c, pack8<T>(w));
                    } else {
                        store8(a.partial + (2LL * gridDim.x + (group == first_group ? 0 : shares) + mine) * a.D + c,
                               pack8<float>(w));
                    }
                }
                if (a.w_post) {
                    if (row_gate) {
                        in.get(here, 4, i, g);
                    } else if (a.gate) {
                        unpack8<T>(load8(static_cast<const T *>(a.gate) + group * a.D + c), g);
                    } else {
#pragma unroll
                        for (int v = 0; v < 8; ++v) g[v] = 1.0f;
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float4 &to = post[(2 * i + q) * THREADS];
                        float4 p = to;
                        p.x = fmaf(g[4 * q], sum_y[i][4 * q] * scale, p.x);
                        p.y = fmaf(g[4 * q + 1], sum_y[i][4 * q + 1] * scale, p.y);
                        p.z = fmaf(g[4 * q + 2], sum_y[i][4 * q + 2] * scale, p.z);
                        p.w = fmaf(g[4 * q + 3], sum_y[i][4 * q + 3] * scale, p.w);
                        to = p;
                    }
                }
#pragma unroll
                for (int v = 0; v < 8; ++v) sum_y[i][v] = 0.0f;
            }
            ++group, group_end += a.per;
            if (m + 1 < last && !row_gate) team_factor<T>(a, in, group, factor);
        }
        if (row_gate) in.fetch(m + STAGES, m + STAGES < last, here);
    }
    if (first == last && a.gate && a.dgate) {       // a share without rows: its piece is read as part of its neighbours' gate row
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (in.col(i) < D) store8(a.partial + (2LL * gridDim.x + mine) * a.D + in.col(i), Eight<float>{});
    }
    // the block's teams add their columns, in order, in the slots' place
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float *block_sums = reinterpret_cast<float *>(slots);
    for (int which = 0; which < 2; ++which) {
        if (which == 0 ? !a.w_post : !a.w_pre) continue;
        float *to = a.partial + ((long long)which * gridDim.x + blockIdx.x) * a.D;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (in.col(i) < D) {
                if (which == 0) {
                    *reinterpret_cast<float4 *>(block_sums + team * D + in.col(i)) = post[2 * i * THREADS];
                    *reinterpret_cast<float4 *>(block_sums + team * D + in.col(i) + 4) = post[(2 * i + 1) * THREADS];
                } else {
                    store8(block_sums + team * D + in.col(i), pack8<float>(sum_pre[i]));
                }
            }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += THREADS) {
            float v = block_sums[c];
#pragma unroll
            for (int t = 1; t < TEAMS; ++t) v += block_sums[t * D + c];
            to[c] = v;
        }
    }
}

struct ColumnArgs {
    long long M, D, per, groups;
    int blocks, shares, grad_f32, f16;
    const float *partial;
    void *dw_post, *dw_pre, *dgate;
};

__device__ __forceinline__ void store_grad(void *p, long long i, float v, int f32, int f16) {
    if (f32)
        static_cast<float *>(p)[i] = v;
    else if (f16)
        static_cast<fp16 *>(p)[i] = from_f32<fp16>(v);
    else
        static_cast<bf16 *>(p)[i] = from_f32<bf16>(v);
}

// Sums of the partial columns, in a fixed order: a warp for 32 columns of a few partial rows, a block's 32 warps joined
// through shared memory.  A few MB from L2: 5 to 15 us, bound by latency.  blockIdx.y = 0: w_post, 1: w_pre, from 2 on:
// gate rows that were split
// between shares.
constexpr int COLUMN_PARTS = 32;
__global__ void __launch_bounds__(32 * COLUMN_PARTS) k_columns(const ColumnArgs a) {
    __shared__ float s[COLUMN_PARTS][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    // 32 warps share out the rows of partial sums: all to one parameter, or `ways` to each of several gate rows
    int ways = COLUMN_PARTS;
    const long long per_block = blockIdx.y < 2 ? 1 : min(a.groups, (long long)COLUMN_PARTS);
    while (ways * per_block > COLUMN_PARTS) ways >>= 1;
    const int slots = COLUMN_PARTS / ways, way = part % ways;
    void *to = blockIdx.y == 0 ? a.dw_post : blockIdx.y == 1 ? a.dw_pre : a.dgate;
    if (!to) return;
    for (long long g0 = blockIdx.y < 2 ? 0 : (blockIdx.y - 2LL) * slots; g0 < (blockIdx.y < 2 ? 1 : a.groups);
         g0 += blockIdx.y < 2 ? 1 : (gridDim.y - 2LL) * slots) {
        float v = 0.0f;
        bool own = true;
        if (blockIdx.y < 2) {
            const float *p = a.partial + (long long)blockIdx.y * a.blocks * a.D + c;
            if (c < a.D) {
#pragma unroll 4
                for (int b = way; b < a.blocks; b += COLUMN_PARTS) v += p[(long long)b * a.D];
            }
        } else {
            const long long g = g0 + part / ways;
            own = g < a.groups;
            if (own) {
                const long long begin = g * a.per, end = min(begin + a.per, a.M);
                // the share that holds a row: the last one that starts at or before it
                auto holder = [&](long long row) {
                    int b = (int)(row * a.shares / a.M);
                    while (b + 1 < a.shares && share(a.M, a.shares, b + 1) <= row) ++b;
                    while (b > 0 && share(a.M, a.shares, b) > row) --b;
                    return b;
                };
                const int b0 = holder(begin), b1 = holder(end - 1);
                own = b0 != b1;         // else one share's own, already written
                const float *p = a.partial + 2LL * a.blocks * a.D + c;
                if (own && c < a.D) {
                    // the first share's first or last piece, the others' first
                    if (way == 0) v = p[((share(a.M, a.shares, b0) / a.per == g ? 0LL : a.shares) + b0) * a.D];
#pragma unroll 4
                    for (int b = b0 + 1 + way; b <= b1; b += ways) v += p[(long long)b * a.D];
                }
            }
        }
        s[part][lane] = v;
        __syncthreads();
        if (way == 0 && own && c < a.D) {
            for (int i = 1; i < ways; ++i) v += s[part + i][lane];
            store_grad(to, (blockIdx.y < 2 ? 0 : (g0 + part / ways) * a.D) + c, v, a.grad_f32, a.f16);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ dropout
// One generator call for eight consecutive elements.  FAST: a thread reads and writes its eight as 16-byte vectors
// (contiguous rows are one long row, whose end may be ragged).  Otherwise a warp takes 256 elements, its lanes draw for
// eight each and then go through them 32 at a time, neighbouring lanes at neighbouring elements, wherever rows end.
// Bound by the bytes: 25.6 M words of binary32 in 34 us, 6.0 TB/s.
struct DropArgs {
    long long rows, cols, ldx, ldy;
    const void *x;
    void *y;
    Dropout drop;
};
template <class T, bool FAST>
__global__ void __launch_bounds__(256) k_dropout(const DropArgs a) {
    // counters c of the calls, from the first element's on; element numbers and so counters go round at 2^64 elements
    const unsigned long long n = (unsigned long long)a.rows * a.cols;
    const unsigned long long c0 = a.drop.offset >> 3, calls = ((a.drop.offset & 7) + n + 7) >> 3;
    const T *x = static_cast<const T *>(a.x);
    T *y = static_cast<T *>(a.y);
    if constexpr (FAST) {
        for (unsigned long long c = blockIdx.x * 256ull + threadIdx.x; c < calls; c += gridDim.x * 256ull) {
            const uint4 w = a.drop.cut ? drop_words(a.drop, (c0 + c) & COUNTERS) : make_uint4(~0u, ~0u, ~0u, ~0u);
            const unsigned long long e = c * 8;
            const long long m = a.rows == 1 ? 0 : (long long)(e / a.cols);
            const long long j = (long long)(e - (unsigned long long)m * a.cols);
            if (j + 8 <= a.cols) {
                float f[8];
                unpack8<T>(load8(x + m * a.ldx + j), f);
#pragma unroll
                for (int v = 0; v < 8; ++v) f[v] = kept(w, v, a.drop.below, f[v] * a.drop.scale);
                store8(y + m * a.ldy + j, pack8<T>(f));
            } else {
#pragma unroll
                for (int v = 0; v < 8; ++v)
                    if (j + v < a.cols) y[m * a.ldy + j + v] = from_f32<T>(kept(w, v, a.drop.below, to_f32<T>(x[m * a.ldx + j + v]) * a.drop.scale));
            }
        }
    } else {
        const int lane = threadIdx.x & 31;
        for (unsigned long long c = (blockIdx.x * 256ull + threadIdx.x) / 32 * 32; c < calls; c += gridDim.x * 256ull) {
            const uint32_t bits = a.drop.cut ? keep_bits(a.drop, (c0 + c + lane) & COUNTERS) : 0xFFu;
            const long long first = (long long)(c * 8) - (long long)(a.drop.offset & 7);    // may lie before the tensor
            const long long base = first > 0 ? first : 0;
            const long long m0 = base / a.cols, j0 = base - m0 * a.cols;
            T v[8];
            long long to[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {           // all loads before the first store
                const long long i = first + 32 * k + lane;
                to[k] = -1;
                if (i < 0 || i >= (long long)n) continue;
                long long m = m0, j = j0 + (i - base);
                if (j >= a.cols) {
                    const long long over = a.cols >= 256 ? 1 : j / a.cols;
                    m += over, j -= over * a.cols;
                }
                to[k] = m * a.ldy + j;
                v[k] = x[m * a.ldx + j];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t keep = __shfl_sync(~0u, bits, 4 * k + (lane >> 3)) >> (lane & 7) & 1;
                if (to[k] >= 0) y[to[k]] = from_f32<T>(keep ? to_f32<T>(v[k]) * a.drop.scale : 0.0f);
            }
        }
    }
}

// ------------------------------------------------------------------ launches
template <class F>
int by_type(int dtype, F f) {
    if (dtype == CCDC_F32) return f(float());
    if (dtype == CCDC_BF16) return f(bf16());
    return f(fp16());
}

bool rows16(const void *p, long long ld, int bytes) { return !p || (aligned_to(p, 16) && ld * bytes % 16 == 0); }

// Shares of the rows in the backward pass.  Teams: W warps of a 256-thread block (one of 16 warps alone), two blocks an
// SM; blocks: two an SM, three of up to 1024 columns.  A share costs a row of partial sums for each parameter, so it gets
// four rows at least.
int team_warps(long long D, int dtype) {
    const int cols = dtype == CCDC_F32 ? 256 : 512;         // of a warp
    int w = 1;
    while (w < 16 && w * cols < D) w *= 2;
    return w * cols >= D ? w : 0;
}
int row_shares(long long M, long long D, int dtype, bool teams, int sms) {
    const int w = teams ? team_warps(D, dtype) : 0;
    const int per_sm = w == 0 ? (D <= 1024 ? 3 : 2) : w == 16 ? 1 : 2 * (8 / w), block = w == 0 || w == 16 ? 1 : 8 / w;
    const long long most = (M + 3) / 4;
    const long long n = std::min<long long>((long long)per_sm * sms, std::max<long long>(1, most));
    return (int)((n + block - 1) / block * block);
}

template <class T, int VEC, int ITEMS, int THREADS>
int launch_forward(const NormArgs &a, cudaStream_t s) {
    const int blocks = (int)std::min<long long>(a.M, 1 << 20);
    k_residual_norm<T, VEC, ITEMS, THREADS><<<blocks, THREADS, 0, s>>>(a);
    return block_launch_status();
}
template <class T, int VEC, int ITEMS, int THREADS>
int launch_back(const NormArgs &a, int blocks, cudaStream_t s) {
    k_residual_norm_back<T, VEC, ITEMS, THREADS><<<blocks, THREADS, 0, s>>>(a);
    return block_launch_status();
}
template <class T, int W, bool BACK>
int launch_team(const NormArgs &a, int shares, cudaStream_t s) {
    constexpr int ITEMS = sizeof(T) == 4 ? 1 : 2, TEAMS = W == 16 ? 1 : 8 / W, THREADS = 32 * W * TEAMS;
    constexpr int SMEM = RowStream<T, ITEMS, W, THREADS, BACK ? 5 : 3, STAGES>::SMEM + (BACK ? ITEMS * 32 * THREADS : 0);
    auto *kernel = BACK ? k_norm_rows_back<T, ITEMS, W, TEAMS> : k_norm_rows<T, ITEMS, W, TEAMS>;
    static std::atomic<unsigned long long> done;
    const int rc = block_allow_smem(reinterpret_cast<const void *>(kernel), SMEM, &done);
    if (rc != CCDC_OK) return rc;
    kernel<<<shares / TEAMS, THREADS, SMEM, s>>>(a);
    return block_launch_status();
}
template <class T, bool BACK>
int launch_teams(const NormArgs &a, int w, int shares, cudaStream_t s) {
    return w == 1   ? launch_team<T, 1, BACK>(a, shares, s)
           : w == 2 ? launch_team<T, 2, BACK>(a, shares, s)
           : w == 4 ? launch_team<T, 4, BACK>(a, shares, s)
           : w == 8 ? launch_team<T, 8, BACK>(a, shares, s) : launch_team<T, 16, BACK>(a, shares, s);
}

template <class T>
int forward(const NormArgs &a, bool vec, int dtype, int sms, cudaStream_t s) {
    const int w = team_warps(a.D, dtype);
    if (vec && w && (a.drop.offset & 7) == 0) {
        const int block = w == 16 ? 1 : 8 / w;      // teams of a block; two blocks an SM, one of 16 warps
        const long long n = std::min<long long>((long long)(w == 16 ? 1 : 2) * block * sms, a.M);
        return launch_teams<T, false>(a, w, (int)((n + block - 1) / block * block), s);
    }
    if (vec) {
        if (a.D <= 1024) return launch_forward<T, 8, 1, 128>(a, s);
        if (a.D <= 8192) return launch_forward<T, 8, 2, 512>(a, s);
        return launch_forward<T, 8, 4, 1024>(a, s);
    }
    if (a.D <= 512) return launch_forward<T, 1, 4, 128>(a, s);
    if (a.D <= 1024) return launch_forward<T, 1, 8, 128>(a, s);
    if (a.D <= 2048) return launch_forward<T, 1, 8, 256>(a, s);
    if (a.D <= 4096) return launch_forward<T, 1, 8, 512>(a, s);
    if (a.D <= 8192) return launch_forward<T, 1, 16, 512>(a, s);
    return launch_forward<T, 1, 32, 1024>(a, s);
}
template <class T>
int backward(const NormArgs &a, bool vec, bool teams, int dtype, int shares, cudaStream_t s) {
    if (teams) return launch_teams<T, true>(a, team_warps(a.D, dtype), shares, s);
    if (vec) {
        if (a.D <= 1024) return launch_back<T, 8, 1, 128>(a, shares, s);
        if (a.D <= 8192) return launch_back<T, 8, 2, 512>(a, shares, s);
        return launch_back<T, 8, 4, 1024>(a, shares, s);
    }
    if (a.D <= 512) return launch_back<T, 1, 4, 128>(a, shares, s);
    if (a.D <= 1024) return launch_back<T, 1, 8, 128>(a, shares, s);
    if (a.D <= 2048) return launch_back<T, 1, 8, 256>(a, shares, s);
    if (a.D <= 4096) return launch_back<T, 1, 8, 512>(a, shares, s);
    if (a.D <= 8192) return launch_back<T, 1, 16, 512>(a, shares, s);
    return launch_back<T, 1, 32, 1024>(a, shares, s);
}

// what forward and backward check alike
int check_norm(long long M, long long D, int dtype, int kind, const void *x, long long ldx, const void *y, long long ldy,
               const void *w_post, const void *gate, long long per, float alpha, double p) {
    if (M < 0 || D < 1 || !is_float_type(dtype) || (kind != CCDC_NORM_RMS && kind != CCDC_NORM_LAYER)) return CCDC_EINVAL;
    if ((M > 0 && !x) || ldx < D || (y && ldy < D) || !(p >= 0.0 && p <= 1.0) || !(alpha == alpha)) return CCDC_EINVAL;
    if (!y && M > 0 && (w_post || gate || p != 0.0)) return CCDC_EINVAL;
    if (gate && per < 1) return CCDC_EINVAL;
    if (D > MAX_D || M > (1LL << 40)) return CCDC_ESIZE;
    return CCDC_OK;
}

}  // namespace

int block_sm_count(int *rc) {
    static std::atomic<int> known[64];          // a device's SM count does not change
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && dev < 64) sms = known[dev].load(std::memory_order_relaxed);
    if (e == cudaSuccess && !sms) {
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess && dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) {
        *rc = ccdc_internal_cuda_fail((int)e);
        return 0;
    }
    *rc = CCDC_OK;
    return sms;
}

int block_allow_smem(const void *kernel, int bytes, std::atomic<unsigned long long> *done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (e == cudaSuccess && (done->load(std::memory_order_relaxed) & bit)) return CCDC_OK;
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    done->fetch_or(bit, std::memory_order_relaxed);
    return CCDC_OK;
}

extern "C" {

int ccdc_residual_norm_forward(long long M, long long D, int dtype, int kind, float eps, const void *x, long long ldx,
                               const void *y, long long ldy, const void *w_post, const void *w_pre, const void *gate,
                               long long rows_per_gate, float alpha, double p, unsigned long long seed,
                               unsigned long long offset, void *out, long long ldo, void *z, long long ldz, void *stats,
                               void *stream) {
    int rc = check_norm(M, D, dtype, kind, x, ldx, y, ldy, w_post, gate, rows_per_gate, alpha, p);
    if (rc != CCDC_OK) return rc;
    if (!(eps >= 0.0f) || (M > 0 && ((out && ldo < D) || (z && ldz < D) || (!w_pre != !z) || (!out && !z))) ||
        !aligned_to(stats, 16))
        return CCDC_EINVAL;
    if (M == 0) return CCDC_OK;
    NormArgs a = {};
    a.M = M, a.D = D, a.x = x, a.y = y, a.w_post = w_post, a.w_pre = w_pre, a.gate = gate;
    a.ldx = ldx, a.ldy = ldy, a.per = gate ? std::min(rows_per_gate, M) : M, a.alpha = alpha, a.eps = eps;
    a.layer = kind == CCDC_NORM_LAYER, a.out = out, a.ldo = ldo, a.z = z, a.ldz = ldz, a.stats = static_cast<float4 *>(stats);
    make_dropout(p, seed, offset, &a.drop);
    const int b = type_bytes(dtype);
    const bool vec = D % 8 == 0 && rows16(x, ldx, b) && rows16(y, ldy, b) && rows16(w_post, D, b) && rows16(w_pre, D, b) &&
                     rows16(gate, D, b) && rows16(out, ldo, b) && rows16(z, ldz, b);
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    return by_type(dtype, [&](auto t) { return forward<decltype(t)>(a, vec, dtype, sms, static_cast<cudaStream_t>(stream)); });
}

size_t ccdc_residual_norm_workspace_bytes(long long M, long long D) {
    if (M < 0 || D < 1 || D > MAX_D) return 0;
    int rc;
    int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) sms = 148;
    // the form that a call takes depends on its tensors: the most that any takes
    int shares = row_shares(M, D, CCDC_F32, false, sms);
    for (int dtype : {CCDC_F32, CCDC_BF16})
        if (team_warps(D, dtype)) shares = std::max(shares, row_shares(M, D, dtype, true, sms));
    return (size_t)4 * shares * round_up((size_t)D, 8) * sizeof(float);
}

int ccdc_residual_norm_backward(long long M, long long D, int dtype, int grad_dtype, int kind, const void *dout,
                                long long lddout, const void *dz, long long lddz, const void *x, long long ldx,
                                const void *y, long long ldy, const void *stats, const void *w_post, const void *w_pre,
                                const void *gate, long long rows_per_gate, float alpha, double p, unsigned long long seed,
                                unsigned long long offset, void *dx, long long lddx, void *dy, long long lddy,
                                void *dw_post, void *dw_pre, void *dgate, void *workspace, size_t workspace_bytes,
                                void *stream) {
    int rc = check_norm(M, D, dtype, kind, x, ldx, y, ldy, w_post, gate, rows_per_gate, alpha, p);
    if (rc != CCDC_OK) return rc;
    if ((grad_dtype != dtype && grad_dtype != CCDC_F32) || (dout && lddout < D) || (dz && lddz < D) || (dx && lddx < D) ||
        (dy && lddy < D))
        return CCDC_EINVAL;
    if (M > 0 && (!stats || (!dout && !dz) || (!dz != !w_pre) || (dy && !y))) return CCDC_EINVAL;
    if ((dw_post && !w_post) || (dw_pre && !w_pre) || (dgate && !gate) || !aligned_to(stats, 16)) return CCDC_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0) {       // no rows: the parameters' gradients are sums over nothing (a gate keeps one row)
        const size_t n = (size_t)D * type_bytes(grad_dtype);
        for (void *g : {dw_post, dw_pre, dgate})
            if (g) {
                const cudaError_t e = cudaMemsetAsync(g, 0, n, s);
                if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
            }
        return CCDC_OK;
    }
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    if (!workspace || !aligned_to(workspace, 16) || workspace_bytes < ccdc_residual_norm_workspace_bytes(M, D))
        return CCDC_EINVAL;
    NormArgs a = {};
    a.M = M, a.D = D, a.x = x, a.y = y, a.w_post = w_post, a.w_pre = w_pre, a.gate = gate;
    a.ldx = ldx, a.ldy = ldy, a.per = gate ? std::min(rows_per_gate, M) : M, a.alpha = alpha;
    a.layer = kind == CCDC_NORM_LAYER, a.stats = const_cast<float4 *>(static_cast<const float4 *>(stats));
    a.dout = dout, a.lddout = lddout, a.dz = dz, a.lddz = lddz, a.dx = dx, a.lddx = lddx, a.dy = dy, a.lddy = lddy;
    a.dgate = dgate, a.grad_f32 = grad_dtype == CCDC_F32, a.partial = static_cast<float *>(workspace);
    make_dropout(p, seed, offset, &a.drop);
    const int b = type_bytes(dtype), gb = type_bytes(grad_dtype);
    const bool vec = D % 8 == 0 && rows16(x, ldx, b) && rows16(y, ldy, b) && rows16(w_post, D, b) && rows16(w_pre, D, b) &&
                     rows16(gate, D, b) && rows16(dout, lddout, b) && rows16(dz, lddz, b) && rows16(dx, lddx, b) &&
                     rows16(dy, lddy, b) && rows16(dgate, D, gb);
    const bool teams = vec && team_warps(D, dtype) && offset % 8 == 0;
    const int blocks = row_shares(M, D, dtype, teams, sms);
    rc = by_type(dtype, [&](auto t) { return backward<decltype(t)>(a, vec, teams, dtype, blocks, s); });
    if (rc != CCDC_OK) return rc;
    const bool split_gate = dgate && a.per > 1;
    if (!dw_post && !dw_pre && !split_gate) return CCDC_OK;
    const int w = teams ? team_warps(D, dtype) : 16;
    ColumnArgs c = {M, D, a.per, split_gate ? (M + a.per - 1) / a.per : 0, blocks / (w == 16 ? 1 : 8 / w), blocks, a.grad_f32, dtype == CCDC_F16, a.partial,
                    dw_post, dw_pre, dgate};
    const dim3 grid((unsigned)((D + 31) / 32), (unsigned)(2 + std::min<long long>((c.groups + 31) / 32, 1024)));
    k_columns<<<grid, 32 * COLUMN_PARTS, 0, s>>>(c);
    return block_launch_status();
}

int ccdc_dropout(long long rows, long long cols, int dtype, const void *x, long long ldx, void *y, long long ldy, double p,
                 unsigned long long seed, unsigned long long offset, void *stream) {
    if (rows < 0 || cols < 0 || !is_float_type(dtype)) return CCDC_EINVAL;
    DropArgs a = {rows, cols, ldx, ldy, x, y, {}};
    if (!make_dropout(p, seed, offset, &a.drop)) return CCDC_EINVAL;
    if (rows == 0 || cols == 0) return CCDC_OK;
    if (!x || !y || ldx < cols || ldy < cols) return CCDC_EINVAL;
    if (rows > (1LL << 46) / cols) return CCDC_ESIZE;
    int rc;
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    const int b = type_bytes(dtype);
    if (rows > 1 && ldx == cols && ldy == cols) a.cols = rows * cols, a.rows = 1, a.ldx = a.ldy = a.cols;
    const bool fast = (a.rows == 1 || a.cols % 8 == 0) && offset % 8 == 0 && aligned_to(x, 16) && aligned_to(y, 16) &&
                      (a.rows == 1 || (rows16(x, ldx, b) && rows16(y, ldy, b)));
    const long long calls = (rows * cols + 14) / 8;
    const int blocks = (int)std::min<long long>((calls + 255) / 256, 64LL * sms);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (fast)
            k_dropout<T, true><<<blocks, 256, 0, s>>>(a);
        else
            k_dropout<T, false><<<blocks, 256, 0, s>>>(a);
        return 0;
    });
    return block_launch_status();
}

}  // extern "C"
