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
// One block owns a row: its columns stay in registers between the passes over them, so every tensor is read
// once and written once.  The sums over rows (w_post, w_pre, gate) are held per column in registers while a
// block walks a contiguous range of rows, and meet through the workspace in block order: no atomics, so that
// a file's gradients have the same bits at every node that maps it.
#include <algorithm>

#include "ccdc_block.h"

namespace {

constexpr long long MAX_D = 32768;      // columns of a row that fit a block's registers

struct NormArgs {
    long long M, D;
    const void *x, *y, *w_post, *w_pre, *gate;
    long long ldx, ldy, per;            // per: rows that share a gate row
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
    float *partial;                     // [4][blocks][D]: w_post, w_pre, first and last piece of a split gate row
};

// first row of block b's share
__host__ __device__ __forceinline__ long long share(long long M, int blocks, int b) { return M * b / blocks; }

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
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) a += s[i].x, b += s[i].y;
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
            keep[i] = c < D ? keep_bits(a.drop.seed, (e0 + c) >> 3, a.drop.cut) : 0;
        }
        return;
    }
    const int shift = (int)(e0 & 7), n = (shift + D + 7) >> 3;
    for (int j = threadIdx.x; j < n; j += THREADS) bytes[j] = (uint8_t)keep_bits(a.drop.seed, (e0 >> 3) + j, a.drop.cut);
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
        const float4 st = a.stats[m];
        float oh[ITEMS][VEC], yh[ITEMS][VEC], cg[ITEMS][VEC], t[ITEMS][VEC];
        R::load(static_cast<const T *>(a.x) + m * a.ldx, D, oh);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int v = 0; v < VEC; ++v) oh[i][v] *= a.alpha, cg[i][v] = 1.0f, yh[i][v] = 0.0f;
        if (a.y) {
            R::load(static_cast<const T *>(a.y) + m * a.ldy, D, yh);
            if (a.drop.cut) {
                uint32_t keep[ITEMS];
                row_keep<VEC, ITEMS, THREADS>(a, m, keep, bytes[parity]);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int v = 0; v < VEC; ++v) cg[i][v] = (keep[i] >> v & 1) ? a.drop.scale : 0.0f;
            }
        }
        float w_post[ITEMS][VEC], gate[ITEMS][VEC];
        if (a.w_post) {
            R::load(static_cast<const T *>(a.w_post), D, w_post);
        }
        if (a.gate) R::load(static_cast<const T *>(a.gate) + m / a.per * a.D, D, gate);
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
        if (a.dout) {
            R::load(static_cast<const T *>(a.dout) + m * a.lddout, D, t);
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int v = 0; v < VEC; ++v) t[i][v] = 0.0f;
        }
        if (a.w_pre) {
            float e[ITEMS][VEC], w[ITEMS][VEC];
            R::load(static_cast<const T *>(a.dz) + m * a.lddz, D, e);
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

struct ColumnArgs {
    long long M, D, per, groups;
    int blocks, grad_f32, f16;
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

// Sums of the blocks' partial columns in block order.  blockIdx.y = 0: w_post, 1: w_pre, 2 + g: gate row g,
// where it was split between blocks.
__global__ void __launch_bounds__(256) k_columns(const ColumnArgs a) {
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    for (long long y = blockIdx.y; y < 2 + a.groups; y += gridDim.y) {
        int b0 = 0, b1 = a.blocks;
        const long long g = y - 2;
        void *to = y == 0 ? a.dw_post : y == 1 ? a.dw_pre : a.dgate;
        if (!to) continue;
        if (y >= 2) {
            const long long begin = g * a.per, end = min(begin + a.per, a.M);
            // the block that holds a row: the last one that starts at or before it
            auto holder = [&](long long row) {
                int b = (int)(row * a.blocks / a.M);
                while (b + 1 < a.blocks && share(a.M, a.blocks, b + 1) <= row) ++b;
                while (b > 0 && share(a.M, a.blocks, b) > row) --b;
                return b;
            };
            b0 = holder(begin), b1 = holder(end - 1) + 1;
            if (b1 - b0 == 1) continue;     // one block's own, already written
        }
        float v = 0.0f;
        if (c < a.D)
            for (int b = b0 + part; b < b1; b += 8) {
                const long long slot = y < 2 ? y : share(a.M, a.blocks, b) / a.per == g ? 2 : 3;
                v += a.partial[(slot * a.blocks + b) * a.D + c];
            }
        s[part][lane] = v;
        __syncthreads();
        if (part == 0 && c < a.D) {
#pragma unroll
            for (int i = 1; i < 8; ++i) v += s[i][lane];
            store_grad(to, (y < 2 ? 0 : g * a.D) + c, v, a.grad_f32, a.f16);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ dropout
// Eight elements, one generator call, a thread.  `fast`: rows are read as 16-byte vectors (contiguous rows are
// one long row); otherwise a thread's eight elements may cross a row's end and go one by one.
struct DropArgs {
    long long rows, cols, ldx, ldy;
    const void *x;
    void *y;
    Dropout drop;
};
template <class T, bool FAST>
__global__ void __launch_bounds__(256) k_dropout(const DropArgs a) {
    const unsigned long long n = (unsigned long long)a.rows * a.cols;
    const unsigned long long c0 = a.drop.offset >> 3, c1 = (a.drop.offset + n + 7) >> 3;
    for (unsigned long long c = c0 + blockIdx.x * 256ull + threadIdx.x; c < c1; c += gridDim.x * 256ull) {
        const uint32_t bits = a.drop.cut ? keep_bits(a.drop.seed, c, a.drop.cut) : 0xFFu;
        if constexpr (FAST) {
            const unsigned long long e = (c - c0) * 8;
            const long long m = a.rows == 1 ? 0 : (long long)(e / a.cols);
            const long long j = (long long)(e - (unsigned long long)m * a.cols);
            float f[8];
            unpack8<T>(load8(static_cast<const T *>(a.x) + m * a.ldx + j), f);
#pragma unroll
            for (int v = 0; v < 8; ++v) f[v] = (bits >> v & 1) ? f[v] * a.drop.scale : 0.0f;
            store8(static_cast<T *>(a.y) + m * a.ldy + j, pack8<T>(f));
        } else {
            for (int v = 0; v < 8; ++v) {
                const unsigned long long e = c * 8 + v;
                if (e < a.drop.offset || e - a.drop.offset >= n) continue;
                const long long i = (long long)(e - a.drop.offset), m = i / a.cols, j = i - m * a.cols;
                const float f = to_f32<T>(static_cast<const T *>(a.x)[m * a.ldx + j]);
                static_cast<T *>(a.y)[m * a.ldy + j] = from_f32<T>((bits >> v & 1) ? f * a.drop.scale : 0.0f);
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

int back_blocks(long long M, long long D, int sms) { return (int)std::min<long long>(M, 2LL * sms); }

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

template <class T>
int forward(const NormArgs &a, bool vec, cudaStream_t s) {
    if (vec) {
        if (a.D <= 256) return launch_forward<T, 8, 1, 32>(a, s);
        if (a.D <= 1024) return launch_forward<T, 8, 1, 128>(a, s);
        if (a.D <= 4096) return launch_forward<T, 8, 2, 256>(a, s);
        if (a.D <= 8192) return launch_forward<T, 8, 2, 512>(a, s);
        if (a.D <= 16384) return launch_forward<T, 8, 4, 512>(a, s);
        return launch_forward<T, 8, 4, 1024>(a, s);
    }
    if (a.D <= 512) return launch_forward<T, 1, 4, 128>(a, s);
    if (a.D <= 2048) return launch_forward<T, 1, 8, 256>(a, s);
    if (a.D <= 8192) return launch_forward<T, 1, 16, 512>(a, s);
    return launch_forward<T, 1, 32, 1024>(a, s);
}
template <class T>
int backward(const NormArgs &a, bool vec, int blocks, cudaStream_t s) {
    if (vec) {
        if (a.D <= 256) return launch_back<T, 8, 1, 32>(a, blocks, s);
        if (a.D <= 1024) return launch_back<T, 8, 1, 128>(a, blocks, s);
        if (a.D <= 4096) return launch_back<T, 8, 1, 512>(a, blocks, s);
        if (a.D <= 8192) return launch_back<T, 8, 2, 512>(a, blocks, s);
        if (a.D <= 16384) return launch_back<T, 8, 4, 512>(a, blocks, s);
        return launch_back<T, 8, 4, 1024>(a, blocks, s);
    }
    if (a.D <= 512) return launch_back<T, 1, 4, 128>(a, blocks, s);
    if (a.D <= 2048) return launch_back<T, 1, 8, 256>(a, blocks, s);
    if (a.D <= 8192) return launch_back<T, 1, 16, 512>(a, blocks, s);
    return launch_back<T, 1, 32, 1024>(a, blocks, s);
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
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) {
        *rc = ccdc_internal_cuda_fail((int)e);
        return 0;
    }
    *rc = CCDC_OK;
    return sms;
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
    a.ldx = ldx, a.ldy = ldy, a.per = gate ? rows_per_gate : M, a.alpha = alpha, a.eps = eps;
    a.layer = kind == CCDC_NORM_LAYER, a.out = out, a.ldo = ldo, a.z = z, a.ldz = ldz, a.stats = static_cast<float4 *>(stats);
    make_dropout(p, seed, offset, &a.drop);
    const int b = type_bytes(dtype);
    const bool vec = D % 8 == 0 && rows16(x, ldx, b) && rows16(y, ldy, b) && rows16(w_post, D, b) && rows16(w_pre, D, b) &&
                     rows16(gate, D, b) && rows16(out, ldo, b) && rows16(z, ldz, b);
    return by_type(dtype, [&](auto t) { return forward<decltype(t)>(a, vec, static_cast<cudaStream_t>(stream)); });
}

size_t ccdc_residual_norm_workspace_bytes(long long M, long long D) {
    if (M < 0 || D < 1 || D > MAX_D) return 0;
    int rc;
    const int sms = block_sm_count(&rc);
    return (size_t)4 * back_blocks(M, D, rc == CCDC_OK ? sms : 148) * round_up((size_t)D, 8) * sizeof(float);
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
    a.ldx = ldx, a.ldy = ldy, a.per = gate ? rows_per_gate : M, a.alpha = alpha;
    a.layer = kind == CCDC_NORM_LAYER, a.stats = const_cast<float4 *>(static_cast<const float4 *>(stats));
    a.dout = dout, a.lddout = lddout, a.dz = dz, a.lddz = lddz, a.dx = dx, a.lddx = lddx, a.dy = dy, a.lddy = lddy;
    a.dgate = dgate, a.grad_f32 = grad_dtype == CCDC_F32, a.partial = static_cast<float *>(workspace);
    make_dropout(p, seed, offset, &a.drop);
    const int b = type_bytes(dtype), gb = type_bytes(grad_dtype);
    const bool vec = D % 8 == 0 && rows16(x, ldx, b) && rows16(y, ldy, b) && rows16(w_post, D, b) && rows16(w_pre, D, b) &&
                     rows16(gate, D, b) && rows16(dout, lddout, b) && rows16(dz, lddz, b) && rows16(dx, lddx, b) &&
                     rows16(dy, lddy, b) && rows16(dgate, D, gb);
    const int blocks = back_blocks(M, D, sms);
    rc = by_type(dtype, [&](auto t) { return backward<decltype(t)>(a, vec, blocks, s); });
    if (rc != CCDC_OK) return rc;
    const bool split_gate = dgate && a.per > 1;
    if (!dw_post && !dw_pre && !split_gate) return CCDC_OK;
    ColumnArgs c = {M, D, a.per, split_gate ? (M + a.per - 1) / a.per : 0, blocks, a.grad_f32, dtype == CCDC_F16, a.partial,
                    dw_post, dw_pre, dgate};
    const dim3 grid((unsigned)((D + 31) / 32), (unsigned)std::min<long long>(2 + c.groups, 1024));
    k_columns<<<grid, 256, 0, s>>>(c);
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
    const bool fast = a.cols % 8 == 0 && offset % 8 == 0 && aligned_to(x, 16) && aligned_to(y, 16) &&
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
