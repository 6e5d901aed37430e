// Distillation loss from a teacher's top logits, and its gradient.
//
// Row m has the student's logits z[V] and k of the teacher's (values v_j at ids_j).  At temperature T
//     t_j  = softmax(v / T) over the slots that are there, or exp(v_j / T - lse) with the whole teacher's lse
//     loss = sum_j t_j (log t_j - log s_id(j)),  s = softmax(z / T)
//     dz   = dloss / T (P s - t),  P = sum_j t_j
// Reading z is all the work: a block takes a row, each thread keeps a running maximum and sum, and a second walk over
// the same row (which L2 still holds) writes the gradient.  The k terms are computed in 64 bits.
#include "ccdc_block.h"

#include <algorithm>

namespace {

constexpr int MAX_TOP = 1024;

struct DistillArgs {
    long long M, V, ldz, lddz;
    int k, id_bytes, values_f32;
    const void *z, *ids, *values;
    const float *lse, *dloss;
    float *loss;
    float2 *stats;              // the row's maximum and the sum of exponentials above it
    void *dz;
    double inv_t;
    float scale;                // log2(e) / T
};

template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

// exp of z / T above the maximum's; 16-bit logits by the approximate exponential (2^-22), which their rounding hides
template <class T>
__device__ __forceinline__ float above(float z, float top, float scale) {
    const float d = (z - top) * scale;      // the difference first: no product of a masked row's lowest value overflows
    if constexpr (sizeof(T) == 4) return exp2f(d);
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d));
    return e;
}
struct Running {
    float top, sum;
};
// the sum's factor when its maximum rises from `from` to `to` (a sum of nothing has -inf)
template <class T>
__device__ __forceinline__ float rebase(float from, float to, float scale) {
    return from == to ? 1.0f : above<T>(from, to, scale);
}
template <class T>
__device__ __forceinline__ Running join(Running a, Running b, float scale) {
    const float top = fmaxf(a.top, b.top);
    return {top, a.sum * rebase<T>(a.top, top, scale) + b.sum * rebase<T>(b.top, top, scale)};
}
template <class T, int COUNT>
__device__ __forceinline__ void add(Running &r, const float (&f)[COUNT], float scale) {
    float top = r.top;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) top = fmaxf(top, f[i]);
    // all -inf so far (or NaN, which fmax leaves out): count from zero, so that -inf adds nothing and NaN stays NaN
    const float from = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) sum += above<T>(f[i], from, scale);
    r.sum = r.sum * rebase<T>(r.top, top, scale) + sum;
    r.top = top;
}

template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double *part) {
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(~0u, v, d);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) s += part[w];
    __syncthreads();
    return s;
}
template <int THREADS>
__device__ __forceinline__ double block_max(double v, double *part) {
#pragma unroll
    for (int d = 16; d; d /= 2) v = fmax(v, __shfl_xor_sync(~0u, v, d));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) s = fmax(s, part[w]);
    __syncthreads();
    return s;
}

// LOSS: computes the statistics, writes loss and (where asked) stats.  GRAD: writes dz, from stats without LOSS.
template <class T, bool LOSS, bool GRAD, int THREADS>
__global__ void __launch_bounds__(THREADS) k_distill(DistillArgs a) {
    constexpr int N = 16 / sizeof(T), AHEAD = 4;
    __shared__ int at[MAX_TOP];             // where the teacher's slots point; -1: not there
    __shared__ double target[MAX_TOP];      // v_j, then t_j
    __shared__ float chosen[MAX_TOP];       // z there, before dz may overwrite it
    __shared__ double part[THREADS / 32];
    __shared__ Running runs[THREADS / 32];
    const int tid = threadIdx.x;
    for (long long m = blockIdx.x; m < a.M; m += gridDim.x) {
        const T *z = static_cast<const T *>(a.z) + m * a.ldz;
        // the teacher's side
        double top = -INFINITY;
        bool mine = false;
        for (int j = tid; j < a.k; j += THREADS) {
            const long long id = a.id_bytes == 8 ? static_cast<const long long *>(a.ids)[m * a.k + j]
                                                 : static_cast<const int *>(a.ids)[m * a.k + j];
            const float v = a.values_f32 ? static_cast<const float *>(a.values)[m * a.k + j]
                                         : to_f32<T>(static_cast<const T *>(a.values)[m * a.k + j]);
            const bool there = id >= 0 && id < a.V && v != -INFINITY;
            at[j] = there ? (int)id : -1;
            target[j] = v;
            chosen[j] = there ? to_f32<T>(z[id]) : 0.0f;
            mine = mine || there;
            if (there) top = fmax(top, (double)v);
        }
        const bool any = __syncthreads_or(mine);
        double log_whole = 0.0, P = 0.0;
        if (any) {
            if (a.lse) {
                log_whole = a.lse[m];
            } else {
                top = block_max<THREADS>(top, part);
                double sum = 0.0;
                for (int j = tid; j < a.k; j += THREADS)
                    if (at[j] >= 0) sum += exp((target[j] - top) * a.inv_t);
                log_whole = top * a.inv_t + log(block_sum<THREADS>(sum, part));
            }
        }
        // t log t and P
        double entropy = 0.0;
        for (int j = tid; j < a.k; j += THREADS) {
            double t = 0.0;
            if (at[j] >= 0) {
                const double log_t = target[j] * a.inv_t - log_whole;
                t = exp(log_t);
                if (t != 0.0) entropy += t * log_t;
            }
            target[j] = t;
            P += t;
        }
        P = any ? block_sum<THREADS>(P, part) : 0.0;
        if (P == 0.0) {                 // a row without targets: padding
            if (LOSS && tid == 0) {
                a.loss[m] = 0.0f;
                if (a.stats) a.stats[m] = make_float2(0.0f, 1.0f);
            }
            if (GRAD) {
                T *dz = static_cast<T *>(a.dz) + m * a.lddz;
                for (long long i = tid; i < a.V; i += THREADS) dz[i] = from_f32<T>(0.0f);
            }
            __syncthreads();
            continue;
        }
        // the row starts anywhere: a head up to a 16-byte boundary, vectors, a tail
        const int head = (int)min(a.V, (long long)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (long long)sizeof(T));
        const long long packs = (a.V - head) / N;
        const int tail = (int)(a.V - head - packs * N);
        const Pack<T, N> *body = reinterpret_cast<const Pack<T, N> *>(z + head);
        const long long rim = tid < head ? tid : tid < head + tail ? head + packs * N + (tid - head) : -1;     // head + tail < THREADS
        Running r = {-INFINITY, 0.0f};
        if constexpr (LOSS) {
            if (rim >= 0) {
                const float f[1] = {to_f32<T>(z[rim])};
                add<T>(r, f, a.scale);
            }
            long long i = tid;
            for (; i + (AHEAD - 1) * THREADS < packs; i += AHEAD * THREADS) {
                Pack<T, N> v[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) v[u] = body[i + u * THREADS];
                float f[AHEAD * N];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                    for (int n = 0; n < N; ++n) f[u * N + n] = to_f32<T>(v[u].v[n]);
                add<T>(r, f, a.scale);
            }
            for (; i < packs; i += THREADS) {
                const Pack<T, N> v = body[i];
                float f[N];
#pragma unroll
                for (int n = 0; n < N; ++n) f[n] = to_f32<T>(v.v[n]);
                add<T>(r, f, a.scale);
            }
#pragma unroll
            for (int d = 1; d < 32; d *= 2)
                r = join<T>(r, {__shfl_xor_sync(~0u, r.top, d), __shfl_xor_sync(~0u, r.sum, d)}, a.scale);
            if ((tid & 31) == 0) runs[tid >> 5] = r;
            __syncthreads();
            r = runs[0];
#pragma unroll 1
            for (int w = 1; w < THREADS / 32; ++w) r = join<T>(r, runs[w], a.scale);
        } else {
            const float2 s = a.stats[m];
            r = {s.x, s.y};
        }
        const float from = r.top == -INFINITY ? 0.0f : r.top;
        if constexpr (LOSS) {
            const double log_sum = log((double)r.sum);
            double cross = 0.0;
            for (int j = tid; j < a.k; j += THREADS)
                if (at[j] >= 0 && target[j] != 0.0)
                    cross += target[j] * (((double)chosen[j] - (double)from) * (double)a.scale * 0.6931471805599453 - log_sum);
            const double loss = block_sum<THREADS>(entropy - cross, part);
            if (tid == 0) {
                a.loss[m] = (float)loss;
                if (a.stats) a.stats[m] = make_float2(r.top, r.sum);
            }
        }
        if constexpr (GRAD) {
            const float c = a.dloss[m] * (float)a.inv_t, cs = (float)((double)a.dloss[m] * a.inv_t * P / (double)r.sum);
            T *dz = static_cast<T *>(a.dz) + m * a.lddz;
            if (rim >= 0) dz[rim] = from_f32<T>(cs * above<T>(to_f32<T>(z[rim]), from, a.scale));
            const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
            Pack<T, N> *out = reinterpret_cast<Pack<T, N> *>(dz + head);
#pragma unroll 4
            for (long long i = tid; i < packs; i += THREADS) {
                Pack<T, N> v = body[i];
#pragma unroll
                for (int n = 0; n < N; ++n) v.v[n] = from_f32<T>(cs * above<T>(to_f32<T>(v.v[n]), from, a.scale));
                if (alike)
                    out[i] = v;
                else
#pragma unroll
                    for (int n = 0; n < N; ++n) dz[head + i * N + n] = v.v[n];
            }
            __syncthreads();            // the targets' elements are written again
            for (int j = tid; j < a.k; j += THREADS) {
                if (at[j] < 0) continue;
                double t = 0.0;         // the slots that name this element add up; the first of them writes it
                bool first = true;
                for (int i = 0; i < a.k; ++i)
                    if (at[i] == at[j]) {
                        if (i < j) first = false;
                        t += target[i];
                    }
                if (first) dz[at[j]] = from_f32<T>(fmaf(-c, (float)t, cs * above<T>(chosen[j], from, a.scale)));
            }
        }
        __syncthreads();
    }
}

template <class T, bool LOSS, bool GRAD>
int launch(const DistillArgs &a, cudaStream_t s) {
    int rc;
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    constexpr int THREADS = 512;
    k_distill<T, LOSS, GRAD, THREADS><<<(unsigned)std::min<long long>(a.M, 2LL * sms), THREADS, 0, s>>>(a);
    return block_launch_status();
}
template <bool LOSS, bool GRAD>
int by_type(const DistillArgs &a, int dtype, cudaStream_t s) {
    return dtype == CCDC_F32    ? launch<float, LOSS, GRAD>(a, s)
           : dtype == CCDC_BF16 ? launch<bf16, LOSS, GRAD>(a, s) : launch<fp16, LOSS, GRAD>(a, s);
}

}  // namespace

extern "C" {

int ccdc_distill(long long M, long long V, int k, int dtype, const void *logits, long long ldz, int id_bytes, const void *ids,
                 int value_dtype, const void *values, const float *teacher_lse, float temperature, const float *dloss, float *loss,
                 void *stats, void *dlogits, long long lddz, void *stream) {
    if (M < 0 || V < 1 || k < 1 || !is_float_type(dtype) || (value_dtype != dtype && value_dtype != CCDC_F32) ||
        (id_bytes != 4 && id_bytes != 8) || !(temperature >= 1e-6f && temperature <= 1e6f))
        return CCDC_EINVAL;
    if (V > 0x7FFFFFFF || k > MAX_TOP) return CCDC_ESIZE;
    if (M == 0) return CCDC_OK;
    if (!logits || ldz < V || !ids || !aligned_to(ids, id_bytes) || !values || !aligned_to(stats, 8)) return CCDC_EINVAL;
    if (dlogits ? !dloss || lddz < V || (!loss && !stats) : !loss) return CCDC_EINVAL;
    DistillArgs a = {};
    a.M = M, a.V = V, a.ldz = ldz, a.lddz = lddz, a.k = k, a.id_bytes = id_bytes, a.values_f32 = value_dtype == CCDC_F32;
    a.z = logits, a.ids = ids, a.values = values, a.lse = teacher_lse, a.dloss = dloss, a.loss = loss;
    a.stats = static_cast<float2 *>(stats), a.dz = dlogits;
    a.inv_t = 1.0 / (double)temperature, a.scale = (float)(1.4426950408889634 / (double)temperature);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return !dlogits ? by_type<true, false>(a, dtype, s) : loss ? by_type<true, true>(a, dtype, s) : by_type<false, true>(a, dtype, s);
}

}  // extern "C"
