// Distillation loss from a teacher's top logits, and its gradient.
//
// Row m has the student's logits z[V] and k of the teacher's (values v_j at ids_j).  At temperature T
//     t_j  = softmax(v / T) over the slots that are there, or exp(v_j / T - lse) with the whole teacher's lse
//     loss = sum_j t_j (log t_j - log s_id(j)),  s = softmax(z / T)
//     dz   = dloss / T (P s - t),  P = sum_j t_j
// Reading z and writing dz is all the work.  A row belongs to one block or to the blocks of a cluster, which keep it in shared
// memory between the walk for maximum and sum and the walk that writes the gradient: z is read from memory once.  Parts are
// small enough for several blocks an SM, so that one row's loads run under another's stores.  Each thread copies 16-byte pieces
// asynchronously and reads only its own, so nothing waits but for them; the blocks of a cluster exchange their maxima and sums.
// The last warp of a block computes the k terms meanwhile, in 64 bits.  Exponentials are the next bound (two for each element).
#include "ccdc_block.h"

#include <algorithm>

namespace {

constexpr int MAX_TOP = 1024, MAX_CLUSTER = 8;
constexpr int AHEAD = 4;                    // slots a lane
constexpr int GROUPS = 4;                   // of copies that are waited for one after the other
constexpr int SMALL_PART = 8 << 10;         // bytes of a row that 64 threads take; more take 256
constexpr int PART = 64 << 10;              // bytes of a part that leave room for three blocks an SM
constexpr int MOST_PART = 192 << 10;

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
    int part_pieces, table;     // room of a block, in pieces of 16 bytes; of the table of ids
};

template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// 16-bit logits by the approximate exponential (2^-22), which their rounding hides
template <class T>
__device__ __forceinline__ float power(float x) {
    if constexpr (sizeof(T) == 4) return exp2f(x);
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}
// exp of z / T above the maximum's.  The difference first: no product of a masked row's lowest value overflows.
template <class T>
__device__ __forceinline__ float above(float z, float top, float scale) {
    return power<T>((z - top) * scale);
}
template <class T>
__device__ __forceinline__ float2 above2(float2 z, float top, float scale) {
    const float2 d = mul2(add2(z, make_float2(-top, -top)), make_float2(scale, scale));
    return make_float2(power<T>(d.x), power<T>(d.y));
}
// the eight (binary32: four) values of a piece of 16 bytes, two by two
template <class T>
__device__ __forceinline__ void values_of(const uint4 &v, float2 (&f)[8 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
        f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
    } else {
        f[0] = unpack2<T>(v.x), f[1] = unpack2<T>(v.y), f[2] = unpack2<T>(v.z), f[3] = unpack2<T>(v.w);
    }
}
template <class T>
__device__ __forceinline__ uint4 piece_of(const float2 (&f)[8 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else
        return make_uint4(pack2<T>(f[0].x, f[0].y), pack2<T>(f[1].x, f[1].y), pack2<T>(f[2].x, f[2].y), pack2<T>(f[3].x, f[3].y));
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
    // the same bits for (a, b) and (b, a): every lane of an exchange gets one result
    return {top, __fadd_rn(__fmul_rn(a.sum, rebase<T>(a.top, top, scale)), __fmul_rn(b.sum, rebase<T>(b.top, top, scale)))};
}
template <class T, int PAIRS>
__device__ __forceinline__ void add(Running &r, const float2 (&f)[PAIRS], float scale) {
    float top = r.top;
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) top = fmaxf(top, fmaxf(f[i].x, f[i].y));
    // all -inf so far (or NaN, which fmax leaves out): count from zero, so that -inf adds nothing and NaN stays NaN
    const float from = top == -INFINITY ? 0.0f : top;
    float2 sum = above2<T>(f[0], from, scale);
#pragma unroll
    for (int i = 1; i < PAIRS; ++i) sum = add2(sum, above2<T>(f[i], from, scale));
    r.sum = r.sum * rebase<T>(r.top, top, scale) + (sum.x + sum.y);
    r.top = top;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(~0u, v, d);
    return v;
}
template <int LEFT>
__device__ __forceinline__ void copies_landed() {       // all but the last LEFT groups of this thread's
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// What the k slots come to, in shared memory
struct Slots {
    double *target;             // exponentials, then t_j
    float *value, *chosen;      // v_j; z at the slot's id, before dz may overwrite it
    int *at;                    // where the slot points; -1: not there
    int *seen;                  // a table of the ids
    int mask;                   // its length - 1, a power of two of at least 2 k - 1
};
inline int table_length(int k) {
    int n = 32;
    while (n < 2 * k) n *= 2;
    return n;
}
struct Teacher {
    double P, entropy;          // sum of t; of t log t
    int twice;                  // whether an id comes more than once
};
// by one warp
template <class T>
__device__ __forceinline__ Teacher teacher_side(const DistillArgs &a, const T *z, long long m, const Slots &s, int lane) {
    for (int i = lane; i <= s.mask; i += 32) s.seen[i] = -1;
    __syncwarp();
    float top = -INFINITY;
    bool twice = false, any = false;
    for (int j0 = lane; j0 < a.k; j0 += 32 * AHEAD) {       // the loads of AHEAD slots are under way together
        long long id[AHEAD];
        float v[AHEAD], c[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + 32 * u;
            const long long from = m * a.k + (j < a.k ? j : j0);
            id[u] = a.id_bytes == 8 ? static_cast<const long long *>(a.ids)[from] : static_cast<const int *>(a.ids)[from];
            v[u] = a.values_f32 ? static_cast<const float *>(a.values)[from] : to_f32<T>(static_cast<const T *>(a.values)[from]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (id[u] < 0 || id[u] >= a.V || v[u] == -INFINITY) id[u] = -1;
            c[u] = to_f32<T>(z[max(id[u], 0LL)]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + 32 * u;
            if (j >= a.k) break;
            s.at[j] = (int)id[u], s.value[j] = v[u], s.chosen[j] = c[u];
            if (id[u] < 0) continue;
            any = true;
            top = fmaxf(top, v[u]);
            for (uint32_t h = (uint32_t)id[u] * 2654435761u >> 7;; ++h) {       // ends: the table has room for twice the slots
                const int there_already = atomicCAS(&s.seen[h & s.mask], -1, (int)id[u]);
                twice = twice || there_already == (int)id[u];
                if (there_already == -1 || there_already == (int)id[u]) break;
            }
        }
    }
    Teacher r = {0.0, 0.0, __any_sync(~0u, twice)};
    if (!__any_sync(~0u, any)) return r;
    // t = e / whole with e = exp(v / T - shift)
    double shift, whole = 1.0;
    if (a.lse) {
        shift = a.lse[m];
    } else {
#pragma unroll
        for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        shift = (double)top * a.inv_t;
    }
    double sum = 0.0;
    for (int j = lane; j < a.k; j += 32) {
        const double e = s.at[j] >= 0 ? exp((double)s.value[j] * a.inv_t - shift) : 0.0;
        s.target[j] = e;
        sum += e;
    }
    sum = warp_sum(sum);
    if (!a.lse) whole = sum;
    const double log_whole = a.lse ? 0.0 : log(whole), scale = 1.0 / whole;
    for (int j = lane; j < a.k; j += 32) {
        const double t = s.target[j] * scale;
        s.target[j] = t;
        if (t != 0.0) r.entropy += t * ((double)s.value[j] * a.inv_t - shift - log_whole);
    }
    r.P = sum * scale, r.entropy = warp_sum(r.entropy);
    return r;
}

// LOSS: computes the statistics, writes loss and (where asked) stats.  GRAD: writes dz, from stats without LOSS.
// A cluster of gridDim.x / M blocks to a row; THREADS that walk the row and one warp for the teacher's side.
template <class T, bool LOSS, bool GRAD, int THREADS>
__global__ void __launch_bounds__(THREADS + 32, THREADS == 256 ? 3 : 10) k_distill(DistillArgs a) {
    constexpr int N = 16 / sizeof(T);       // elements of a piece
    extern __shared__ uint4 row[];          // this block's pieces, then the slots
    Slots slots;
    slots.target = reinterpret_cast<double *>(row + a.part_pieces);
    slots.value = reinterpret_cast<float *>(slots.target + a.k), slots.chosen = slots.value + a.k;
    slots.at = reinterpret_cast<int *>(slots.chosen + a.k);
    slots.seen = slots.at + a.k, slots.mask = a.table - 1;
    __shared__ Running runs[THREADS / 32], whole;
    __shared__ Teacher told;
    const int tid = threadIdx.x, lane = tid & 31;
    const bool walks = tid < THREADS;
    const unsigned blocks = (unsigned)(gridDim.x / a.M), rank = blockIdx.x % blocks;
    const long long m = blockIdx.x / blocks;
    const T *z = static_cast<const T *>(a.z) + m * a.ldz;
    // The row in pieces from the 16-byte boundary below its start: element i of piece p is z[p N + i - skew].
    const int skew = (int)(reinterpret_cast<uintptr_t>(z) & 15) / (int)sizeof(T);
    const long long pieces = (a.V + skew + N - 1) / N, first = pieces * rank / blocks;
    const int count = (int)(pieces * (rank + 1) / blocks - first);
    const int each = (count + THREADS - 1) / THREADS, group = (each + GROUPS - 1) / GROUPS;

    Running r = {-INFINITY, 0.0f};
    if (walks) {
        const uint4 *from = reinterpret_cast<const uint4 *>(z - skew) + first;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            for (int j = g * group; j < min(each, (g + 1) * group); ++j)
                if (tid + j * THREADS < count)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                                 ::"r"((uint32_t)__cvta_generic_to_shared(row + tid + j * THREADS)), "l"(from + tid + j * THREADS) : "memory");
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        if constexpr (LOSS) {
            constexpr int PAIRS = N / 2;
            // two pieces at a time, one rise of the maximum for both
            const auto use = [&](int g) {
                for (int j = g * group; j < min(each, (g + 1) * group); j += 2) {
                    float2 f[2 * PAIRS];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int p = tid + (j + u) * THREADS;
                        float2(&h)[PAIRS] = *reinterpret_cast<float2(*)[PAIRS]>(f + u * PAIRS);
                        if (p >= count || j + u >= min(each, (g + 1) * group)) {
#pragma unroll
                            for (int i = 0; i < PAIRS; ++i) h[i] = make_float2(-INFINITY, -INFINITY);
                            continue;
                        }
                        values_of<T>(row[p], h);
                        if (first + p == 0 || first + p == pieces - 1) {        // may reach over the row's ends
                            const long long e = (first + p) * N - skew;
#pragma unroll
                            for (int i = 0; i < PAIRS; ++i) {
                                if (e + 2 * i < 0 || e + 2 * i >= a.V) h[i].x = -INFINITY;
                                if (e + 2 * i + 1 < 0 || e + 2 * i + 1 >= a.V) h[i].y = -INFINITY;
                            }
                        }
                    }
                    add<T>(r, f, a.scale);
                }
            };
            copies_landed<3>(), use(0), copies_landed<2>(), use(1), copies_landed<1>(), use(2), copies_landed<0>(), use(3);
#pragma unroll
            for (int d = 1; d < 32; d *= 2)
                r = join<T>(r, {__shfl_xor_sync(~0u, r.top, d), __shfl_xor_sync(~0u, r.sum, d)}, a.scale);
            if (lane == 0) runs[tid >> 5] = r;
        } else {
            copies_landed<0>();
        }
    } else {
        const Teacher t = teacher_side<T>(a, z, m, slots, lane);
        if (lane == 0) told = t;
    }
    __syncthreads();
    if constexpr (LOSS) {
        r = runs[lane & (THREADS / 32 - 1)];
#pragma unroll
        for (int d = 1; d < THREADS / 32; d *= 2)
            r = join<T>(r, {__shfl_xor_sync(~0u, r.top, d), __shfl_xor_sync(~0u, r.sum, d)}, a.scale);
        if (blocks > 1 && tid == 0) whole = r;
    } else {
        const float2 s = a.stats[m];
        r = {s.x, s.y};
    }
    if (blocks > 1) {
        // every block has its sums, and has read what others may overwrite from here on
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if constexpr (LOSS) {
            for (unsigned b = 0; b < blocks; ++b) {
                uint32_t p;
                Running o;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"((uint32_t)__cvta_generic_to_shared(&whole)), "r"(b));
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(o.top), "=f"(o.sum) : "r"(p) : "memory");
                r = b ? join<T>(r, o, a.scale) : o;
            }
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // waited for at the end
        }
    }
    const float base = r.top == -INFINITY ? 0.0f : r.top;
    const double P = told.P;
    const bool empty = P == 0.0;                // a row without targets: padding
    if (LOSS && rank == 0 && !walks) {
        const double log_sum = log((double)r.sum);
        double loss = 0.0;
        for (int j = lane; j < a.k; j += 32)
            if (slots.at[j] >= 0 && slots.target[j] != 0.0)
                loss -= slots.target[j] * (((double)slots.chosen[j] - (double)base) * (double)a.scale * 0.6931471805599453 - log_sum);
        loss = warp_sum(loss) + told.entropy;
        if (lane == 0) {
            a.loss[m] = empty ? 0.0f : (float)loss;
            if (a.stats) a.stats[m] = make_float2(r.top, r.sum);
        }
    }
    if constexpr (GRAD) {
        const float c = a.dloss[m] * (float)a.inv_t, cs = (float)((double)a.dloss[m] * a.inv_t * P / (double)r.sum);
        T *dz = static_cast<T *>(a.dz) + m * a.lddz;
        const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
        for (int j = 0; walks && j < each; ++j) {
            const int p = tid + j * THREADS;
            if (p >= count) break;
            const long long e = (first + p) * N - skew;
            float2 f[N / 2];
            values_of<T>(row[p], f);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f[i] = empty ? make_float2(0.0f, 0.0f) : mul2(above2<T>(f[i], base, a.scale), make_float2(cs, cs));
            const uint4 v = piece_of<T>(f);
            if (alike && e >= 0 && e + N <= a.V) {
                *reinterpret_cast<uint4 *>(dz + e) = v;
            } else {
                const Pack<T, N> w = *reinterpret_cast<const Pack<T, N> *>(&v);
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (e + i >= 0 && e + i < a.V) dz[e + i] = w.v[i];
            }
        }
        __syncthreads();            // the targets' elements are written again, by the block that wrote them
        const long long e0 = first * N - skew, e1 = (first + count) * N - skew;
        const bool twice = told.twice;
        for (int j = tid; !empty && j < a.k; j += THREADS + 32) {
            const int id = slots.at[j];
            if (id < 0 || id < e0 || id >= e1) continue;
            double t = slots.target[j];
            bool lead = true;
            if (twice) {            // the slots that name this element add up; the first of them writes it
                t = 0.0;
                for (int i = 0; i < a.k; ++i)
                    if (slots.at[i] == id) {
                        if (i < j) lead = false;
                        t += slots.target[i];
                    }
            }
            if (lead) dz[id] = from_f32<T>(fmaf(-c, (float)t, cs * above<T>(slots.chosen[j], base, a.scale)));
        }
    }
    __syncwarp();
    if (LOSS && blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // `whole` has been read
}

template <class T, bool LOSS, bool GRAD, int THREADS>
int launch(DistillArgs &a, int blocks, cudaStream_t s) {
    auto *kernel = k_distill<T, LOSS, GRAD, THREADS>;
    static std::atomic<unsigned long long> done;
    const int rc = block_allow_smem(reinterpret_cast<const void *>(kernel), MOST_PART + 32 + 28 * MAX_TOP, &done);
    if (rc != CCDC_OK) return rc;
    a.table = table_length(a.k);
    a.part_pieces = (int)((a.V * (long long)sizeof(T) + 30) / 16 / blocks) + 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.M * blocks)), cfg.blockDim = dim3(THREADS + 32);
    cfg.dynamicSmemBytes = 16 * (size_t)a.part_pieces + 20 * a.k + 4 * a.table, cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = blocks, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    return block_launch_status();
}
template <class T, bool LOSS, bool GRAD>
int launch(DistillArgs &a, cudaStream_t s) {
    int rc;
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    // parts that leave room for several blocks an SM; smaller ones where rows are few
    const long long bytes = a.V * (long long)sizeof(T);
    int blocks = 1;
    while (blocks < MAX_CLUSTER && (bytes > (long long)PART * blocks || (a.M * blocks * 2 <= sms && bytes > (long long)SMALL_PART * blocks)))
        blocks *= 2;
    if (bytes > (long long)MOST_PART * blocks || a.M * blocks > 0x7FFFFFFF) return CCDC_ESIZE;
    return bytes <= (long long)SMALL_PART * blocks ? launch<T, LOSS, GRAD, 64>(a, blocks, s) : launch<T, LOSS, GRAD, 256>(a, blocks, s);
}
template <bool LOSS, bool GRAD>
int by_type(DistillArgs &a, int dtype, cudaStream_t s) {
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
    if (V * type_bytes(dtype) > MOST_PART * MAX_CLUSTER || V > 0x7FFFFFFF || k > MAX_TOP) return CCDC_ESIZE;
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
