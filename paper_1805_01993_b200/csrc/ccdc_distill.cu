// Distillation loss from a teacher's top logits, and its gradient.
//
// Row m has the student's logits z[V] and k of the teacher's (values v_j at ids_j).  At temperature T
//     t_j  = softmax(v / T) over the slots that are there, or exp(v_j / T - lse) with the whole teacher's lse
//     loss = sum_j t_j (log t_j - log s_id(j)),  s = softmax(z / T)
//     dz   = dloss / T (P s - t),  P = sum_j t_j
// Reading z and writing dz is all the work.  A row belongs to one block or to the blocks of a cluster, which keep it in shared
// memory between the walk for maximum and sum and the walk that writes the gradient: z is read from memory once.  Blocks stay and
// take row after row: a thread copies 16-byte pieces asynchronously and reads only its own, so the copy of the next row's piece
// starts as soon as a piece has been read for the last time, and nothing waits but for copies.  The blocks of a cluster exchange
// their maxima and sums.  The last warp of a block computes the next row's k terms meanwhile, in 64 bits.
//
// Measured (one B200): 4096 x 131072 bf16 in one pass 557 us, 3.9 TB/s of z and dz; the loss alone 325 us, the gradient alone
// 420 us; 1024 x 32000 binary32 38 and 56 us.  Instructions and their latency bound it (27 warps an SM, 0.6 of the issue slots):
// the walk for the sum takes 5 a bf16 element and 700 a row and warp beside, the other 7 and 400.  Slower: 512 threads a block (726 us),
// 128 (635), parts of 52 KiB by four blocks an SM (613) or 42 by five (728), rows read again from L2 instead of kept (777).
#include "ccdc_block.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int MAX_TOP = 1024, MAX_CLUSTER = 8;
// Slots that a lane has under way.  Four: 579 us for 557 at 4096 x 131072 bf16 in one pass, 23.7 for 23.1 at 300 x 50257 fp16; but
// 120 for 137 at 1024 x 32000 binary32 with 400 slots.
constexpr int AHEAD = 2;
constexpr int GROUPS = 4;                   // of copies that are waited for one after the other
constexpr int SMALL_PART = 8 << 10;         // bytes of a row that 64 threads take
constexpr int PART = 65 << 10;              // bytes of a part that leave room for three blocks an SM
constexpr int MOST_PART = 176 << 10, MOST_SMEM = MOST_PART + 32 + 48 * MAX_TOP;

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
    int group;                  // pieces of a thread in a group of copies
    int part_pieces, table;     // room of a block, in pieces of 16 bytes; of the table of ids
    int blocks;                 // to a row
};

template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
        "fma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
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
// 2^(z * scale) relative to a reference `top` (a row's or a thread's largest value).  16-bit logits: 2^(z * scale - b), one
// fused operation for each, with b = top * scale rounded once: its rounding is the same in every term, and a factor of 2^-0.5 to
// 2^0.5 as long as |b| < 2^24.  Further out (masks of -1e9, low temperatures) it would be a factor of hundreds of octaves, infinity
// or 0.  There, and for binary32: 2^((z - top) * scale).  A reference that rises from one form to the other passes 2^13 octaves at
// least, the distance of neighbours among 16-bit values so far out: the sum's factor is 0 in either form.
template <class T>
struct Above {
    float top, scale, b;
    bool fused;
    __device__ __forceinline__ Above(float top_, float scale_) : top(top_ == -INFINITY ? 0.0f : top_), scale(scale_) {
        b = __fmul_rn(top, scale);
        fused = sizeof(T) == 2 && fabsf(b) < 0x1p24f;
    }
    __device__ __forceinline__ float exponent(float z) const { return fused ? fmaf(z, scale, -b) : (z - top) * scale; }
    __device__ __forceinline__ float operator()(float z) const { return power<T>(exponent(z)); }
    template <bool FUSED>
    __device__ __forceinline__ float2 two(float2 z) const {
        const float2 d = FUSED ? fma2(z, make_float2(scale, scale), make_float2(-b, -b))
                               : mul2(add2(z, make_float2(-top, -top)), make_float2(scale, scale));
        return make_float2(power<T>(d.x), power<T>(d.y));
    }
    // the exponent in 64 bits, of the same products
    __device__ __forceinline__ double exact(float z) const {
        return fused ? (double)z * (double)scale - (double)b : ((double)z - (double)top) * (double)scale;
    }
};
// the eight (binary32: four) values of a piece of 16 bytes, two by two
template <class T>
__device__ __forceinline__ void values_of(const uint4 &v, float2 (&f)[8 / (int)sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
        f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
    } else {
        f[0] = unpack2<T>(v.x), f[1] = unpack2<T>(v.y), f[2] = unpack2<T>(v.z), f[3] = unpack2<T>(v.w);
    }
}
template <class T>
__device__ __forceinline__ uint4 piece_of(const float2 (&f)[8 / (int)sizeof(T)]) {
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else
        return make_uint4(pack2<T>(f[0].x, f[0].y), pack2<T>(f[1].x, f[1].y), pack2<T>(f[2].x, f[2].y), pack2<T>(f[3].x, f[3].y));
}

struct Running {
    float top, sum;
};
// the sum's factor when its reference rises from `from` to `to` (a sum of nothing has -inf)
template <class T>
__device__ __forceinline__ float rebase(float from, float to, float scale) {
    if (from == to || from == -INFINITY) return 1.0f;
    const Above<T> lo(from, scale), hi(to, scale);
    return power<T>(lo.fused && hi.fused ? lo.b - hi.b : (from - to) * scale);
}
// The lanes' sums together, in groups of LANES: every lane of a group gets the same bits.
template <class T>
__device__ __forceinline__ Running join(Running r, float scale, int lanes) {
    float top = r.top;
    for (int d = 1; d < lanes; d *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
    float sum = r.sum * rebase<T>(r.top, top, scale);
    for (int d = 1; d < lanes; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
    return {top, sum};
}
// Largest values piece by piece, 16-bit ones two by two as they lie in memory.  NaN is left out, and shows in the sum.
template <class T>
struct Largest {
    using T2 = typename std::conditional<std::is_same<T, bf16>::value, __nv_bfloat162, __half2>::type;
    T2 two;
    __device__ __forceinline__ Largest() : two(T2(from_f32<T>(-INFINITY), from_f32<T>(-INFINITY))) {}
    __device__ __forceinline__ void take(const uint4 &v) {
        const T2 *w = reinterpret_cast<const T2 *>(&v);
        two = __hmax2(two, __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3])));
    }
    __device__ __forceinline__ float value() const { return fmaxf(to_f32<T>(two.x), to_f32<T>(two.y)); }
};
template <>
struct Largest<float> {
    float one = -INFINITY;
    __device__ __forceinline__ void take(const uint4 &v) {
        one = fmaxf(one, fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w))));
    }
    __device__ __forceinline__ float value() const { return one; }
};

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
// by one warp; TWICE: looks for ids that come more than once
template <class T, bool TWICE>
__device__ __forceinline__ Teacher teacher_side(const DistillArgs &a, const T *z, long long m, const Slots &s, int lane) {
    if constexpr (TWICE) {
        for (int i = lane; i <= s.mask; i += 32) s.seen[i] = -1;
        __syncwarp();
    }
    float top = -INFINITY;
    bool twice = false, any = false;
    for (int k0 = 0; k0 < a.k; k0 += 32 * AHEAD) {          // the loads of AHEAD slots are under way together
        const int j0 = k0 + lane;
        long long id[AHEAD];
        float v[AHEAD], c[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + 32 * u;
            const long long from = m * a.k + min(j, a.k - 1);
            id[u] = a.id_bytes == 8 ? static_cast<const long long *>(a.ids)[from] : static_cast<const int *>(a.ids)[from];
            v[u] = a.values_f32 ? static_cast<const float *>(a.values)[from] : to_f32<T>(static_cast<const T *>(a.values)[from]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (id[u] < 0 || id[u] >= a.V || v[u] == -INFINITY || j0 + 32 * u >= a.k) id[u] = -1;
            c[u] = to_f32<T>(z[max(id[u], 0LL)]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + 32 * u;
            if (j < a.k) s.at[j] = (int)id[u], s.value[j] = v[u], s.chosen[j] = c[u];
            if (id[u] < 0) continue;
            any = true;
            top = fmaxf(top, v[u]);
        }
        if constexpr (TWICE) {
            // Into the table, AHEAD slots at a time (one after the other, a warp waits for the longest way of 32 each time: loss and
            // gradient of 4096 x 131072 bf16 with 128 slots 450 us, 419 so).  Ends: the table has room for twice the slots.
            uint32_t at[AHEAD];
            bool open[AHEAD], more;
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) at[u] = (uint32_t)id[u] * 2654435761u >> 7, open[u] = id[u] >= 0;
            do {
                int old[AHEAD];
                more = false;
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    if (k0 + 32 * u < a.k) old[u] = atomicCAS(&s.seen[at[u]++ & s.mask], open[u] ? -1 : -2, (int)id[u]);    // no entry is -2
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    twice = twice || (open[u] && old[u] == (int)id[u]);
                    open[u] = open[u] && old[u] != -1 && old[u] != (int)id[u];
                    more = more || open[u];
                }
            } while (__any_sync(~0u, more));
        }
    }
    Teacher r = {0.0, 0.0, TWICE && __any_sync(~0u, twice)};
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

// A block's share of a row, in pieces from the 16-byte boundary below the row's start: element i of piece p is z[at + p N + i].
template <class T>
struct Share {
    static constexpr int N = 16 / sizeof(T);
    const uint4 *from;
    int at, count, low, high;   // low, high: pieces that may reach over the row's ends, or -1
    __device__ __forceinline__ Share(const DistillArgs &a, const T *z, int rank) {
        const int skew = (int)(reinterpret_cast<uintptr_t>(z) & 15) / (int)sizeof(T);
        const int pieces = ((int)a.V + skew + N - 1) / N, first = rank * a.part_pieces;
        count = max(0, min(a.part_pieces, pieces - first)), at = first * N - skew;
        from = reinterpret_cast<const uint4 *>(z + at);
        low = rank ? -1 : 0, high = first + count == pieces ? count - 1 : -1;
    }
    __device__ __forceinline__ bool edge(int p) const { return p == low || p == high; }
    // what lies outside counts as -inf
    __device__ __forceinline__ uint4 inside(const DistillArgs &a, uint4 v, int p) const {
        Pack<T, N> w = *reinterpret_cast<const Pack<T, N> *>(&v);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + p * N + i < 0 || at + p * N + i >= (int)a.V) w.v[i] = from_f32<T>(-INFINITY);
        return *reinterpret_cast<const uint4 *>(&w);
    }
};
__device__ __forceinline__ void copy_piece(uint4 *to, const uint4 *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
// the elements of a piece that fall into [low, high)
template <class T>
__device__ __forceinline__ void put_some(const DistillArgs &a, T *dz, int e, const uint4 &v, int low, int high) {
    const Pack<T, 16 / sizeof(T)> w = *reinterpret_cast<const Pack<T, 16 / sizeof(T)> *>(&v);
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i)
        if (e + i >= low && e + i < high) dz[e + i] = w.v[i];
}
// 16 bytes of two pieces, from element `shift` of the first on
template <class T>
__device__ __forceinline__ uint4 cut(const uint4 &lo, const uint4 &hi, int shift) {
    const int bytes = shift * (int)sizeof(T);
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 7; ++i) w[i] = bytes & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = bytes & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (bytes & 2));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// LOSS: computes the statistics, writes loss and (where asked) stats.  GRAD: writes dz, from stats without LOSS.
// `blocks` to a row (a cluster); THREADS that walk rows and one warp for the teacher's side.
template <class T, bool LOSS, bool GRAD, int THREADS>
__global__ void __launch_bounds__(THREADS + 32, THREADS == 256 ? 3 : THREADS == 128 ? 6 : THREADS == 64 ? 12 : 16) k_distill(DistillArgs a) {
    constexpr int N = 16 / sizeof(T), PAIRS = N / 2;        // elements of a piece
    extern __shared__ uint4 row[];          // this block's pieces, then the slots of two rows
    __shared__ Running runs[2][THREADS / 32], whole[2];
    __shared__ Teacher told[2];
    const int tid = threadIdx.x, lane = tid & 31;
    const bool walks = tid < THREADS;
    const int blocks = a.blocks, rank = (int)(blockIdx.x % (unsigned)blocks);
    const long long step = gridDim.x / (unsigned)blocks;
    const auto slots_of = [&](int which) {
        Slots s;
        s.target = reinterpret_cast<double *>(row + a.part_pieces) + which * a.k;
        s.value = reinterpret_cast<float *>(reinterpret_cast<double *>(row + a.part_pieces) + 2 * a.k) + which * 2 * a.k, s.chosen = s.value + a.k;
        s.at = reinterpret_cast<int *>(reinterpret_cast<double *>(row + a.part_pieces) + 4 * a.k) + which * a.k;
        s.seen = reinterpret_cast<int *>(reinterpret_cast<double *>(row + a.part_pieces) + 5 * a.k), s.mask = a.table - 1;
        return s;
    };
    const auto row_of = [&](long long m) { return static_cast<const T *>(a.z) + m * a.ldz; };

    long long m = blockIdx.x / (unsigned)blocks;
    if (m < a.M) {
        if (walks) {
            const Share<T> own(a, row_of(m), rank);
            for (int g = 0; g < GROUPS; ++g) {
                for (int p = tid + g * a.group * THREADS; p < min(own.count, tid + (g + 1) * a.group * THREADS); p += THREADS)
                    copy_piece(row + p, own.from + p);
                copies_end();
            }
        } else {
            const Teacher t = teacher_side<T, GRAD>(a, row_of(m), m, slots_of(0), lane);
            if (lane == 0) told[0] = t;
        }
    }
    for (int which = 0; m < a.M; m += step, which ^= 1) {
        const T *z = row_of(m);
        const bool more = m + step < a.M;
        const Share<T> own(a, z, rank), next(a, row_of(more ? m + step : m), rank);
        const int group = a.group;
        const Slots slots = slots_of(which);
        const int next_count = more ? next.count : 0;
        Running r = {-INFINITY, 0.0f};
        if (walks) {
            if constexpr (LOSS) {
                // the pieces' maximum first: one rise of the reference for all of them
                const auto use = [&](int begin, int end) {
                    Largest<T> largest;
                    for (int p = begin; p < end; p += THREADS) {
                        if (own.edge(p)) row[p] = own.inside(a, row[p], p);
                        largest.take(row[p]);
                    }
                    const float top = fmaxf(r.top, largest.value());
                    r.sum *= rebase<T>(r.top, top, a.scale), r.top = top;
                    const Above<T> above(top, a.scale);     // all -inf: counted from zero, so that -inf adds nothing and NaN stays NaN
                    const auto sum_up = [&](auto fused) {
                        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll 2
                        for (int p = begin; p < end; p += THREADS) {
                            float2 f[PAIRS], e[PAIRS];
                            values_of<T>(row[p], f);
#pragma unroll
                            for (int i = 0; i < PAIRS; ++i) e[i] = above.template two<decltype(fused)::value>(f[i]);
#pragma unroll
                            for (int d = PAIRS / 2; d; d /= 2)
#pragma unroll
                                for (int i = 0; i < d; ++i) e[i] = add2(e[i], e[i + d]);
                            sum = add2(sum, e[0]);
                        }
                        r.sum += sum.x + sum.y;
                    };
                    if (sizeof(T) == 2 && above.fused)
                        sum_up(std::true_type());
                    else
                        sum_up(std::false_type());
                };
                // group by group in either form, so that the loss has the same bits with and without the gradient
                static_assert(GROUPS == 4, "waits");
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const int begin = tid + g * group * THREADS, end = begin + group * THREADS;
                    if (!GRAD || g == 0)
                        copies_landed<3>();
                    else if (g == 1)
                        copies_landed<2>();
                    else if (g == 2)
                        copies_landed<1>();
                    else
                        copies_landed<0>();
                    use(begin, min(own.count, end));
                    if constexpr (!GRAD) {      // the next row's copies take the place of a group's as soon as it has been used
                        for (int p = begin; p < min(next_count, end); p += THREADS) copy_piece(row + p, next.from + p);
                        copies_end();
                    }
                }
                r = join<T>(r, a.scale, 32);
                if (lane == 0) runs[which][tid >> 5] = r;
            } else {
                copies_landed<0>();
            }
        }
        __syncthreads();
        if constexpr (LOSS) {
            r = join<T>(runs[which][lane & (THREADS / 32 - 1)], a.scale, THREADS / 32);
            if (blocks > 1 && tid == 0) whole[which] = r;
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
                const int b = lane & (MAX_CLUSTER - 1);
                r = {-INFINITY, 0.0f};
                if (b < blocks) {
                    uint32_t p;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                                 : "=r"(p) : "r"((uint32_t)__cvta_generic_to_shared(&whole[which])), "r"(b));
                    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(r.top), "=f"(r.sum) : "r"(p) : "memory");
                }
                r = join<T>(r, a.scale, MAX_CLUSTER);
            }
        }
        const Above<T> above(r.top, a.scale);
        const double P = told[which].P;
        const bool empty = P == 0.0;                // a row without targets: padding
        if (!walks) {
            if (LOSS && rank == 0) {
                const double log_sum = log((double)r.sum);
                double loss = 0.0;
                for (int j = lane; j < a.k; j += 32)
                    if (slots.at[j] >= 0 && slots.target[j] != 0.0)
                        loss -= slots.target[j] * (above.exact(slots.chosen[j]) * 0.6931471805599453 - log_sum);
                loss = warp_sum(loss) + told[which].entropy;
                if (lane == 0) {
                    a.loss[m] = empty ? 0.0f : (float)loss;
                    if (a.stats) a.stats[m] = make_float2(r.top, r.sum);
                }
            }
            if (more) {
                const Teacher t = teacher_side<T, GRAD>(a, row_of(m + step), m + step, slots_of(which ^ 1), lane);
                if (lane == 0) told[which ^ 1] = t;
            }
        } else if constexpr (GRAD) {
            const float c = a.dloss[m] * (float)a.inv_t, cs = c * ((float)P / r.sum);
            T *dz = static_cast<T *>(a.dz) + m * a.lddz;
            const bool alike = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
            const auto gradient = [&](const uint4 &v, auto fused) {
                float2 f[PAIRS];
                values_of<T>(v, f);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) f[i] = mul2(above.template two<decltype(fused)::value>(f[i]), make_float2(cs, cs));
                return piece_of<T>(f);
            };
            const auto write = [&](auto fused) {
                for (int g = 0; g < GROUPS; ++g) {
                    const int from = tid + g * group * THREADS, to = from + group * THREADS;
#pragma unroll 2
                    for (int p = from; p < min(own.count, to); p += THREADS) {
                        const uint4 v = empty ? make_uint4(0, 0, 0, 0) : gradient(row[p], fused);
                        if (!alike) {
                            row[p] = v;
                            continue;
                        }
                        if (p < next_count) copy_piece(row + p, next.from + p);
                        const int e = own.at + p * N;
                        if (!own.edge(p))
                            *reinterpret_cast<uint4 *>(dz + e) = v;
                        else
                            put_some<T>(a, dz, e, v, 0, (int)a.V);
                    }
                    if (!alike) continue;
                    // the next row may have a piece more
                    if (own.count >= from && own.count < to && own.count < next_count && (own.count - from) % THREADS == 0)
                        copy_piece(row + own.count, next.from + own.count);
                    copies_end();
                }
                if (alike) return;
                // Rows of z and dz that lie differently to 16 bytes: the gradient's pieces, which are in shared memory now, leave cut
                // anew.  Only then may the next row come.
                asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
                const int low = max(0, own.at), high = min((int)a.V, own.at + own.count * N);
                const int skew = (int)(reinterpret_cast<uintptr_t>(dz) & 15) / (int)sizeof(T), first = (low + skew) / N;
                const int shift = (first * N - skew - own.at) & (N - 1);        // of a cut piece in those it comes from
                for (int q = first + tid; q * N - skew < high; q += THREADS) {
                    const int e = q * N - skew, p = (e - own.at) >> (N == 8 ? 3 : 2);
                    const uint4 v = cut<T>(row[max(p, 0)], row[min(p + 1, own.count - 1)], shift);
                    if (e >= low && e + N <= high)
                        *reinterpret_cast<uint4 *>(dz + e) = v;
                    else
                        put_some<T>(a, dz, e, v, low, high);
                }
                asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
                for (int g = 0; g < GROUPS; ++g) {
                    for (int p = tid + g * group * THREADS; p < min(next_count, tid + (g + 1) * group * THREADS); p += THREADS)
                        copy_piece(row + p, next.from + p);
                    copies_end();
                }
            };
            if (sizeof(T) == 2 && above.fused)
                write(std::true_type());
            else
                write(std::false_type());
            // the targets' elements are written again, by the block that wrote them
            asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
            const int e0 = own.at, e1 = own.at + own.count * N;
            const bool twice = told[which].twice;
            for (int j = tid; !empty && j < a.k; j += THREADS) {
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
                if (lead) dz[id] = from_f32<T>(fmaf(-c, (float)t, cs * above(slots.chosen[j])));
            }
        }
    }
    if (LOSS && blocks > 1) {           // no block leaves while another reads its sums
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

template <class T, bool LOSS, bool GRAD, int THREADS>
int launch(DistillArgs &a, int blocks, cudaStream_t s) {
    auto *kernel = k_distill<T, LOSS, GRAD, THREADS>;
    static std::atomic<unsigned long long> done;
    const int rc = block_allow_smem(reinterpret_cast<const void *>(kernel), MOST_SMEM, &done);
    if (rc != CCDC_OK) return rc;
    a.table = table_length(a.k), a.blocks = blocks;
    // a row has (V + 2 (N - 1)) / N pieces at most
    a.part_pieces = (int)(((a.V * (long long)sizeof(T) + 30) / 16 + blocks - 1) / blocks);
    a.group = (a.part_pieces + GROUPS * THREADS - 1) / (GROUPS * THREADS);
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(THREADS + 32);
    cfg.dynamicSmemBytes = 16 * (size_t)a.part_pieces + 40 * a.k + 4 * a.table, cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = blocks, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 1;
    // As many clusters as run at once; more would wait for whole blocks to end.  The answer for the last shape that was asked for
    // is kept: device, blocks and shared memory in the upper bits, clusters in the lower 16.
    static std::atomic<unsigned long long> known;
    int dev = 0, clusters = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const unsigned long long shape = ((unsigned long long)dev << 32 | (unsigned)blocks << 24 | (unsigned)cfg.dynamicSmemBytes) << 16;
    const unsigned long long last = known.load(std::memory_order_relaxed);
    cfg.gridDim = dim3((unsigned)blocks);
    if (last >> 16 == shape >> 16 && (last & 0xFFFF)) {
        clusters = (int)(last & 0xFFFF);
    } else if (e == cudaSuccess) {
        e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
        clusters = std::min(std::max(clusters, 1), 0xFFFF);
        if (e == cudaSuccess) known.store(shape | (unsigned)clusters, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    cfg.gridDim = dim3((unsigned)(std::min<long long>(a.M, clusters) * blocks));
    e = cudaLaunchKernelEx(&cfg, kernel, a);
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
    int blocks = (int)std::min<long long>(MAX_CLUSTER, (bytes + PART - 1) / PART);
    while (2 * blocks <= MAX_CLUSTER && a.M * blocks * 2 <= sms && bytes > (long long)SMALL_PART * blocks) blocks *= 2;
    if (bytes > (long long)MOST_PART * blocks) return CCDC_ESIZE;
    // Few threads to a small part: what a row costs beside its bytes is paid by each warp.  (8192 x 8192 bf16 in one pass: 97 us
    // with 128 threads, 114 with 256; 8192 x 32000: 261 and 231.)
    const long long part = bytes / blocks;
    return part <= SMALL_PART / 2   ? launch<T, LOSS, GRAD, 32>(a, blocks, s)
           : part <= SMALL_PART     ? launch<T, LOSS, GRAD, 64>(a, blocks, s)
           : part <= 4 * SMALL_PART ? launch<T, LOSS, GRAD, 128>(a, blocks, s) : launch<T, LOSS, GRAD, 256>(a, blocks, s);
}
template <bool LOSS, bool GRAD>
int by_type(DistillArgs &a, int dtype, cudaStream_t s) {
    return dtype == CCDC_F32    ? launch<float, LOSS, GRAD>(a, s)
           : dtype == CCDC_BF16 ? launch<bf16, LOSS, GRAD>(a, s) : launch<fp16, LOSS, GRAD>(a, s);
}

}  // namespace

extern "C" {

int ccdc_distill(long long M, long long V, int k, int dtype, const void *logits, long long ldz, int id_bytes, const void *ids,
                 int value_dtype, const void *values, const float *teacher_lse, double temperature, const float *dloss, float *loss,
                 void *stats, void *dlogits, long long lddz, void *stream) {
    if (M < 0 || V < 1 || k < 1 || !is_float_type(dtype) || (value_dtype != dtype && value_dtype != CCDC_F32) ||
        (id_bytes != 4 && id_bytes != 8) || !(temperature >= 1e-6 && temperature <= 1e6))
        return CCDC_EINVAL;
    if (V * type_bytes(dtype) > MOST_PART * MAX_CLUSTER || V > 0x7FFFFFFF || k > MAX_TOP) return CCDC_ESIZE;
    if (M == 0) return CCDC_OK;
    if (!logits || ldz < V || !ids || !aligned_to(ids, id_bytes) || !values || !aligned_to(stats, 8)) return CCDC_EINVAL;
    if (dlogits ? !dloss || lddz < V || (!loss && !stats) : !loss) return CCDC_EINVAL;
    DistillArgs a = {};
    a.M = M, a.V = V, a.ldz = ldz, a.lddz = lddz, a.k = k, a.id_bytes = id_bytes, a.values_f32 = value_dtype == CCDC_F32;
    a.z = logits, a.ids = ids, a.values = values, a.lse = teacher_lse, a.dloss = dloss, a.loss = loss;
    a.stats = static_cast<float2 *>(stats), a.dz = dlogits;
    a.inv_t = 1.0 / temperature, a.scale = (float)(1.4426950408889634 / temperature);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return !dlogits ? by_type<true, false>(a, dtype, s) : loss ? by_type<true, true>(a, dtype, s) : by_type<false, true>(a, dtype, s);
}

}  // extern "C"
