// Tokens sorted by expert and back, with weights applied, and the gradients.
//
// Slot s = m k + j is token m's j-th expert.  The sort is a stable counting sort: offsets[e] = slots of experts before e, the
// place of a slot = offsets[e] + slots of the same expert before it.  Everything has one order (atomics count whole numbers
// alone), so replicas of a file agree bit by bit.  A slot whose expert lies outside [0, E) is dropped: place -1.
#include "ccdc_block.h"

#include <algorithm>

namespace {

constexpr int MAX_EXPERTS = 4096;
constexpr int SORT_CLUSTER = 8, SORT_MOST = 16;     // blocks of a sort of many slots, and of very many (where the GPU has room)
constexpr int SORT_VERY_MANY = 32768;
constexpr int SORT_ONE_BLOCK = 4096;        // slots that one block sorts alone
constexpr int BATCH = 4;

struct SortArgs {
    long long slots;
    int experts, bits;
    const void *ids;
    int *offsets, *slot_at, *place_of;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a word of another block's shared memory
__device__ __forceinline__ int remote(const int *p, uint32_t rank) {
    uint32_t at;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// One launch of one block, or of one cluster of blocks.  Each warp owns a run of consecutive slots and counts its experts in
// shared memory; the counts become starting positions by prefix sums over warps, over the cluster's blocks (read from one
// another's shared memory) and over experts; the same walk again, in which lanes with the same expert find one another by
// ballots, then places every slot.  Instructions bound it, on the few SMs of a cluster: 131072 slots over 64 experts 13 us with
// 16 blocks, 18 with 8.
template <class I>
__global__ void __launch_bounds__(1024) k_expert_sort(SortArgs a) {
    extern __shared__ int smem[];
    const int E = a.experts, warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *count = smem, *total = count + warps * E, *base = total + E, *sums = base + E;     // [warps][E], [E], [E], [33]
    const int blocks = gridDim.x, rank = blocks > 1 ? (int)cluster_rank() : 0;
    for (int i = threadIdx.x; i < warps * E; i += blockDim.x) count[i] = 0;
    __syncthreads();
    const long long run = ((a.slots + (long long)blocks * warps - 1) / ((long long)blocks * warps) + 31) / 32 * 32;
    const long long from = min(a.slots, run * ((long long)rank * warps + warp)), to = min(a.slots, from + run);
    const I *ids = static_cast<const I *>(a.ids);
    int *mine = count + warp * E;
    // experts of the warp's slots, BATCH loads under way at a time; -1 where dropped, -2 behind the run
    const auto walk = [&](auto use) {
        for (long long s0 = from; s0 < to; s0 += 32 * BATCH) {
            I id[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) id[u] = s0 + 32 * u + lane < to ? ids[s0 + 32 * u + lane] : (I)-2;
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                if (s0 + 32 * u >= to) break;
                use(s0 + 32 * u + lane, id[u] >= 0 && id[u] < (I)E ? (int)id[u] : s0 + 32 * u + lane < to ? -1 : -2);
            }
        }
    };
    walk([&](long long, int e) {        // whole numbers: any order of these additions gives the same counts
        if (e >= 0) atomicAdd(&mine[e], 1);
    });
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        int sum = 0;
        for (int w = 0; w < warps; ++w) {
            const int c = count[w * E + e];
            count[w * E + e] = sum;
            sum += c;
        }
        total[e] = sum;
    }
    if (blocks > 1)
        cluster_sync();
    else
        __syncthreads();
    // base[e]: slots of experts before e, and of e in the cluster's earlier blocks
    int carry = 0;
    for (int first = 0; first < E; first += blockDim.x) {
        const int e = first + threadIdx.x;
        int all = 0, before = 0;
        if (e < E)
            for (int b = 0; b < blocks; ++b) {
                const int v = blocks > 1 ? remote(total + e, b) : total[e];
                before += b < rank ? v : 0;
                all += v;
            }
        int scan = all;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(~0u, scan, d);
            if (lane >= d) scan += v;
        }
        if (lane == 31) sums[warp] = scan;
        __syncthreads();
        if (warp == 0) {
            int v = lane < warps ? sums[lane] : 0;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int u = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v += u;
            }
            sums[lane] = v;
        }
        __syncthreads();
        const int start = carry + (warp ? sums[warp - 1] : 0) + scan - all;
        if (e < E) {
            base[e] = start + before;
            if (rank == 0) a.offsets[e] = start;
        }
        carry += sums[31];
        __syncthreads();
    }
    if (rank == 0 && threadIdx.x == 0) a.offsets[E] = carry;
    for (int i = threadIdx.x; i < warps * E; i += blockDim.x) count[i] += base[i % E];
    __syncthreads();
    walk([&](long long s, int e) {
        // the lanes with the same expert: one ballot a bit (a match of all values took 1 us a step)
        uint32_t same = __ballot_sync(~0u, e >= 0);
#pragma unroll 4
        for (int bit = 0; bit < a.bits; ++bit) {
            const bool set = e >> bit & 1;
            const uint32_t all = __ballot_sync(~0u, set);
            same &= set ? all : ~all;
        }
        int place = -1;
        if (e >= 0) {
            place = mine[e] + __popc(same & ((1u << lane) - 1));
            a.slot_at[place] = (int)s;
        }
        __syncwarp();
        if (e >= 0 && (same >> lane) == 1) mine[e] += __popc(same);     // the last of them, for all
        __syncwarp();
        if (e > -2) a.place_of[s] = place;
    });
    // positions behind the last expert's hold nothing
    for (long long i = carry + (long long)rank * blockDim.x + threadIdx.x; i < a.slots; i += (long long)blocks * blockDim.x)
        a.slot_at[i] = -1;
    if (blocks > 1) cluster_sync();         // no block leaves while another reads its totals
}

// ------------------------------------------------------------- rows there and back
// Rows are read and written N elements at a time: 16 bytes where the sorted rows are aligned to them, else one.  The tokens' rows,
// which are fewer, may then still start anywhere (APART: a padded batch), and go element by element into and out of the same
// registers.  (Cutting whole pieces out of rows that start elsewhere was slower for its registers: 8192 x 8 rows of 1001 bf16
// there, 42 us one by one and 68 cut.)
// Words stay as they lie in memory until they are used: as elements, 16-bit ones would take a register each.
template <class T, int N>
struct Pack {
    uint4 v = {0, 0, 0, 0};
    __device__ __forceinline__ void get(float (&f)[N]) const {
        if constexpr (sizeof(T) == 4) {
            f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
        } else {
            unpack8<T>(Eight<T>{{v}}, f);
        }
    }
    template <bool APART>
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (!APART) {
            v = *reinterpret_cast<const uint4 *>(p);
        } else if constexpr (sizeof(T) == 4) {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(p);
            v = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
            v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
    }
    template <bool APART>
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (!APART) {
            *reinterpret_cast<uint4 *>(p) = v;
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if constexpr (sizeof(T) == 4)
                    reinterpret_cast<uint32_t *>(p)[i] = w[i];
                else
                    reinterpret_cast<uint16_t *>(p)[2 * i] = (uint16_t)w[i], reinterpret_cast<uint16_t *>(p)[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[N]) {
        if constexpr (sizeof(T) == 4)
            v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        else
            v = pack8<T>(f).v[0];
    }
};
template <class T>
struct Pack<T, 1> {
    T v = from_f32<T>(0.0f);
    template <bool APART>
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    template <bool APART>
    __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32<T>(v); }
    __device__ __forceinline__ void set(const float (&f)[1]) { v = from_f32<T>(f[0]); }
};

struct RowArgs {
    long long M, rows;          // tokens, slots
    int k, D, weights_f32;
    const void *x;              // what is read by token (dispatch: x; backward of combine: dy)
    const void *ys;             // what is read by place
    void *out;                  // xs, y or dys
    long long ldx, ldys, ldo;
    const int *slots, *places;
    const void *weights;
    void *dweights;
};
template <class T>
__device__ __forceinline__ float weight_of(const RowArgs &a, long long slot) {
    if (!a.weights) return 1.0f;
    return a.weights_f32 ? static_cast<const float *>(a.weights)[slot] : to_f32<T>(static_cast<const T *>(a.weights)[slot]);
}
// xs[place] = x[m] for the token's places, and zeros in as many of the rows behind the last expert's.  A token's row is read
// once.  blockDim.x threads to a row, blockDim.y tokens to a block, ITEMS accesses a thread.  16384 x 8 rows of 4096 bf16: 193 us,
// 6.3 TB/s.
template <class T, int N, int ITEMS, bool APART>
__global__ void __launch_bounds__(256) k_expert_dispatch(RowArgs a) {
    const long long m = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    if (m >= a.M) return;
    using P = Pack<T, N>;
    const int c0 = (blockIdx.y * ITEMS * blockDim.x + threadIdx.x) * N, step = blockDim.x * N;
    const T *x = static_cast<const T *>(a.x) + m * a.ldx;
    P v[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (c0 + i * step < a.D) v[i].template load<APART>(x + c0 + i * step);
    for (int j = 0; j < a.k; ++j) {
        const long long s = m * a.k + j;
        const int place = a.places[s];
        const bool empty = a.slots[s] < 0;
        if (place >= 0 && place < a.rows) {
            T *out = static_cast<T *>(a.out) + place * a.ldo;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (c0 + i * step < a.D) *reinterpret_cast<P *>(out + c0 + i * step) = v[i];
        }
        if (empty) {
            T *out = static_cast<T *>(a.out) + s * a.ldo;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (c0 + i * step < a.D) *reinterpret_cast<P *>(out + c0 + i * step) = P();
        }
    }
}

// y[m] = sum over j of w[m][j] ys[place], j ascending, dropped slots left out; 0 for a token without slots.  What bounds it is the
// bytes in flight, since a row's address has to be read first.  So blocks stay and take token after token: eight lanes ask for the
// next slots' places and weights while this token's rows are on their way, and share them by shuffles; AHEAD rows of ITEMS
// accesses a thread are asked for together.  16384 x 8 rows of 4096 bf16: 188 us, 6.4 TB/s (437 us a token a block).
template <class T, int N, int AHEAD, int ITEMS, bool APART>
__global__ void __launch_bounds__(256, 3) k_expert_combine(RowArgs a) {
    using P = Pack<T, N>;
    constexpr int SLOTS = 8;            // known ahead
    const int lane8 = threadIdx.x & (SLOTS - 1), c0 = (blockIdx.y * ITEMS * blockDim.x + threadIdx.x) * N, width = blockDim.x * N;
    const long long step = (long long)gridDim.x * blockDim.y;
    int next_place;
    float next_w;
    const auto know = [&](long long m, int j) {
        const bool there = m < a.M && j + lane8 < a.k;
        next_place = there ? a.places[m * a.k + j + lane8] : -1;
        if (next_place >= a.rows) next_place = -1;
        next_w = there ? weight_of<T>(a, m * a.k + j + lane8) : 0.0f;
    };
    long long m = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    know(m, 0);
    // all threads of a warp take the same number of steps: the shuffles need them
    for (long long first = (long long)blockIdx.x * blockDim.y; first < a.M; first += step, m += step) {
        float sum[ITEMS][N] = {};
        for (int j0 = 0; j0 < a.k; j0 += SLOTS) {
            const int place8 = next_place;
            const float w8 = next_w;
            if (j0 + SLOTS < a.k)
                know(m, j0 + SLOTS);
            else
                know(m + step, 0);
#pragma unroll
            for (int h = 0; h < SLOTS; h += AHEAD) {
                if (j0 + h >= a.k) break;
                P v[AHEAD][ITEMS];
                int place[AHEAD];
                float w[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    place[u] = __shfl_sync(~0u, place8, h + u, SLOTS);
                    w[u] = __shfl_sync(~0u, w8, h + u, SLOTS);
                    const T *ys = static_cast<const T *>(a.ys) + place[u] * a.ldys;
#pragma unroll
                    for (int i = 0; i < ITEMS; ++i)
                        if (place[u] >= 0 && c0 + i * width < a.D) v[u][i] = *reinterpret_cast<const P *>(ys + c0 + i * width);
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u)
                    if (place[u] >= 0)
#pragma unroll
                        for (int i = 0; i < ITEMS; ++i) {
                            float f[N];
                            v[u][i].get(f);
#pragma unroll
                            for (int n = 0; n < N; ++n) sum[i][n] = fmaf(w[u], f[n], sum[i][n]);
                        }
            }
        }
        T *out = static_cast<T *>(a.out) + m * a.ldo;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (m < a.M && c0 + i * width < a.D) {
                P r;
                r.set(sum[i]);
                r.template store<APART>(out + c0 + i * width);
            }
    }
}

// dys[place] = w dy[m] and dw = <dy[m], ys[place]>: `lanes` of a warp to a slot, so that the product is summed by shuffles.  The
// lanes of a token's k slots read its dy at about the same time, from L1 or L2.  16384 x 8 rows of 4096 bf16: 344 us, 6.6 TB/s.
template <class T, int N, int ITEMS, bool APART>
__global__ void __launch_bounds__(256) k_expert_combine_back(RowArgs a, int lanes) {
    using P = Pack<T, N>;
    const long long s = ((long long)blockIdx.x * 256 + threadIdx.x) / lanes;
    const int lane = threadIdx.x & (lanes - 1);
    float dot = 0.0f;
    if (s < a.rows) {
        const long long m = s / a.k;
        const int place = a.places[s];
        const float w = weight_of<T>(a, s);
        if (a.out && a.slots[s] < 0) {
            T *out = static_cast<T *>(a.out) + s * a.ldo;
            for (int c = lane * N; c < a.D; c += lanes * N) *reinterpret_cast<P *>(out + c) = P();
        }
        if (place >= 0 && place < a.rows) {
            const T *dy = static_cast<const T *>(a.x) + m * a.ldx, *ys = static_cast<const T *>(a.ys) + place * a.ldys;
            T *out = static_cast<T *>(a.out) + place * a.ldo;
            for (int c0 = lane * N; c0 < a.D; c0 += lanes * N * ITEMS) {
                P g[ITEMS], v[ITEMS];
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int c = c0 + lanes * N * i;
                    if (c >= a.D) break;
                    g[i].template load<APART>(dy + c);
                    if (a.dweights) v[i] = *reinterpret_cast<const P *>(ys + c);
                }
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) {
                    const int c = c0 + lanes * N * i;
                    if (c >= a.D) break;
                    float d[N], y[N];
                    g[i].get(d);
                    if (a.dweights) {
                        v[i].get(y);
#pragma unroll
                        for (int n = 0; n < N; ++n) dot = fmaf(d[n], y[n], dot);
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) d[n] *= w;
                    P r;
                    r.set(d);
                    if (a.out) *reinterpret_cast<P *>(out + c) = r;
                }
            }
        }
    }
    if (!a.dweights) return;
    for (int d = lanes / 2; d; d /= 2) dot += __shfl_xor_sync(~0u, dot, d);
    if (lane == 0 && s < a.rows) {
        if (a.weights_f32)
            static_cast<float *>(a.dweights)[s] = dot;
        else
            static_cast<T *>(a.dweights)[s] = from_f32<T>(dot);
    }
}

enum Which { DISPATCH, COMBINE, COMBINE_BACK };

template <class T, int N, int AHEAD, int ITEMS, bool APART>
int launch_rows(Which which, const RowArgs &a, int sms, cudaStream_t s) {
    const int packs = (a.D + N - 1) / N;
    int x = 8;
    while (x < 256 && x * ITEMS < packs) x *= 2;
    dim3 block(x, 256 / x), grid((unsigned)((a.M + block.y - 1) / block.y), (unsigned)((packs + x * ITEMS - 1) / (x * ITEMS)));
    if (which == DISPATCH) {
        k_expert_dispatch<T, N, ITEMS, APART><<<grid, block, 0, s>>>(a);
    } else {
        const unsigned at_once = 3 * sms;       // blocks that stay
        grid.x = std::min(grid.x, std::max(1u, at_once / std::min(grid.y, at_once)));
        k_expert_combine<T, N, AHEAD, ITEMS, APART><<<grid, block, 0, s>>>(a);
    }
    return block_launch_status();
}
template <class T, int N, bool APART>
int launch_type(Which which, const RowArgs &a, int sms, cudaStream_t s) {
    if (which == COMBINE_BACK) {
        // four accesses a lane, eight lanes at least
        const int packs = (a.D + N - 1) / N, lanes = packs <= 32 ? 8 : packs <= 64 ? 16 : 32;
        k_expert_combine_back<T, N, 4, APART><<<(unsigned)((a.rows * lanes + 255) / 256), 256, 0, s>>>(a, lanes);
        return block_launch_status();
    }
    if constexpr (N == 1) {
        return launch_rows<T, 1, 4, 4, APART>(which, a, sms, s);
    } else {
        if (a.D < 256 * N) return launch_rows<T, N, 4, 1, APART>(which, a, sms, s);
        // one or two slots a token leave fewer rows to ask for: more of each
        return which == DISPATCH || a.k > 2 ? launch_rows<T, N, 4, 2, APART>(which, a, sms, s)
               : a.k == 2 ? launch_rows<T, N, 2, 4, APART>(which, a, sms, s) : launch_rows<T, N, 1, 4, APART>(which, a, sms, s);
    }
}
template <class T>
int launch_type(Which which, const RowArgs &a, int sms, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const auto aligned = [&](const void *p, long long ld) { return aligned_to(p, 16) && (!p || ld * sizeof(T) % 16 == 0); };
    const bool x = aligned(a.x, a.ldx), ys = aligned(a.ys, a.ldys), out = aligned(a.out, a.ldo);
    // dispatch: x by token, out sorted; combine: out by token, ys sorted; its backward pass: x by token, the others sorted
    const bool token = which == COMBINE ? out : x, sorted = ys && (which == COMBINE || out);
    if (a.D % N || !sorted) return launch_type<T, 1, false>(which, a, sms, s);
    return token ? launch_type<T, N, false>(which, a, sms, s) : launch_type<T, N, true>(which, a, sms, s);
}
int launch(Which which, RowArgs &a, int dtype, cudaStream_t s) {
    int rc;
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    return dtype == CCDC_F32    ? launch_type<float>(which, a, sms, s)
           : dtype == CCDC_BF16 ? launch_type<bf16>(which, a, sms, s) : launch_type<fp16>(which, a, sms, s);
}
int check(long long M, int k, long long D, int dtype, int weight_dtype) {
    if (M < 0 || k < 1 || D < 1 || !is_float_type(dtype) || (weight_dtype != dtype && weight_dtype != CCDC_F32))
        return CCDC_EINVAL;
    return M > 0x7FFFFFFF / k || D > (1 << 20) ? CCDC_ESIZE : CCDC_OK;
}

}  // namespace

extern "C" {

int ccdc_expert_sort(long long M, int k, int experts, int id_bytes, const void *ids, int *offsets, int *slots, int *places,
                     void *stream) {
    if (M < 0 || k < 1 || experts < 1 || (id_bytes != 4 && id_bytes != 8) || !offsets || !aligned_to(ids, id_bytes) ||
        !aligned_to(offsets, 4) || !aligned_to(slots, 4) || !aligned_to(places, 4))
        return CCDC_EINVAL;
    if (M > 0 && (!ids || !slots || !places)) return CCDC_EINVAL;
    if (M > 0x7FFFFFFF / k || experts > MAX_EXPERTS) return CCDC_ESIZE;
    int bits = 0;
    while (1 << bits < experts) ++bits;
    SortArgs a = {M * k, experts, bits, ids, offsets, slots, places};
    const int warps = experts <= 1024 ? 32 : 8;             // the counts of all warps fit the shared memory
    const int smem = (warps * experts + 2 * experts + 33) * (int)sizeof(int);
    static std::atomic<unsigned long long> done[2];
    constexpr int MOST = (32 * 1024 + 2 * MAX_EXPERTS + 33) * (int)sizeof(int);
    const void *kernel = id_bytes == 4 ? (const void *)k_expert_sort<int> : (const void *)k_expert_sort<long long>;
    const int rc = block_allow_smem(kernel, MOST, &done[id_bytes / 8]);
    if (rc != CCDC_OK) return rc;
    int blocks = a.slots <= SORT_ONE_BLOCK ? 1 : SORT_CLUSTER;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(32 * warps), cfg.dynamicSmemBytes = smem, cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
    cfg.attrs = at, cfg.numAttrs = 1;
    if (a.slots >= SORT_VERY_MANY) {
        // whether the device runs clusters of this size; the answer is kept, a bit for each device
        static std::atomic<unsigned long long> asked[2], possible[2];
        int dev = 0, clusters = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
        const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
        if (bit && !(asked[id_bytes / 8].load() & bit)) {
            cudaLaunchConfig_t most = cfg;
            most.gridDim = dim3(SORT_MOST), most.blockDim = dim3(1024), most.dynamicSmemBytes = MOST;
            at[0].val.clusterDim.x = SORT_MOST;
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &most);
            if (e == cudaSuccess && clusters > 0)
                possible[id_bytes / 8].fetch_or(bit);
            else
                cudaGetLastError();
            asked[id_bytes / 8].fetch_or(bit);
        }
        if (possible[id_bytes / 8].load() & bit) blocks = SORT_MOST;
    }
    cfg.gridDim = dim3(blocks);
    at[0].val.clusterDim.x = blocks;
    const cudaError_t e = id_bytes == 4 ? cudaLaunchKernelEx(&cfg, k_expert_sort<int>, a)
                                        : cudaLaunchKernelEx(&cfg, k_expert_sort<long long>, a);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    return block_launch_status();
}

int ccdc_expert_dispatch(long long M, int k, long long D, int dtype, const void *x, long long ldx, const int *slots,
                         const int *places, void *xs, long long ldxs, void *stream) {
    const int rc = check(M, k, D, dtype, dtype);
    if (rc != CCDC_OK) return rc;
    if (M == 0) return CCDC_OK;
    if (!x || !slots || !places || !xs || ldx < D || ldxs < D) return CCDC_EINVAL;
    RowArgs a = {};
    a.M = M, a.rows = M * k, a.k = k, a.D = (int)D, a.x = x, a.ldx = ldx, a.slots = slots, a.places = places;
    a.out = xs, a.ldo = ldxs;
    return launch(DISPATCH, a, dtype, static_cast<cudaStream_t>(stream));
}

int ccdc_expert_combine(long long M, int k, long long D, int dtype, const void *ys, long long ldys, const int *places,
                        const void *weights, int weight_dtype, void *y, long long ldy, void *stream) {
    const int rc = check(M, k, D, dtype, weights ? weight_dtype : dtype);
    if (rc != CCDC_OK) return rc;
    if (M == 0) return CCDC_OK;
    if (!ys || !places || !y || ldys < D || ldy < D) return CCDC_EINVAL;
    RowArgs a = {};
    a.M = M, a.rows = M * k, a.k = k, a.D = (int)D, a.ys = ys, a.ldys = ldys, a.places = places, a.weights = weights;
    a.weights_f32 = weight_dtype == CCDC_F32, a.out = y, a.ldo = ldy;
    return launch(COMBINE, a, dtype, static_cast<cudaStream_t>(stream));
}

int ccdc_expert_combine_backward(long long M, int k, long long D, int dtype, const void *dy, long long lddy, const void *ys,
                                 long long ldys, const int *slots, const int *places, const void *weights, int weight_dtype,
                                 void *dys, long long lddys, void *dweights, void *stream) {
    const int rc = check(M, k, D, dtype, weight_dtype);
    if (rc != CCDC_OK) return rc;
    if (M == 0) return CCDC_OK;
    if (!dy || !slots || !places || lddy < D || (!dys && !dweights) || (dys && lddys < D) ||
        (dweights && (!ys || ldys < D)))
        return CCDC_EINVAL;
    RowArgs a = {};
    a.M = M, a.rows = M * k, a.k = k, a.D = (int)D, a.x = dy, a.ldx = lddy, a.ys = ys, a.ldys = ldys, a.slots = slots;
    a.places = places, a.weights = weights, a.weights_f32 = weight_dtype == CCDC_F32, a.out = dys, a.ldo = lddys;
    a.dweights = dweights;
    return launch(COMBINE_BACK, a, dtype, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
