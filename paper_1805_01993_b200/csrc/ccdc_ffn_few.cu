// Backward products of a binary32 feed-forward block for up to 32 rows.
//
// The tensor cores would need every weight split into three planes first (3.5 times the bytes of reading it once), so
// few rows run on plain multiply-adds: 32 rows are 16 operations a byte, about where the plain cores and the memory
// take the same time.  Weights are read once, gradients written once; sums cut along k are added in order.
// Measured: one row at 4096 x 16384 backward 0.37 ms for 1.6 GB, 4.3 TB/s; 32 rows at 2048 x 8192 about 0.35 ms, bound by the
// multiply-adds and their shared-memory reads.
#include <algorithm>

#include "ccdc_ffn.h"
#include "ccdc_ffn_few.h"
#include "ccdc_ffn_mma.h"

namespace {

__device__ __forceinline__ float4 load4(const float *row, long long c, long long C, bool wide) {
    if (wide && c + 4 <= C) return *reinterpret_cast<const float4 *>(row + c);
    float4 v = make_float4(0, 0, 0, 0);
    if (c < C) v.x = row[c];
    if (c + 1 < C) v.y = row[c + 1];
    if (c + 2 < C) v.z = row[c + 2];
    if (c + 3 < C) v.w = row[c + 3];
    return v;
}
__device__ __forceinline__ bool rows_of_16(const void *p, long long ld) {
    return ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

constexpr int ACROSS_THREADS = 128, CHUNK = 32, AHEAD = 8;

// A thread owns four columns and all rows; the block's share of k goes by in chunks whose p sits in shared memory, read
// by all threads at once; AHEAD weight rows are in flight a thread.
template <int TOKENS>
__global__ void __launch_bounds__(ACROSS_THREADS) k_few_across(const FewAcross a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ __align__(16) float s[CHUNK][TOKENS];
    const long long n = ((long long)blockIdx.x * ACROSS_THREADS + threadIdx.x) * 4;
    const long long all = a.K * a.terms;
    const long long k0 = all * blockIdx.y / a.splits, k1 = all * (blockIdx.y + 1) / a.splits;
    float4 acc[TOKENS];
#pragma unroll
    for (int m = 0; m < TOKENS; ++m) acc[m] = make_float4(0, 0, 0, 0);
    for (long long k = k0; k < k1; k += CHUNK) {
        const int count = (int)min((long long)CHUNK, k1 - k);
        __syncthreads();
        for (int i = threadIdx.x; i < CHUNK * TOKENS; i += ACROSS_THREADS) {
            const int j = i % CHUNK, m = i / CHUNK;
            const int t = k + j >= a.K ? 1 : 0;
            s[j][m] = j < count && m < a.M ? a.p[t][m * a.ldp + (k + j - t * a.K)] : 0.0f;
        }
        __syncthreads();
        for (int j0 = 0; j0 < count; j0 += AHEAD) {
            float4 w[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const long long kk = k + j0 + j;
                const int t = kk >= a.K ? 1 : 0;
                const float *row = a.w[t] + (kk - t * a.K) * a.ldw;
                w[j] = j0 + j < count && n < a.N ? load4(row, n, a.N, rows_of_16(a.w[t], a.ldw)) : make_float4(0, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (j0 + j >= count) break;
#pragma unroll
                for (int m = 0; m < TOKENS; m += 4) {
                    const float4 p = *reinterpret_cast<const float4 *>(&s[j0 + j][m]);
                    const float f[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[m + e].x = fmaf(f[e], w[j].x, acc[m + e].x);
                        acc[m + e].y = fmaf(f[e], w[j].y, acc[m + e].y);
                        acc[m + e].z = fmaf(f[e], w[j].z, acc[m + e].z);
                        acc[m + e].w = fmaf(f[e], w[j].w, acc[m + e].w);
                    }
                }
            }
        }
    }
    if (n < a.N) {      // rows of the parts are padded to four columns
        float *to = a.parts + (long long)blockIdx.y * a.M * a.ldo + n;
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
            if (m < a.M) *reinterpret_cast<float4 *>(to + m * a.ldo) = acc[m];
    }
}

__global__ void __launch_bounds__(256) k_few_gate_back(const FewGateBack a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long groups = ffn_saved_groups(a.N), n = a.M * groups;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
        const long long m = i / groups, f = (i - m * groups) * 4;
        const float *p = a.parts + m * a.ld + f;
        float4 d = *reinterpret_cast<const float4 *>(p);
        for (int s = 1; s < a.splits; ++s) {
            const float4 o = *reinterpret_cast<const float4 *>(p + s * a.M * a.ld);
            d.x += o.x, d.y += o.y, d.z += o.z, d.w += o.w;
        }
        const long long at = ffn_saved_index(m, f, groups) / 4;
        const float4 h = reinterpret_cast<const float4 *>(a.h)[at], u = reinterpret_cast<const float4 *>(a.u)[at];
        float4 dh, du;
        act_apply<true>(a.act, [&](auto act) {
            float slope;
            du.x = d.x * act(h.x, &slope), dh.x = d.x * u.x * slope;
            du.y = d.y * act(h.y, &slope), dh.y = d.y * u.y * slope;
            du.z = d.z * act(h.z, &slope), dh.z = d.z * u.z * slope;
            du.w = d.w * act(h.w, &slope), dh.w = d.w * u.w * slope;
        });
        *reinterpret_cast<float4 *>(a.dh + m * a.ld + f) = dh;
        *reinterpret_cast<float4 *>(a.du + m * a.ld + f) = du;
    }
}

// 64 rows by 128 columns a block, a thread eight rows by four columns
__global__ void __launch_bounds__(256) k_few_outer(const FewOuters a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ __align__(16) float sp[FEW_MOST][64], sq[FEW_MOST][128];
    const FewOuter &o = a.o[blockIdx.z];
    const bool wide = rows_of_16(o.out, o.C);
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, M = (int)a.M;
    const long long c0 = (long long)blockIdx.x * 128;
    if (c0 >= o.C) return;
    for (int i = threadIdx.x; i < M * 128; i += 256) {
        const long long c = c0 + (i & 127);
        sq[i >> 7][i & 127] = c < o.C ? o.q[(i >> 7) * o.ldq + c] : 0.0f;
    }
    for (long long r0 = (long long)blockIdx.y * 64; r0 < o.R; r0 += gridDim.y * 64LL) {
        __syncthreads();
        for (int i = threadIdx.x; i < M * 64; i += 256) {
            const long long r = r0 + (i & 63);
            sp[i >> 6][i & 63] = r < o.R ? o.p[(i >> 6) * o.ldp + r] : 0.0f;
        }
        __syncthreads();
        float4 acc[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) acc[r] = make_float4(0, 0, 0, 0);
        for (int m = 0; m < M; ++m) {
            const float4 q = *reinterpret_cast<const float4 *>(&sq[m][4 * x]);
            const float4 p0 = *reinterpret_cast<const float4 *>(&sp[m][8 * y]), p1 = *reinterpret_cast<const float4 *>(&sp[m][8 * y + 4]);
            const float p[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                acc[r].x = fmaf(p[r], q.x, acc[r].x), acc[r].y = fmaf(p[r], q.y, acc[r].y);
                acc[r].z = fmaf(p[r], q.z, acc[r].z), acc[r].w = fmaf(p[r], q.w, acc[r].w);
            }
        }
        const long long c = c0 + 4 * x;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const long long row = r0 + 8 * y + r;
            if (row >= o.R || c >= o.C) continue;
            float *to = o.out + row * o.C + c;
            if (wide && c + 4 <= o.C) {
                *reinterpret_cast<float4 *>(to) = acc[r];
            } else {
                to[0] = acc[r].x;
                if (c + 1 < o.C) to[1] = acc[r].y;
                if (c + 2 < o.C) to[2] = acc[r].z;
                if (c + 3 < o.C) to[3] = acc[r].w;
            }
        }
    }
}

template <class P>
int launch(void (*kernel)(P), const P &p, dim3 grid, int threads, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}

}  // namespace

int few_across_splits(long long M, long long N, long long K, int terms, int sms) {
    // four blocks an SM (two, where they multiply more than they wait), of four chunks at least
    const long long columns = (N + 4 * ACROSS_THREADS - 1) / (4 * ACROSS_THREADS);
    return (int)std::max<long long>(1, std::min((M <= 8 ? 4LL : 2LL) * sms / columns, K * terms / (4 * CHUNK)));
}
int few_across(const FewAcross &a, cudaStream_t s) {
    const dim3 grid((unsigned)((a.N + 4 * ACROSS_THREADS - 1) / (4 * ACROSS_THREADS)), (unsigned)a.splits);
    return launch(a.M <= 8 ? k_few_across<8> : k_few_across<32>, a, grid, ACROSS_THREADS, s);
}
int few_gate_back(const FewGateBack &a, cudaStream_t s) {
    const long long items = a.M * ffn_saved_groups(a.N);
    return launch(k_few_gate_back, a, dim3((unsigned)std::min<long long>((items + 255) / 256, 2048)), 256, s);
}
int few_outer(const FewOuters &a, cudaStream_t s) {
    long long columns = 1, rows = 1;
    for (int i = 0; i < a.count; ++i) columns = std::max(columns, a.o[i].C), rows = std::max(rows, a.o[i].R);
    const dim3 grid((unsigned)((columns + 127) / 128), (unsigned)std::min<long long>((rows + 63) / 64, 64), (unsigned)a.count);
    return launch(k_few_outer, a, grid, 256, s);
}
