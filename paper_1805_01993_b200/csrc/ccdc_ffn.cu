// Gated feed-forward block, forward and backward: the products, with the activation, its derivative and the
// elementwise products in their epilogues.
#include <algorithm>

#include "ccdc_ffn.h"

namespace {

// C[m][n] = sum over segments s and k of A_s(m, k) B_s(n, k); strides in elements.
struct Operand {
    const void *p;
    long long rs, ks;
};
enum Epilogue { STORE, GATE, GATE_BACK };
struct Product {
    long long M, N, K;
    int segments;               // GATE: the two products stay apart
    Operand a[2], b[2];
    void *c;                    // STORE
    long long ldc;
    int c_f32;
    float *h, *u;               // GATE: out (may be NULL); GATE_BACK: in
    void *v;                    // GATE: a
    void *dh, *du;
    long long ldf;
    int act;
};

constexpr int TILE = 64, STEP = 16;

template <class T, int EPI>
__global__ void __launch_bounds__(256) k_product(const Product p) {
    __shared__ float sa[STEP][TILE + 1], sb[2][STEP][TILE + 1];
    constexpr int NB = EPI == GATE ? 2 : 1;
    const long long m0 = (long long)blockIdx.y * TILE, n0 = (long long)blockIdx.x * TILE;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[NB][4][4] = {};
    for (int s = 0; s < (EPI == GATE ? 1 : p.segments); ++s)
        for (long long k0 = 0; k0 < p.K; k0 += STEP) {
            for (int i = threadIdx.x; i < TILE * STEP; i += 256) {
                // neighbouring threads along the operand's contiguous direction
                auto fetch = [&](const Operand &o, long long r0, long long rows, float *to) {
                    const int r = o.ks == 1 ? i / STEP : i % TILE, k = o.ks == 1 ? i % STEP : i / TILE;
                    const bool in = r0 + r < rows && k0 + k < p.K;
                    to[k * (TILE + 1) + r] = in ? to_f32<T>(static_cast<const T *>(o.p)[(r0 + r) * o.rs + (k0 + k) * o.ks]) : 0.0f;
                };
                fetch(p.a[s], m0, p.M, &sa[0][0]);
#pragma unroll
                for (int j = 0; j < NB; ++j) fetch(p.b[EPI == GATE ? j : s], n0, p.N, &sb[j][0][0]);
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < STEP; ++k)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[j][y][x] += sa[k][ty + 16 * y] * sb[j][k][tx + 16 * x];
            __syncthreads();
        }
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const long long m = m0 + ty + 16 * y, n = n0 + tx + 16 * x;
            if (m >= p.M || n >= p.N) continue;
            if constexpr (EPI == STORE) {
                if (p.c_f32)
                    static_cast<float *>(p.c)[m * p.ldc + n] = acc[0][y][x];
                else
                    static_cast<T *>(p.c)[m * p.ldc + n] = from_f32<T>(acc[0][y][x]);
            } else if constexpr (EPI == GATE) {
                const float h = acc[0][y][x], u = acc[NB - 1][y][x];
                float slope;
                const float f = act_value(p.act, h, &slope);
                if (p.h) {
                    p.h[m * p.ldf + n] = h;
                    p.u[m * p.ldf + n] = u;
                }
                static_cast<T *>(p.v)[m * p.ldf + n] = from_f32<T>(f * u);
            } else {
                const float h = p.h[m * p.ldf + n], u = p.u[m * p.ldf + n];
                float slope;
                const float f = act_value(p.act, h, &slope), d = acc[0][y][x];
                static_cast<T *>(p.dh)[m * p.ldf + n] = from_f32<T>(d * u * slope);
                static_cast<T *>(p.du)[m * p.ldf + n] = from_f32<T>(d * f);
            }
        }
}

template <class T, int EPI>
int launch(const Product &p, cudaStream_t s) {
    if (p.M == 0 || p.N == 0) return CCDC_OK;
    const dim3 grid((unsigned)((p.N + TILE - 1) / TILE), (unsigned)((p.M + TILE - 1) / TILE));
    k_product<T, EPI><<<grid, 256, 0, s>>>(p);
    return block_launch_status();
}

template <class F>
int by_type(int dtype, F f) {
    if (dtype == CCDC_F32) return f(float());
    if (dtype == CCDC_BF16) return f(bf16());
    return f(fp16());
}

// planes of [M][F] between the products, rows padded to 16 bytes
long long inner_stride(long long F) { return (long long)round_up((size_t)F, 8); }
size_t plane_bytes(long long M, long long F, int dtype) {
    return round_up((size_t)M * inner_stride(F) * type_bytes(dtype), 256);
}

int check_ffn(long long M, long long D, long long F, int dtype, int act) {
    if (M < 0 || D < 1 || F < 1 || !is_float_type(dtype) || act < CCDC_ACT_SILU || act > CCDC_ACT_RELU) return CCDC_EINVAL;
    if (M > (1LL << 21) || D > (1LL << 20) || F > (1LL << 20)) return CCDC_ESIZE;
    return CCDC_OK;
}

}  // namespace

extern "C" {

size_t ccdc_ffn_saved_bytes(long long M, long long F, int dtype) {
    if (check_ffn(M, 1, F, dtype, 0) != CCDC_OK) return 0;
    return 2 * plane_bytes(M, F, CCDC_F32) + plane_bytes(M, F, dtype);
}

size_t ccdc_ffn_workspace_bytes(long long M, long long D, long long F, int dtype, int backward, int aligned) {
    if (check_ffn(M, D, F, dtype, 0) != CCDC_OK) return 0;
    (void)aligned;
    return (backward ? 2 : 1) * plane_bytes(M, F, dtype);
}

int ccdc_ffn_forward(long long M, long long D, long long F, int dtype, int act, const void *x, long long ldx,
                     const void *w_gate, const void *w_up, long long ldw, const void *w_down, long long ldd, void *y,
                     long long ldy, void *saved, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_ffn(M, D, F, dtype, act);
    if (rc != CCDC_OK) return rc;
    if (M == 0) return CCDC_OK;
    if (!x || !w_gate || !w_up || !w_down || !y || !workspace || ldx < D || ldw < D || ldd < F || ldy < D ||
        !aligned_to(saved, 16) || !aligned_to(workspace, 16))
        return CCDC_EINVAL;
    if (workspace_bytes < ccdc_ffn_workspace_bytes(M, D, F, dtype, 0, 0)) return CCDC_ESIZE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long ldf = inner_stride(F);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        Product p = {};
        p.M = M, p.N = F, p.K = D, p.segments = 2, p.act = act, p.ldf = ldf;
        p.a[0] = p.a[1] = {x, ldx, 1}, p.b[0] = {w_gate, ldw, 1}, p.b[1] = {w_up, ldw, 1};
        char *keep = static_cast<char *>(saved);
        const size_t wide = plane_bytes(M, F, CCDC_F32);
        if (keep) p.h = reinterpret_cast<float *>(keep), p.u = reinterpret_cast<float *>(keep + wide);
        p.v = keep ? static_cast<void *>(keep + 2 * wide) : workspace;
        int r = launch<T, GATE>(p, s);
        if (r != CCDC_OK) return r;
        Product q = {};
        q.M = M, q.N = D, q.K = F, q.segments = 1;
        q.a[0] = {p.v, ldf, 1}, q.b[0] = {w_down, ldd, 1}, q.c = y, q.ldc = ldy, q.c_f32 = dtype == CCDC_F32;
        return launch<T, STORE>(q, s);
    });
}

int ccdc_ffn_backward(long long M, long long D, long long F, int dtype, int grad_dtype, int act, const void *dy,
                      long long lddy, const void *x, long long ldx, const void *w_gate, const void *w_up, long long ldw,
                      const void *w_down, long long ldd, const void *saved, void *dx, long long lddx, void *dw_gate,
                      void *dw_up, void *dw_down, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_ffn(M, D, F, dtype, act);
    if (rc != CCDC_OK) return rc;
    if (grad_dtype != dtype && grad_dtype != CCDC_F32) return CCDC_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0) {
        for (void *g : {dw_gate, dw_up, dw_down})
            if (g) {
                const cudaError_t e = cudaMemsetAsync(g, 0, (size_t)D * F * type_bytes(grad_dtype), s);
                if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
            }
        return CCDC_OK;
    }
    if (!dy || !x || !w_gate || !w_up || !w_down || !saved || !workspace || lddy < D || ldx < D || ldw < D || ldd < F ||
        (dx && lddx < D) || !aligned_to(saved, 16) || !aligned_to(workspace, 16))
        return CCDC_EINVAL;
    if (workspace_bytes < ccdc_ffn_workspace_bytes(M, D, F, dtype, 1, 0)) return CCDC_ESIZE;
    const size_t plane = plane_bytes(M, F, dtype);
    const long long ldf = inner_stride(F);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        char *keep = const_cast<char *>(static_cast<const char *>(saved));
        const size_t wide = plane_bytes(M, F, CCDC_F32);
        char *dh = static_cast<char *>(workspace), *du = dh + plane;
        Product p = {};
        p.M = M, p.N = F, p.K = D, p.segments = 1, p.act = act, p.ldf = ldf;
        p.a[0] = {dy, lddy, 1}, p.b[0] = {w_down, 1, ldd};
        p.h = reinterpret_cast<float *>(keep), p.u = reinterpret_cast<float *>(keep + wide), p.dh = dh, p.du = du;
        int r = launch<T, GATE_BACK>(p, s);
        auto product = [&](long long m, long long n, long long k, Operand a, Operand b, void *c, long long ldc, int f32) {
            if (r != CCDC_OK || !c) return;
            Product q = {};
            q.M = m, q.N = n, q.K = k, q.segments = 1, q.a[0] = a, q.b[0] = b, q.c = c, q.ldc = ldc, q.c_f32 = f32;
            r = launch<T, STORE>(q, s);
        };
        const int g32 = grad_dtype == CCDC_F32;
        if (r == CCDC_OK && dx) {
            Product q = {};
            q.M = M, q.N = D, q.K = F, q.segments = 2, q.c = dx, q.ldc = lddx, q.c_f32 = dtype == CCDC_F32;
            q.a[0] = {dh, ldf, 1}, q.b[0] = {w_gate, 1, ldw}, q.a[1] = {du, ldf, 1}, q.b[1] = {w_up, 1, ldw};
            r = launch<T, STORE>(q, s);
        }
        product(F, D, M, {dh, 1, ldf}, {x, 1, ldx}, dw_gate, D, g32);
        product(F, D, M, {du, 1, ldf}, {x, 1, ldx}, dw_up, D, g32);
        product(D, F, M, {dy, 1, lddy}, {keep + 2 * wide, 1, ldf}, dw_down, F, g32);
        return r;
    });
}

}  // extern "C"
