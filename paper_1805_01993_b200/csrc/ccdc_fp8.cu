// 8-bit products with a scale for each block of 128: quantisation, and the entry of the product.
//
// A block of 128 elements of a row (activations) or of 128 x 128 (weights) is held as e4m3 values q and one binary32
// scale: x ~ q * scale.  The scale made here is the least power of two that brings the block's largest magnitude to 448 at
// most.  Quotients by it are exact, so every q has one value whichever way it is computed.  A finer scale would not change the
// relative error of q's normal values (2^-6 to 448); what lies below them (under 2^-6 scale) has a fixed
// step, which a scale of up to twice the least possible one makes up to one bit coarser.
#include "ccdc_block.h"
#include "ccdc_fp8.h"

#include <cuda_fp8.h>

#include <algorithm>

namespace {

constexpr int BLOCK = 128;

struct QuantArgs {
    long long M, K;             // of one group
    const void *x;
    long long ldx, x_group;
    uint8_t *q;
    long long ldq, q_group;
    float *scales;
    long long s_group, s_row, s_col;
};

// eight elements of a row, zeros beyond its end
template <class T, bool VEC>
__device__ __forceinline__ void row8(const T *row, long long c, long long K, float (&f)[8]) {
    if (VEC && c + 8 <= K) {
        unpack8<T>(load8<T>(row + c), f);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < K ? to_f32<T>(row[c + i]) : 0.0f;
}
// the magnitudes' largest as an integer, in which a NaN is larger than infinity and both than any number
__device__ __forceinline__ uint32_t largest(const float (&f)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7FFFFFFFu);
    return m;
}
// 2^e with the least e >= -126 for which the magnitude is at most 448 * 2^e = 1.75 * 2^(e + 8); NaN for a block that holds an
// infinity or a NaN
__device__ __forceinline__ float block_scale(uint32_t magnitude, float *inverse) {
    if (magnitude >= 0x7F800000u) return *inverse = __uint_as_float(0x7FC00000u);
    const int e = max((int)((magnitude + 0x1FFFFFu) >> 23) - 8, 1);         // biased
    *inverse = __uint_as_float((uint32_t)(254 - e) << 23);
    return __uint_as_float((uint32_t)e << 23);
}
__device__ __forceinline__ void put8(uint8_t *row, long long c, long long K, const float (&f)[8], float inverse) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * h] * inverse, f[4 * h + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * h + 2] * inverse, f[4 * h + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
        w[h] = lo | hi << 16;
    }
    if (c + 8 <= K) {
        *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < K) row[c + i] = (uint8_t)(w[i >> 2] >> 8 * (i & 3));
}

// Blocks of one row: 16 lanes to a block, a warp to 256 elements of a row.  The warps of a thread block take neighbouring rows,
// so that scales that are stored by column leave in whole sectors.  8192 x 8192 bf16: 46 us, 4.4 TB/s (two rows a warp the
// same, four 64 us; neighbouring segments of one row in a block 53 us).
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_quantize_rows(QuantArgs a, unsigned segments) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // a product that follows may set itself up
    const unsigned group = blockIdx.x / segments;
    const long long c = (blockIdx.x - group * segments) * 256 + lane * 8, m = (long long)group * 8 + warp;
    if (m >= a.M) return;
    float f[8];
    row8<T, VEC>(static_cast<const T *>(a.x) + m * a.ldx, c, a.K, f);
    uint32_t most = largest(f);
#pragma unroll
    for (int d = 8; d; d /= 2) most = max(most, __shfl_xor_sync(~0u, most, d));
    float inverse;
    const float scale = block_scale(most, &inverse);
    if ((lane & 15) == 0 && c < a.K) a.scales[m * a.s_row + c / BLOCK * a.s_col] = scale;
    put8(a.q + m * a.ldq, c, a.K, f, inverse);
}

// Blocks of 128 x 128: a block of threads each, eight rows a thread.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_quantize_tiles(QuantArgs a) {
    __shared__ uint32_t most_of[8];
    const long long g = blockIdx.z, c = (long long)blockIdx.x * BLOCK + (threadIdx.x & 15) * 8;
    const long long m0 = (long long)blockIdx.y * BLOCK + (threadIdx.x >> 4);
    float f[8][8];
    uint32_t most = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        if (m0 + 16 * r >= a.M) break;
        row8<T, VEC>(static_cast<const T *>(a.x) + g * a.x_group + (m0 + 16 * r) * a.ldx, c, a.K, f[r]);
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (m0 + 16 * r < a.M) most = max(most, largest(f[r]));
    most = __reduce_max_sync(~0u, most);
    if ((threadIdx.x & 31) == 0) most_of[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) most = max(most, most_of[w]);
    float inverse;
    const float scale = block_scale(most, &inverse);
    if (threadIdx.x == 0) a.scales[g * a.s_group + blockIdx.y * a.s_row + blockIdx.x * a.s_col] = scale;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (m0 + 16 * r < a.M) put8(a.q + g * a.q_group + (m0 + 16 * r) * a.ldq, c, a.K, f[r], inverse);
}

template <class T, bool VEC>
int launch_quantize(const QuantArgs &a, long long groups, int block_rows, cudaStream_t s) {
    if (block_rows == 1) {
        const long long segments = (a.K + 255) / 256, blocks = (a.M + 7) / 8 * segments;
        if (blocks > 0x7FFFFFFF) return CCDC_ESIZE;
        k_quantize_rows<T, VEC><<<(unsigned)blocks, 256, 0, s>>>(a, (unsigned)segments);
    } else {
        const dim3 grid((unsigned)((a.K + BLOCK - 1) / BLOCK), (unsigned)((a.M + BLOCK - 1) / BLOCK), (unsigned)groups);
        k_quantize_tiles<T, VEC><<<grid, 256, 0, s>>>(a);
    }
    return block_launch_status();
}
template <class T>
int launch_quantize(const QuantArgs &a, long long groups, int block_rows, bool vec, cudaStream_t s) {
    return vec ? launch_quantize<T, true>(a, groups, block_rows, s) : launch_quantize<T, false>(a, groups, block_rows, s);
}

}  // namespace

extern "C" {

int ccdc_quantize_fp8(long long groups, long long M, long long K, int block_rows, int dtype, const void *x, long long x_group,
                      long long ldx, void *q, long long q_group, long long ldq, float *scales, long long scale_group,
                      long long scale_row, long long scale_col, void *stream) {
    if (groups < 0 || M < 0 || K < 1 || !is_float_type(dtype) || (block_rows != 1 && block_rows != BLOCK) ||
        (block_rows == 1 && groups > 1))
        return CCDC_EINVAL;
    if (groups > 65535 || M > (block_rows == 1 ? 0x7FFFFFFFLL : 65535LL * BLOCK) || K > (1LL << 23)) return CCDC_ESIZE;
    if (groups == 0 || M == 0) return CCDC_OK;
    if (!x || !q || !scales || ldx < K || ldq < K || !aligned_to(q, 16) || ldq % 16 || (groups > 1 && q_group % 16)) return CCDC_EINVAL;
    QuantArgs a = {M, K, x, ldx, x_group, static_cast<uint8_t *>(q), ldq, q_group, scales, scale_group, scale_row, scale_col};
    const int b = type_bytes(dtype);
    const bool vec = aligned_to(x, 16) && ldx * b % 16 == 0 && (groups == 1 || x_group * b % 16 == 0);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == CCDC_F32    ? launch_quantize<float>(a, groups, block_rows, vec, s)
           : dtype == CCDC_BF16 ? launch_quantize<bf16>(a, groups, block_rows, vec, s)
                                : launch_quantize<fp16>(a, groups, block_rows, vec, s);
}

int ccdc_matmul_fp8(long long M, long long N, long long K, int experts, const void *x, long long ldx, const float *x_scales,
                    long long x_scale_row, long long x_scale_col, const void *w, long long w_expert, long long ldw,
                    const float *w_scales, const int *offsets, void *y, int y_dtype, long long ldy, void *stream) {
    if (M < 0 || N < 1 || K < 1 || experts < 1 || !is_float_type(y_dtype) || (experts > 1 && !offsets)) return CCDC_EINVAL;
    if (M > (1 << 30) || N > (1 << 22) || K > (1 << 23) || experts > 1024) return CCDC_ESIZE;
    if (M == 0) return CCDC_OK;
    if (!x || !x_scales || !w || !w_scales || !y || ldx < K || ldw < K || ldy < N || !aligned_to(x, 16) || !aligned_to(w, 16) ||
        ldx % 16 || ldw % 16 || (experts > 1 && (w_expert % 16 || w_expert <= 0)))
        return CCDC_EINVAL;
    int rc;
    const int sms = block_sm_count(&rc);
    if (rc != CCDC_OK) return rc;
    const Fp8Product p = {M, N, K, experts, static_cast<const uint8_t *>(x), static_cast<const uint8_t *>(w), ldx, ldw, w_expert, x_scales,
                          w_scales, x_scale_row, x_scale_col, offsets, y, y_dtype, ldy};
    return fp8_mma_launch(p, sms, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
