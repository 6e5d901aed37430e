// What the block operators (feed-forward, norms, dropout) share: element types, launch helpers and the
// counter-based generator.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "ccdc.h"
#include "ccdc_internal.h"

using bf16 = __nv_bfloat16;
using fp16 = __half;

template <class T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<bf16>(bf16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<fp16>(fp16 v) { return __half2float(v); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ fp16 from_f32<fp16>(float v) { return __float2half_rn(v); }

// two values to one 32-bit word of a 16-bit type, the first in the low half
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<bf16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack2<fp16>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <class T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<bf16>(uint32_t w) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w));
}
template <>
__device__ __forceinline__ float2 unpack2<fp16>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// eight consecutive elements as they lie in memory (16 bytes of a 16-bit type, 32 of binary32)
template <class T>
struct Eight {
    uint4 v[sizeof(T) / 2];
};
template <class T>
__device__ __forceinline__ Eight<T> load8(const T *p) {
    Eight<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = reinterpret_cast<const uint4 *>(p)[i];
    return r;
}
template <class T>
__device__ __forceinline__ void unpack8(const Eight<T> &r, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(&r.v[0]), b = *reinterpret_cast<const float4 *>(&r.v[1]);
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
        const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = unpack2<T>(w[i]);
            f[2 * i] = p.x, f[2 * i + 1] = p.y;
        }
    }
}
template <class T>
__device__ __forceinline__ Eight<T> pack8(const float (&f)[8]) {
    Eight<T> r;
    if constexpr (sizeof(T) == 4) {
        r.v[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        r.v[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else {
        r.v[0] = make_uint4(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
    }
    return r;
}
template <class T>
__device__ __forceinline__ void store8(T *p, const Eight<T> &r) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(p)[i] = r.v[i];
}

// The generator of the dropout masks: Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel
// Random Numbers: As Easy as 1, 2, 3", 2011).  Key = the two words of the seed; counter = (element / 8, 0),
// so that eight elements share one call and an element's number depends on (seed, element) alone: every
// replica of a file draws the same mask wherever and in whatever order it is computed.  Element numbers are taken modulo
// 2^64, counters modulo 2^61 (COUNTERS).
constexpr unsigned long long COUNTERS = ~0ull >> 3;
// A probability in 1/65536 steps, and the factor of kept elements: that of the rounded probability, so that the
// expectation is exact.  p = 1 drops everything.
struct Dropout {
    unsigned long long seed, offset;
    uint32_t cut;       // 0: no dropout
    uint32_t below;     // cut * 65536 - 1: 16 bits in the upper half of a word are kept where the word is above this
    float scale;
    uint32_t key[20];   // the generator's keys, round by round
};
inline bool make_dropout(double p, unsigned long long seed, unsigned long long offset, Dropout *d) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d->seed = seed, d->offset = offset;
    d->cut = (uint32_t)(p * 65536.0 + 0.5);
    d->below = d->cut ? (uint32_t)(((unsigned long long)d->cut << 16) - 1) : 0;
    d->scale = d->cut >= 65536u ? 0.0f : (float)(65536.0 / (65536.0 - d->cut));
    for (uint32_t i = 0; i < 10; ++i) {
        d->key[2 * i] = (uint32_t)seed + i * 0x9E3779B9u;
        d->key[2 * i + 1] = (uint32_t)(seed >> 32) + i * 0xBB67AE85u;
    }
    return true;
}
// one call of the generator: 128 bits for the eight elements that share the counter
__device__ __forceinline__ uint4 drop_words(const Dropout &d, unsigned long long counter) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ d.key[2 * i];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ d.key[2 * i + 1];
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// v where element `e` of the eight that share `w` is kept, else 0
__device__ __forceinline__ float kept(const uint4 &w, int e, uint32_t below, float v) {
    const uint32_t word = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
    return ((e & 1) ? word : word << 16) > below ? v : 0.0f;
}
// the same as bits: bit e is set where element e is kept
__device__ __forceinline__ uint32_t keep_bits(const Dropout &d, unsigned long long counter) {
    const uint4 w = drop_words(d, counter);
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t word = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
        bits |= (uint32_t)(((e & 1) ? word : word << 16) > d.below) << e;
    }
    return bits;
}

inline bool is_16bit(int dtype) { return dtype == CCDC_BF16 || dtype == CCDC_F16; }
inline bool is_float_type(int dtype) { return dtype == CCDC_F32 || is_16bit(dtype); }
inline int type_bytes(int dtype) { return dtype == CCDC_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline size_t round_up(size_t v, size_t n) { return (v + n - 1) / n * n; }

// SM count of the current device; 0 on failure (status in *rc)
int block_sm_count(int *rc);
// allows a kernel `bytes` of dynamic shared memory on the current device; `done` remembers the devices it was asked on
int block_allow_smem(const void *kernel, int bytes, std::atomic<unsigned long long> *done);

inline int block_launch_status() {
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return ccdc_internal_cuda_fail((int)e);
    ccdc_internal_count_launch();
    return CCDC_OK;
}
