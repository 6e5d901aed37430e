// Matrix products of the feed-forward block on the fifth-generation tensor cores, as the host sees them.
#pragma once

#include "ccdc_block.h"

// A row-major matrix of 16-bit elements in `planes` equal planes (a binary32 matrix is held as three bf16 planes
// whose sum it is).  Address and row pitch are multiples of 16 bytes.
struct MmaMatrix {
    const void *p;
    long long rows, cols, ld;       // ld in elements
    int planes;                     // plane stride: rows * ld elements
};
// One side of a product: the matrix as it lies ([index][k]) or transposed ([k][index]).
struct MmaSide {
    MmaMatrix m;
    bool transposed;
};
enum MmaEpilogue { MMA_STORE = 0, MMA_GATE = 1, MMA_GATE_BACK = 2 };

// C = sum over terms of A_t B_t^T.
// GATE: two B sides and one A: h = A B_0^T and u = A B_1^T.
struct MmaProduct {
    long long M, N, K;
    int terms;
    MmaSide a[2], b[2];
    // STORE
    void *c;
    long long ldc;
    int c_type;                     // CCDC_F32, CCDC_BF16, CCDC_F16
    int splits;                     // > 1: binary32 partial products [splits][M][ldc] at c
    // GATE and GATE_BACK
    int act;
    float *h, *u;                   // saved values, see ffn_saved_index; GATE: may be NULL
    MmaMatrix out[2];               // GATE: a; GATE_BACK: dh, du
};

// h and u are kept in blocks of 32 rows by 4 columns, row after row, so that the 32 threads that hold one row each
// read and write 512 consecutive bytes.
__host__ __device__ __forceinline__ long long ffn_saved_index(long long m, long long f, long long groups) {
    return (((m >> 5) * groups + (f >> 2)) * 32 + (m & 31)) * 4 + (f & 3);
}
__host__ __device__ __forceinline__ long long ffn_saved_groups(long long F) { return (F + 3) / 4; }

// Tile shapes: two SMs to 256 x 512 or 256 x 256, one SM to 128 x 128; binary32 blocks: two SMs to 256 x 128.
enum MmaTile { MMA_WIDE = 0, MMA_PAIR = 1, MMA_SINGLE = 2, MMA_PLANES = 3 };
inline int mma_tile_rows(MmaTile t) { return t == MMA_SINGLE ? 128 : 256; }
inline int mma_tile_columns(MmaTile t) {        // GATE: of h and u together
    return t == MMA_WIDE ? 512 : t == MMA_PAIR ? 256 : 128;
}

// All products of a call go through one launch: `type` CCDC_BF16 or CCDC_F16.  Matrices of three planes take
// MMA_PLANES, others one of the first three.
int mma_launch(const MmaProduct *products, int count, MmaEpilogue epilogue, int type, MmaTile tile, int sms, cudaStream_t s);
int mma_status(int *failed);     // *failed: whether a wait ever ran out on the current device
