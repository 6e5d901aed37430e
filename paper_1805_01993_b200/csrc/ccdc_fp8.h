// The 8-bit product on tcgen05, behind ccdc_matmul_fp8 (which has checked the arguments).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

struct Fp8Product {
    long long M, N, K;
    int experts;
    const uint8_t *x, *w;               // [M][K]; [experts][N][K]
    long long ldx, ldw, w_expert;
    const float *xs, *ws;
    long long xs_row, xs_col;
    const int *offsets;
    void *y;
    int y_type;
    long long ldy;
};

int fp8_mma_launch(const Fp8Product &p, int sms, cudaStream_t s);
// *failed: whether a bounded wait of any call ran out on the current device
int fp8_mma_status(int *failed);
