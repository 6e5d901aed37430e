// Products of the feed-forward block for few rows: bound by reading the weights once.
#pragma once

#include "ccdc_block.h"
#include "ccdc_ffn_few.h"

// out[m][n] = sum_k x[m][k] w[n][k] for m < M, n < N; with a second matrix w2 the two products h and u make
// a = act(h) u.  dtype for x, w and the output; h, u: NULL or where they are kept (ffn_saved_index).
struct RowsProduct {
    long long M, N, K;
    const void *x, *w, *w2;
    long long ldx, ldw;
    void *out;
    long long ldo;
    float *h, *u;
    int act, dtype;
    bool weights_early;     // the launch before this one does not write the weights
};
inline long long rows_most(int dtype) { return dtype == CCDC_F32 ? FEW_MOST : 8; }      // the most rows served
int rows_launch(const RowsProduct &p, int sms, cudaStream_t s);
