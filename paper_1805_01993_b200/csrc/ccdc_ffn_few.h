// Backward products of a binary32 feed-forward block for few rows, on the plain cores.
#pragma once

#include "ccdc_block.h"

// the most rows these and the forward products of few rows (binary32) serve
constexpr long long FEW_MOST = 32;

// parts[s][m][n] = the s-th share along k of sum over terms t and k of p_t[m][k] w_t[k][n]
struct FewAcross {
    long long M, N, K;
    int terms, splits;
    const float *p[2], *w[2];
    long long ldp, ldw, ldo;
    float *parts;
};
int few_across_splits(long long M, long long N, long long K, int terms, int sms);
int few_across(const FewAcross &a, cudaStream_t s);

// da = the sum of the parts; dh = da u act'(h), du = da act(h)
struct FewGateBack {
    long long M, N, ld;
    int splits, act;
    const float *parts, *h, *u;
    float *dh, *du;
};
int few_gate_back(const FewGateBack &a, cudaStream_t s);

// out[r][c] = sum over m of p[m][r] q[m][c], for up to three matrices in one launch
struct FewOuter {
    const float *p, *q;
    long long ldp, ldq, R, C;
    float *out;
};
struct FewOuters {
    FewOuter o[3];
    long long M;
    int count;
};
int few_outer(const FewOuters &a, cudaStream_t s);
