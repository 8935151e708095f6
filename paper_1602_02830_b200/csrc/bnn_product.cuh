// The 16-bit matrix product behind the dense layer and the gated projections (internal interface).
#pragma once
#include "bnn_real.cuh"

enum BnnEpilogue {
    BNN_EPI_LINEAR,       // z = sum + bias; pre = z; out0 = add + act(z)
    BNN_EPI_LINEAR_BACK,  // out0 = add * act'(sum + bias)
    BNN_EPI_GATED,        // g, u: pre = (g, u); out0 = act(g) u
    BNN_EPI_GATED_BACK    // out0 = add u act'(g), out1 = add act(g)
};
enum { BNN_CHEAPEST = 0, BNN_PAIR = 1, BNN_FEW = 2 };
// One operand: rows of `ld` elements.  Its rows run along the output's rows (columns) and its columns along the sum, or, with
// BnnProduct::a_mn / b_mn, the other way round.
struct BnnOperand { const void *p; int64_t ld; };
struct BnnProduct {
    int dtype;                    // BNN_F16 or BNN_BF16
    int epilogue;
    BnnOperand a[2], b[2];
    int a_mn, b_mn;
    int pairs;                    // 2: out = a0 b0 + a1 b1 (linear epilogues)
    int64_t M, N, K;              // K: of each pair
    const void *bias;             // N or NULL
    const void *add; int64_t ld_add;
    void *out[2]; int64_t ldo[2];
    float *pre; int64_t ldp;      // EPI_GATED: [2][M][ldp]
    int act;
    int kernel;                   // BNN_CHEAPEST, or the one to use
};
// Up to three products in one launch (several: linear epilogue without bias, add or pre).  Every operand must satisfy bnn_rows16.
// M, N > 0; K = 0 is the empty sum.
int bnn_product(bnn_ctx *ctx, const BnnProduct *list, int count);
// Whether several products are made faster apart than in one launch of the pair kernel; few[i]: product i on the kernel for few rows.
bool bnn_product_apart(const bnn_ctx *ctx, const BnnProduct *list, int n, bool *few);
