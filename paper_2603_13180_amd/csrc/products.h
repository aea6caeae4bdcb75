// products.h -- what the composed MXNormLinear calls use of the entry points'
// implementation (internal; not part of the C ABI): the entry points' argument
// checks, which launch nothing, and the parts of the backward that share a
// launch, whose arguments the caller has checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mxnorm.h"

namespace mxk {

// mxnorm_mx_fwd's and mx_cast_fwd's checks; coef <= 0 becomes the table's.
mx_status check_mxnorm(const void *x, int64_t T, int64_t d, int block, int elem, int p, float &coef,
                       float eps, int scale_mode, const uint8_t *codes, const uint8_t *scales,
                       const float *rho);
mx_status check_cast(const void *x, const void *gamma, int64_t T, int64_t d, int block, int elem,
                     int scale_mode, const uint8_t *codes, const uint8_t *scales);

} // namespace mxk

namespace mxg {

// out = dec(a) dec(b)^T (times gain per column), as mx_matmul_fwd's arguments;
// M, N > 0.
struct Product {
    const uint8_t *a, *as, *b, *bs;
    int64_t M, N, K;
    const void *gain;
    void *out;
};

// mx_matmul_fwd's checks.
mx_status check_product(const Product &P, int block, int elem, int out_dtype);

// mx_gated_fwd's arguments and checks.
struct GatedProduct {
    const uint8_t *a, *as, *w, *ws;
    int64_t M, F, K;
    int act, mode, out_dtype;
    void *out;
    uint8_t *out_scales;
    void *gu;
};
mx_status check_gated(const GatedProduct &P, int block, int elem);
// mxnorm_gated_fwd's norm: x bf16 [M, K] in place of the product's operand.
struct RowNorm {
    const void *x;
    float *rho;
    int p;
    float coef, eps;
};
// The norm and the product (M, F > 0, both checked) in one launch, with the
// bits of two, where so few rows allow it; false: nothing was launched.
bool normed_product(const GatedProduct &P, const RowNorm &n, int elem, hipStream_t stream, mx_status &st);
// mx_gated_bwd's checks.
mx_status check_gated_bwd(const void *grad_h, const void *gu, int64_t T, int64_t F, int act,
                          const void *grad_gu);

// A product with output of type out0 and one with bf16 output that do not
// depend on each other, on one stream: within mx_matmul_fwd's bound, in one
// launch or two, so the sums may be taken in another order than by two
// mx_matmul_fwd calls.  may_split: the second's also as four partial sums, where
// that is faster.
mx_status matmul_pair(const Product &first, int out0, const Product &bf16, int elem, bool may_split,
                      hipStream_t stream);

} // namespace mxg

namespace mxb {

// mx_cast_t_fwd's and mxnorm_ste_bwd's checks.
mx_status check_cast_t(const void *x, const float *rho, int64_t R, int64_t C, int block, int elem,
                       int scale_mode, const uint8_t *codes, const uint8_t *scales);
mx_status check_ste(const void *x, const void *grad_z, const void *gamma, const float *rho,
                    int64_t T, int64_t d, int out_dtype, const void *grad_x, const float *grad_gamma,
                    const void *workspace, size_t workspace_bytes);

// mxnorm_ste_bwd after its checks, T > 0, with grad_gamma in gamma_dtype.
mx_status ste(const void *x, const void *grad_z, const void *gamma, const float *rho, int64_t T,
              int64_t d, int out_dtype, void *grad_x, int gamma_dtype, void *grad_gamma,
              void *workspace, hipStream_t stream);

// Codes and scales of the backward's casts, laid out as the entry points of
// the single casts do (RCEIL, blocks of 32).
struct BackwardCasts {
    uint8_t *gh, *gh_s;   // grad_H [T, N] along N
    uint8_t *ght, *ght_s; // grad_H^T [N, T] along T
    uint8_t *wt, *wt_s;   // W^T [d, N] along N
    uint8_t *xt, *xt_s;   // (rho X)^T [d, T] along T
};

// The casts along T are of T rows and then zeros up to Tp.  Tp and N multiples
// of 128, d of 16; grad_h, x, w 16-byte aligned.  With a gate grad_h is H's
// gradient [T, N/2], and what is cast are both projections' gradients [T, N],
// mx_gated_bwd's values.
struct Gate {
    const void *gu;
    int act;
};
mx_status backward_casts(const void *grad_h, const void *x, const float *rho, const void *w,
                         int64_t T, int64_t Tp, int64_t N, int64_t d, int elem,
                         const BackwardCasts &o, const Gate *gate, hipStream_t stream);

} // namespace mxb
