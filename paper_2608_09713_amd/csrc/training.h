// Arguments of the operators of a training step: the cross entropy of a linear
// layer, the norms around a block, and the AdamW step.
#pragma once

#include "rows.h"

namespace spsyrk {

// a column per row; outside [0, V): padding
struct Targets {
    const void* p = nullptr;
    int64_t stride = 1;
    int bytes = 8;
};

// ---- crossentropy.hip
// loss (and lse, may be null) of every row of X against the rows of W.
size_t linear_cross_entropy_tmp_bytes(const DenseRows& X, const DenseRows& W);
void linear_cross_entropy(const DenseRows& X, const DenseRows& W, const Targets& t, float scale, float* loss,
                          float* lse, void* tmp, hipStream_t s);
// loss, and the gradients of sum weight loss (weight null: 1)
size_t linear_cross_entropy_grad_tmp_bytes(const DenseRows& X, const DenseRows& W);
void linear_cross_entropy_grad(const DenseRows& X, const DenseRows& W, const Targets& t, float scale,
                               const float* weight, float* loss, const DenseRows& dX, const DenseRows& dW, void* tmp,
                               hipStream_t s);

// ---- blocknorm.hip
// The gate of a block: a row for every `per` (at least 1) rows, or (own) for
// every row, of 32-bit floats (wide) or of the rows' type; p null: ones.
struct BlockGate {
    const void* p = nullptr;
    int64_t rows = 0, ld = 0, per = 1;
    bool own = false, wide = false;
};
// weights of the norms, of 32-bit floats (wide) or of the rows' type; null: ones
struct BlockParams {
    const void *post = nullptr, *pre = nullptr;
    bool wide = false;
};
void block_norm(const DenseRows& X, const DenseRows& B, const BlockGate& gate, float scale, const BlockParams& par,
                bool normed, float eps, const DenseRows& Y, const DenseRows& H, float* rstd_post, float* rstd_pre,
                hipStream_t s);
size_t block_norm_grad_tmp_bytes(int64_t m, int64_t d, int dt, const BlockGate& gate);
// DY.p null: no gradient of y; rstd_post null: the block has no norm of its own
void block_norm_grad(const DenseRows& DY, const DenseRows& DH, const DenseRows& Y, const DenseRows& B,
                     const float* rstd_post, const float* rstd_pre, const BlockGate& gate, float scale,
                     const BlockParams& par, const DenseRows& DX, const DenseRows& DB, void* dgate, int64_t lddg,
                     void* dpost, void* dpre, void* tmp, hipStream_t s);

// ---- adamw.hip
// elements that share a scale in 8-bit states
constexpr int kAdamBlock = 256;
struct AdamTensor {
    int64_t n;
    void* p;
    const void* g;
    float* master;            // 32-bit copy of the parameters, or null
    void *m, *v;              // floats, or codes of 8 bits
    float *m_scale, *v_scale; // of 8-bit states: a float per kAdamBlock elements
};
struct AdamRates {
    float lr_decay, lr_m;  // lr decay, lr / (1 - b1^t)
    float b1, a1, b2, a2;  // rates, and 1 - rates
    float inv_v, eps;      // 1 / (1 - b2^t)
    double d1, d2;         // the rates in 64 bits
    const float* grad_scale;
};
void adamw(const AdamTensor* t, int64_t count, int param_dtype, int grad_dtype, int bits, bool master,
           const AdamRates& r, hipStream_t s);
// m into t.p, v into t.master, both floats
void adam_values(const AdamTensor* t, int64_t count, hipStream_t s);

}  // namespace spsyrk
