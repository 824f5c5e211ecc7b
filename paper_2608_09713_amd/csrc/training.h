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

}  // namespace spsyrk
