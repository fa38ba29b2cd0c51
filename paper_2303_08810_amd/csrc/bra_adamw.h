// AdamW over many tensors (internal).
#pragma once

#include "bra_common.h"

namespace bra {

struct AdamwSteps {
    float beta1, rest1, beta2, rest2, eps;      // rest: 1 - beta
    float away, root;                           // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    const float *scalars;                       // where the step's number is on the device: `away` and `root` from here
    const float *grad_scale;
};

int adamw_step(const bra_adamw_tensor *tensors, int count, const bra_adamw_args &A, hipStream_t st);

}  // namespace bra
