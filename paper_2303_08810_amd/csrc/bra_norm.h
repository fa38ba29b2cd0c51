// Norms around a residual sum: what both passes take (internal).
#pragma once

#include "bra_common.h"

namespace bra {

struct NormSizes {
    long rows, per_group;       // per_group rows share a row of the gate
    int C, groups;
    bool f32, layer, post;
    float eps;
    bool vec;                   // rows are whole 16-byte pieces, pointers aligned
};

struct NormIn {
    const void *X, *Y, *gate;
    const float *gamma, *beta, *post_gamma, *post_beta, *scale;
};

int norm_forward(const NormSizes &S, const NormIn &I, void *R, void *N, hipStream_t st);

struct NormGrads {
    void *dX, *dY, *dgate;
    float *dgamma, *dbeta, *dpost_gamma, *dpost_beta, *dscale;
};
size_t norm_backward_workspace_bytes(const NormSizes &S);
// I.X is the sum that the forward returned.
int norm_backward(const NormSizes &S, const NormIn &I, const void *dN, const void *dR, const NormGrads &G, void *ws, hipStream_t st);

}  // namespace bra
