// Norms and position rotation of queries and keys: what both passes take (internal).
#pragma once

#include "bra_attention.h"

namespace bra {

struct QkNormSizes {
    long tokens;                // B N
    int N, heads, kv_heads;     // kv_heads 0: queries alone
    int d, turned, table_rows;
    bool f32, halves;
    float eps;
};

struct QkNormIn {
    att::Rows Q, K;
    const float *q_gamma, *k_gamma;         // or NULL: no norm
    const float *cos, *sin;
    const int *positions;                   // or NULL: a token's place in its sequence
};

int qk_norm_forward(const QkNormSizes &S, const QkNormIn &I, const att::Rows &Qout, const att::Rows &Kout, hipStream_t st);
size_t qk_norm_backward_workspace_bytes(const QkNormSizes &S);
int qk_norm_backward(const QkNormSizes &S, const QkNormIn &I, const att::Rows &gQ, const att::Rows &gK, const att::Rows &dQ, const att::Rows &dK, float *dq_gamma,
                     float *dk_gamma, void *ws, hipStream_t st);

}  // namespace bra
