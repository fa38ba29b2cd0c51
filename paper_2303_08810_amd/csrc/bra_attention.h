// Attention between whole sequences: what its passes take (internal).
#pragma once

#include "bra_common.h"

namespace bra {
namespace att {

// A [B, N, heads, d] tensor, strides in bytes.
struct Rows {
    char *p;
    long batch, token, head;
};

struct Sizes {
    int B, Nq, Nk, H, Hk, d;
    bool f32, causal;
    float scale;
    const int *q_lens, *k_lens;             // or NULL
    int group() const { return H / Hk; }
    // Queries of the heads that share a key head are rows of one matrix: row = query * group + head within the group.
    long rows() const { return (long)Nq * group(); }
    int width() const { return (d + 31) / 32 * 32; }
};

}  // namespace att

size_t attention_workspace_bytes(const att::Sizes &S);
int attention_forward(const att::Sizes &S, const att::Rows &Q, const att::Rows &K, const att::Rows &V, const att::Rows &O, float *lse, void *ws, hipStream_t st);
size_t attention_backward_workspace_bytes(const att::Sizes &S);
int attention_backward(const att::Sizes &S, const att::Rows &Q, const att::Rows &K, const att::Rows &V, const att::Rows &O, const float *lse, const att::Rows &dO,
                       const att::Rows &dQ, const att::Rows &dK, const att::Rows &dV, void *ws, hipStream_t st);

}  // namespace bra
