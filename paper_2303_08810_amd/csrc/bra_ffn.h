// The gated feed-forward block's sizes and operands, as both of its passes use them (internal).
#pragma once

#include "bra_common.h"

namespace bra {
namespace ffn {

struct Sizes {
    long M;
    int C, h, act;
    bool f32;
    int Cp, hp;         // rounded up to multiples of 8: pitches of what lies in the workspace
    bool copies() const { return f32 || Cp != C || hp != h; }      // operands are laid out anew (k_operands)
    int terms() const { return f32 ? 3 : 1; }
};

// An operand of a product, pitch ld, the contraction of K; with three terms they are `plane` elements apart.
struct Operand {
    const bf16_t *p;
    long ld, plane;
    int K;              // beyond it reads as zero
};

// Out [M, N] = A B + bias: A's contraction inside, B's outside (`outer`) or inside.  Out in bf16, or float32 where the operands have three terms.
int product(const Operand &A, const Operand &Bm, bool outer, long M, int N, void *Out, const float *bias, bool f32, int kernel_id, hipStream_t st);

// Side of the tiles (256, 128 or 64) for a product of M x N outputs.
inline int tile_size(long M, long N)
{
    auto tiles = [&](long side) { return ((M + side - 1) / side) * ((N + side - 1) / side); };
    return tiles(256) >= 192 ? 256 : tiles(128) >= 192 ? 128 : 64;
}

// A matrix of `blocks` column blocks of `cols` columns laid out anew: each block padded with zeros to `cols_p` columns, float32 as three
// planes of terms.
struct Layout {
    const void *src;
    bf16_t *dst;
    long rows, plane;
    int blocks, cols, cols_p;
};
struct Layouts {
    Layout job[4];
    long end[4];        // pieces of 8 columns up to each job's end
    int count;
};
int lay_out(const Layouts &J, bool f32, hipStream_t st);
inline void add_layout(Layouts &J, const void *src, bf16_t *dst, long rows, int blocks, int cols, int cols_p, long plane)
{
    const long before = J.count ? J.end[J.count - 1] : 0;
    J.job[J.count] = Layout{src, dst, rows, plane, blocks, cols, cols_p};
    J.end[J.count++] = before + rows * blocks * (cols_p / 8);
}

}  // namespace ffn

size_t ffn_workspace_bytes(const ffn::Sizes &S);
int ffn_forward(const ffn::Sizes &S, const void *X, const void *W1, const float *b1, const void *W2, const float *b2, void *Y, void *pre, void *ws, hipStream_t st);
size_t ffn_backward_workspace_bytes(const ffn::Sizes &S);
int ffn_backward(const ffn::Sizes &S, const void *X, const void *W1, const float *b1, const void *W2, const void *pre, const void *dY, void *dX, void *dW1, void *dW2,
                 void *db1, void *db2, bool grads_f32, void *ws, hipStream_t st);

}  // namespace bra
