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

// Sides of the tiles (256, 128 or 64), by the number of tiles there would be: large ones multiply faster (one workgroup per compute unit,
// 1.2 PFLOP/s in long loops, against 0.9 and 0.5), small ones fill the chip.  Measured (us with 256 / 128 / 64):
//   k_gated    4096 x 512 x 1368 (176 large tiles) 22.8 / 25.0 / 27.7, 12544 x 128 x 256 (98; 392 of 128) 12.9 / 9.8 / 11.9,
//              1024 x 768 x 2048 (256 of 128) 26.1 / 17.8 / 15.2
//   k_product  12544 x 768 x 2048 (147) 48.8 / 65.2 / 70.9, 12544 x 512 x 1368 (98; 392) 38.7 / 29.8 / 42.5, 4096 x 768 x 2048 (192 of 128) 45.8 / 30.9 / 27.3
//              12544 x 256 (196 of 128; 784 of 64 are more than three to a compute unit, a second round) with a contraction of 512 - / 10.4 / 12.1, 2048 - / 30.5 / 32.0,
//              12288 x 256 (192; 768) 512 - / 10.2 / 10.8, 1024 - / 17.1 / 16.8, 2048 - / 30.1 / 28.1
//   k_hidden   given G | U, bound by its reads and stores: 12544 x 768 (392) 99 / 103 / 119, 12544 x 512 (294) 75.9 / 64.4 / 63.5,
//              4096 x 256 (128 of 128) 29.1 / 16.2 / 10.4;  otherwise 12544 x 128 (196 of 128) - / 15.2 / 17.1, 4096 x 256 (128) - / 16.8 / 13.4
inline long tiles(long M, long N, long side) { return ((M + side - 1) / side) * ((N + side - 1) / side); }
inline int gated_side(const Sizes &S) { return tiles(S.M, 2L * S.hp, 256) >= 160 ? 256 : tiles(S.M, 2L * S.hp, 128) >= 300 ? 128 : 64; }
inline int product_side(long M, long N) { return tiles(M, N, 256) >= 140 ? 256 : tiles(M, N, 128) >= 195 ? 128 : 64; }
inline int hidden_side(const Sizes &S, bool given)
{
    const long t = tiles(S.M, S.hp, 128);
    if (!given) return t >= 170 ? 128 : 64;
    return S.C >= 512 && tiles(S.M, S.hp, 256) >= 350 ? 256 : t >= 300 ? 128 : 64;
}

// Whether the forward goes to k_few: up to 128 rows it is the faster one at every width (us, k_few / tiles: 1 x 768 x 2048 8.8 / 21.2,
// 128 x 768 x 2048 15.2 / 21.9, 128 x 1024 x 4096 29 / 34).
inline bool few_rows(const Sizes &S) { return !S.f32 && S.M <= 128; }

// And to k_few_f32, whose vector instructions take a time that grows with the rows (us, k_few_f32 / tiles: 1 x 768 x 2048 18 / 43, 32 rows 37 / 44, 64 rows 53 / 45;
// 32 x 1024 x 2816 62 / 57; 128 x 256 x 512 19 / 29, 48 x 512 x 1368 37 / 36).
inline bool few_rows_f32(const Sizes &S) { return S.f32 && (S.M <= 32 || (S.M <= 128 && (double)S.M * S.C * S.h <= 32e6)); }

// Workgroups of 256 in a launch: 2^32 threads and more cannot be launched.
constexpr long kMaxBlocks = 1L << 23;

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
