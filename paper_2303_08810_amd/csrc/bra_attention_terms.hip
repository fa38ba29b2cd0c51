// float32 operands of attention as three bf16 terms each, hi + mid + lo, in planes that the products' tiles are loaded from: keys and values a head after
// the other, queries and dO as rows (query, head) of a key head.  Zero behind the lengths, behind the last row up to a multiple of 32, and behind a head's
// channels up to the pitch, so that the tiles need no bounds.  Bound by memory.
#include "bra_attention_dev.h"

#include <algorithm>

namespace bra {
namespace att {
namespace {

struct Tensors {
    Rows R[4];              // K, V, Q, dO
    char *planes[4];
    unsigned blocks[4];     // workgroups of the tensors up to this one
    int n;
};

// A workgroup has 128 pieces of 8 channels of a head.  2 x 1295 tokens of 8 / 2 heads of 72: K, V, Q and dO 9 us, 40 MB written.
template <int P>
__global__ __launch_bounds__(128) void k_attention_terms(Call A, Tensors X, unsigned first)
{
    constexpr int kPieces = P / 8, kRows = 128 / kPieces;
    unsigned block = first + blockIdx.x;
    int which = 0;
    while (which + 1 < X.n && block >= X.blocks[which]) ++which;
    if (which) block -= X.blocks[which - 1];
    const bool keys = which < 2;
    const unsigned per = (unsigned)(keys ? A.key_rows : A.row_rows) / kRows;
    const int hb = (int)(block / per), row = (int)(block - hb * per) * kRows + threadIdx.x / kPieces, piece = threadIdx.x % kPieces, b = hb / A.Hk, hk = hb - b * A.Hk;
    const long i = (long)block * 128 + threadIdx.x;
    const Sequence seq(A, b);
    const Rows &R = X.R[which];
    int token = row, head = hk;
    bool there = row < seq.nk;
    if (!keys) {
        token = row_query(A, row);
        head = hk * A.G + row - token * A.G;
        there = token < seq.nq;
    }
    float v[8] = {};
    if (there && 8 * piece < A.d) {
        const char *p = R.p + b * R.batch + token * R.token + head * R.head + 32 * piece;
        const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(p + 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = v0[e];
            v[4 + e] = v1[e];
        }
    }
    bf16x8 t[3];
    split3(v, t);
    char *out = X.planes[which] + i * 16;
#pragma unroll
    for (int k = 0; k < 3; ++k) *(bf16x8 *)(out + k * (keys ? A.key_plane : A.row_plane)) = t[k];
}

int pitch(const Sizes &S) { return S.width() <= 32 ? 32 : S.width() <= 64 ? 64 : 128; }
long padded(long rows) { return (rows + 31) / 32 * 32; }
long plane_bytes(const Sizes &S, long rows) { return (long)S.B * S.Hk * padded(rows) * pitch(S) * 2; }

}  // namespace

size_t terms_bytes(const Sizes &S, bool backward) { return align256(2 * 3 * (plane_bytes(S, S.Nk) + (backward ? plane_bytes(S, S.rows()) : 0))); }

int make_terms(const Sizes &S, Call &A, bool backward, void *ws, hipStream_t st)
{
    A.key_rows = (int)padded(S.Nk);
    A.row_rows = (int)padded(S.rows());
    A.key_plane = plane_bytes(S, S.Nk);
    A.row_plane = plane_bytes(S, S.rows());
    Tensors X{};
    char *p = (char *)ws;
    X.n = backward ? 4 : 2;
    long blocks = 0;
    const Rows all[4] = {A.K, A.V, A.Q, A.dO};
    for (int i = 0; i < X.n; ++i) {
        X.R[i] = all[i];
        X.planes[i] = p;
        const long plane = i < 2 ? A.key_plane : A.row_plane;
        blocks += plane / 16 / 128;             // (32 rows of 4 pieces at least: whole workgroups)
        X.blocks[i] = (unsigned)blocks;
        p += 3 * plane;
    }
    if (blocks >= 1L << 32) return BRA_ERR_UNSUPPORTED;
    A.pK = X.planes[0];
    A.pV = X.planes[1];
    A.pQ = X.planes[2];
    A.pG = X.planes[3];
    for (long first = 0; first < blocks; first += kMaxBlocks) {
        const unsigned n = (unsigned)std::min(kMaxBlocks, blocks - first);
        const ProfScope scope(st, K_ATTENTION_TERMS);
        if (pitch(S) == 32) k_attention_terms<32><<<n, 128, 0, st>>>(A, X, (unsigned)first);
        else if (pitch(S) == 64) k_attention_terms<64><<<n, 128, 0, st>>>(A, X, (unsigned)first);
        else k_attention_terms<128><<<n, 128, 0, st>>>(A, X, (unsigned)first);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

}  // namespace att
}  // namespace bra
