// Gradients of the gated feed-forward block.
//
//   k_hidden      dA = dY W2^T and, from it and G | U, dG | dU and A in bf16 (float32: three terms).  G | U are read, or formed
//                 again in the same tile by a second product, so that they are not rounded and not stored
//   k_product     dX = [dG | dU] W1^T
//   k_weights     dW1 = X^T [dG | dU] and dW2 = A^T dY, contractions over all tokens in shares, in one launch
//   k_columns     sums over the tokens for the biases' gradients
//   k_shares      the shares' sums, in order, in the type that is asked for
#include "bra_ffn.h"
#include "bra_ffn_dev.h"

namespace bra {
namespace ffn {

namespace {

// TD: the tile of dA, columns are hidden units; TG: that of G | U, the same rows and wavefronts.
template <class TD, class TG, int TERMS, int ACT, bool GIVEN, typename E>
__global__ __launch_bounds__(TD::kThreads, TD::kMinWaves) void k_hidden(Operand dY, Operand W2, Operand X, Operand W1, const float *__restrict__ b1, const E *__restrict__ pre,
                                                           bf16_t *__restrict__ Act, long plane_a, bf16_t *__restrict__ dP, long plane_p, long M, int h, int hp)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *lds = (bf16_t *)smem;
    constexpr int BJ = TD::BN, PW = 32 * TD::NT;         // hidden units of a tile, of a wavefront
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int mt0, nt0;
    tile_of(blockIdx.x, (int)((M + TD::BM - 1) / TD::BM), (hp + BJ - 1) / BJ, mt0, nt0);
    const long m0 = (long)mt0 * TD::BM;
    const int j0 = nt0 * BJ, last = hp - 8 - j0, rows = (int)min((long)TD::BM, M - m0);
    f32x16 acc[TD::NT][TD::MT];
    clear<TD>(acc);
    {
        const Loads<TD, TD::BM, false, false> la(wave, lane, dY.ld, [&](int row) { return (long)min(row, rows - 1); });
        const Loads<TD, TD::BN, false, true> lb(wave, lane, W2.ld, [&](int i) { return (long)min(i, h - 1 - j0); });
        multiply<TD, false, false, TERMS>(dY, W2, dY.p + m0 * dY.ld, W2.p + j0 * W2.ld, la, lb, 0, (dY.K + 63) / 64, lds, acc);
    }
    f32x16 gu[GIVEN ? 1 : TG::NT][TG::MT];
    if constexpr (!GIVEN) {
        clear<TG>(gu);
        const Loads<TG, TG::BM, false, false> la(wave, lane, X.ld, [&](int row) { return (long)min(row, rows - 1); });
        const Loads<TG, TG::BN, true, true> lb(wave, lane, W1.ld, [&](int col) {
            const int w = col / (2 * PW), in = col % (2 * PW);
            return (long)(min(w * PW + in % PW, last) + (in >= PW ? hp : 0));
        });
        multiply<TG, false, true, TERMS>(X, W1, X.p + m0 * X.ld, W1.p + j0, la, lb, 0, (X.K + 63) / 64, lds, gu);
    }
    const int hi = lane / 32, c = lane % 32, wm = (wave / TD::WC) * (32 * TD::MT), wj = j0 + (wave % TD::WC) * PW;
    const bool vec = h % 8 == 0;
    constexpr int P = PW / 8;
    // 32 rows at a time through this wavefront's part of LDS: G and U in, dG and dU in their places, then A
    bf16_t *const own = lds + wave * (2 * 32 * PW);
    const Rows<P> first{own}, second{own + 32 * PW};
    const bool whole = GIVEN && TERMS == 1 && vec && h >= 8;
#pragma unroll
    for (int mt = 0; mt < TD::MT; ++mt) {
        const int r0 = wm + 32 * mt, row = r0 + c;
        if (GIVEN && TERMS == 1 && whole) {
            // (pieces and rows that do not exist: the last ones again)
            lds_reads_done();
#pragma unroll
            for (int r = 0; r < 32; r += 64 / P) {
                const int in = r + lane / P, piece = (lane % P) ^ (in * P / 16 % P);
                const bf16_t *g = (const bf16_t *)pre + (size_t)(m0 + min(r0 + in, rows - 1)) * 2 * h + min(wj + 8 * piece, h - 8);
                load_to_lds_untracked(g, lds_address(own) + r * P * 16);
                load_to_lds_untracked(g + h, lds_address(own) + (32 + r) * P * 16);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        bf16x8 held[TD::NT][2][TERMS];
        auto pieces = [&](int q) {
#pragma unroll
            for (int nt = 0; nt < TD::NT; ++nt)
#pragma unroll
                for (int run = 0; run < 2; ++run) {
                    const int piece = 4 * nt + 2 * run + hi, j = wj + 8 * piece, n = h - j;
                    float g[8], u[8], a[8], dg[8], du[8];
                    if constexpr (GIVEN) {
                        if (TERMS == 1 && whole) {
                            load8((const bf16_t *)first.at(c, piece), g, 8, true);
                            load8((const bf16_t *)second.at(c, piece), u, 8, true);
                        } else {
                            const E *p = pre + (size_t)(m0 + min(row, rows - 1)) * 2 * h + j;
                            load8(p, g, n, vec);
                            load8(p + h, u, n, vec);
                        }
                    } else {
                        float bg[8], bu[8];
                        if (b1 && n > 0) {
                            load8(b1 + j, bg, n, false);
                            load8(b1 + h + j, bu, n, false);
                        } else
#pragma unroll
                            for (int e = 0; e < 8; ++e) bg[e] = bu[e] = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) { g[e] = gu[nt][mt][8 * run + e] + bg[e]; u[e] = gu[TD::NT + nt][mt][8 * run + e] + bu[e]; }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float f, slope;
                        activation_slope<ACT>(g[e], f, slope);
                        const float d = acc[nt][mt][8 * run + e];
                        a[e] = e < n ? f * u[e] : 0.f;
                        dg[e] = e < n ? d * u[e] * slope : 0.f;
                        du[e] = e < n ? d * f : 0.f;
                    }
                    bf16x8 t[TERMS];
                    operand<TERMS>(dg, t);
                    first.put(c, piece, t[q]);
                    operand<TERMS>(du, t);
                    second.put(c, piece, t[q]);
                    operand<TERMS>(a, held[nt][run]);
                }
        };
#pragma unroll
        for (int q = 0; q < TERMS; ++q) {
            pieces(q);
            auto flush = [&](const Rows<P> &from, bf16_t *to, long ld) {
                from.each(32, lane, [&](int in, int piece, bf16x8 v) {
                    if (r0 + in < rows && wj + 8 * piece < hp) *(bf16x8 *)(to + (size_t)(m0 + r0 + in) * ld + wj + 8 * piece) = v;
                });
            };
            flush(first, dP + q * plane_p, 2L * hp);
            flush(second, dP + q * plane_p + hp, 2L * hp);
#pragma unroll
            for (int nt = 0; nt < TD::NT; ++nt)
#pragma unroll
                for (int run = 0; run < 2; ++run) first.put(c, 4 * nt + 2 * run + hi, held[nt][run][q]);
            flush(first, Act + q * plane_a, hp);
        }
    }
}

// A contraction over the tokens: Part[share][rows][cols] = A^T B over the share's tokens; rows and cols as in the workspace (padded).
struct Contraction {
    Operand A, B;
    float *part;
    int rows, cols;
};

template <class T, int TERMS>
__global__ __launch_bounds__(T::kThreads, T::kMinWaves) void k_weights(Contraction J0, Contraction J1, int tiles0, int tiles1, int shares)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *lds = (bf16_t *)smem;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int share = blockIdx.x / (tiles0 + tiles1), i = blockIdx.x % (tiles0 + tiles1);
    const Contraction &J = i < tiles0 ? J0 : J1;
    int mt0, nt0;
    tile_of(i < tiles0 ? i : i - tiles0, (J.rows + T::BM - 1) / T::BM, (J.cols + T::BN - 1) / T::BN, mt0, nt0);
    const int r0 = mt0 * T::BM, c0 = nt0 * T::BN;
    const Loads<T, T::BM, true, false> la(wave, lane, J.A.ld, [&](int row) { return (long)min(row, J.rows - 8 - r0); });
    const Loads<T, T::BN, true, true> lb(wave, lane, J.B.ld, [&](int col) { return (long)min(col, J.cols - 8 - c0); });
    const int chunks = (J.A.K + 63) / 64, first = (int)((long)chunks * share / shares), end = (int)((long)chunks * (share + 1) / shares);
    f32x16 acc[T::NT][T::MT];
    clear<T>(acc);
    if (end > first) multiply<T, true, true, TERMS>(J.A, J.B, J.A.p + r0, J.B.p + c0, la, lb, first, end, lds, acc);
    const int hi = lane / 32, c = lane % 32, wm = (wave / T::WC) * (32 * T::MT), wn = (wave % T::WC) * (32 * T::NT);
    float *part = J.part + (size_t)share * J.rows * J.cols;
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
        for (int run = 0; run < 2; ++run) {
            const int col = c0 + wn + 32 * nt + 16 * run + 8 * hi;
            if (col >= J.cols) continue;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
                const int row = r0 + wm + 32 * mt + c;
                if (row >= J.rows) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[nt][mt][8 * run + e];
                store8(part + (size_t)row * J.cols + col, v, 8, true);
            }
        }
}

// Part[share][col] = sum over the share's rows of the columns of two maps (each the sum of its planes), 8 columns per thread, 32 rows
// of threads per workgroup.
struct Columns {
    const bf16_t *map;
    long ld, plane;
    float *part;
    int cols;
};
template <int TERMS>
__global__ __launch_bounds__(256) void k_columns(Columns J0, Columns J1, int groups0, long M, int shares)
{
    __shared__ float sums[32][64 + 4];
    const Columns J = (int)blockIdx.x < groups0 ? J0 : J1;
    const int group = (int)blockIdx.x < groups0 ? blockIdx.x : blockIdx.x - groups0, share = blockIdx.y;
    const int piece = threadIdx.x % 8, slot = threadIdx.x / 8, col = 64 * group + 8 * piece;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    if (col < J.cols)
        for (long m = M * share / shares + slot; m < M * (share + 1) / shares; m += 32)
#pragma unroll
            for (int q = TERMS - 1; q >= 0; --q) {
                float v[8];
                load8(J.map + q * J.plane + m * J.ld + col, v, 8, true);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += v[e];
            }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[slot][8 * piece + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < 64 && 64 * group + (int)threadIdx.x < J.cols) {
        float s = 0.f;
        for (int r = 0; r < 32; ++r) s += sums[r][threadIdx.x];
        J.part[(size_t)share * J.cols + 64 * group + threadIdx.x] = s;
    }
}

// out[row][block * cols + col] = sum over the shares of part[share][row][block * cols_p + col], 8 columns per thread.
struct Shares {
    const float *part;
    void *out;
    long size;          // of a share
    int blocks, cols, cols_p, shares;
};
struct SharesList {
    Shares job[4];
    long end[4];
    int count;
};
template <typename E>
__global__ __launch_bounds__(256) void k_shares(SharesList L)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    int j = 0;
    while (j < L.count && i >= L.end[j]) ++j;
    if (j == L.count) return;
    const Shares S = L.job[j];
    const long p = i - (j ? L.end[j - 1] : 0);
    const int per = S.cols_p / 8, piece = (int)(p % per);
    const long line = p / per;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    for (int s = 0; s < S.shares; ++s) {
        float v[8];
        load8(S.part + s * S.size + line * S.cols_p + 8 * piece, v, 8, true);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += v[e];
    }
    store8((E *)S.out + line * S.cols + 8 * piece, acc, S.cols - 8 * piece, S.cols % 8 == 0);
}

template <class TD, class TG, int TERMS, int ACT, bool GIVEN, typename E>
int launch_hidden(const Operand &dY, const Operand &W2, const Operand &X, const Operand &W1, const float *b1, const void *pre, bf16_t *Act, long plane_a, bf16_t *dP,
                  long plane_p, const Sizes &S, hipStream_t st)
{
    constexpr size_t bytes = GIVEN || TD::kLds > TG::kLds ? TD::kLds : TG::kLds;
    if (allow_lds<k_hidden<TD, TG, TERMS, ACT, GIVEN, E>>(bytes) != BRA_OK) return BRA_ERR_LAUNCH;
    const long tiles = ((S.M + TD::BM - 1) / TD::BM) * ((S.hp + TD::BN - 1) / TD::BN);
    k_hidden<TD, TG, TERMS, ACT, GIVEN, E><<<(unsigned)tiles, TD::kThreads, bytes, st>>>(dY, W2, X, W1, b1, (const E *)pre, Act, plane_a, dP, plane_p, S.M, S.h, S.hp);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <int TERMS, int ACT, typename E>
int pick_hidden(const Operand &dY, const Operand &W2, const Operand &X, const Operand &W1, const float *b1, const void *pre, bf16_t *Act, long pa, bf16_t *dP, long pp,
                const Sizes &S, hipStream_t st)
{
    if (pre) {
        switch (tile_size(S.M, S.hp)) {
        case 256: return launch_hidden<Tile<256, 256, 4, 2>, Tile<256, 256, 4, 2>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        case 128: return launch_hidden<Tile<128, 128, 2, 2>, Tile<128, 128, 2, 2>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        default: return launch_hidden<Tile<64, 64, 2, 2>, Tile<64, 64, 2, 2>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        }
    }
    if (tile_size(S.M, S.hp) >= 128)
        return launch_hidden<Tile<128, 128, 2, 4>, Tile<128, 256, 2, 4>, TERMS, ACT, false, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
    return launch_hidden<Tile<64, 64, 2, 2>, Tile<64, 128, 2, 2>, TERMS, ACT, false, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
}

template <class T, int TERMS>
int launch_weights(const Contraction &J0, const Contraction &J1, int shares, hipStream_t st)
{
    if (allow_lds<k_weights<T, TERMS>>(T::kLds) != BRA_OK) return BRA_ERR_LAUNCH;
    auto tiles = [](const Contraction &J) { return ((J.rows + T::BM - 1) / T::BM) * ((J.cols + T::BN - 1) / T::BN); };
    const int t0 = tiles(J0), t1 = tiles(J1);
    k_weights<T, TERMS><<<(unsigned)((t0 + t1) * shares), T::kThreads, T::kLds, st>>>(J0, J1, t0, t1, shares);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

// Tiles of the weights' gradients and the shares of the tokens: workgroups for every compute unit, in rounds that are
// nearly full, each with at least four chunks of 64 tokens.
struct WeightsPlan {
    int side, shares;
    WeightsPlan(const Sizes &S)
    {
        const int chunks = (int)((S.M + 63) / 64);
        auto tiles = [&](int side) {
            auto n = [&](int v) { return (v + side - 1) / side; };
            return (long)n(S.Cp) * n(2 * S.hp) + (long)n(S.hp) * n(S.Cp);
        };
        side = tiles(256) * std::min(8, std::max(1, chunks / 8)) >= 192 ? 256 : 128;
        const int resident = side == 256 ? 256 : 512;        // workgroups that run at once
        const long t = tiles(side);
        const int most = (int)std::max(1L, std::min<long>({(long)std::max(1, chunks / 4), 64L, 4 * resident / t + 1}));
        double best = 0;
        shares = 1;
        for (int s = 1; s <= most; ++s) {
            const long w = t * s;
            const double use = (double)w / (double)((w + resident - 1) / resident * resident) * (1 - 0.01 * s);
            if (use > best) { best = use; shares = s; }
        }
    }
};

constexpr int kColumnShares = 32;

struct BackwardPlan {
    size_t X, W1, W2, dY, Act, dP, parts1, parts2, cols1, cols2, total;
    BackwardPlan(const Sizes &S, const WeightsPlan &P)
    {
        size_t at = 0;
        auto take = [&](size_t bytes) {
            const size_t here = at;
            at += align256(bytes);
            return here;
        };
        const size_t e = S.terms() * sizeof(bf16_t), M = (size_t)S.M;
        X = S.copies() ? take(M * S.Cp * e) : 0;
        W1 = S.copies() ? take((size_t)S.C * 2 * S.hp * e) : 0;
        W2 = S.copies() ? take((size_t)S.h * S.Cp * e) : 0;
        dY = S.copies() ? take(M * S.Cp * e) : 0;
        Act = take(M * S.hp * e);
        dP = take(M * 2 * S.hp * e);
        parts1 = take((size_t)P.shares * S.Cp * 2 * S.hp * 4);
        parts2 = take((size_t)P.shares * S.hp * S.Cp * 4);
        cols1 = take((size_t)kColumnShares * 2 * S.hp * 4);
        cols2 = take((size_t)kColumnShares * S.Cp * 4);
        total = at;
    }
};

}  // namespace
}  // namespace ffn

using namespace ffn;

size_t ffn_backward_workspace_bytes(const Sizes &S) { return BackwardPlan(S, WeightsPlan(S)).total; }

int ffn_backward(const Sizes &S, const void *X, const void *W1, const float *b1, const void *W2, const void *pre, const void *dY, void *dX, void *dW1, void *dW2,
                 void *db1, void *db2, bool grads_f32, void *ws, hipStream_t st)
{
    const WeightsPlan W(S);
    const BackwardPlan P(S, W);
    auto at = [&](size_t offset) { return (bf16_t *)((char *)ws + offset); };
    const long pX = S.M * S.Cp, pW1 = (long)S.C * 2 * S.hp, pW2 = (long)S.h * S.Cp, pA = S.M * S.hp, pP = 2 * pA;
    int rc = BRA_OK;
    if (S.M > 0) {
        if (S.copies()) {
            Layouts J{};
            add_layout(J, X, at(P.X), S.M, 1, S.C, S.Cp, pX);
            add_layout(J, W1, at(P.W1), S.C, 2, S.h, S.hp, pW1);
            add_layout(J, W2, at(P.W2), S.h, 1, S.C, S.Cp, pW2);
            add_layout(J, dY, at(P.dY), S.M, 1, S.C, S.Cp, pX);
            rc = lay_out(J, S.f32, st);
            if (rc != BRA_OK) return rc;
            X = at(P.X); W1 = at(P.W1); W2 = at(P.W2); dY = at(P.dY);
        }
        Operand oX{(const bf16_t *)X, S.Cp, pX, S.Cp}, oW1{(const bf16_t *)W1, 2L * S.hp, pW1, S.C}, oW2{(const bf16_t *)W2, S.Cp, pW2, S.Cp},
            odY{(const bf16_t *)dY, S.Cp, pX, S.Cp};
        {
            ProfScope prof(st, K_FFN_HIDDEN_GRADS);
            bf16_t *A = at(P.Act), *dP = at(P.dP);
            if (S.f32) rc = S.act == BRA_SILU ? pick_hidden<3, BRA_SILU, float>(odY, oW2, oX, oW1, b1, pre, A, pA, dP, pP, S, st)
                                              : pick_hidden<3, BRA_GELU, float>(odY, oW2, oX, oW1, b1, pre, A, pA, dP, pP, S, st);
            else rc = S.act == BRA_SILU ? pick_hidden<1, BRA_SILU, bf16_t>(odY, oW2, oX, oW1, b1, pre, A, pA, dP, pP, S, st)
                                        : pick_hidden<1, BRA_GELU, bf16_t>(odY, oW2, oX, oW1, b1, pre, A, pA, dP, pP, S, st);
            if (rc != BRA_OK) return rc;
        }
        const Operand odP{at(P.dP), 2L * S.hp, pP, 2 * S.hp};
        Operand iW1 = oW1;
        iW1.K = 2 * S.hp;
        rc = product(odP, iW1, false, S.M, S.C, dX, nullptr, S.f32, K_FFN_PRODUCT, st);
        if (rc != BRA_OK) return rc;
        // over the tokens
        ProfScope prof(st, K_FFN_WEIGHT_GRADS);
        const int M = (int)S.M;
        const Contraction J0{{(const bf16_t *)X, S.Cp, pX, M}, {at(P.dP), 2L * S.hp, pP, M}, (float *)at(P.parts1), S.Cp, 2 * S.hp};
        const Contraction J1{{at(P.Act), S.hp, pA, M}, {(const bf16_t *)dY, S.Cp, pX, M}, (float *)at(P.parts2), S.hp, S.Cp};
        if (W.side == 256) rc = S.f32 ? launch_weights<Tile<256, 256, 4, 2>, 3>(J0, J1, W.shares, st) : launch_weights<Tile<256, 256, 4, 2>, 1>(J0, J1, W.shares, st);
        else rc = S.f32 ? launch_weights<Tile<128, 128, 2, 2>, 3>(J0, J1, W.shares, st) : launch_weights<Tile<128, 128, 2, 2>, 1>(J0, J1, W.shares, st);
        if (rc != BRA_OK) return rc;
        if (db1 || db2) {
            const Columns C0{at(P.dP), 2L * S.hp, pP, (float *)at(P.cols1), 2 * S.hp}, C1{(const bf16_t *)dY, S.Cp, pX, (float *)at(P.cols2), S.Cp};
            const int g0 = db1 ? (2 * S.hp + 63) / 64 : 0, g1 = db2 ? (S.Cp + 63) / 64 : 0;
            const dim3 grid(g0 + g1, kColumnShares);
            if (S.f32) k_columns<3><<<grid, 256, 0, st>>>(C0, C1, g0, S.M, kColumnShares);
            else k_columns<1><<<grid, 256, 0, st>>>(C0, C1, g0, S.M, kColumnShares);
            if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
        }
    }
    ProfScope prof(st, K_FFN_SUMS);
    SharesList L{};
    auto add = [&](const float *part, void *out, int rows, int rows_p, int blocks, int cols, int cols_p, int shares) {
        if (!out) return;
        const long before = L.count ? L.end[L.count - 1] : 0;
        L.job[L.count] = Shares{part, out, (long)rows_p * blocks * cols_p, blocks, cols, cols_p, S.M > 0 ? shares : 0};
        L.end[L.count++] = before + (long)rows * blocks * (cols_p / 8);
    };
    add((const float *)at(P.parts1), dW1, S.C, S.Cp, 2, S.h, S.hp, W.shares);
    add((const float *)at(P.parts2), dW2, S.h, S.hp, 1, S.C, S.Cp, W.shares);
    add((const float *)at(P.cols1), db1, 1, 1, 2, S.h, S.hp, kColumnShares);
    add((const float *)at(P.cols2), db2, 1, 1, 1, S.C, S.Cp, kColumnShares);
    const unsigned blocks = (unsigned)((L.end[L.count - 1] + 255) / 256);
    if (grads_f32) k_shares<float><<<blocks, 256, 0, st>>>(L);
    else k_shares<bf16_t><<<blocks, 256, 0, st>>>(L);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

}  // namespace bra
