// Gradients of the gated feed-forward block.
//
//   k_hidden      dA = dY W2^T and, from it and G | U, dG | dU and A in bf16 (float32: three terms).  G | U are read, or formed
//                 again in the same tile by a second product, so that they are not rounded and not stored
//   k_gradients   dX = [dG | dU] W1^T in tiles, dW1 = X^T [dG | dU] and dW2 = A^T dY in parts of the contraction over all tokens, and the
//                 columns' sums for the biases: one launch, none of them waits for another
//   k_sums        the parts' sums, in order, in the type that is asked for
#include "bra_ffn.h"
#include "bra_ffn_dev.h"

#include <algorithm>

namespace bra {
namespace ffn {

namespace {

// TD: the tile of dA, columns are hidden units; TG: that of G | U, the same rows and wavefronts.
// Given G | U bound by what it reads and stores behind a short product: 16384 x 1024 x 2816 187 us for 95 GFLOP and 0.50 GB, matrix cores busy in 28 %
// of the cycles.  Forming G | U again 12544 x 128 x 256 takes 17 us: one round of 196 workgroups, half of it the slope's arithmetic.
template <class TD, class TG, int TERMS, int ACT, bool GIVEN, typename E>
__global__ __launch_bounds__(TD::kThreads, TD::kMinWaves) void k_hidden(Operand dY, Operand W2, Operand X, Operand W1, const float *__restrict__ b1, const E *__restrict__ pre,
                                                           bf16_t *__restrict__ Act, long plane_a, bf16_t *__restrict__ dP, long plane_p, long M, int h, int hp,
                                                           int first_tile)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *lds = (bf16_t *)smem;
    constexpr int BJ = TD::BN, PW = 32 * TD::NT;         // hidden units of a tile, of a wavefront
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int mt0, nt0;
    tile_of(first_tile + blockIdx.x, (int)((M + TD::BM - 1) / TD::BM), (hp + BJ - 1) / BJ, mt0, nt0);
    const long m0 = (long)mt0 * TD::BM;
    const int j0 = nt0 * BJ, last = hp - 8 - j0, rows = (int)min((long)TD::BM, M - m0);
    f32x16 acc[TD::NT][TD::MT];
    clear<TD>(acc);
    {
        const Loads<TD, TD::BM, false> la(wave, lane, dY.ld, [&](int row) { return (long)min(row, rows - 1); });
        const Loads<TD, TD::BN, false> lb(wave, lane, W2.ld, [&](int i) { return (long)min(i, h - 1 - j0); });
        multiply<TD, false, false, TERMS>(dY, W2, dY.p + m0 * dY.ld, W2.p + j0 * W2.ld, la, lb, 0, (dY.K + 63) / 64, lds, acc);
    }
    f32x16 gu[GIVEN ? 1 : TG::NT][TG::MT];
    if constexpr (!GIVEN) {
        clear<TG>(gu);
        const Loads<TG, TG::BM, false> la(wave, lane, X.ld, [&](int row) { return (long)min(row, rows - 1); });
        const Loads<TG, TG::BN, true> lb(wave, lane, W1.ld, [&](int col) {
            const int w = col / (2 * PW), in = col % (2 * PW);
            return (long)(min(w * PW + in % PW, last) + (in >= PW ? hp : 0));
        });
        multiply<TG, false, true, TERMS>(X, W1, X.p + m0 * X.ld, W1.p + j0, la, lb, 0, (X.K + 63) / 64, lds, gu);
    }
    const int hi = lane / 32, c = lane % 32, wm = (wave / TD::WC) * (32 * TD::MT), wj = j0 + (wave % TD::WC) * PW;
    const bool vec = h % 8 == 0, vec_b = vec && (uintptr_t)b1 % 16 == 0;
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
        // A waits in registers, and with it all terms of dG and dU where they fit: otherwise they are formed again for each term
        constexpr bool kHold = TERMS > 1 && TD::NT <= 2;
        bf16x8 held[TD::NT][2][TERMS], held_g[kHold ? TD::NT : 1][2][TERMS], held_u[kHold ? TD::NT : 1][2][TERMS];
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
                            load8(b1 + j, bg, n, vec_b);
                            load8(b1 + h + j, bu, n, vec_b);
                        } else
#pragma unroll
                            for (int e = 0; e < 8; ++e) bg[e] = bu[e] = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) { g[e] = gu[nt][mt][8 * run + e] + bg[e]; u[e] = gu[TD::NT + nt][mt][8 * run + e] + bu[e]; }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float f, slope;
                        activation_slope<ACT, TERMS != 1>(g[e], f, slope);
                        const float d = acc[nt][mt][8 * run + e];
                        a[e] = e < n ? f * u[e] : 0.f;
                        dg[e] = e < n ? d * u[e] * slope : 0.f;
                        du[e] = e < n ? d * f : 0.f;
                    }
                    operand<TERMS>(a, held[nt][run]);
                    if constexpr (kHold) {
                        operand<TERMS>(dg, held_g[nt][run]);
                        operand<TERMS>(du, held_u[nt][run]);
                    } else {
                        bf16x8 t[TERMS];
                        operand<TERMS>(dg, t);
                        first.put(c, piece, t[q]);
                        operand<TERMS>(du, t);
                        second.put(c, piece, t[q]);
                    }
                }
        };
#pragma unroll
        for (int q = 0; q < TERMS; ++q) {
            if (!kHold || q == 0) pieces(q);
            if constexpr (kHold)
#pragma unroll
                for (int nt = 0; nt < TD::NT; ++nt)
#pragma unroll
                    for (int run = 0; run < 2; ++run) {
                        first.put(c, 4 * nt + 2 * run + hi, held_g[nt][run][q]);
                        second.put(c, 4 * nt + 2 * run + hi, held_u[nt][run][q]);
                    }
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

// Contractions over the tokens, dW = A^T B, rows x cols as they lie in the workspace (padded).  The tiles of both stand in one row, each with
// `chunks` chunks.  The first `main` tiles come in `shares` equal shares, as many as there are workgroups at once (or whole, some to each
// workgroup); those of one share next to each other on an XCD read the same tokens at the same time.  The chunks of the tiles that are left go
// to all workgroups in equal parts, so that all end together.  One share per tile more than fits took a second round for 8 of 132 tiles;
// all tiles in equal parts, wherever those begin, shared nothing in the L2 (dW and dX of 16384 x 1024 x 2816: 478 us).
// Sums go to slots: a share to its own, a part of what is left to (tile + workgroup) behind them, which no two have the same.
struct Contraction {
    Operand A, B;
    int rows, cols;
};
struct Weights {
    Contraction job[2];
    float *part;            // slots of BM x BN sums in the order of the wavefronts' registers
    int tiles0, tiles, chunks, main, shares, per, workgroups;
};
// Tile i of the row: its job and where it lies.
template <class T>
__device__ __forceinline__ void weight_tile(const Weights &W, int i, int &job, int &r0, int &c0)
{
    job = i >= W.tiles0;
    const Contraction &J = W.job[job];
    const int t = i - (job ? W.tiles0 : 0), mtiles = (J.rows + T::BM - 1) / T::BM, ntiles = (J.cols + T::BN - 1) / T::BN;
    const int g = t / (4 * ntiles), ms = min(4, mtiles - 4 * g), r = t - g * 4 * ntiles;
    r0 = (4 * g + r % ms) * T::BM;
    c0 = r / ms * T::BN;
}

template <class T, int TERMS>
__device__ __forceinline__ void weights_part(const Weights &W, int workgroup, bf16_t *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    long at = (long)workgroup * W.per;
    const long end = min(at + W.per, (long)(W.tiles - W.main) * W.chunks);
    for (int i = workgroup;;) {
        int tile, first, last, slot;
        if (i < W.main * W.shares) {
            const int share = i / W.main;
            tile = i % W.main;
            first = (int)((long)W.chunks * share / W.shares);
            last = (int)((long)W.chunks * (share + 1) / W.shares);
            slot = i;
            i += W.workgroups;
        } else if (at < end) {
            const int t = (int)(at / W.chunks);
            tile = W.main + t;
            first = (int)(at % W.chunks);
            last = (int)min((long)W.chunks, first + end - at);
            slot = W.main * W.shares + t + workgroup;
            at += last - first;
        } else return;
        int job, r0, c0;
        weight_tile<T>(W, tile, job, r0, c0);
        const Operand A = W.job[job].A, B = W.job[job].B;
        const int rows = W.job[job].rows, cols = W.job[job].cols;
        const Loads<T, T::BM, true> la(wave, lane, A.ld, [&](int row) { return (long)min(row, rows - 8 - r0); });
        const Loads<T, T::BN, true> lb(wave, lane, B.ld, [&](int col) { return (long)min(col, cols - 8 - c0); });
        f32x16 acc[T::NT][T::MT];
        clear<T>(acc);
        multiply<T, true, true, TERMS>(A, B, A.p + r0, B.p + c0, la, lb, first, last, lds, acc);
        store_slot<T>(W.part + (size_t)slot * kSlot<T>, acc, wave, lane);
    }
}

// Part[share][col] = sum over the share's rows of a map's columns (the sum of its planes), 8 columns per thread, 64 per workgroup.
struct Columns {
    const bf16_t *map;
    long ld, plane;
    float *part;
    int cols, groups;
};
template <int TERMS>
__device__ __forceinline__ void columns_part(const Columns &J, int group, int share, int shares, long M, float *sums)
{
    constexpr int kPitch = 64 + 4;
    const int piece = threadIdx.x % 8, slot = threadIdx.x / 8, slots = blockDim.x / 8, col = 64 * group + 8 * piece;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
    if (col < J.cols)
        for (long m = M * share / shares + slot; m < M * (share + 1) / shares; m += slots)
#pragma unroll
            for (int q = TERMS - 1; q >= 0; --q) {
                float v[8];
                load8(J.map + q * J.plane + m * J.ld + col, v, 8, true);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += v[e];
            }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[slot * kPitch + 8 * piece + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < 64 && 64 * group + (int)threadIdx.x < J.cols) {
        float s = 0.f;
        for (int r = 0; r < slots; ++r) s += sums[r * kPitch + threadIdx.x];
        J.part[(size_t)share * J.cols + 64 * group + threadIdx.x] = s;
    }
}

// Everything that follows from dG | dU and A, in one launch: the weights' parts, dX = [dG | dU] W1^T in tiles (or, few of them, shares of
// their long contraction, to slots that k_sums joins), the columns' sums.
struct Gradients {
    Weights W;
    Operand dP, W1;
    void *dX;
    long M;
    int C, product_tiles, product_shares;
    float *product_part;    // share s of tile i in slot (s * product_tiles + i)
    int product_first;      // dX's tiles ahead of the weights' parts: whichever takes a workgroup longer
    Columns columns[2];
    int shares;
};
// Bound by the matrix cores: 16384 x 1024 x 2816 447 to 462 us for 472 GFLOP, 1.02 to 1.06 PFLOP/s, busy in 61 % of the cycles.
template <class T, int TERMS, typename E>
__global__ __launch_bounds__(T::kThreads, T::kMinWaves) void k_gradients(Gradients G)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *lds = (bf16_t *)smem;
    int block = blockIdx.x;
    const int products = G.product_tiles * G.product_shares;
    auto product = [&] {
        if (G.product_shares == 1) {
            product_tile<T, false, TERMS, E>(G.dP, G.W1, nullptr, (E *)G.dX, G.M, G.C, block, lds);
            return;
        }
        const int chunks = (G.dP.K + 63) / 64, share = block / G.product_tiles;
        f32x16 acc[T::NT][T::MT];
        product_sums<T, false, TERMS>(G.dP, G.W1, G.M, G.C, block % G.product_tiles, (int)((long)chunks * share / G.product_shares),
                                      (int)((long)chunks * (share + 1) / G.product_shares), lds, acc);
        store_slot<T>(G.product_part + (size_t)block * kSlot<T>, acc, threadIdx.x / 64, threadIdx.x % 64);
    };
    if (G.product_first) {
        if (block < products) return product();
        block -= products;
    }
    if (block < G.W.workgroups) {
        // workgroups of an XCD have neighbouring parts
        const int xcd = block % 8, per = G.W.workgroups / 8, rest = G.W.workgroups % 8;
        weights_part<T, TERMS>(G.W, xcd * per + min(xcd, rest) + block / 8, lds);
        return;
    }
    block -= G.W.workgroups;
    if (!G.product_first) {
        if (block < products) return product();
        block -= products;
    }
    const int j = block >= G.columns[0].groups * G.shares;
    if (j) block -= G.columns[0].groups * G.shares;
    columns_part<TERMS>(G.columns[j], block / G.shares, block % G.shares, G.shares, G.M, (float *)smem);
}

// The parts' sums, in order: a thread has 8 columns of a row of a tile, in the place where its wavefront had them; behind the tiles the columns.
// Bound by memory: 16384 x 1024 x 2816 25 us for 84 MB of parts and 17 MB of gradients.
struct SumsArgs {
    Weights W;
    void *dW[2];
    int rows[2], blocks[2], cols[2], cols_p[2];         // as they are returned; column blocks of cols_p columns in the workspace
    void *db[2];
    const float *columns[2];
    int shares, tile_blocks;
    // dX [M, C], if its tiles came in shares; `product_blocks` workgroups behind the weights'
    const float *product_part;
    void *dX;
    long M;
    int C, product_tiles, product_shares, product_blocks;
    bool f32;
};
template <class T, typename E>
__global__ __launch_bounds__(256) void k_sums(SumsArgs S)
{
    if ((int)blockIdx.x < S.tile_blocks) {
        constexpr int kPer = kSlot<T> / 8 / 256;        // workgroups per tile
        const int tile = blockIdx.x / kPer, i = blockIdx.x % kPer * 256 + threadIdx.x, lane = i % 64, run = i / 64 % 2, frag = i / 128;
        const int mt = frag % T::MT, nt = frag / T::MT % T::NT, wave = frag / (T::MT * T::NT);
        int job, r0, c0;
        weight_tile<T>(S.W, tile, job, r0, c0);
        const int row = r0 + (wave / T::WC) * (32 * T::MT) + 32 * mt + lane % 32, col = c0 + (wave % T::WC) * (32 * T::NT) + 32 * nt + 16 * run + 8 * (lane / 32);
        if (row >= S.rows[job] || col >= S.W.job[job].cols) return;
        const int t = tile - S.W.main;          // of those that are left
        int first = tile, apart = S.W.main, count = S.W.shares;
        if (t >= 0) {
            const int w0 = (int)((long)t * S.W.chunks / S.W.per), w1 = (int)(((long)(t + 1) * S.W.chunks - 1) / S.W.per);
            first = S.W.main * S.W.shares + t + w0;
            apart = 1;
            count = w1 - w0 + 1;
        }
        float acc[8];
        sum_slots<T>(S.W.part, first, apart, count, frag, run, lane, acc);
        const int block = col / S.cols_p[job], in = col % S.cols_p[job], n = S.cols[job] - in;
        store8((E *)S.dW[job] + ((size_t)row * S.blocks[job] + block) * S.cols[job] + in, acc, n, S.cols[job] % 8 == 0);
        return;
    }
    int i = ((int)blockIdx.x - S.tile_blocks) * 256 + threadIdx.x;
    if ((int)blockIdx.x < S.tile_blocks + S.product_blocks) {
        constexpr int kEach = kSlot<T> / 8;
        const int tile = i / kEach, in = i % kEach, lane = in % 64, run = in / 64 % 2, frag = in / 128;
        const int mt = frag % T::MT, nt = frag / T::MT % T::NT, wave = frag / (T::MT * T::NT);
        int mt0, nt0;
        tile_of(tile, (int)((S.M + T::BM - 1) / T::BM), (S.C + T::BN - 1) / T::BN, mt0, nt0);
        const long row = (long)mt0 * T::BM + (wave / T::WC) * (32 * T::MT) + 32 * mt + lane % 32;
        const int col = nt0 * T::BN + (wave % T::WC) * (32 * T::NT) + 32 * nt + 16 * run + 8 * (lane / 32);
        if (row >= S.M || col >= S.C) return;
        float acc[8];
        sum_slots<T>(S.product_part, tile, S.product_tiles, S.product_shares, frag, run, lane, acc);
        if (S.f32) store8((float *)S.dX + (size_t)row * S.C + col, acc, S.C - col, S.C % 8 == 0);
        else store8((bf16_t *)S.dX + (size_t)row * S.C + col, acc, S.C - col, S.C % 8 == 0);
        return;
    }
    i -= S.product_blocks * 256;
    for (int j = 0; j < 2; ++j) {
        const int count = S.db[j] ? S.blocks[j] * S.cols[j] : 0;
        if (i < count) {
            const int at = i / S.cols[j] * S.cols_p[j] + i % S.cols[j];
            float s = 0.f;
#pragma unroll 8
            for (int p = 0; p < S.shares; ++p) s += S.columns[j][(size_t)p * S.blocks[j] * S.cols_p[j] + at];
            store_from_f32((E *)S.db[j] + i, s);
            return;
        }
        i -= count;
    }
}

template <typename E>
__global__ __launch_bounds__(256) void k_zero(E *p, long n)
{
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += 256L * gridDim.x) store_from_f32(p + i, 0.f);
}

template <class TD, class TG, int TERMS, int ACT, bool GIVEN, typename E>
int launch_hidden(const Operand &dY, const Operand &W2, const Operand &X, const Operand &W1, const float *b1, const void *pre, bf16_t *Act, long plane_a, bf16_t *dP,
                  long plane_p, const Sizes &S, hipStream_t st)
{
    constexpr size_t bytes = GIVEN || TD::kLds > TG::kLds ? TD::kLds : TG::kLds;
    if (allow_lds<k_hidden<TD, TG, TERMS, ACT, GIVEN, E>>(bytes) != BRA_OK) return BRA_ERR_LAUNCH;
    const long tiles = ((S.M + TD::BM - 1) / TD::BM) * ((S.hp + TD::BN - 1) / TD::BN);
    // (one launch but for close to 2^30 tokens, whose tiles make 2^32 threads)
    constexpr long kMost = kMaxBlocks * 256 / TD::kThreads;
    for (long first = 0; first < tiles; first += kMost) {
        k_hidden<TD, TG, TERMS, ACT, GIVEN, E>
            <<<(unsigned)std::min(tiles - first, kMost), TD::kThreads, bytes, st>>>(dY, W2, X, W1, b1, (const E *)pre, Act, plane_a, dP, plane_p, S.M, S.h, S.hp, (int)first);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <int TERMS, int ACT, typename E>
int pick_hidden(const Operand &dY, const Operand &W2, const Operand &X, const Operand &W1, const float *b1, const void *pre, bf16_t *Act, long pa, bf16_t *dP, long pp,
                const Sizes &S, hipStream_t st)
{
    if (pre) {
        switch (hidden_side(S, true)) {
        case 256: return launch_hidden<Tile<256, 256, 4, 2, 2>, Tile<256, 256, 4, 2, 2>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        case 128: return launch_hidden<Tile<128, 128, 2, 2, 2>, Tile<128, 128, 2, 2, 2>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        default: return launch_hidden<Tile<64, 64, 2, 2, 4>, Tile<64, 64, 2, 2, 4>, TERMS, ACT, true, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
        }
    }
    if (hidden_side(S, false) == 128)
        return launch_hidden<Tile<128, 128, 2, 4, 2>, Tile<128, 256, 2, 4, 2>, TERMS, ACT, false, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
    return launch_hidden<Tile<64, 64, 2, 2, 4>, Tile<64, 128, 2, 2, 3>, TERMS, ACT, false, E>(dY, W2, X, W1, b1, pre, Act, pa, dP, pp, S, st);
}

constexpr int kColumnShares = 32;

template <class T, int TERMS, typename E>
int launch_gradients(Gradients G, bool columns, hipStream_t st)
{
    constexpr size_t bytes = std::max<size_t>(T::kLds, T::kThreads / 8 * 68 * 4);
    if (allow_lds<k_gradients<T, TERMS, E>>(bytes) != BRA_OK) return BRA_ERR_LAUNCH;
    G.product_tiles = (int)(((G.M + T::BM - 1) / T::BM) * ((G.C + T::BN - 1) / T::BN));
    G.product_first = (G.dP.K + 63) / 64 / G.product_shares > G.W.chunks / std::max(1, G.W.shares);
    const int groups = columns ? G.columns[0].groups + G.columns[1].groups : 0;
    k_gradients<T, TERMS, E><<<(unsigned)(G.W.workgroups + G.product_tiles * G.product_shares + groups * G.shares), T::kThreads, bytes, st>>>(G);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <class T>
int launch_sums(SumsArgs S, bool grads_f32, hipStream_t st)
{
    S.tile_blocks = S.W.tiles * (kSlot<T> / 8 / 256);
    S.product_tiles = (int)(((S.M + T::BM - 1) / T::BM) * ((S.C + T::BN - 1) / T::BN));
    S.product_blocks = S.product_shares > 1 ? S.product_tiles * (kSlot<T> / 8 / 256) : 0;
    const int columns = (S.db[0] ? S.blocks[0] * S.cols[0] : 0) + (S.db[1] ? S.cols[1] : 0);
    const unsigned blocks = (unsigned)(S.tile_blocks + S.product_blocks + (columns + 255) / 256);
    if (grads_f32) k_sums<T, float><<<blocks, 256, 0, st>>>(S);
    else k_sums<T, bf16_t><<<blocks, 256, 0, st>>>(S);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

// Side of the tiles of k_gradients, and how the weights' tiles are shared out (see Weights).
struct WeightsPlan {
    int side, tiles0, tiles, chunks, main, shares, per, workgroups, product_shares;
    WeightsPlan(const Sizes &S)
    {
        chunks = (int)((S.M + 63) / 64);
        // By the operations and, because dX's tiles have the long contraction, their number (us with 256 / 128 / 64): 12544 x 768 x 2048 (147 large
        // tiles) 212 / 265 / 353, 12544 x 512 x 1368 (98; 392) 141 / 133 / 172, 1024 x 768 x 2048 (48 of 128) 109 / 70 / 45, 32768 x 128 x 256 (13 GFLOP) 69 / 47 / 32
        const double flops = 12.0 * (double)S.M * S.Cp * S.hp;
        side = flops >= 2e11 && ffn::tiles(S.M, S.C, 256) >= 140 ? 256 : flops >= 1.5e10 && ffn::tiles(S.M, S.C, 128) >= 190 ? 128 : 64;
        tiles0 = (int)ffn::tiles(S.Cp, 2 * S.hp, side);
        tiles = tiles0 + (int)ffn::tiles(S.hp, S.Cp, side);
        const int at_once = side == 256 ? 256 : 512, least = S.f32 ? 1 : 2;     // chunks of a share (of float32 a chunk is six)
        per = 0;
        if (tiles >= at_once) {
            shares = 1;
            main = tiles / at_once * at_once;
        } else {
            shares = std::min((at_once + tiles - 1) / tiles, std::max(1, chunks / least));
            main = std::min(tiles, at_once / shares);
        }
        // dX's few tiles of a long contraction are shared out (us with one share / these: 129 x 768 x 2048 244 / 149 in float32, 46 / 42 in bf16, whose chunks are
        // soon done: shares of 4 at least, and not more than one per compute unit; with 2 and two 1024 x 256 x 512 took 27.1 for 25.4)
        const int products = (int)ffn::tiles(S.M, S.C, side), long_chunks = (2 * S.hp + 63) / 64;
        product_shares = side != 64 || products == 0 ? 1 : std::max(1, std::min({(S.f32 ? 512 : 256) / products, long_chunks / (S.f32 ? 1 : 4), 16}));
        workgroups = std::min(at_once, main * shares);
        if (main < tiles) {
            workgroups = at_once;
            // (more than 16 parts of a tile took k_sums longer than they saved here: 53 us against 28, with 64)
            per = std::max({(int)(((long)(tiles - main) * chunks + at_once - 1) / at_once), least, (chunks + 15) / 16});
        }
    }
    int slots() const { return main * shares + (main < tiles ? tiles - main + workgroups : 0); }
};

struct BackwardPlan {
    size_t X, W1, W2, dY, Act, dP, parts, products, cols1, cols2, total;
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
        parts = take((size_t)P.slots() * P.side * P.side * 4);
        products = P.product_shares > 1 ? take((size_t)ffn::tiles(S.M, S.C, P.side) * P.product_shares * P.side * P.side * 4) : 0;
        cols1 = take((size_t)kColumnShares * 2 * S.hp * 4);
        cols2 = take((size_t)kColumnShares * S.Cp * 4);
        total = at;
    }
};

}  // namespace
}  // namespace ffn

using namespace ffn;

typedef Tile<256, 256, 4, 2, 2> T256;
typedef Tile<128, 128, 2, 2, 2> T128;
typedef Tile<64, 64, 2, 2, 4> T64;

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
        Gradients G{};
        const int M = (int)S.M;
        G.W.job[0] = Contraction{{(const bf16_t *)X, S.Cp, pX, M}, {at(P.dP), 2L * S.hp, pP, M}, S.Cp, 2 * S.hp};
        G.W.job[1] = Contraction{{at(P.Act), S.hp, pA, M}, {(const bf16_t *)dY, S.Cp, pX, M}, S.hp, S.Cp};
        G.W.part = (float *)at(P.parts);
        G.W.tiles0 = W.tiles0; G.W.tiles = W.tiles; G.W.chunks = W.chunks; G.W.main = W.main; G.W.shares = W.shares; G.W.per = W.per; G.W.workgroups = W.workgroups;
        G.dP = odP;
        G.W1 = oW1;
        G.W1.K = 2 * S.hp;
        G.product_shares = W.product_shares;
        G.product_part = (float *)at(P.products);
        G.dX = dX; G.M = S.M; G.C = S.C; G.shares = kColumnShares;
        G.columns[0] = Columns{at(P.dP), 2L * S.hp, pP, (float *)at(P.cols1), 2 * S.hp, db1 ? (2 * S.hp + 63) / 64 : 0};
        G.columns[1] = Columns{(const bf16_t *)dY, S.Cp, pX, (float *)at(P.cols2), S.Cp, db2 ? (S.Cp + 63) / 64 : 0};
        {
            ProfScope prof(st, K_FFN_WEIGHT_GRADS);
            const bool columns = db1 || db2;
            if (S.f32) rc = W.side == 256 ? launch_gradients<T256, 3, float>(G, columns, st) : W.side == 128 ? launch_gradients<T128, 3, float>(G, columns, st)
                                                                                                 : launch_gradients<T64, 3, float>(G, columns, st);
            else rc = W.side == 256 ? launch_gradients<T256, 1, bf16_t>(G, columns, st) : W.side == 128 ? launch_gradients<T128, 1, bf16_t>(G, columns, st)
                                                                                                : launch_gradients<T64, 1, bf16_t>(G, columns, st);
            if (rc != BRA_OK) return rc;
        }
        ProfScope prof(st, K_FFN_SUMS);
        SumsArgs A{};
        A.W = G.W;
        A.dW[0] = dW1; A.dW[1] = dW2; A.db[0] = db1; A.db[1] = db2;
        A.rows[0] = S.C; A.rows[1] = S.h;
        A.blocks[0] = 2; A.blocks[1] = 1;
        A.cols[0] = S.h; A.cols[1] = S.C;
        A.cols_p[0] = S.hp; A.cols_p[1] = S.Cp;
        A.columns[0] = (const float *)at(P.cols1); A.columns[1] = (const float *)at(P.cols2);
        A.shares = kColumnShares;
        A.product_part = G.product_part;
        A.dX = dX; A.M = S.M; A.C = S.C; A.product_shares = W.product_shares; A.f32 = S.f32;
        return W.side == 256 ? launch_sums<T256>(A, grads_f32, st) : W.side == 128 ? launch_sums<T128>(A, grads_f32, st) : launch_sums<T64>(A, grads_f32, st);
    }
    ProfScope prof(st, K_FFN_SUMS);
    const struct { void *p; long n; } all[4] = {{dW1, (long)S.C * 2 * S.h}, {dW2, (long)S.h * S.C}, {db1, 2L * S.h}, {db2, S.C}};
    for (const auto &z : all) {
        if (!z.p) continue;
        const unsigned blocks = (unsigned)std::min((z.n + 255) / 256, kMaxBlocks);
        if (grads_f32) k_zero<float><<<blocks, 256, 0, st>>>((float *)z.p, z.n);
        else k_zero<bf16_t><<<blocks, 256, 0, st>>>((bf16_t *)z.p, z.n);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

}  // namespace bra
