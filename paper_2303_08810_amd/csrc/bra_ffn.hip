// Gated feed-forward block: Y = (act(X Wg + bg) * (X Wu + bu)) Wd + bd, W1 = [Wg | Wu].
//
//   k_few         up to 128 rows (k_few_f32: few float32 rows): both products by workgroups of few columns
//   k_operands    float32 operands as three bf16 terms, operands of odd sizes padded to multiples of 8 (other calls skip it)
//   k_gated       A = act(G) * U with G | U = X W1 + b1: the tile's columns are half of G and half of U, so that a lane holds both of a
//                 hidden unit and nothing but A (and, where the caller wants it, G | U) is written
//   k_product     Y = A W2 + b2
//   k_split, k_join   either of them where tiles are few and the contraction long
#include "bra_ffn.h"
#include "bra_ffn_dev.h"

#include <algorithm>

namespace bra {
namespace ffn {

namespace {

template <typename E>
__global__ __launch_bounds__(256) void k_operands(Layouts J)
{
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < J.end[J.count - 1]; i += 256L * gridDim.x) {
        int j = 0;
        while (i >= J.end[j]) ++j;
        const Layout L = J.job[j];
        const long p = i - (j ? J.end[j - 1] : 0);
        const int per = L.cols_p / 8, piece = (int)(p % per);
        const long line = p / per;                       // row * blocks + block
        float v[8];
        load8((const E *)L.src + line * L.cols + 8 * piece, v, L.cols - 8 * piece, false);
        store_operand<sizeof(E) == 4 ? 3 : 1>(L.dst + line * L.cols_p + 8 * piece, L.plane, v);
    }
}

// Bound by the matrix cores and, with G | U stored, by the epilogue that they wait for: 32768 x 1024 x 2816 430 to 447 us, 0.87 PFLOP/s, matrix
// cores busy in 49 % of the cycles at a clock that their power brings down to 1.8 GHz.  12544 x 256 x 512, one round of 196 workgroups: 17 us.
template <class T, int TERMS, int ACT, typename E>
__global__ __launch_bounds__(T::kThreads, T::kMinWaves) void k_gated(Operand X, Operand W1, const float *__restrict__ b1, E *__restrict__ pre, bf16_t *__restrict__ Act,
                                                         long plane, long M, int h, int hp)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *lds = (bf16_t *)smem;
    constexpr int BJ = T::BN / 2, PW = 16 * T::NT;       // hidden units of a tile, of a wavefront
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int mt0, nt0;
    tile_of(blockIdx.x, (int)((M + T::BM - 1) / T::BM), (hp + BJ - 1) / BJ, mt0, nt0);
    const long m0 = (long)mt0 * T::BM;
    const int j0 = nt0 * BJ, last = hp - 8 - j0, rows = (int)min((long)T::BM, M - m0);
    const Loads<T, T::BM, false> la(wave, lane, X.ld, [&](int row) { return (long)min(row, rows - 1); });
    const Loads<T, T::BN, true> lb(wave, lane, W1.ld, [&](int col) {
        const int w = col / (2 * PW), in = col % (2 * PW);
        return (long)(min(w * PW + in % PW, last) + (in >= PW ? hp : 0));
    });
    f32x16 acc[T::NT][T::MT];
    clear<T>(acc);
    multiply<T, false, true, TERMS>(X, W1, X.p + m0 * X.ld, W1.p + j0, la, lb, 0, (X.K + 63) / 64, lds, acc);
    const int hi = lane / 32, c = lane % 32, wm = (wave / T::WC) * (32 * T::MT), wj = j0 + (wave % T::WC) * PW;
    const bool vec = h % 8 == 0, vec_b = vec && (uintptr_t)b1 % 16 == 0;
    constexpr int P = PW / 8;
    bf16_t *const own = lds + wave * (32 * T::MT * 2 * PW);      // this wavefront's part of what the chunks have left
    const Rows<P> first{own}, second{own + 32 * T::MT * PW};
#pragma unroll
    for (int nt = 0; nt < T::NT / 2; ++nt)
#pragma unroll
        for (int run = 0; run < 2; ++run) {
            const int piece = 4 * nt + 2 * run + hi, j = wj + 8 * piece, n = h - j;
            float bg[8], bu[8];
            if (b1 && n > 0) {
                load8(b1 + j, bg, n, vec_b);
                load8(b1 + h + j, bu, n, vec_b);
            } else
#pragma unroll
                for (int e = 0; e < 8; ++e) bg[e] = bu[e] = 0.f;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
                const int row = wm + 32 * mt + c;
                f32x16 &G = acc[nt][mt], &U = acc[T::NT / 2 + nt][mt];
                float g[8], u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) { g[e] = G[8 * run + e] + bg[e]; u[e] = U[8 * run + e] + bu[e]; }
                if (pre) {
                    if constexpr (TERMS == 1) {
                        first.put(32 * mt + c, piece, pack8(g));
                        second.put(32 * mt + c, piece, pack8(u));
                    } else if (row < rows) {
                        store8(pre + (size_t)(m0 + row) * 2 * h + j, g, n, vec);
                        store8(pre + (size_t)(m0 + row) * 2 * h + h + j, u, n, vec);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) G[8 * run + e] = e < n ? activation<ACT, TERMS != 1>(g[e]) * u[e] : 0.f;      // A, in G's place
            }
        }
    if constexpr (TERMS == 1)
        if (pre) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
                (half ? second : first).each(32 * T::MT, lane, [&](int row, int piece, bf16x8 v) {
                    if (wm + row < rows) store_piece(pre + (size_t)(m0 + wm + row) * 2 * h + half * h + wj + 8 * piece, v, h - wj - 8 * piece, vec);
                });
        }
#pragma unroll
    for (int q = 0; q < TERMS; ++q) {
#pragma unroll
        for (int nt = 0; nt < T::NT / 2; ++nt)
#pragma unroll
            for (int run = 0; run < 2; ++run)
#pragma unroll
                for (int mt = 0; mt < T::MT; ++mt) {
                    float v[8];
                    bf16x8 t[TERMS];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = acc[nt][mt][8 * run + e];
                    operand<TERMS>(v, t);
                    first.put(32 * mt + c, 4 * nt + 2 * run + hi, t[q]);
                }
        first.each(32 * T::MT, lane, [&](int row, int piece, bf16x8 v) {
            if (wm + row < rows && wj + 8 * piece < hp) *(bf16x8 *)(Act + q * plane + (size_t)(m0 + wm + row) * hp + wj + 8 * piece) = v;
        });
    }
}

// 32768 x 2816 x 1024: 195 us, 0.97 PFLOP/s, matrix cores busy in 52 % of the cycles (the library's product of these sizes 145).
template <class T, int TERMS, typename E>
__global__ __launch_bounds__(T::kThreads, T::kMinWaves) void k_product(Operand A, Operand Bm, const float *__restrict__ bias, E *__restrict__ Out, long M, int N)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    product_tile<T, true, TERMS, E>(A, Bm, bias, Out, M, N, blockIdx.x, (bf16_t *)smem);
}

// Few rows: 32 x 32 outputs per workgroup, the contraction's chunks shared out to its kFewWaves wavefronts, each with a ring of its own and no
// barrier before the sums meet in LDS.  Few columns per workgroup spread the weights over the chip; the direct loads of all wavefronts
// are on their way at once.  Of X only ROWS rows are read (the rest of the tile is whatever LDS holds: a row's results depend on no
// other).  ACT < 0: Out = X W + b; otherwise the 32 columns are those of G and U of 16 hidden units, 16 registers apart in a lane, and Out = act(G) U.
constexpr int kFewWaves = 8, kFewRing = 2;
typedef Tile<32, 32, 1, 1, kFewRing> TFew;
template <int ACT, int ROWS>
__global__ __launch_bounds__(64 * kFewWaves, 2) void k_few(Operand X, Operand W, const float *__restrict__ bias, bf16_t *__restrict__ pre, bf16_t *__restrict__ Out, int M, int N, int Np)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr bool GATED = ACT >= 0;
    constexpr int LA = ROWS / 8, LB = Loads<TFew, 32, true>::L, kLoads = LA + LB, kChunk = TFew::kChunkA + TFew::kChunkB;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    // an XCD has neighbouring columns: they lie in the same lines
    const int xcd = blockIdx.x % 8, per = gridDim.x / 8, rest = gridDim.x % 8, tile = xcd * per + min(xcd, rest) + blockIdx.x / 8;
    const int c0 = tile * (GATED ? 16 : 32), m0 = blockIdx.y * 32, rows = min(M - m0, 32), last = Np - 8 - c0;
    const Loads<TFew, 32, false> la(0, lane, X.ld, [&](int row) { return (long)min(row, rows - 1); });
    const Loads<TFew, 32, true> lb(0, lane, W.ld, [&](int col) { return (long)(GATED ? min(col % 16, last) + (col >= 16 ? Np : 0) : min(col, last)); });
    bf16_t *const ring = (bf16_t *)smem + wave * (kFewRing * kChunk);
    const unsigned at = lds_address(ring);
    const bf16_t *const a0 = X.p + m0 * X.ld, *const b0 = W.p + c0;
    const int chunks = (X.K + 63) / 64, mine = (chunks - wave + kFewWaves - 1) / kFewWaves;
    auto ask = [&](int i) {
        const int k0 = 64 * (wave + i * kFewWaves);
        const unsigned to = at + (i % kFewRing) * (kChunk * 2);
#pragma unroll
        for (int u = 0; u < LA; ++u) la.request(u, a0 + k0, X.K - k0, to, 0, lane);
#pragma unroll
        for (int u = 0; u < LB; ++u) lb.request(u, b0 + k0 * W.ld, W.K - k0, to + 2 * TFew::kChunkA, 0, lane);
    };
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    for (int i = 0; i < min(mine, kFewRing); ++i) ask(i);
    for (int i = 0; i < mine; ++i) {
        if (i + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" : : "n"((kFewRing - 1) * kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const bf16_t *As = ring + (i % kFewRing) * kChunk, *Bs = As + TFew::kChunkA;
        bf16x8 x[4], w[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            w[ks] = fragment<32, true, true>(Bs, 0, ks, lane);
            x[ks] = fragment<32, false, false>(As, 0, ks, lane);
        }
        lds_reads_done();
        __builtin_amdgcn_sched_barrier(0);
        if (i + kFewRing < mine) ask(i + kFewRing);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) acc = mfma32(w[ks], x[ks], acc);
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15");
    __builtin_amdgcn_sched_barrier(0);
    // the wavefronts' sums, [wave][quarter of the registers][lane][4]; then a wavefront has a quarter (GATED: one of G's and the same of U's)
    __syncthreads();
    f32x4 *const sums = (f32x4 *)smem;
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[(wave * 4 + q) * 64 + lane] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    if (wave >= (GATED ? 2 : 4)) return;
    auto total = [&](int q) {
        f32x4 s = sums[q * 64 + lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) s += sums[(w * 4 + q) * 64 + lane];
        return s;
    };
    const int row = lane % 32, col = c0 + 16 * (wave / 2) + 8 * (lane / 32) + 4 * (wave % 2);
    // (N columns exist; an operand of a later product has its columns up to Np written, with zeros)
    f32x4 g = total(wave);
    if (row >= rows || col >= (GATED ? Np : N)) return;
    const size_t m = (size_t)(m0 + row);
    const int n = N - col;
    auto put = [&](bf16_t *p, f32x4 v) {
        if (N % 8 == 0) {
            *(u32x2 *)p = pack4(v);
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = f32_to_bf16(v[e]);
    };
    if (bias)
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] += e < n ? bias[col + e] : 0.f;
    if constexpr (GATED) {
        f32x4 u = total(wave + 2);
        if (bias)
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] += e < n ? bias[N + col + e] : 0.f;
        if (pre) {
            put(pre + m * 2 * N + col, g);
            put(pre + m * 2 * N + N + col, u);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = e < n ? activation<GATED ? ACT : 0, false>(g[e]) * u[e] : 0.f;
        *(u32x2 *)(Out + m * Np + col) = pack4(g);
    } else put(Out + m * N + col, g);
}

template <int ACT>
int few(const Operand &X, const Operand &W, const float *bias, void *pre, bf16_t *Out, int M, int N, int Np, hipStream_t st)
{
    constexpr size_t bytes = kFewWaves * kFewRing * (size_t)(TFew::kChunkA + TFew::kChunkB) * 2;
    const dim3 grid((Np + (ACT >= 0 ? 15 : 31)) / (ACT >= 0 ? 16 : 32), (M + 31) / 32);
    if (M <= 8) {
        if (allow_lds<k_few<ACT, 8>>(bytes) != BRA_OK) return BRA_ERR_LAUNCH;
        k_few<ACT, 8><<<grid, 64 * kFewWaves, bytes, st>>>(X, W, bias, (bf16_t *)pre, Out, M, N, Np);
    } else {
        if (allow_lds<k_few<ACT, 32>>(bytes) != BRA_OK) return BRA_ERR_LAUNCH;
        k_few<ACT, 32><<<grid, 64 * kFewWaves, bytes, st>>>(X, W, bias, (bf16_t *)pre, Out, M, N, Np);
    }
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

// Few rows in float32, the weights read once and as they lie (no terms, no copies): 8 rows x 32 columns per workgroup, a lane has 4 columns and every
// 64th group of 4 of the contraction; the rows wait in LDS, kFewK of the contraction at a time.  Bound by the weights' bytes.  Columns as in k_few.
constexpr int kFewK = 2048, kFewRows = 8;
template <int ACT>
__global__ __launch_bounds__(512, 2) void k_few_f32(const float *__restrict__ X, const float *__restrict__ W, const float *__restrict__ bias, float *__restrict__ pre,
                                                   float *__restrict__ Out, int M, int K, int N)
{
    constexpr bool GATED = ACT >= 0;
    constexpr int cols = GATED ? 16 : 32;
    typedef f32x4 f32x4u __attribute__((aligned(4)));
    __shared__ __attribute__((aligned(16))) float xs[kFewRows][kFewK];
    __shared__ float sums[8][8][kFewRows * 4];
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, piece = lane % 8, group = wave * 8 + lane / 8;
    const int xcd = blockIdx.x % 8, per = gridDim.x / 8, rest = gridDim.x % 8, tile = xcd * per + min(xcd, rest) + blockIdx.x / 8;
    const int c0 = tile * (GATED ? 16 : 32), m0 = blockIdx.y * kFewRows, rows = min(M - m0, kFewRows);
    const int ld = GATED ? 2 * N : N, unit = c0 + (GATED ? 4 * (piece % 4) : 4 * piece), n = N - unit;      // columns from `unit` on
    const float *const w = W + unit + (GATED && piece >= 4 ? N : 0);
    float acc[kFewRows][4];
#pragma unroll
    for (int m = 0; m < kFewRows; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][e] = 0.f;
    for (int k0 = 0; k0 < K; k0 += kFewK) {
        const int kn = min(kFewK, K - k0);
        if (k0) __syncthreads();
        if (wave < rows)
            for (int k = lane; k < (kn + 3) / 4 * 4; k += 64) xs[wave][k] = k < kn ? X[(size_t)(m0 + wave) * K + k0 + k] : 0.f;
        __syncthreads();
        auto add = [&](int k, const f32x4 (&v)[4]) {
#pragma unroll
            for (int m = 0; m < kFewRows; ++m) {
                if (m >= rows) continue;
                const f32x4 x = *(const f32x4 *)&xs[m][k];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][e] = fmaf(x[j], v[j][e], acc[m][e]);
            }
        };
        int k = 4 * group;
        if (c0 + cols <= N) {
            // four groups' loads on their way at a time, without a question in between
            const float *p = w + (size_t)(k0 + k) * ld;
            const size_t row = ld, step = 256 * row;
            for (; k + 3 * 256 + 4 <= kn; k += 4 * 256, p += 4 * step) {
                f32x4 v[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][j] = *(const f32x4u *)(p + i * step + j * row);
#pragma unroll
                for (int i = 0; i < 4; ++i) add(k + 256 * i, v[i]);
            }
        }
        for (; k < kn; k += 256) {
            f32x4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *p = w + (size_t)(k0 + min(k + j, kn - 1)) * ld;
                if (n >= 4) v[j] = *(const f32x4u *)p;
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][e] = e < n ? p[e] : 0.f;
                if (k + j >= kn) v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            add(k, v);
        }
    }
    // over the groups of a wavefront, then over the wavefronts
#pragma unroll
    for (int m = 0; m < kFewRows; ++m) {
        if (m >= rows) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float s = cross_row_sum(dpp_fadd<0x128>(acc[m][e]));      // lanes 8 apart, then rows of 16
            if (lane < 8) sums[wave][lane][4 * m + e] = s;
        }
    }
    __syncthreads();
    auto total = [&](int p, int i) {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += sums[q][p][i];
        return s;
    };
    const int m = tid / cols, col = tid % cols;
    if (m >= rows || c0 + col >= N) return;
    float g = total(col / 4, 4 * m + col % 4) + (bias ? bias[c0 + col] : 0.f);
    const size_t row = (size_t)(m0 + m);
    if constexpr (GATED) {
        const float u = total(4 + col / 4, 4 * m + col % 4) + (bias ? bias[N + c0 + col] : 0.f);
        if (pre) {
            pre[row * 2 * N + c0 + col] = g;
            pre[row * 2 * N + N + c0 + col] = u;
        }
        g = activation<GATED ? ACT : 0, true>(g) * u;
    }
    Out[row * N + c0 + col] = g;
}

template <int ACT>
int few_f32(const void *X, const void *W, const float *bias, void *pre, void *Out, int M, int K, int N, hipStream_t st)
{
    const dim3 grid((N + (ACT >= 0 ? 15 : 31)) / (ACT >= 0 ? 16 : 32), (M + kFewRows - 1) / kFewRows);
    k_few_f32<ACT><<<grid, 512, 0, st>>>((const float *)X, (const float *)W, bias, (float *)pre, (float *)Out, M, K, N);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

// Few tiles and a long contraction: each tile in `shares` shares of it, the sums joined (with all that follows them) by k_join.  GATED: the columns of
// k_gated's tiles, N of them hidden units (padded); otherwise those of a product.  Tile i of share s in slot (s * tiles + i).
template <class T, bool GATED, int TERMS>
__global__ __launch_bounds__(T::kThreads, T::kMinWaves) void k_split(Operand A, Operand Bm, float *__restrict__ part, long M, int N, int tiles, int shares)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, share = blockIdx.x / tiles, i = blockIdx.x % tiles;
    const int chunks = (A.K + 63) / 64, first = (int)((long)chunks * share / shares), last = (int)((long)chunks * (share + 1) / shares);
    f32x16 acc[T::NT][T::MT];
    if constexpr (GATED) {
        constexpr int BJ = T::BN / 2, PW = 16 * T::NT;
        int mt0, nt0;
        tile_of(i, (int)((M + T::BM - 1) / T::BM), (N + BJ - 1) / BJ, mt0, nt0);
        const long m0 = (long)mt0 * T::BM;
        const int j0 = nt0 * BJ, rows = (int)min((long)T::BM, M - m0), most = N - 8 - j0;
        const Loads<T, T::BM, false> la(wave, lane, A.ld, [&](int row) { return (long)min(row, rows - 1); });
        const Loads<T, T::BN, true> lb(wave, lane, Bm.ld, [&](int col) {
            const int w = col / (2 * PW), in = col % (2 * PW);
            return (long)(min(w * PW + in % PW, most) + (in >= PW ? N : 0));
        });
        clear<T>(acc);
        multiply<T, false, true, TERMS>(A, Bm, A.p + m0 * A.ld, Bm.p + j0, la, lb, first, last, (bf16_t *)smem, acc);
    } else product_sums<T, true, TERMS>(A, Bm, M, N, i, first, last, (bf16_t *)smem, acc);
    store_slot<T>(part + (size_t)blockIdx.x * kSlot<T>, acc, wave, lane);
}

// N columns exist, Np in the rows that a later product reads.
template <class T, int ACT, int TERMS, typename E>
__global__ __launch_bounds__(256) void k_join(const float *__restrict__ part, const float *__restrict__ bias, E *__restrict__ pre, void *__restrict__ Out, long plane, long M, int N, int Np,
                                             int tiles, int shares)
{
    constexpr bool GATED = ACT >= 0;
    constexpr int BJ = GATED ? T::BN / 2 : T::BN, NT = GATED ? T::NT / 2 : T::NT, kPer = T::BM * BJ / 8 / 256;      // workgroups per tile
    const int tile = blockIdx.x / kPer, i = blockIdx.x % kPer * 256 + threadIdx.x, lane = i % 64, run = i / 64 % 2, f = i / 128;
    const int mt = f % T::MT, nt = f / T::MT % NT, wave = f / (T::MT * NT);
    int mt0, nt0;
    tile_of(tile, (int)((M + T::BM - 1) / T::BM), ((GATED ? Np : N) + BJ - 1) / BJ, mt0, nt0);
    const long m = (long)mt0 * T::BM + (wave / T::WC) * (32 * T::MT) + 32 * mt + lane % 32;
    const int col = nt0 * BJ + (wave % T::WC) * (32 * NT) + 32 * nt + 16 * run + 8 * (lane / 32), n = N - col;
    if (m >= M || col >= (GATED ? Np : N)) return;
    const bool vec_b = N % 8 == 0 && (uintptr_t)bias % 16 == 0;
    float g[8], b[8];
    sum_slots<T>(part, tile, tiles, shares, (wave * T::NT + nt) * T::MT + mt, run, lane, g);
    if (bias) {
        load8(bias + col, b, n, vec_b);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] += b[e];
    }
    if constexpr (GATED) {
        float u[8];
        sum_slots<T>(part, tile, tiles, shares, (wave * T::NT + NT + nt) * T::MT + mt, run, lane, u);
        if (bias) {
            load8(bias + N + col, b, n, vec_b);
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] += b[e];
        }
        if (pre) {
            store8(pre + (size_t)m * 2 * N + col, g, n, N % 8 == 0);
            store8(pre + (size_t)m * 2 * N + N + col, u, n, N % 8 == 0);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = e < n ? activation<GATED ? ACT : 0, TERMS != 1>(g[e]) * u[e] : 0.f;
        store_operand<TERMS>((bf16_t *)Out + (size_t)m * Np + col, plane, g);
    } else store8((E *)Out + (size_t)m * N + col, g, n, N % 8 == 0);
}

template <class T, int ACT, int TERMS, typename E>
int split(const Operand &A, const Operand &Bm, const float *bias, void *pre, void *Out, long plane, long M, int N, int Np, int shares, float *part, hipStream_t st)
{
    constexpr bool GATED = ACT >= 0;
    constexpr int BJ = GATED ? T::BN / 2 : T::BN;
    if (allow_lds<k_split<T, GATED, TERMS>>(T::kLds) != BRA_OK) return BRA_ERR_LAUNCH;
    const int count = (int)(((M + T::BM - 1) / T::BM) * (((GATED ? Np : N) + BJ - 1) / BJ));
    k_split<T, GATED, TERMS><<<(unsigned)(count * shares), T::kThreads, T::kLds, st>>>(A, Bm, part, M, GATED ? Np : N, count, shares);
    if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    k_join<T, ACT, TERMS, E><<<(unsigned)(count * (T::BM * BJ / 8 / 256)), 256, 0, st>>>(part, bias, (E *)pre, Out, plane, M, N, Np, count, shares);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <class T, int TERMS, typename E>
int launch_product(const Operand &A, const Operand &Bm, long M, int N, void *Out, const float *bias, hipStream_t st)
{
    if (allow_lds<k_product<T, TERMS, E>>(T::kLds) != BRA_OK) return BRA_ERR_LAUNCH;
    const long tiles = ((M + T::BM - 1) / T::BM) * ((N + T::BN - 1) / T::BN);
    k_product<T, TERMS, E><<<(unsigned)tiles, T::kThreads, T::kLds, st>>>(A, Bm, bias, (E *)Out, M, N);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

// Out [M, N] = A B + bias: A's contraction inside, B's outside.
template <int TERMS, typename E>
int product(const Operand &A, const Operand &Bm, long M, int N, void *Out, const float *bias, hipStream_t st)
{
    switch (product_side(M, N)) {
    case 256: return launch_product<Tile<256, 256, 4, 2, 2>, TERMS, E>(A, Bm, M, N, Out, bias, st);
    case 128: return launch_product<Tile<128, 128, 2, 2, 2>, TERMS, E>(A, Bm, M, N, Out, bias, st);
    default: return launch_product<Tile<64, 64, 2, 2, 4>, TERMS, E>(A, Bm, M, N, Out, bias, st);
    }
}

template <class T, int TERMS, int ACT, typename E>
int launch_gated(const Operand &X, const Operand &W1, const float *b1, void *pre, bf16_t *Act, long plane, const Sizes &S, hipStream_t st)
{
    if (allow_lds<k_gated<T, TERMS, ACT, E>>(T::kLds) != BRA_OK) return BRA_ERR_LAUNCH;
    const long tiles = ((S.M + T::BM - 1) / T::BM) * ((S.hp + T::BN / 2 - 1) / (T::BN / 2));
    k_gated<T, TERMS, ACT, E><<<(unsigned)tiles, T::kThreads, T::kLds, st>>>(X, W1, b1, (E *)pre, Act, plane, S.M, S.h, S.hp);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <int TERMS, int ACT, typename E>
int pick_gated(const Operand &X, const Operand &W1, const float *b1, void *pre, bf16_t *Act, long plane, const Sizes &S, hipStream_t st)
{
    switch (gated_side(S)) {
    case 256: return launch_gated<Tile<256, 256, 4, 2, 2>, TERMS, ACT, E>(X, W1, b1, pre, Act, plane, S, st);
    case 128: return launch_gated<Tile<128, 128, 2, 2, 2>, TERMS, ACT, E>(X, W1, b1, pre, Act, plane, S, st);
    default: return launch_gated<Tile<64, 128, 2, 2, 3>, TERMS, ACT, E>(X, W1, b1, pre, Act, plane, S, st);
    }
}

}  // namespace

int lay_out(const Layouts &J, bool f32, hipStream_t st)
{
    const long pieces = J.count ? J.end[J.count - 1] : 0;
    if (!pieces) return BRA_OK;
    ProfScope prof(st, K_FFN_OPERANDS);
    const unsigned blocks = (unsigned)std::min((pieces + 255) / 256, kMaxBlocks);
    if (f32) k_operands<float><<<blocks, 256, 0, st>>>(J);
    else k_operands<bf16_t><<<blocks, 256, 0, st>>>(J);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

}  // namespace ffn

using namespace ffn;

namespace {

typedef Tile<64, 128, 2, 2, 3> TSplitGated;
typedef Tile<64, 64, 2, 2, 4> TSplit;

// Shares of the contraction of K for `count` tiles: for two workgroups per compute unit, if that saves more than the joining launch costs.  A chunk takes about
// 0.25 us where a compute unit has one or two workgroups (six of them in float32).  Forward, us, whole / shared out: float32 129 x 768 x 2048 134 / 58,
// 129 x 256 x 512 42 / 29, 1024 x 512 x 1368 104 / 77; bf16 129 x 1024 x 2816 27.4 / 22.2, 512 x 768 x 2048 23.5 / 22.4.
int split_shares(const Sizes &S, long count, int K)
{
    const int chunks = (K + 63) / 64, shares = (int)std::min<long>({512 / std::max(1L, count), chunks, 16});
    return shares > 1 && 0.25 * chunks * (S.f32 ? 6 : 1) * (1 - 1.0 / shares) > 6 ? shares : 1;
}

// What the forward keeps in the workspace.
struct ForwardPlan {
    size_t X, W1, W2, Act, parts, total;
    int gated_shares, product_shares;
    ForwardPlan(const Sizes &S)
    {
        auto tiles = [](long M, int BM, long N, int BN) { return ((M + BM - 1) / BM) * ((N + BN - 1) / BN); };
        const bool few = few_rows(S) || few_rows_f32(S);
        gated_shares = few || gated_side(S) != 64 ? 1 : split_shares(S, tiles(S.M, 64, S.hp, 64), S.Cp);
        product_shares = few || product_side(S.M, S.C) != 64 ? 1 : split_shares(S, tiles(S.M, 64, S.C, 64), S.hp);
        size_t at = 0;
        auto take = [&](size_t elements) {
            const size_t here = at;
            at += align256(elements * S.terms() * sizeof(bf16_t));
            return here;
        };
        X = S.copies() ? take((size_t)S.M * S.Cp) : 0;
        W1 = S.copies() ? take((size_t)S.C * 2 * S.hp) : 0;
        W2 = S.copies() ? take((size_t)S.h * S.Cp) : 0;
        Act = take((size_t)S.M * S.hp);
        auto slots = [](long count, int shares, size_t floats) { return shares > 1 ? (size_t)count * shares * floats * 4 : 0; };
        parts = at;
        at += std::max(slots(tiles(S.M, 64, S.hp, 64), gated_shares, kSlot<TSplitGated>), slots(tiles(S.M, 64, S.C, 64), product_shares, kSlot<TSplit>));
        total = at;
    }
};

template <int TERMS, int ACT, typename E>
int gated(const Operand &X, const Operand &W1, const float *b1, void *pre, bf16_t *Act, long plane, const Sizes &S, const ForwardPlan &P, void *parts, hipStream_t st)
{
    if (P.gated_shares > 1) return split<TSplitGated, ACT, TERMS, E>(X, W1, b1, pre, Act, plane, S.M, S.h, S.hp, P.gated_shares, (float *)parts, st);
    return pick_gated<TERMS, ACT, E>(X, W1, b1, pre, Act, plane, S, st);
}

}  // namespace

size_t ffn_workspace_bytes(const Sizes &S) { return ForwardPlan(S).total; }

int ffn_forward(const Sizes &S, const void *X, const void *W1, const float *b1, const void *W2, const float *b2, void *Y, void *pre, void *ws, hipStream_t st)
{
    if (S.M == 0) return BRA_OK;
    const ForwardPlan P(S);
    auto at = [&](size_t offset) { return (bf16_t *)((char *)ws + offset); };
    const long pX = S.M * S.Cp, pW1 = (long)S.C * 2 * S.hp, pW2 = (long)S.h * S.Cp, pA = S.M * S.hp;
    if (few_rows_f32(S)) {
        ProfScope prof(st, K_FFN_FEW);
        float *A = (float *)at(P.Act);
        const int rc = S.act == BRA_SILU ? few_f32<BRA_SILU>(X, W1, b1, pre, A, (int)S.M, S.C, S.h, st) : few_f32<BRA_GELU>(X, W1, b1, pre, A, (int)S.M, S.C, S.h, st);
        return rc != BRA_OK ? rc : few_f32<-1>(A, W2, b2, nullptr, Y, (int)S.M, S.h, S.C, st);
    }
    if (S.copies()) {
        Layouts J{};
        add_layout(J, X, at(P.X), S.M, 1, S.C, S.Cp, pX);
        add_layout(J, W1, at(P.W1), S.C, 2, S.h, S.hp, pW1);
        add_layout(J, W2, at(P.W2), S.h, 1, S.C, S.Cp, pW2);
        const int rc = lay_out(J, S.f32, st);
        if (rc != BRA_OK) return rc;
        X = at(P.X); W1 = at(P.W1); W2 = at(P.W2);
    }
    const Operand oX{(const bf16_t *)X, S.Cp, pX, S.Cp}, oW1{(const bf16_t *)W1, 2L * S.hp, pW1, S.C}, oW2{(const bf16_t *)W2, S.Cp, pW2, S.h},
        oA{at(P.Act), S.hp, pA, S.hp};
    int rc;
    if (few_rows(S)) {
        ProfScope prof(st, K_FFN_FEW);
        rc = S.act == BRA_SILU ? few<BRA_SILU>(oX, oW1, b1, pre, at(P.Act), (int)S.M, S.h, S.hp, st) : few<BRA_GELU>(oX, oW1, b1, pre, at(P.Act), (int)S.M, S.h, S.hp, st);
        if (rc != BRA_OK) return rc;
        return few<-1>(oA, oW2, b2, nullptr, (bf16_t *)Y, (int)S.M, S.C, S.Cp, st);
    }
    {
        ProfScope prof(st, K_FFN_GATED);
        if (S.f32) rc = S.act == BRA_SILU ? gated<3, BRA_SILU, float>(oX, oW1, b1, pre, at(P.Act), pA, S, P, at(P.parts), st)
                                          : gated<3, BRA_GELU, float>(oX, oW1, b1, pre, at(P.Act), pA, S, P, at(P.parts), st);
        else rc = S.act == BRA_SILU ? gated<1, BRA_SILU, bf16_t>(oX, oW1, b1, pre, at(P.Act), pA, S, P, at(P.parts), st)
                                    : gated<1, BRA_GELU, bf16_t>(oX, oW1, b1, pre, at(P.Act), pA, S, P, at(P.parts), st);
    }
    if (rc != BRA_OK) return rc;
    ProfScope prof(st, K_FFN_PRODUCT);
    if (P.product_shares > 1) {
        float *part = (float *)at(P.parts);
        return S.f32 ? split<TSplit, -1, 3, float>(oA, oW2, b2, nullptr, Y, 0, S.M, S.C, S.Cp, P.product_shares, part, st)
                     : split<TSplit, -1, 1, bf16_t>(oA, oW2, b2, nullptr, Y, 0, S.M, S.C, S.Cp, P.product_shares, part, st);
    }
    return S.f32 ? product<3, float>(oA, oW2, S.M, S.C, Y, b2, st) : product<1, bf16_t>(oA, oW2, S.M, S.C, Y, b2, st);
}

}  // namespace bra
