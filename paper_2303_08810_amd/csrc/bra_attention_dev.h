// Building blocks of attention between whole sequences (internal).
//
// Every product is formed with the index that a lane keeps in the matrix instruction's columns: S^T = K Q^T has a query per lane (and half of
// the keys, four and four), O^T = V^T P^T takes that result as its right operand as it stands in the registers, since the order of the contraction
// is free: step kk takes the keys 16 kk + 4 h + 0..3 and 16 kk + 8 + 4 h + 0..3 from half h of the wavefront, and V^T is read from LDS in
// the same order.  No value of S or P moves between lanes.  The backward pass does the same with keys in the columns.
// bf16: 32x32x16 instructions, the transposed operand by the transposing LDS read.  float32 with many rows: three bf16 terms to a value, x = hi + mid +
// lo, and the six products of terms that matter (2^-23 of a product is left out), the small ones first: on the float32 instruction, which few rows take, a
// product takes 16 bf16 ones' time, this way 6.
#pragma once

#include "bra_attention.h"
#include "bra_attn_dev.h"

#include <type_traits>

namespace bra {
namespace att {

using namespace mfma;

// What tiles read beyond a sequence's end and a head's width.
alignas(16) static __device__ bf16_t zeros[8];

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

struct Call {
    Rows Q, K, V, O;
    const int *q_lens, *k_lens;
    int Nq, Nk, G, Hk, d;           // G query heads to a key head
    unsigned magic;                 // division by G
    int rows;                       // Nq G
    int causal;
    float scale, c;                 // c = scale log2 e
    int tiles, splits;
    long first, blocks;             // this launch's first workgroup, and how many there are over all launches
    long whole;                     // workgroups of the heads in whole groups of 8
    int whole_heads;                // those heads
    float *lse;                     // [B, heads, Nq]
    float *part, *part_ml;          // of the splits
    // the backward pass
    Rows dO, dQ, dK, dV;
    const float *lse_in;
    float *row_lse, *row_delta;     // [B Hk, rows]: lse log2 e, and sum of dO O
    // float32 as three planes of bf16 terms, [B Hk][rows rounded up to 32][pitch] each, zero behind lengths and widths
    const char *pK, *pV, *pQ, *pG;
    long key_plane, row_plane;      // bytes from a plane to the next
    int key_rows, row_rows;         // of a head in a plane
};

// row / G: the product with 2^32 / G, rounded up, is too large by one at most.
__device__ __forceinline__ int row_query(const Call &A, int row)
{
    if (A.G == 1) return row;
    const int q = (int)__umulhi((unsigned)row, A.magic);
    return q - (q * A.G > row);
}

// Lengths and masks of a sequence: query q sees the keys below limit(q).
struct Sequence {
    int nq, nk, off;
    bool causal;
    __device__ __forceinline__ Sequence(const Call &A, int b)
        : nq(A.q_lens ? min(max(A.q_lens[b], 0), A.Nq) : A.Nq), nk(A.k_lens ? min(max(A.k_lens[b], 0), A.Nk) : A.Nk), off(nk - nq), causal(A.causal) {}
    __device__ __forceinline__ int limit(int q) const { return q >= nq ? 0 : causal ? min(max(q + off + 1, 0), nk) : nk; }
};

// What workgroup `block` works on: `per` workgroups to a head, those of a head on one XCD, where they meet in its L2, heads next to each other on
// different ones, since those of a batch's long sequences would otherwise come to one.  The last heads, fewer than XCDs, are dealt out evenly, a part of a head
// to an XCD, or, where sequences have lengths of their own, every head to all of them.
struct Place {
    int head, inner;
    __device__ __forceinline__ Place(const Call &A, long block, int per)
    {
        long i = block;
        if (block < A.whole) {
            const unsigned xcd = (unsigned)block % 8;
            const long j = block / 8;
            const long group = j >> 32 ? j / per : (unsigned)j / (unsigned)per;        // (the long division takes 0.3 us)
            head = (int)(group * 8 + xcd);
            inner = (int)(j - group * per);
            return;
        }
        if (!A.q_lens && !A.k_lens) {
            const unsigned left = (unsigned)(A.blocks - A.whole), j = (unsigned)(block - A.whole), xcd = j % 8;
            i = A.whole + xcd * (left / 8) + min(xcd, left % 8) + j / 8;
        }
        const unsigned rest = (unsigned)(i - A.whole);          // of fewer than 8 heads
        head = (int)(rest / (unsigned)per);
        inner = (int)(rest - head * (unsigned)per);
        head += A.whole_heads;
    }
};

// Elements E, heads of up to D channels: rows of P elements in LDS.
template <class E, int D_>
struct Geometry {
    static constexpr bool kF32 = sizeof(E) == 4;
    static constexpr int D = D_, P = D <= 32 ? 32 : D <= 64 ? 64 : 128, kPitch = P * (int)sizeof(E), kPieces = kPitch / 16;
    static constexpr int kSteps = D * (int)sizeof(E) / 32;      // pairs of 16-byte pieces of a row
    static constexpr int NT = D / 32;
    typedef typename std::conditional<kF32, f32x4, bf16x8>::type Piece;
    // Swizzle of a row's pieces: 16 rows' reads of one piece, and the four rows that a transposing read touches, lie in different banks.
    __device__ static __forceinline__ int turn(int row)
    {
        if (kPieces >= 16) return 2 * row % 16 + row / 8 % 2;
        if (kPieces == 8) return row % 8 / 2 * 2 % 8 + row / 8 % 2;
        return row / 4 % 4;
    }
};

// Direct loads of a tile of ROWS rows by THREADS threads (whole wavefronts).
template <class G, int ROWS, int THREADS>
struct Stage {
    static constexpr int L = ROWS * G::kPieces / THREADS;
    static_assert(L * THREADS == ROWS * G::kPieces, "whole loads");
    // at(row): address of a row of the tile; rows from `rows` on and pieces from `pieces` on read as zero
    template <class F>
    __device__ static __forceinline__ void request(F at, int rows, int pieces, unsigned lds, int thread)
    {
        const unsigned base = lds + 1024 * __builtin_amdgcn_readfirstlane(thread / 64);
#pragma unroll
        for (int u = 0; u < L; ++u) {
            const int i = thread + THREADS * u, row = i / G::kPieces, piece = i % G::kPieces ^ G::turn(row);
            const char *p = row < rows && piece < pieces ? at(row) + 16 * piece : (const char *)zeros;
            load_to_lds_untracked((const bf16_t *)p, base + 16 * THREADS * u);
        }
    }
};

// A row of a tensor (or zeros) as a column operand: pieces 2 ks + h.
template <class G>
__device__ __forceinline__ void load_columns(const char *p, bool valid, int pieces, int h, typename G::Piece (&x)[G::kSteps])
{
#pragma unroll
    for (int ks = 0; ks < G::kSteps; ++ks) {
        const int piece = 2 * ks + h;
        x[ks] = *(const typename G::Piece *)(valid && piece < pieces ? p + 16 * piece : (const char *)zeros);
    }
}

// The operands have arrived.  Without it the compiler, which does not count the direct loads, waits for the registers' loads at their first use in
// the loop over the tiles, and with them for the tile that is on its way, every time.
template <class G>
__device__ __forceinline__ void arrived(typename G::Piece (&x)[G::kSteps])
{
#pragma unroll
    for (int ks = 0; ks < G::kSteps; ++ks) asm volatile("" : "+v"(x[ks]));
}

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// acc += (rows row0 .. row0 + 31 of a tile) (columns in registers)
template <class G>
__device__ __forceinline__ void multiply_rows(f32x16 &acc, const char *tile, int row0, const typename G::Piece (&x)[G::kSteps], int lane)
{
    const int h = lane / 32, c = lane % 32;
    const char *row = tile + (row0 + c) * G::kPitch;
#pragma unroll
    for (int ks = 0; ks < G::kSteps; ++ks) {
        const auto a = *(const typename G::Piece *)(row + 16 * ((2 * ks + h) ^ G::turn(c)));
        if constexpr (G::kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = mfma_f32(a[e], x[ks][e], acc);
        } else acc = mfma32(a, x[ks], acc);
    }
}

// acc[t] += (columns 32 t .. of rows row0 .. row0 + 31 of a tile, transposed) (p: 32 values of the contraction as the products leave them).
// The middle quads of 16 columns are exchanged: registers 8 a .. 8 a + 7 of a result are the channels 32 t + 16 a + 8 h ...
template <class G>
__device__ __forceinline__ void multiply_columns(f32x16 (&acc)[G::NT], const char *tile, int row0, const f32x16 &p, int lane)
{
    const int h = lane / 32, c = lane % 32;
    if constexpr (G::kF32) {
        const int channel = c / 16 * 16 + c / 4 % 2 * 8 + c / 8 % 2 * 4 + c % 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = 8 * (r / 4) + 4 * h + r % 4;
#pragma unroll
            for (int t = 0; t < G::NT; ++t) {
                const int o = 32 * t + channel;
                const float a = *(const float *)(tile + (row0 + row) * G::kPitch + 16 * ((o / 4) ^ G::turn(row)) + 4 * (o % 4));
                acc[t] = mfma_f32(a, p[r], acc[t]);
            }
        }
    } else {
        const int s = lane % 16, q = lane / 16, col4 = s % 2 * 2 + s % 4 / 2;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const bf16x8 b = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(p[8 * kk], p[8 * kk + 1]), pack_bf16(p[8 * kk + 2], p[8 * kk + 3]),
                                                              pack_bf16(p[8 * kk + 4], p[8 * kk + 5]), pack_bf16(p[8 * kk + 6], p[8 * kk + 7])});
#pragma unroll
            for (int t = 0; t < G::NT; ++t) {
                const int o = 32 * t + 16 * (q % 2) + 4 * col4;
                u32x2 r[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int row = 16 * kk + 8 * half + 4 * h + s / 4;
                    r[half] = __builtin_bit_cast(u32x2, lds_read_tr16((const bf16_t *)(tile + (row0 + row) * G::kPitch + 16 * ((o / 8) ^ G::turn(row))) + o % 8));
                }
                acc[t] = mfma32(__builtin_bit_cast(bf16x8, u32x4{r[0][0], r[0][1], r[1][0], r[1][1]}), b, acc[t]);
            }
        }
    }
}

// A column's 8 channels 32 t + 16 a + 8 h .. to memory.
template <class E>
__device__ __forceinline__ void store8(char *p, const float (&v)[8])
{
    if constexpr (sizeof(E) == 2) *(bf16x8 *)p = pack8(v);
    else {
        *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4 *)(p + 16) = f32x4{v[4], v[5], v[6], v[7]};
    }
}
template <class E, class G>
__device__ __forceinline__ void store_columns(char *p, const f32x16 (&acc)[G::NT], float factor, int d, int h)
{
#pragma unroll
    for (int t = 0; t < G::NT; ++t)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int channel = 32 * t + 16 * a + 8 * h;
            if (channel >= d) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[t][8 * a + e] * factor;
            store8<E>(p + channel * sizeof(E), v);
        }
}

template <int N>
__device__ __forceinline__ void clear(f32x16 (&acc)[N])
{
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
}

// A wavefront's reads of a tile in LDS, as offsets from its first row, for subtiles of 32 rows from a multiple of 32 on.
template <class G>
struct Reader {
    unsigned row[G::kSteps], column[2 * G::NT];
    __device__ __forceinline__ explicit Reader(int lane)
    {
        const int h = lane / 32, c = lane % 32, s = lane % 16, q = lane / 16, col4 = s % 2 * 2 + s % 4 / 2;
#pragma unroll
        for (int ks = 0; ks < G::kSteps; ++ks) row[ks] = c * G::kPitch + 16 * ((2 * ks + h) ^ G::turn(c));
#pragma unroll
        for (int t = 0; t < G::NT; ++t)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int r = 8 * half + 4 * h + s / 4, o = 32 * t + 16 * (q % 2) + 4 * col4;
                column[2 * t + half] = r * G::kPitch + 16 * ((o / 8) ^ G::turn(r)) + 2 * (o % 8);
            }
    }
};

template <int N, class F, int I = 0>
__device__ __forceinline__ void unrolled(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<N, F, I + 1>(f);
    }
}

// One product of a subtile: slot f of kRows multiplies rows into s, slot f of kColumns columns into acc.  T terms to a value, whose tiles are PLANE bytes apart.
template <class G, int T, int PLANE>
struct Slots {
    static constexpr int kRows = G::kSteps, kColumns = 2 * G::NT;
    static constexpr bool kLeaves = T == 3;         // the last step of rows is left out where heads have no channels there: six products for a branch
    struct Operand {
        u32x4 v[T];
    };
    struct Columns {            // what a wavefront keeps: 32 rows as column operands
        bf16x8 v[T][G::kSteps];
    };
    struct Weights {            // 32 values of the contraction
        u32x4 v[T][2];
    };
    // MIRROR: the terms' products in the order in which they come with the operands exchanged, so that both sides of a gradient have the same bits of a score.
    template <bool MIRROR = false>
    __device__ static __forceinline__ f32x16 product(const Operand &a, const bf16x8 (&b)[T], f32x16 c)
    {
        auto one = [&](int i, int j) __attribute__((always_inline)) { c = mfma32(__builtin_bit_cast(bf16x8, a.v[MIRROR ? j : i]), b[MIRROR ? i : j], c); };
        if constexpr (T == 3) {
            one(2, 0);
            one(0, 2);
            one(1, 1);
            one(1, 0);
            one(0, 1);
        }
        one(0, 0);
        return c;
    }
    __device__ static __forceinline__ void read_rows(Operand &o, const char *tile, const Reader<G> &R, int f)
    {
#pragma unroll
        for (int t = 0; t < T; ++t) o.v[t] = *(const u32x4 *)(tile + t * PLANE + R.row[f]);
    }
    __device__ static __forceinline__ void read_columns(Operand &o, const char *tile, const Reader<G> &R, int f)
    {
        const int kk = f / G::NT, n = f % G::NT;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            u32x2 r[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) r[half] = __builtin_bit_cast(u32x2, lds_read_tr16((const bf16_t *)(tile + t * PLANE + 16 * kk * G::kPitch + R.column[2 * n + half])));
            o.v[t] = u32x4{r[0][0], r[0][1], r[1][0], r[1][1]};
        }
    }
    template <bool MIRROR = false>
    __device__ static __forceinline__ void rows(f32x16 &s, const Operand &o, const Columns &x, int f)
    {
        bf16x8 b[T];
#pragma unroll
        for (int t = 0; t < T; ++t) b[t] = x.v[t][f];
        s = product<MIRROR>(o, b, s);
    }
    __device__ static __forceinline__ void columns(f32x16 (&acc)[G::NT], const Operand &o, const Weights &p, int f)
    {
        bf16x8 b[T];
#pragma unroll
        for (int t = 0; t < T; ++t) b[t] = __builtin_bit_cast(bf16x8, p.v[t][f / G::NT]);
        acc[f % G::NT] = product(o, b, acc[f % G::NT]);
    }
    // Values r - 1 and r of the weights.
    __device__ static __forceinline__ void keep(Weights &p, const f32x16 &s, int r)
    {
        float a = s[r - 1], b = s[r];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const unsigned u = pack_bf16(a, b);
            p.v[t][r / 8][r % 8 / 2] = u;
            a -= bf16_lo(u);
            b -= bf16_hi(u);
        }
    }
    // A row of a tensor (or zeros), pieces 2 ks + h of 8 channels of `pieces`.
    template <class E>
    __device__ static __forceinline__ void load(const char *p, bool valid, int pieces, int h, Columns &x)
    {
#pragma unroll
        for (int ks = 0; ks < G::kSteps; ++ks) {
            const int piece = 2 * ks + h;
            const bool there = valid && piece < pieces;
            if constexpr (T == 1) x.v[0][ks] = *(const bf16x8 *)(there ? p + 16 * piece : (const char *)zeros);
            else {
                const f32x4 v0 = *(const f32x4 *)(there ? p + 32 * piece : (const char *)zeros), v1 = *(const f32x4 *)(there ? p + 32 * piece + 16 : (const char *)zeros);
                const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
                bf16x8 t[3];
                split3(v, t);
#pragma unroll
                for (int i = 0; i < T; ++i) x.v[i][ks] = t[i];
            }
        }
    }
    // The operands have arrived.  Without it the compiler, which does not count the direct loads, waits for the registers' loads at their first use in
    // the loop over the tiles, and with them for the tile that is on its way, every time.
    __device__ static __forceinline__ void arrived(Columns &x)
    {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int ks = 0; ks < G::kSteps; ++ks) asm volatile("" : "+v"(x.v[t][ks]));
    }
};

// sum over a row's channels of a b, this lane's pieces of them; all loads are on their way at once
template <class E, int STEPS>
__device__ __forceinline__ float row_product(const char *a, const char *b, bool valid, int pieces, int h)
{
    constexpr int W = sizeof(E) == 2 ? 1 : 2;       // loads of 16 bytes to 8 channels
    u32x4 x[STEPS * W], y[STEPS * W];
#pragma unroll
    for (int i = 0; i < STEPS * W; ++i) {
        const int piece = 2 * (i / W) + h;
        const bool there = valid && piece < pieces;
        x[i] = *(const u32x4 *)(there ? a + 16 * (W * piece + i % W) : (const char *)zeros);
        y[i] = *(const u32x4 *)(there ? b + 16 * (W * piece + i % W) : (const char *)zeros);
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS * W; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (W == 1) sum = fmaf(bf16_lo(x[i][e]), bf16_lo(y[i][e]), fmaf(bf16_hi(x[i][e]), bf16_hi(y[i][e]), sum));
            else sum = fmaf(__builtin_bit_cast(f32x4, x[i])[e], __builtin_bit_cast(f32x4, y[i])[e], sum);
        }
    return sum;
}

// Where tiles of keys (rows) of a head come from: the tensor itself, or its planes of terms, which have whole rows and zeros behind the end.
struct Source {
    const char *p;
    long token, plane;
    int rows, pieces;
};
template <class G, int T>
__device__ __forceinline__ Source key_source(const Call &A, const Rows &R, const char *planes, int b, int hb, int nk)
{
    if constexpr (T == 1) return Source{R.p + b * R.batch + (hb - b * A.Hk) * R.head, R.token, 0, nk, A.d / 8};
    else return Source{planes + (long)hb * A.key_rows * G::kPitch, G::kPitch, A.key_plane, A.key_rows, G::kPieces};
}
template <class G>
__device__ __forceinline__ Source row_source(const Call &A, const char *planes, int hb)
{
    return Source{planes + (long)hb * A.row_rows * G::kPitch, G::kPitch, A.row_plane, A.row_rows, G::kPieces};
}

// Direct loads of its tiles of ROWS rows one after the other, from row `first` on: a lane's pointers go on by a tile each time.  Rows that do not fill the pitch select zeros at
// every load (8 x 1024 tokens of 12 heads in bf16, of 56 / 64 channels 38.5 / 36.8 us, of 80 / 96 / 104 / 120 / 128 55.0 / 55.9 / 65.4 / 69.0 / 63.6).
template <class G, int T, int ROWS, int THREADS>
struct Walk {
    static constexpr int kLoads = ROWS * G::kPieces, L = (kLoads + THREADS - 1) / THREADS, kTile = ROWS * G::kPitch;
    static_assert(kLoads % THREADS == 0 || (kLoads < THREADS && kLoads % 64 == 0), "whole loads of a wavefront");
    const char *at[L];
    long step, plane;
    unsigned wave;          // LDS offset of this wavefront's part
    int left, pieces;       // rows from the next tile on; pieces of a row
    __device__ __forceinline__ Walk(const Source &S, int first, int thread)
        : step(ROWS * S.token), plane(S.plane), wave(1024 * __builtin_amdgcn_readfirstlane(thread / 64)), left(S.rows - first), pieces(S.pieces)
    {
#pragma unroll
        for (int u = 0; u < L; ++u) {
            const int i = thread + THREADS * u, row = i / G::kPieces, piece = i % G::kPieces ^ G::turn(row);
            at[u] = S.p + (first + row) * S.token + 16 * piece;
        }
    }
    __device__ __forceinline__ void request(unsigned lds, int thread)
    {
        if (kLoads < THREADS && wave >= kLoads * 16) return;        // the first wavefronts load it all
        if (T > 1 || (pieces == G::kPieces && left >= ROWS)) {
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int u = 0; u < L; ++u) load_to_lds_untracked((const bf16_t *)(at[u] + t * plane), lds + wave + t * kTile + 16 * THREADS * u);
        } else {
#pragma unroll
            for (int u = 0; u < L; ++u) {
                const int i = thread + THREADS * u, row = i / G::kPieces, piece = i % G::kPieces ^ G::turn(row);
                load_to_lds_untracked((const bf16_t *)(row < left && piece < pieces ? at[u] : (const char *)zeros), lds + wave + 16 * THREADS * u);
            }
        }
#pragma unroll
        for (int u = 0; u < L; ++u) at[u] += step;
        left -= ROWS;
    }
};

// A head's rows, which lie at place(row), to LDS; zeros behind `rows`.
template <class E, class F, class P>
__device__ __forceinline__ void load_short(char *tile, int rows, int pieces, P place)
{
    typedef typename F::G G;
    constexpr int kLoads = F::kPlane / 16, L = (kLoads + F::kThreads - 1) / F::kThreads;
    const unsigned at = lds_address(tile) + 1024 * __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
    for (int u = 0; u < L; ++u) {
        const int i = threadIdx.x + F::kThreads * u, row = i / G::kPieces, piece = i % G::kPieces ^ G::turn(row);
        if (kLoads % F::kThreads != 0 && i >= kLoads) break;         // (whole wavefronts)
        const bool there = row < rows && piece < pieces;
        const char *p = there ? place(row) + (int)sizeof(E) * 8 * piece : (const char *)zeros;
        if constexpr (F::T == 1) load_to_lds_untracked((const bf16_t *)p, at + 16 * F::kThreads * u);
        else {
            const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(there ? p + 16 : p);
            const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            bf16x8 t[3];
            split3(v, t);
#pragma unroll
            for (int k = 0; k < 3; ++k) *(bf16x8 *)(tile + k * F::kPlane + 16 * i) = t[k];
        }
    }
}

// The same for one term and rows whose places are at(row), `step` bytes further on with every tile, or (0) anywhere.  Gradients of 2 x 2048 tokens of 4 key heads of 128 with 2, 4 and
// 8 heads to each, which have a step, 524 / 642 / 683 TFLOP/s; with 3, 5, 6 and 7, which form every place anew, 514 / 519 / 550 / 552 (heads of 64 478 / 599 / 655 and 508 / 563 / 595 / 580).
template <class G, int ROWS, int THREADS>
struct Tiles {
    static constexpr int kLoads = ROWS * G::kPieces, L = (kLoads + THREADS - 1) / THREADS;
    static_assert(kLoads % THREADS == 0 || (kLoads < THREADS && kLoads % 64 == 0), "whole loads of a wavefront");
    static constexpr int kLoaders = kLoads < THREADS ? kLoads / 64 : THREADS / 64;      // wavefronts that load
    const char *place[L];
    long step;
    int wave, row, end;     // this wavefront; the next tile's first row, where rows end
    bool whole;             // rows fill the pitch
    __device__ static __forceinline__ int row_of(int u, int thread) { return (thread + THREADS * u) / G::kPieces; }
    __device__ static __forceinline__ int piece_of(int u, int thread) { return (thread + THREADS * u) % G::kPieces ^ G::turn(row_of(u, thread)); }
    template <class F>
    __device__ __forceinline__ Tiles(F at, long step_, int first, int end_, int pieces, int thread)
        : step(step_), wave(__builtin_amdgcn_readfirstlane(thread / 64)), row(first), end(end_), whole(pieces == G::kPieces)
    {
#pragma unroll
        for (int u = 0; u < L; ++u) place[u] = at(first + row_of(u, thread)) + 16 * piece_of(u, thread);
    }
    template <class F>
    __device__ __forceinline__ void request(unsigned lds, int pieces, int thread, F at)
    {
        const unsigned to = lds + 1024 * wave;
#pragma unroll
        for (int u = 0; u < L; ++u)
            load_to_lds_untracked((const bf16_t *)(row + row_of(u, thread) < end && piece_of(u, thread) < pieces ? place[u] : (const char *)zeros), to + 16 * THREADS * u);
        row += ROWS;
#pragma unroll
        for (int u = 0; u < L; ++u) place[u] = step ? place[u] + step : at(row + row_of(u, thread)) + 16 * piece_of(u, thread);
    }
    // the same where the tile and its rows are whole and places go on by `step`
    __device__ __forceinline__ void request_whole(unsigned lds)
    {
        const unsigned to = lds + 1024 * wave;
#pragma unroll
        for (int u = 0; u < L; ++u) load_to_lds_untracked((const bf16_t *)place[u], to + 16 * THREADS * u);
        row += ROWS;
#pragma unroll
        for (int u = 0; u < L; ++u) place[u] += step;
    }
};

// Whether the one key that a row sees has all of its weight, as far as the roundings of its score and of lse (both in powers of two) tell: O is that key's value then, and
// dS = dO V - dO O is zero.  What float32 leaves of the difference of the two sums would be all that dQ, and dK of a sequence of one key, consist of.  The score
// is asked, not the number of keys alone: with the lse of a longer sequence, of whose keys a call has one, the weight is less and dS is what the formula gives.
__device__ __forceinline__ bool all_weight(float s, float c, float lse) { return fabsf(fmaf(s, c, -lse)) < 0x1p-16f * (1.f + fabsf(lse)); }

// Of the two lanes of a column.
__device__ __forceinline__ float pair_max(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float pair_sum(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
// Over the columns of a wavefront.
__device__ __forceinline__ int columns_min(int v)
{
#pragma unroll
    for (int o = 16; o; o /= 2) v = min(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int columns_max(int v)
{
#pragma unroll
    for (int o = 16; o; o /= 2) v = max(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}

// Softmax statistics of a column, in powers of two: m, from which its weights are taken (the same in both of its lanes), l this lane's share of their
// sum.
struct Running {
    float m, base, bar, l = 0.f;        // base: m, or 0 where there is none yet; bar: what a lane's weights of 32 keys may sum up to
    // `sees`: whether any key is visible to the column; one that sees none needs no m
    __device__ __forceinline__ explicit Running(bool sees) : m(sees ? -INFINITY : 0.f), base(0.f), bar(sees ? -1.f : kMost) {}
    static constexpr float kMost = 8192.f;
    // S -> P of 32 keys.  Weights are taken from the m that there is; only where a lane's sum shows that one has grown too large, or where there is none
    // yet, the maximum is looked for, and m raised to it.  Sums are float32 and stay below 2^13 a step.  The largest weight of a row's first tile is
    // one, which bf16 holds: a row of one key is that key's value, and in rows of few keys the weight that counts most is not rounded.  The maximum of every tile took a sixth of the vector instructions, which bound heads of 64 channels.
    template <int NT>
    __device__ __forceinline__ void weights(f32x16 &s, float c, f32x16 (&acc)[NT])
    {
        f32x16 e;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -base));
            sum += e[r];
        }
        if (__builtin_amdgcn_ballot_w64(sum > bar) != 0) {
            float top = fmaxf(s[0], s[1]);
#pragma unroll
            for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
            const float next = fmaxf(m, pair_max(top) * c), alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - next);
            m = next;
            base = next == -INFINITY ? 0.f : next;
            bar = next == -INFINITY ? -1.f : kMost;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
            sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -base));
                sum += e[r];
            }
        }
        l += sum;
        s = e;
    }
};

// The row that 16 registers of a product's result stand for.
__device__ __forceinline__ int result_row(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

Call make_call(const Sizes &S);

// The grid: `tiles` x `splits` workgroups to a head.
inline void set_grid(Call &A, long heads, long tiles, int splits)
{
    A.tiles = (int)tiles;
    A.splits = splits;
    A.blocks = tiles * splits * heads;
    A.whole_heads = (int)(heads / 8 * 8);
    A.whole = tiles * splits * A.whole_heads;
}

// float32: the planes of terms of keys and values, in the backward pass of queries and dO too (bra_attention_terms.hip).
size_t terms_bytes(const Sizes &S, bool backward);
int make_terms(const Sizes &S, Call &A, bool backward, void *ws, hipStream_t st);

constexpr long kMaxBlocks = 1L << 22;       // of a launch: fewer than 2^32 threads

}  // namespace att
}  // namespace bra
