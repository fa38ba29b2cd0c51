// Building blocks of attention between whole sequences (internal).
//
// Every product is formed with the index that a lane keeps in the matrix instruction's columns: S^T = K Q^T has a query per lane (and half of
// the keys, four and four), O^T = V^T P^T takes that result as its right operand as it stands in the registers, since the order of the contraction
// is free: step kk takes the keys 16 kk + 4 h + 0..3 and 16 kk + 8 + 4 h + 0..3 from half h of the wavefront, and V^T is read from LDS in
// the same order.  No value of S or P moves between lanes.  The backward pass does the same with keys in the columns.
// bf16: 32x32x16 instructions, the transposed operand by the transposing LDS read.  float32: 32x32x2 instructions, the same layouts.
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
    float *lse;                     // [B, heads, Nq]
    float *part, *part_ml;          // of the splits
    // the backward pass
    Rows dO, dQ, dK, dV;
    const float *lse_in;
    float *row_lse, *row_delta;     // [B Hk, rows]: lse log2 e, and sum of dO O
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
// different ones, since those of a batch's long sequences would otherwise come to one.  The workgroups of the last heads, fewer than XCDs, are dealt out evenly.
struct Place {
    int head, inner;
    __device__ __forceinline__ Place(long block, long blocks, long per)
    {
        const long whole = blocks / per / 8 * 8 * per;
        long i;
        if (block < whole) {
            const long j = block / 8;
            i = (j / per * 8 + block % 8) * per + j % per;
        } else {
            const long left = blocks - whole, j = block - whole, xcd = j % 8, each = left / 8, rest = left % 8;
            i = whole + xcd * each + min(xcd, rest) + j / 8;
        }
        head = (int)(i / per);
        inner = (int)(i - head * per);
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
    unsigned row[G::kSteps], column[G::kF32 ? 2 : 2 * G::NT];
    __device__ __forceinline__ explicit Reader(int lane)
    {
        const int h = lane / 32, c = lane % 32;
#pragma unroll
        for (int ks = 0; ks < G::kSteps; ++ks) row[ks] = c * G::kPitch + 16 * ((2 * ks + h) ^ G::turn(c));
        if constexpr (!G::kF32) {
            const int s = lane % 16, q = lane / 16, col4 = s % 2 * 2 + s % 4 / 2;
#pragma unroll
            for (int t = 0; t < G::NT; ++t)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = 8 * half + 4 * h + s / 4, o = 32 * t + 16 * (q % 2) + 4 * col4;
                    column[2 * t + half] = r * G::kPitch + 16 * ((o / 8) ^ G::turn(r)) + 2 * (o % 8);
                }
        } else {
            // rows 8 a + 4 h + b of a subtile, a channel of 32: turn() of the row is that of 4 h with b in front of it and a % 2 behind
            const int channel = c / 16 * 16 + c / 4 % 2 * 8 + c / 8 % 2 * 4 + c % 4;
            column[0] = 4 * h * G::kPitch + 4 * (channel % 4);
            column[1] = channel / 4 ^ G::turn(4 * h);
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

// One product of a subtile: slot f of kRowSlots multiplies rows into s, slot f of kColumnSlots columns into acc.  A slot's operand is read some
// slots before.
template <class G>
struct Slots {
    static constexpr int kRows = G::kSteps, kColumns = G::kF32 ? 16 : 2 * G::NT;
    struct Operand {
        typename std::conditional<G::kF32, f32x4, u32x4>::type v;
    };
    __device__ static __forceinline__ void read_rows(Operand &o, const char *tile, const Reader<G> &R, const int f) { o.v = *(const decltype(o.v) *)(tile + R.row[f]); }
    __device__ static __forceinline__ void read_columns(Operand &o, const char *tile, const Reader<G> &R, int f)
    {
        if constexpr (G::kF32) {
            const int row = 8 * (f / 4) + f % 4;            // + 4 h
#pragma unroll
            for (int t = 0; t < G::NT; ++t) {
                const int piece = (8 * t) ^ (R.column[1] ^ G::turn(row));
                o.v[t] = *(const float *)(tile + R.column[0] + row * G::kPitch + 16 * piece);
            }
        } else {
            const int kk = f / G::NT, t = f % G::NT;
            u32x2 r[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) r[half] = __builtin_bit_cast(u32x2, lds_read_tr16((const bf16_t *)(tile + 16 * kk * G::kPitch + R.column[2 * t + half])));
            o.v = u32x4{r[0][0], r[0][1], r[1][0], r[1][1]};
        }
    }
    __device__ static __forceinline__ void rows(f32x16 &s, const Operand &o, const typename G::Piece (&x)[G::kSteps], int f)
    {
        if constexpr (G::kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s = mfma_f32(o.v[e], x[f][e], s);
        } else s = mfma32(__builtin_bit_cast(bf16x8, o.v), x[f], s);
    }
    typedef typename std::conditional<G::kF32, f32x16, u32x4[2]>::type Weights;        // 32 values of the contraction: float32, or bf16 pairs
    __device__ static __forceinline__ void copy(Weights &p, const Weights &q)
    {
        if constexpr (G::kF32) p = q;
        else {
            p[0] = q[0];
            p[1] = q[1];
        }
    }
    // Values r - 1 and r of them.
    __device__ static __forceinline__ void keep(Weights &p, const f32x16 &s, int r)
    {
        if constexpr (G::kF32) {
            p[r - 1] = s[r - 1];
            p[r] = s[r];
        } else p[r / 8][r % 8 / 2] = pack_bf16(s[r - 1], s[r]);
    }
    __device__ static __forceinline__ void columns(f32x16 (&acc)[G::NT], const Operand &o, const Weights &p, int f)
    {
        if constexpr (G::kF32) {
#pragma unroll
            for (int t = 0; t < G::NT; ++t) acc[t] = mfma_f32(o.v[t], p[f], acc[t]);
        } else acc[f % G::NT] = mfma32(__builtin_bit_cast(bf16x8, o.v), __builtin_bit_cast(bf16x8, p[f / G::NT]), acc[f % G::NT]);
    }
};

// Direct loads of a tensor's tiles of ROWS rows one after the other: a lane's pointers go on by a tile each time.
template <class G, int ROWS, int THREADS>
struct Walk {
    static constexpr int L = ROWS * G::kPieces / THREADS;
    static_assert(L * THREADS == ROWS * G::kPieces, "whole loads");
    const char *at[L];
    long step;
    unsigned wave;          // LDS offset of this wavefront's part
    int left;               // rows from the next tile on
    bool whole;             // rows fill the pitch
    __device__ __forceinline__ Walk(const char *first, long token, int rows, int pieces, int thread) : step(ROWS * token), wave(1024 * __builtin_amdgcn_readfirstlane(thread / 64)), left(rows), whole(pieces == G::kPieces)
    {
#pragma unroll
        for (int u = 0; u < L; ++u) {
            const int i = thread + THREADS * u, row = i / G::kPieces, piece = i % G::kPieces ^ G::turn(row);
            at[u] = first + row * token + 16 * piece;
        }
    }
    __device__ __forceinline__ void request(unsigned lds, int pieces, int thread)
    {
        if (whole && left >= ROWS) {
#pragma unroll
            for (int u = 0; u < L; ++u) load_to_lds_untracked((const bf16_t *)at[u], lds + wave + 16 * THREADS * u);
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

// The same for rows whose places are at(row), `step` bytes further on with every tile, or (0) anywhere.
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
        if (wave < kLoaders) {
            if (whole && row + ROWS <= end) {
#pragma unroll
                for (int u = 0; u < L; ++u) load_to_lds_untracked((const bf16_t *)place[u], to + 16 * THREADS * u);
            } else {
#pragma unroll
                for (int u = 0; u < L; ++u)
                    load_to_lds_untracked((const bf16_t *)(row + row_of(u, thread) < end && piece_of(u, thread) < pieces ? place[u] : (const char *)zeros), to + 16 * THREADS * u);
            }
        }
        row += ROWS;
#pragma unroll
        for (int u = 0; u < L; ++u) place[u] = step ? place[u] + step : at(row + row_of(u, thread)) + 16 * piece_of(u, thread);
    }
};

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

// Softmax statistics of a column, in powers of two: m, from which its weights are taken (a whole number, the same in both of its lanes), l this lane's
// share of their sum.
struct Running {
    float m, base, bar, l = 0.f;        // base: m, or 0 where there is none yet; bar: what a lane's weights of 32 keys may sum up to
    // `sees`: whether any key is visible to the column; one that sees none needs no m
    __device__ __forceinline__ explicit Running(bool sees) : m(sees ? -INFINITY : 0.f), base(0.f), bar(sees ? -1.f : kMost) {}
    static constexpr float kMost = 8192.f;
    // S -> P of 32 keys.  Weights are taken from the m that there is; only where a lane's sum shows that one has grown too large, or where there is none
    // yet, the maximum is looked for, and m raised to it: what is in acc follows by a power of two, so that nothing is rounded.  Sums are float32
    // and stay below 2^13 a step.  The maximum of every tile took a sixth of the vector instructions, which bound heads of 64 channels.
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
            const float next = fmaxf(m, ceilf(pair_max(top) * c)), alpha = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - next);
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

constexpr long kMaxBlocks = 1L << 22;       // of a launch: fewer than 2^32 threads

}  // namespace att
}  // namespace bra
