// Building blocks of the gated feed-forward block's products (internal).
//
// A tile of BM rows m x BN columns n of a product, the contraction in chunks of 64 that direct loads bring into a ring of
// buffers in LDS while one of them is multiplied.  Either operand may lie with the contraction axis inside (rows of k) or
// outside (rows of m or n): the second kind is read by the transposing LDS read, so that no product of the forward or the
// backward pass needs a transposed copy.  The product is formed transposed (rows n, columns m of the 32x32x16 instruction), the two
// middle bits of n exchanged, so that a lane ends up with 8 consecutive columns of one row.
// float32 operands enter as three exact bf16 terms hi + mid + lo, each a plane of its own in memory; the six products of terms whose
// sizes matter (2^-24 of the product is left out) are further rounds over the contraction into the same accumulators, the small
// ones first.  On the float32 matrix instruction a product would take 16 bf16 ones' time, this way it takes 6.
#pragma once

#include "bra_attn_dev.h"
#include "bra_ffn.h"

namespace bra {
namespace ffn {

using namespace mfma;

// What chunks read beyond the contraction's end.
alignas(16) static __device__ bf16_t zeros[8];

// BM x BN outputs by WR x WC wavefronts, MT x NT 32 x 32 tiles each, NB buffers.
template <int BM_, int BN_, int WR_, int WC_, int NB_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WR = WR_, WC = WC_, NB = NB_, kWaves = WR * WC, kThreads = 64 * kWaves;
    static constexpr int MT = BM / (32 * WR), NT = BN / (32 * WC);
    static constexpr int kChunkA = BM * 64, kChunkB = BN * 64;                  // elements of a chunk
    static constexpr int kMinWaves = MT * NT > 8 ? 1 : 2;                       // per SIMD, of the register budget
    static constexpr size_t kLds = NB * (size_t)(kChunkA + kChunkB) * 2;
};

// Swizzle of the 16-byte pieces of a row: by rows of k where the contraction is outside (the four rows that a transposing
// read touches lie in different quarters of the banks), else differently for the 8 rows that 8 lanes next to each other read.
template <int B>
__device__ __forceinline__ int turn_outer(int k) { return B >= 128 ? 4 * (k % 4) : B == 64 ? 4 * (k / 2 % 2) : 0; }
__device__ __forceinline__ int turn_inner(int row) { return row / 2 % 8; }

// A wavefront's direct loads of one operand's chunks: B rows (or columns) of the tile, OUTER: contraction outside.
template <class T, int B, bool OUTER>
struct Loads {
    static constexpr int L = B / 8 / T::kWaves, CH = B / 8, RPI = 64 / CH;
    static_assert(L * 8 * T::kWaves == B, "a chunk is a whole number of loads per wavefront");
    unsigned off[L];                    // bytes from the chunk's origin
    // at(i): where row (column) i of the tile lies, relative to the origin; for OUTER asked for multiples of 8
    template <class F>
    __device__ __forceinline__ Loads(int wave, int lane, long ld, F at)
    {
#pragma unroll
        for (int u = 0; u < L; ++u) {
            if (OUTER) {
                const int k = RPI * (wave * L + u) + lane / CH;
                off[u] = 2u * (unsigned)(k * ld + at(8 * ((lane % CH) ^ turn_outer<B>(k))));
            } else {
                const int row = 8 * (wave * L + u) + lane / 8;
                off[u] = 2u * (unsigned)(at(row) * ld + 8 * ((lane % 8) ^ turn_inner(row)));
            }
        }
    }
    // load u of the chunk whose first element is `origin` (the same for all lanes), `left` of the contraction from there on, to LDS address `at`
    __device__ __forceinline__ void request(int u, const bf16_t *origin, int left, unsigned at, int wave, int lane) const
    {
        at += 1024 * (wave * L + u);
        if (left >= 64) {
            load_to_lds_untracked(origin, off[u], at);
            return;
        }
        const int row = 8 * (wave * L + u) + lane / 8;
        const int k = OUTER ? RPI * (wave * L + u) + lane / CH : 8 * ((lane % 8) ^ turn_inner(row));
        const bf16_t *p = (const bf16_t *)((const char *)origin + off[u]);
        load_to_lds_untracked(k < left ? p : zeros, at);
    }
};

// Operand of the matrix instruction: 32 rows (columns) from `first` on of the chunk, step ks of 16.
template <int B, bool OUTER, bool PERMUTED>
__device__ __forceinline__ bf16x8 fragment(const bf16_t *S, int first, int ks, int lane)
{
    const int h = lane / 32, c = lane % 32;
    if (!OUTER) {
        const int row = first + (PERMUTED ? (c & 0x13) + ((c & 4) << 1) + ((c & 8) >> 1) : c);
        return *(const bf16x8 *)(S + row * 64 + 8 * ((2 * ks + h) ^ turn_inner(row)));
    }
    // lane s of a 16-lane group q gives the address of 4 columns of row k
    const int s = lane % 16, q = lane / 16, col4 = PERMUTED ? (s % 2) * 2 + s % 4 / 2 : s % 4;
    u32x2 r[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int k = 16 * ks + 8 * (q / 2) + 4 * half + s / 4, o = first + 16 * (q % 2) + 4 * col4;
        r[half] = __builtin_bit_cast(u32x2, lds_read_tr16(S + k * B + 8 * ((o / 8) ^ turn_outer<B>(k)) + o % 8));
    }
    return __builtin_bit_cast(bf16x8, u32x4{r[0][0], r[0][1], r[1][0], r[1][1]});
}

template <class T>
__device__ __forceinline__ void clear(f32x16 (&acc)[T::NT][T::MT])
{
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[nt][mt][e] = 0.f;
}

// acc += A^T-or-A B over the contraction's chunks [first, end).  a0, b0: origins of the tile at k = 0 in the first plane.
// One barrier per chunk: it stands in the middle of the chunk's last quarter, whose operands are in registers by then, so that
// the buffer just read is free for the chunk after next, and the next chunk is there; the quarter's
// second half of products runs while the next chunk's first operands are read.  Reads and loads stand one by one between the products: in
// bursts they held up the products behind them.
template <class T, bool AO, bool BO, int TERMS>
__device__ __forceinline__ void multiply(const Operand &A, const Operand &Bm, const bf16_t *a0, const bf16_t *b0, const Loads<T, T::BM, AO> &la,
                                         const Loads<T, T::BN, BO> &lb, int first, int end, bf16_t *lds, f32x16 (&acc)[T::NT][T::MT])
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int wm = (wave / T::WC) * (32 * T::MT), wn = (wave % T::WC) * (32 * T::NT);
    const unsigned base = lds_address(lds);
    constexpr unsigned kBuffer = 2 * (T::kChunkA + T::kChunkB);
    constexpr int LA = Loads<T, T::BM, AO>::L, LB = Loads<T, T::BN, BO>::L, kLoads = LA + LB;
    const int rounds = end - first, total = TERMS == 1 ? rounds : 6 * rounds;
    // the chunk that is being asked for
    const bf16_t *an = a0, *bn = b0;
    int left_a = 0, left_b = 0;
    unsigned to = 0;
    auto aim = [&](int chunk, int buffer) {
        long pa = 0, pb = 0;
        int c = chunk;
        if (TERMS > 1) {
            const int round = chunk / rounds;
            c -= round * rounds;
            // (lo, hi), (hi, lo), (mid, mid), (mid, hi), (hi, mid), (hi, hi)
            pa = ((0x001102 >> (4 * round)) & 3) * A.plane;
            pb = ((0x010120 >> (4 * round)) & 3) * Bm.plane;
        }
        const int k0 = 64 * (first + c);
        an = a0 + pa + (AO ? k0 * A.ld : (long)k0);
        bn = b0 + pb + (BO ? k0 * Bm.ld : (long)k0);
        left_a = A.K - k0;
        left_b = Bm.K - k0;
        to = base + buffer * kBuffer;
    };
    auto ask = [&](int u) {
        if (u < LA) la.request(u, an, left_a, to, wave, lane);
        else if (u < kLoads) lb.request(u - LA, bn, left_b, to + 2 * T::kChunkA, wave, lane);
    };
    constexpr int kReads = T::NT + T::MT;
    if constexpr (T::MT * T::NT <= 2) {
        // Few products per chunk: a whole chunk's operands are in registers before its first product, read while the chunk before is multiplied.
        // Quarter by quarter, each waiting for LDS, a chunk of a 64 x 64 tile took 0.45 us.
        bf16x8 x[2][4][T::MT], w[2][4][T::NT];
        auto read = [&](int buffer, int reg) {
            const bf16_t *As = lds + buffer * (T::kChunkA + T::kChunkB), *Bs = As + T::kChunkA;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
                for (int nt = 0; nt < T::NT; ++nt) w[reg][ks][nt] = fragment<T::BN, BO, true>(Bs, wn + 32 * nt, ks, lane);
#pragma unroll
                for (int mt = 0; mt < T::MT; ++mt) x[reg][ks][mt] = fragment<T::BM, AO, false>(As, wm + 32 * mt, ks, lane);
            }
        };
        __builtin_amdgcn_s_barrier();              // the buffers are free
        for (int i = 0; i < min(T::NB, total); ++i) {
            aim(i, i);
#pragma unroll
            for (int u = 0; u < kLoads; ++u) ask(u);
        }
        if (total >= T::NB) asm volatile("s_waitcnt vmcnt(%0)" : : "n"((T::NB - 1) * kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, 0);
        int buffer = 0;
        auto turn = [&](int i, int reg) {
            const int next = buffer + 1 == T::NB ? 0 : buffer + 1;
            // the next chunk is there, and this one is in registers everywhere
            if (i + T::NB <= total) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((T::NB - 2) * kLoads) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            read(next, reg ^ 1);                   // (behind the last chunk: what is there, which nobody uses)
            if (i + T::NB < total) {
                aim(i + T::NB, buffer);
#pragma unroll
                for (int u = 0; u < kLoads; ++u) ask(u);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int mt = 0; mt < T::MT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < T::NT; ++nt) acc[nt][mt] = mfma32(w[reg][ks][nt], x[reg][ks][mt], acc[nt][mt]);
            __builtin_amdgcn_sched_barrier(0);
            buffer = next;
        };
        for (int i = 0; i < total; i += 2) {
            turn(i, 0);
            if (i + 1 < total) turn(i + 1, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        return;
    }
    bf16x8 xf[2][T::MT], wf[2][T::NT];
    // operand r of a step: buffer, quarter, and the registers it goes to
    auto read = [&](int r, int buffer, int ks, int reg) {
        const bf16_t *As = lds + buffer * (T::kChunkA + T::kChunkB), *Bs = As + T::kChunkA;
        if (r < T::NT) wf[reg][r] = fragment<T::BN, BO, true>(Bs, wn + 32 * r, ks, lane);
        else xf[reg][r - T::NT] = fragment<T::BM, AO, false>(As, wm + 32 * (r - T::NT), ks, lane);
    };
    // The products of the row tiles [mt0, mt1) with what is in registers `reg`; between them the reads of a step and the loads [u0, u1), as
    // evenly as they go.
    auto step = [&](int reg, int mt0, int mt1, bool reading, int buffer, int ks, int u0, int u1, bool asking) {
        const int n = (mt1 - mt0) * T::NT, side = (reading ? kReads : 0) + u1 - u0, reads = reading ? kReads : 0;
        int d = 0, s = 0;
#pragma unroll
        for (int mt = mt0; mt < mt1; ++mt)
#pragma unroll
            for (int nt = 0; nt < T::NT; ++nt) {
                acc[nt][mt] = mfma32(wf[reg][nt], xf[reg][mt], acc[nt][mt]);
                __builtin_amdgcn_sched_barrier(0);
                ++d;
#pragma unroll
                for (; s * n < side * d; ++s) {
                    if (s < reads) read(s, buffer, ks, reg ^ 1);
                    else if (asking) ask(u0 + s - reads);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    static_assert(T::MT * T::NT <= 2 || (T::MT > 1 && T::NB == 2), "the products of a step's second half cover the next chunk's first reads");
    constexpr int kHalf = T::MT / 2, kFirst = kLoads / 4;
    __builtin_amdgcn_s_barrier();                  // the buffers are free
    for (int i = 0; i < min(T::NB, total); ++i) {
        aim(i, i);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) ask(u);
    }
    if (total >= T::NB) asm volatile("s_waitcnt vmcnt(%0)" : : "n"((T::NB - 1) * kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int r = 0; r < kReads; ++r) read(r, 0, 0, 0);
    bool asking = false;
    for (int i = 0, buffer = 0; i < total; ++i) {
        const int next = buffer + 1 == T::NB ? 0 : buffer + 1;
        step(0, 0, T::MT, true, buffer, 1, kFirst, kLoads, asking);
        step(1, 0, T::MT, true, buffer, 2, 0, 0, false);
        step(0, 0, T::MT, true, buffer, 3, 0, 0, false);
        step(1, 0, kHalf, false, 0, 0, 0, 0, false);
        // the next chunk is there
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        asking = i + T::NB < total;
        if (asking) aim(i + T::NB, buffer);
        // (behind the last chunk the reads find what is there, which nobody uses)
        step(1, kHalf, T::MT, true, next, 0, 0, kFirst, asking);
        buffer = next;
    }
    // the wait between the last products and the first use of their results, spelled out: where a branch lies between them the
    // compiler has left it short
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15");
    __builtin_amdgcn_sched_barrier(0);
}

// Tile (m, n) of workgroup `block`: an XCD takes neighbouring tiles, in groups of 4 tiles along m, so that what its workgroups read at the
// same time fits its L2.
__device__ __forceinline__ void tile_of(int block, int mtiles, int ntiles, int &m, int &n)
{
    const int tiles = mtiles * ntiles, xcd = block % 8, per = tiles / 8, rest = tiles % 8;
    const int i = xcd * per + min(xcd, rest) + block / 8;
    const int group = 4 * ntiles, g = i / group, m0 = 4 * g, ms = min(4, mtiles - m0), r = i - g * group;
    m = m0 + r % ms;
    n = r / ms;
}

// Rows x 8 P bf16 of one wavefront, on their way between the products' layout (a lane has 8 columns of a row) and rows as they
// lie in memory, where a whole row of the wavefront's goes in one piece: stored from the products' layout, lines were written in pieces of 32
// bytes, and G | U of 32768 x 5632 took 160 us where its bytes take 75.
template <int P>
struct Rows {
    bf16_t *base;
    __device__ __forceinline__ bf16_t *at(int row, int piece) const { return base + (row * P + (piece ^ (row * P / 16 % P))) * 8; }
    __device__ __forceinline__ void put(int row, int piece, bf16x8 v) const { *(bf16x8 *)at(row, piece) = v; }
    // to(row, piece, value) for every piece of `rows` rows
    template <class F>
    __device__ __forceinline__ void each(int rows, int lane, F to) const
    {
#pragma unroll
        for (int r = 0; r < rows; r += 64 / P) {
            const int row = r + lane / P, piece = lane % P;
            to(row, piece, *(const bf16x8 *)at(row, piece));
        }
    }
};

// A piece of a row to memory: `n` of its 8 values exist, `vec`: rows are whole pieces.
__device__ __forceinline__ void store_piece(bf16_t *p, bf16x8 v, int n, bool vec)
{
    if (vec && n >= 8) {
        *(bf16x8 *)p = v;
        return;
    }
    const u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = (bf16_t)(u[e / 2] >> (16 * (e % 2)));
}

// A wavefront's sums to a slot of BM x BN floats, in the order of its registers.
template <class T>
constexpr int kSlot = T::BM * T::BN;
template <class T>
__device__ __forceinline__ void store_slot(float *slot, const f32x16 (&acc)[T::NT][T::MT], int wave, int lane)
{
    f32x4 *part = (f32x4 *)slot + wave * (T::NT * T::MT * 256) + lane;
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < T::MT; ++mt)
#pragma unroll
            for (int q = 0; q < 4; ++q) part[((nt * T::MT + mt) * 4 + q) * 64] = f32x4{acc[nt][mt][4 * q], acc[nt][mt][4 * q + 1], acc[nt][mt][4 * q + 2], acc[nt][mt][4 * q + 3]};
}
// The sum over `count` slots, `apart` from each other, of the 8 columns that lane `lane` has of 32 x 32 tile `frag` (of the workgroup's: wave, nt, mt), run `run`.
template <class T>
__device__ __forceinline__ void sum_slots(const float *part, size_t first, size_t apart, int count, int frag, int run, int lane, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 8
    for (int k = 0; k < count; ++k) {
        const f32x4 *p = (const f32x4 *)(part + (first + k * apart) * kSlot<T>) + (frag * 4 + 2 * run) * 64 + lane;
        const f32x4 a = p[0], b = p[64];
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] += a[e]; v[4 + e] += b[e]; }
    }
}

// 8 consecutive values; `n` of them exist, `vec`: in whole 16-byte pieces.
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8], int n, bool vec)
{
    if (vec && n >= 8) {
        *(u32x4 *)p = __builtin_bit_cast(u32x4, pack8(v));
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = f32_to_bf16(v[e]);
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8], int n, bool vec)
{
    if (vec && n >= 8) {
        *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = v[e];
}
__device__ __forceinline__ void load8(const bf16_t *p, float (&v)[8], int n, bool vec)
{
    if (vec && n >= 8) {
        const u32x4 t = *(const u32x4 *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(t[e]); v[2 * e + 1] = bf16_hi(t[e]); }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_to_f32(p[e]) : 0.f;
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8], int n, bool vec)
{
    if (vec && n >= 8) {
        const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
}

// 8 values of an operand that a later product reads: one bf16 rounding, or three terms.
template <int TERMS>
__device__ __forceinline__ void operand(const float (&v)[8], bf16x8 (&t)[TERMS])
{
    if constexpr (TERMS == 1) t[0] = pack8(v);
    else split3(v, t);
}
template <int TERMS>
__device__ __forceinline__ void store_operand(bf16_t *p, long plane, const float (&v)[8])
{
    bf16x8 t[TERMS];
    operand<TERMS>(v, t);
#pragma unroll
    for (int q = 0; q < TERMS; ++q) *(bf16x8 *)(p + q * plane) = t[q];
}

// The activations' distribution functions: act(g) = g F(g), act'(g) = F(g) + g F'(g).
//   silu: F = 1 / (1 + e^-g), F' = F (1 - F);  gelu: F = Phi, F' = e^(-g^2 / 2) / sqrt(2 pi).
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g)); }

// Phi for float32 results: Phi(-a) = e^(-a^2 / 2) t P(t), t = 1 / (1 + 0.35 a), a = |g|.  P, of degree 8, is the least maximum relative error of the
// rest on a <= 14.5 (by linear programming), 1.2 units of 2^-24 with its coefficients rounded; with the arithmetic's the value is within 2 g^2 + 36 units.
// 0.5 + 0.5 erf has lost the digits of Phi(g) below 0 (10 % of it at -5), the polynomial of gelu_f32 is within 7e-7 of 1, not of the value (2.6e-5 of it
// close to 0, 0.3 % at -4), and the library's erfc has branches that keep the epilogues' loops from being unrolled.
__device__ __forceinline__ float phi(float g)
{
    const float a = fabsf(g), t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.f));
    float p = fmaf(-2.915759198e-02f, t, 1.440297663e-01f);
    p = fmaf(p, t, -2.558371425e-01f);
    p = fmaf(p, t, 1.593181789e-01f);
    p = fmaf(p, t, -2.321167663e-02f);
    p = fmaf(p, t, 1.055523455e-01f);
    p = fmaf(p, t, 1.198213026e-01f);
    p = fmaf(p, t, 1.398635209e-01f);
    p = fmaf(p, t, 1.396213025e-01f);
    const float q = p * t * __builtin_amdgcn_exp2f(-0.72134752044448170f * (a * a));
    return g > 0.f ? 1.f - q : q;
}
// (-infinity gives 0)
__device__ __forceinline__ float gelu_exact(float g, float f) { return fmaxf(g, -16.f) * f; }

// EXACT: for float32 results.
template <int ACT, bool EXACT>
__device__ __forceinline__ float activation(float g)
{
    return ACT == BRA_SILU ? g * sigmoid(g) : EXACT ? gelu_exact(g, phi(g)) : gelu_f32(g);
}

// EXACT as above; else log2 Phi(-a) by the polynomial of gelu_f32, within 1.4e-5, a 280th of a bf16 step, for half the instructions (gradients of
// 12544 x 128 x 256 with GELU are bound by them).
template <int ACT, bool EXACT>
__device__ __forceinline__ void activation_slope(float g, float &a, float &slope)
{
    if (ACT == BRA_SILU) {
        const float f = sigmoid(g);
        a = g * f;
        slope = f + a * (1.f - f);
    } else {
        float f;
        if (EXACT) f = phi(g);
        else {
            const float x = fminf(fabsf(g), 16.0f);
            float p = fmaf(-4.732939124e-04f, x, 7.084460463e-03f);
            p = fmaf(p, x, -5.182716623e-02f);
            p = fmaf(p, x, -4.599926472e-01f);
            p = fmaf(p, x, -1.150787711e+00f);
            p = fmaf(p, x, -1.000037670e+00f);
            const float q = __builtin_amdgcn_exp2f(p);
            f = g > 0.f ? 1.f - q : q;
            f = g != g ? g : f;
        }
        a = EXACT ? gelu_exact(g, f) : g * f;
        slope = f + g * 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g);
    }
}

// The sums of tile `block` of A B [M, N] over chunks [first, last) of the contraction: A's inside, B's outside (BO) or inside.
template <class T, bool BO, int TERMS>
__device__ __forceinline__ void product_sums(const Operand &A, const Operand &Bm, long M, int N, int block, int first, int last, bf16_t *lds, f32x16 (&acc)[T::NT][T::MT])
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int mt0, nt0;
    tile_of(block, (int)((M + T::BM - 1) / T::BM), (N + T::BN - 1) / T::BN, mt0, nt0);
    const long m0 = (long)mt0 * T::BM;
    const int n0 = nt0 * T::BN, rows = (int)min((long)T::BM, M - m0), most = BO ? (N + 7) / 8 * 8 - 8 - n0 : N - 1 - n0;
    const Loads<T, T::BM, false> la(wave, lane, A.ld, [&](int row) { return (long)min(row, rows - 1); });
    const Loads<T, T::BN, BO> lb(wave, lane, Bm.ld, [&](int i) { return (long)min(i, most); });
    clear<T>(acc);
    multiply<T, false, BO, TERMS>(A, Bm, A.p + m0 * A.ld, Bm.p + n0 * (BO ? 1 : Bm.ld), la, lb, first, last, lds, acc);
}

// Tile `block` of Out = A B + bias.
template <class T, bool BO, int TERMS, typename E>
__device__ __forceinline__ void product_tile(const Operand &A, const Operand &Bm, const float *__restrict__ bias, E *__restrict__ Out, long M, int N, int block, bf16_t *lds)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int mt0, nt0;
    tile_of(block, (int)((M + T::BM - 1) / T::BM), (N + T::BN - 1) / T::BN, mt0, nt0);
    const long m0 = (long)mt0 * T::BM;
    const int n0 = nt0 * T::BN, rows = (int)min((long)T::BM, M - m0);
    f32x16 acc[T::NT][T::MT];
    product_sums<T, BO, TERMS>(A, Bm, M, N, block, 0, (A.K + 63) / 64, lds, acc);
    const int hi = lane / 32, c = lane % 32, wm = (wave / T::WC) * (32 * T::MT), wn = n0 + (wave % T::WC) * (32 * T::NT);
    const bool vec = N % 8 == 0, vec_b = (uintptr_t)bias % 16 == 0;
    const Rows<4 * T::NT> out{lds + wave * (32 * T::MT * 32 * T::NT)};
#pragma unroll
    for (int nt = 0; nt < T::NT; ++nt)
#pragma unroll
        for (int run = 0; run < 2; ++run) {
            const int piece = 4 * nt + 2 * run + hi, col = wn + 8 * piece, n = N - col;
            float b[8];
            if (bias && n > 0) load8(bias + col, b, n, vec_b);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = 0.f;
#pragma unroll
            for (int mt = 0; mt < T::MT; ++mt) {
                const int row = wm + 32 * mt + c;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[nt][mt][8 * run + e] + b[e];
                if constexpr (TERMS == 1) out.put(32 * mt + c, piece, pack8(v));
                else if (row < rows) store8(Out + (size_t)(m0 + row) * N + col, v, n, vec);
            }
        }
    if constexpr (TERMS == 1)
        out.each(32 * T::MT, lane, [&](int row, int piece, bf16x8 v) {
            if (wm + row < rows) store_piece(Out + (size_t)(m0 + wm + row) * N + wn + 8 * piece, v, N - wn - 8 * piece, vec);
        });
}

}  // namespace ffn
}  // namespace bra
