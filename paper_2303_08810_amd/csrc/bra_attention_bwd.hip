// Attention between whole sequences, backward, with the probabilities formed again from the row sums that the forward kept:
//     P = exp(S - lse),  delta = sum dO O,  dS = P (dO V^T - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
// k_query_grads has 32 rows (queries of the heads that share a key head) in the lanes of a wavefront and walks over the keys; it leaves delta.
// k_key_grads has 32 keys in the lanes of a wavefront and walks over the rows of all heads that share them.  Two more products than one kernel
// would need; every sum is formed in registers in a fixed order, so that a repeat gives the same bits.
#include "bra_attention_dev.h"

#include <algorithm>

namespace bra {
namespace att {
namespace {

template <class E, int D, int TILE, int WAVES>
struct Backward {
    typedef Geometry<E, D> G;
    static constexpr int kThreads = 64 * WAVES, kRows = 32 * WAVES;
    static constexpr int kTile = TILE * G::kPitch, kBuffer = 2 * kTile, kQueryLds = 2 * kBuffer, kKeyBuffer = kBuffer + 2 * TILE * 4, kKeyLds = 2 * kKeyBuffer;
    typedef Stage<G, TILE, kThreads> Loads;
};

template <class E, int D, int KT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, sizeof(E) == 4 && D > 64 ? 1 : 2) void k_query_grads(Call A)
{
    typedef Backward<E, D, KT, WAVES> F;
    typedef typename F::G G;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A.first + blockIdx.x, A.blocks, (long)A.tiles * A.splits);
    const int tile = A.tiles - 1 - place.inner % A.tiles, split = place.inner / A.tiles;
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d * (int)sizeof(E) / 16;

    const int first_row = tile * F::kRows, row = first_row + 32 * wave + c, some = min(row, A.rows - 1);
    const bool valid = row < A.rows;
    const int query = row_query(A, some), head = hk * A.G + some - query * A.G, limit = valid ? seq.limit(query) : 0;
    const int least = columns_min(limit), most = columns_max(limit);
    int end = 0;
    if (row_query(A, first_row) < seq.nq) end = seq.limit(min(row_query(A, min(first_row + F::kRows, A.rows) - 1), seq.nq - 1));
    const int all = (end + KT - 1) / KT, share = (all + A.splits - 1) / A.splits, from = split * share, last = min(all, from + share);

    const unsigned ring_at = lds_address(lds);
    const char *keys = A.K.p + b * A.K.batch + hk * A.K.head, *values = A.V.p + b * A.V.batch + hk * A.V.head;
    auto request = [&](int t, int buffer) {
        const int k0 = t * KT;
        const char *k = keys + k0 * A.K.token, *v = values + k0 * A.V.token;
        F::Loads::request([&](int r) { return k + r * A.K.token; }, seq.nk - k0, pieces, ring_at + buffer * F::kBuffer, threadIdx.x);
        F::Loads::request([&](int r) { return v + r * A.V.token; }, seq.nk - k0, pieces, ring_at + buffer * F::kBuffer + F::kTile, threadIdx.x);
    };
    if (from < last) request(from, 0);

    typename G::Piece x[G::kSteps], g[G::kSteps];
    load_columns<G>(A.Q.p + b * A.Q.batch + query * A.Q.token + head * A.Q.head, limit > 0, pieces, h, x);
    load_columns<G>(A.dO.p + b * A.dO.batch + query * A.dO.token + head * A.dO.head, limit > 0, pieces, h, g);
    float delta = 0.f, lse = 0.f;
    {
        typename G::Piece o[G::kSteps];
        load_columns<G>(A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head, limit > 0, pieces, h, o);
#pragma unroll
        for (int ks = 0; ks < G::kSteps; ++ks)
#pragma unroll
            for (int e = 0; e < 16 / (int)sizeof(E); ++e) delta = fmaf((float)g[ks][e], (float)o[ks][e], delta);
        delta = pair_sum(delta);
        if (limit > 0) lse = A.lse_in[((long)b * A.Hk * A.G + head) * A.Nq + query];
        lse = lse == -INFINITY ? INFINITY : lse * kLog2e;       // (no weight at all)
        if (valid && h == 0 && split == 0) {
            A.row_lse[(long)hb * A.rows + row] = lse;
            A.row_delta[(long)hb * A.rows + row] = delta;
        }
    }

    arrived<G>(x);
    arrived<G>(g);

    f32x16 acc[G::NT];
    clear(acc);
    for (int t = from, buffer = 0; t < last; ++t, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < last) request(t + 1, buffer ^ 1);
        const int k0 = t * KT;
        if (k0 >= most) continue;
        const char *kt = lds + buffer * F::kBuffer, *vt = kt + F::kTile;
        const bool masked = k0 + KT > least;
#pragma unroll
        for (int i = 0; i < KT / 32; ++i) {
            f32x16 s[2];
            clear(s);
            multiply_rows<G>(s[0], kt, 32 * i, x, lane);
            multiply_rows<G>(s[1], vt, 32 * i, g, lane);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], A.c, -lse)) * (s[1][r] - delta);
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = k0 + 32 * i + result_row(r, h) < limit ? s[0][r] : 0.f;
            }
            multiply_columns<G>(acc, kt, 32 * i, s[0], lane);
        }
    }
    if (A.splits > 1) {
        if (valid) store_columns<float, G>((char *)(A.part + (((long)hb * A.splits + split) * A.rows + row) * D), acc, A.scale, D, h);
    } else if (valid) store_columns<E, G>(A.dQ.p + b * A.dQ.batch + query * A.dQ.token + head * A.dQ.head, acc, A.scale, A.d, h);
}

template <class E, int D, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 64 || (sizeof(E) == 4 && D > 32) ? 1 : 2) void k_key_grads(Call A)
{
    typedef Backward<E, D, RT, WAVES> F;
    typedef typename F::G G;
    static_assert(RT == 64 && WAVES >= 2, "a wavefront each loads a tile's lse and delta");
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A.first + blockIdx.x, A.blocks, (long)A.tiles * A.splits);
    const int tile = place.inner % A.tiles, split = place.inner / A.tiles;      // those of a causal mask's long columns first
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d * (int)sizeof(E) / 16;

    // rows begin .. end - 1 see this lane's key
    const int first_key = tile * F::kRows, key = first_key + 32 * wave + c, end = seq.nq * A.G;
    auto begin_of = [&](int k) { return seq.causal ? min(max(k - seq.off, 0), seq.nq) * A.G : 0; };
    const bool live = key < seq.nk;
    const int begin = live ? begin_of(key) : end;
    const int wave_key = first_key + 32 * wave, least = begin_of(wave_key), most = wave_key + 31 < seq.nk ? begin_of(wave_key + 31) : end;

    typename G::Piece kx[G::kSteps], vx[G::kSteps];
    const int some = live ? key : 0;
    load_columns<G>(A.K.p + b * A.K.batch + some * A.K.token + hk * A.K.head, live, pieces, h, kx);
    load_columns<G>(A.V.p + b * A.V.batch + some * A.V.token + hk * A.V.head, live, pieces, h, vx);

    const unsigned ring_at = lds_address(lds);
    const char *queries = A.Q.p + b * A.Q.batch + hk * A.G * A.Q.head, *grads = A.dO.p + b * A.dO.batch + hk * A.G * A.dO.head;
    const float *row_lse = A.row_lse + (long)hb * A.rows, *row_delta = A.row_delta + (long)hb * A.rows;
    auto request = [&](int t, int buffer) {
        const int r0 = t * RT;
        const unsigned at = ring_at + buffer * F::kKeyBuffer;
        F::Loads::request([&](int r) { const int q = row_query(A, r0 + r); return queries + q * A.Q.token + (r0 + r - q * A.G) * A.Q.head; }, end - r0, pieces, at, threadIdx.x);
        F::Loads::request([&](int r) { const int q = row_query(A, r0 + r); return grads + q * A.dO.token + (r0 + r - q * A.G) * A.dO.head; }, end - r0, pieces, at + F::kTile,
                          threadIdx.x);
        if (wave < 2) load4_to_lds_untracked((wave ? row_delta : row_lse) + min(r0 + lane, A.rows - 1), at + F::kBuffer + 4 * RT * wave);
    };
    const int front = begin_of(first_key) / RT, all = first_key < seq.nk ? max((end + RT - 1) / RT - front, 0) : 0, share = (all + A.splits - 1) / A.splits;
    const int from = front + split * share, last = front + min(all, (split + 1) * share);
    f32x16 dk[G::NT], dv[G::NT];
    clear(dk);
    clear(dv);
    if (from < last) request(from, 0);
    arrived<G>(kx);
    arrived<G>(vx);
    for (int t = from, buffer = 0; t < last; ++t, buffer ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < last) request(t + 1, buffer ^ 1);
        const int r0 = t * RT;
        if (r0 + RT <= least || wave_key >= seq.nk) continue;
        const char *qt = lds + buffer * F::kKeyBuffer, *gt = qt + F::kTile;
        const float *ls = (const float *)(qt + F::kBuffer), *ds = ls + RT;
        const bool masked = r0 < most || r0 + RT > end;
#pragma unroll
        for (int i = 0; i < RT / 32; ++i) {
            f32x16 s[2];
            clear(s);
            multiply_rows<G>(s[0], qt, 32 * i, kx, lane);
            multiply_rows<G>(s[1], gt, 32 * i, vx, lane);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 l4 = *(const f32x4 *)(ls + 32 * i + 8 * q + 4 * h), d4 = *(const f32x4 *)(ds + 32 * i + 8 * q + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * q + e;
                    s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], A.c, -l4[e]));
                    s[1][r] = s[0][r] * (s[1][r] - d4[e]);
                }
            }
            if (masked) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = r0 + 32 * i + result_row(r, h);
                    const bool see = at >= begin && at < end;
                    s[0][r] = see ? s[0][r] : 0.f;
                    s[1][r] = see ? s[1][r] : 0.f;
                }
            }
            multiply_columns<G>(dv, gt, 32 * i, s[0], lane);
            multiply_columns<G>(dk, qt, 32 * i, s[1], lane);
        }
    }
    if (key >= A.Nk) return;
    if (A.splits > 1) {
        float *part = A.part + ((((long)hb * A.splits + split) * A.Nk + key) * 2) * D;
        store_columns<float, G>((char *)part, dk, A.scale, D, h);
        store_columns<float, G>((char *)(part + D), dv, 1.f, D, h);
    } else {
        store_columns<E, G>(A.dK.p + b * A.dK.batch + key * A.dK.token + hk * A.dK.head, dk, A.scale, A.d, h);
        store_columns<E, G>(A.dV.p + b * A.dV.batch + key * A.dV.token + hk * A.dV.head, dv, 1.f, A.d, h);
    }
}

// The splits' sums put together, in their order: dQ, [heads][splits][rows][D], or dK and dV, [heads][splits][Nk][2][D].
template <class E, int D, bool KEYS>
__global__ __launch_bounds__(256) void k_grads_join(Call A)
{
    constexpr int CH = D / 8, W = KEYS ? 2 : 1;
    const long i = (A.first + blockIdx.x) * 256 + threadIdx.x, each = KEYS ? A.Nk : A.rows, n = A.blocks * each * W;      // here blocks: sequences x key heads
    const int ch = 8 * (int)(i % CH);
    const long r = i / CH;
    if (r >= n || ch >= A.d) return;
    const int which = (int)(r % W), row = (int)(r / W % each), hb = (int)(r / W / each), b = hb / A.Hk, hk = hb % A.Hk;
    const float *p = A.part + (((long)hb * A.splits * each + row) * W + which) * D + ch;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < A.splits; ++s, p += each * W * D) {
        const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] += v0[e];
            v[4 + e] += v1[e];
        }
    }
    if (KEYS) {
        const Rows &R = which ? A.dV : A.dK;
        store8<E>(R.p + b * R.batch + row * R.token + hk * R.head + ch * sizeof(E), v);
    } else {
        const int query = row_query(A, row), head = hk * A.G + row - query * A.G;
        store8<E>(A.dQ.p + b * A.dQ.batch + query * A.dQ.token + head * A.dQ.head + ch * sizeof(E), v);
    }
}

constexpr int kWaves = 4, kRowTile = 64;
int key_tile(const Sizes &S) { return S.f32 ? 32 : 64; }

// Shares of the keys (of the rows) that workgroups walk over, where there are few of them, or a causal mask makes them of different lengths.
int splits_of(const Sizes &S, bool keys)
{
    const long mine = keys ? S.Nk : S.rows(), walked = keys ? S.rows() : S.Nk;
    const long blocks = (mine + 32 * kWaves - 1) / (32 * kWaves) * S.B * S.Hk, tiles = (walked + (keys ? kRowTile : key_tile(S)) - 1) / (keys ? kRowTile : key_tile(S));
    if (blocks == 0) return 1;
    const long want = S.causal ? 1024 : 512;
    return (int)std::max(1L, std::min({want / blocks, tiles / 4, 16L}));
}
size_t part_bytes(const Sizes &S)
{
    const size_t q = splits_of(S, false), k = splits_of(S, true), row = sizeof(float) * S.width() * S.B * S.Hk;
    return std::max(q > 1 ? q * S.rows() * row : 0, k > 1 ? k * S.Nk * 2 * row : 0);
}

template <class E, int D, bool KEYS>
int join(Call A, long heads, hipStream_t st)
{
    A.blocks = heads;
    const long blocks = (heads * (KEYS ? 2L * A.Nk : (long)A.rows) * (D / 8) + 255) / 256;
    for (A.first = 0; A.first < blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_JOIN);
        k_grads_join<E, D, KEYS><<<(unsigned)std::min(kMaxBlocks, blocks - A.first), 256, 0, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D>
int run(const Sizes &S, Call A, hipStream_t st)
{
    constexpr int KT = sizeof(E) == 4 ? 32 : 64;
    typedef Backward<E, D, KT, kWaves> FQ;
    typedef Backward<E, D, kRowTile, kWaves> FK;
    const long heads = (long)S.B * S.Hk;
    int rc = allow_lds<k_query_grads<E, D, KT, kWaves>>(FQ::kQueryLds);
    if (rc == BRA_OK) rc = allow_lds<k_key_grads<E, D, kRowTile, kWaves>>(FK::kKeyLds);
    if (rc != BRA_OK) return rc;
    A.tiles = (A.rows + FQ::kRows - 1) / FQ::kRows;
    A.splits = splits_of(S, false);
    A.blocks = A.tiles * A.splits * heads;
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_QUERY_GRADS);
        k_query_grads<E, D, KT, kWaves><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), FQ::kThreads, FQ::kQueryLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    if (A.splits > 1 && (rc = join<E, D, false>(A, heads, st)) != BRA_OK) return rc;
    A.tiles = (A.Nk + FK::kRows - 1) / FK::kRows;
    A.splits = splits_of(S, true);
    A.blocks = A.tiles * A.splits * heads;
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_KEY_GRADS);
        k_key_grads<E, D, kRowTile, kWaves><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), FK::kThreads, FK::kKeyLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return A.splits > 1 ? join<E, D, true>(A, heads, st) : BRA_OK;
}

template <class E>
int run(const Sizes &S, const Call &A, hipStream_t st)
{
    switch (S.width()) {
    case 32: return run<E, 32>(S, A, st);
    case 64: return run<E, 64>(S, A, st);
    case 96: return run<E, 96>(S, A, st);
    default: return run<E, 128>(S, A, st);
    }
}

}  // namespace
}  // namespace att

using namespace att;

size_t attention_backward_workspace_bytes(const Sizes &S) { return 2 * align256(sizeof(float) * S.rows() * S.B * S.Hk) + align256(part_bytes(S)); }

int attention_backward(const Sizes &S, const Rows &Q, const Rows &K, const Rows &V, const Rows &O, const float *lse, const Rows &dO, const Rows &dQ, const Rows &dK,
                       const Rows &dV, void *ws, hipStream_t st)
{
    Call A = make_call(S);
    A.Q = Q;
    A.K = K;
    A.V = V;
    A.O = O;
    A.dO = dO;
    A.dQ = dQ;
    A.dK = dK;
    A.dV = dV;
    A.lse_in = lse;
    A.row_lse = (float *)ws;
    A.row_delta = (float *)((char *)ws + align256(sizeof(float) * S.rows() * S.B * S.Hk));
    A.part = (float *)((char *)A.row_delta + align256(sizeof(float) * S.rows() * S.B * S.Hk));
    return S.f32 ? run<float>(S, A, st) : run<bf16_t>(S, A, st);
}

}  // namespace bra
