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

// dQ, and delta for the key side.  8192 causal tokens of 16 / 4 heads of 128: 455 us, 0.9 PFLOP/s, bound by the matrix cores (60 % of the cycles) at the 1.3 to 1.4 GHz
// that the card's power leaves them.
template <class E, int D, int WAVES>
struct Queries {
    static constexpr int T = sizeof(E) == 4 ? 3 : 1, kThreads = 64 * WAVES, kMine = 32 * WAVES, KT = T == 3 ? 32 : 64;
    typedef Geometry<bf16_t, D> G;
    static constexpr int kPlane = KT * G::kPitch, kTile = T * kPlane, kSub = 32 * G::kPitch, kLds = 4 * kTile;       // K, V, K, V
    typedef Slots<G, T, kPlane> S;
    typedef Walk<G, T, KT, kThreads> Loads;
};

template <class E, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, sizeof(E) == 4 && D > 64 ? 1 : 2) void k_query_grads(Call A)
{
    typedef Queries<E, D, WAVES> F;
    typedef typename F::G G;
    typedef typename F::S S;
    constexpr int KT = F::KT;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.tiles * A.splits);
    const int tile = A.tiles - 1 - place.inner % A.tiles, split = place.inner / A.tiles;
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d / 8;

    const int first_row = tile * F::kMine, row = first_row + 32 * wave + c, some = min(row, A.rows - 1);
    const bool valid = row < A.rows;
    const int query = row_query(A, some), head = hk * A.G + some - query * A.G, limit = valid ? seq.limit(query) : 0;
    const int least = columns_min(limit), most = columns_max(limit);
    int end = 0;
    if (row_query(A, first_row) < seq.nq) end = seq.limit(min(row_query(A, min(first_row + F::kMine, A.rows) - 1), seq.nq - 1));
    const int all = (end + KT - 1) / KT, share = (all + A.splits - 1) / A.splits, first = split * share, last = min(all, first + share);

    const unsigned at = lds_address(lds);
    typename F::Loads keys(key_source<G, F::T>(A, A.K, A.pK, b, hb, seq.nk), first * KT, threadIdx.x), values(key_source<G, F::T>(A, A.V, A.pV, b, hb, seq.nk), first * KT, threadIdx.x);
    if (first < last) {
        keys.request(at, threadIdx.x);
        values.request(at + F::kTile, threadIdx.x);
    }
    typename S::Columns x, g;
    const char *dO = A.dO.p + b * A.dO.batch + query * A.dO.token + head * A.dO.head;
    S::template load<E>(A.Q.p + b * A.Q.batch + query * A.Q.token + head * A.Q.head, limit > 0, pieces, h, x);
    S::template load<E>(dO, limit > 0, pieces, h, g);
    float delta = 0.f, lse = 0.f;
    {
        delta = row_product<E, G::kSteps>(dO, A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head, limit > 0, pieces, h);
        if (limit > 0) lse = A.lse_in[((long)b * A.Hk * A.G + head) * A.Nq + query];
        delta = pair_sum(delta);
        lse = lse == -INFINITY ? INFINITY : lse * kLog2e;       // (no weight at all)
        if (valid && h == 0 && split == 0) {
            A.row_lse[(long)hb * A.rows + row] = lse;
            A.row_delta[(long)hb * A.rows + row] = delta;
        }
    }
    S::arrived(x);
    S::arrived(g);

    const Reader<G> reader(lane);
    f32x16 acc[G::NT];
    clear(acc);
    // tile t, which lies in the buffers B
    auto body = [&](auto B, int t) __attribute__((always_inline)) {
        constexpr int kMine = decltype(B)::value * 2 * F::kTile, kOther = 2 * F::kTile - kMine;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < last) {
            keys.request(at + kOther, threadIdx.x);
            values.request(at + kOther + F::kTile, threadIdx.x);
        }
        const int k0 = t * KT;
        if (k0 >= most) return;
        const bool masked = k0 + KT > least;
        unrolled<KT / 32>([&](auto i) __attribute__((always_inline)) {
            const char *kt = lds + kMine + i * F::kSub, *vt = kt + F::kTile;
            f32x16 s{}, d{};
            unrolled<2 * S::kRows>([&](auto f) __attribute__((always_inline)) {
                if (S::kLeaves && f / 2 == S::kRows - 1 && 16 * (f / 2) >= A.d) return;
                typename S::Operand o;
                S::read_rows(o, f % 2 ? vt : kt, reader, f / 2);
                S::rows(f % 2 ? d : s, o, f % 2 ? g : x, f / 2);
            });
            if (masked) {
                if (i == 0 && k0 == 0 && limit == 1 && all_weight(s[0], A.c, lse)) {
                    // dS = 0 here; the key side, whose dO V has the same bits, subtracts it from itself
                    lse = INFINITY;
                    if (h == 0) A.row_delta[(long)hb * A.rows + row] = d[0];
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = k0 + 32 * i + result_row(r, h) < limit ? s[r] : -INFINITY;
            }
            typename S::Weights w;
            unrolled<16>([&](auto i) __attribute__((always_inline)) {
                constexpr int r = i;
                d[r] = __builtin_amdgcn_exp2f(fmaf(s[r], A.c, -lse)) * (d[r] - delta);
                if constexpr (r % 2) S::keep(w, d, r);
            });
            unrolled<S::kColumns>([&](auto f) __attribute__((always_inline)) {
                typename S::Operand o;
                S::read_columns(o, kt, reader, f);
                S::columns(acc, o, w, f);
            });
        });
    };
    for (int t = first; t < last; t += 2) {
        body(std::integral_constant<int, 0>{}, t);
        if (t + 1 < last) body(std::integral_constant<int, 1>{}, t + 1);
    }
    if (!valid) return;
    if (limit == 0) clear(acc);             // it sees nothing: zeros, also where the keys that others see are not finite
    if (A.splits > 1) store_columns<float, G>((char *)(A.part + (((long)hb * A.splits + split) * A.rows + row) * D), acc, A.scale, A.d, h);
    else store_columns<E, G>(A.dQ.p + b * A.dQ.batch + query * A.dQ.token + head * A.dQ.head, acc, A.scale, A.d, h);
}

// k_key_grads walks over subtiles of 32 rows, kRing of which are in LDS: while the weights of one are formed, the products of the one before with its
// weights are on their way, a product between every few of the other instructions; then come the products of the next one with what the wavefront keeps
// in registers.  With heads of 128 a wavefront's sums, keys and values take 224 registers: one wavefront to a SIMD, so nothing but this order hides a latency, and
// every instruction counts (matrix cores 44 % of the cycles, issue 57 %).  8192 causal tokens of 16 / 4 heads of 128: 555 us, 0.99 PFLOP/s.
template <int D, int WAVES>
struct Backward {
    typedef Geometry<bf16_t, D> G;
    typedef Slots<G, 1, 0> S;
    static constexpr int kThreads = 64 * WAVES, kMine = 32 * WAVES;
    static constexpr int kRing = 5;
    static constexpr int kTile = 32 * G::kPitch, kSlot = 2 * kTile + 256, kLds = kRing * kSlot;      // two tensors, lse and delta
    typedef Tiles<G, 32, kThreads> Loads;
};

// A wavefront's registers over the subtiles.
template <class G>
struct Pipe {
    typedef Slots<G, 1, 0> S;
    typedef typename S::Columns X;
    static constexpr int kColumns = 2 * S::kColumns, kScores = 2 * S::kRows, kAhead = kScores < 8 ? kScores : 8;
    f32x16 s[2];                                // scores and dP of a subtile
    typename S::Weights p, ds;                  // of the subtile before
    f32x16 sum[2][G::NT];                       // dV and dK
    typename S::Operand ahead[kAhead];          // the first operands of the sums of the subtile before

    // s of a subtile
    __device__ __forceinline__ void scores(const char *t0, const char *t1, const Reader<G> &R, const X &x, const X &g)
    {
        s[0] = s[1] = f32x16{};
        unrolled<kScores>([&](auto f) __attribute__((always_inline)) {
            typename S::Operand o;
            S::read_rows(o, f % 2 ? t1 : t0, R, f / 2);
            S::rows(s[f % 2], o, f % 2 ? g : x, f / 2);
        });
    }
    // one product of the sums of the subtile before, whose tiles are t0 and t1
    template <int F>
    __device__ __forceinline__ void read_column(typename S::Operand &o, const char *t0, const char *t1, const Reader<G> &R)
    {
        S::read_columns(o, F % 2 ? t0 : t1, R, F / 2);
    }
    template <int F>
    __device__ __forceinline__ void product(const typename S::Operand &o)
    {
        S::columns(sum[F % 2], o, F % 2 ? ds : p, F / 2);
    }
    __device__ __forceinline__ void sums(const char *t0, const char *t1, const Reader<G> &R)
    {
        unrolled<kColumns>([&](auto f) __attribute__((always_inline)) {
            typename S::Operand o;
            if constexpr (f < kAhead) o = ahead[f];
            else this->template read_column<f>(o, t0, t1, R);
            this->template product<f>(o);
        });
    }
    // s -> p, ds; with COLUMNS the sums of the subtile before, in b0, b1, on the way; then s of the next one, in n0, n1, of which nothing is read before
    // arrive().  weights(r): value r's -lse log2 e and delta.  Operands are read kAhead products ahead, also those of the next step, which
    // come from this subtile, in h0, h1.
    template <bool COLUMNS, class W, class Arrive>
    __device__ __forceinline__ void step(const char *b0, const char *b1, const char *h0, const char *h1, const char *n0, const char *n1, const Reader<G> &R, const X &x, const X &g, float c,
                                         W weights, Arrive arrive)
    {
        constexpr int N = COLUMNS ? kColumns : kAhead, all = N + kScores;
        typename S::Operand o[all];
        typename S::Weights np, nds;
        auto read = [&](auto f) __attribute__((always_inline)) {
            if constexpr (f >= all) this->template read_column<f - all>(ahead[f - all], h0, h1, R);
            else if constexpr (f >= N) S::read_rows(o[f], (f - N) % 2 ? n1 : n0, R, (f - N) / 2);
            else if constexpr (COLUMNS) this->template read_column<f>(o[f], b0, b1, R);
        };
        if constexpr (COLUMNS) unrolled<kAhead>([&](auto f) __attribute__((always_inline)) { o[f] = ahead[f]; });
        unrolled<N>([&](auto f) __attribute__((always_inline)) {
            if constexpr (f + kAhead == N) arrive();
            read(std::integral_constant<int, f + kAhead>{});
            if constexpr (COLUMNS) this->template product<f>(o[f]);
            unrolled<16 * (f + 1) / N - 16 * f / N>([&](auto i) __attribute__((always_inline)) {
                constexpr int r = 16 * f / N + i;
                float minus_lse, delta;
                weights(std::integral_constant<int, r>{}, minus_lse, delta);
                s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, minus_lse));
                s[1][r] = s[0][r] * (s[1][r] - delta);
                if constexpr (r % 2) {
                    S::keep(np, s[0], r);
                    S::keep(nds, s[1], r);
                    if constexpr (N > kAhead) {         // formed here, not in the block behind arrive()
                        unsigned a = np.v[0][r / 8][r % 8 / 2], b = nds.v[0][r / 8][r % 8 / 2];
                        asm volatile("" : "+v"(a), "+v"(b));
                        np.v[0][r / 8][r % 8 / 2] = a;
                        nds.v[0][r / 8][r % 8 / 2] = b;
                    }
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        p = np;
        ds = nds;
        s[0] = s[1] = f32x16{};
        unrolled<kScores>([&](auto i) __attribute__((always_inline)) {
            constexpr int f = N + i;
            read(std::integral_constant<int, f + kAhead>{});
            S::rows(s[i % 2], o[f], i % 2 ? g : x, i / 2);
            __builtin_amdgcn_sched_barrier(0);
        });
    }
};

// A workgroup's subtiles [0, n), of which this wavefront works on [from, to).  Turn j makes sure that subtile j + 1 has arrived and that nobody reads j - 2 any
// more, in whose place it asks for j + 3.  `loads`: whether this wavefront loads.
template <class F, class Scores, class Weights, class Sums, class Request>
__device__ __forceinline__ void take_turns(int n, int from, int to, bool loads, Scores scores, Weights weights, Sums sums, Request request)
{
    static_assert(F::kRing == 5, "three subtiles that are worked on, two on their way");
    if (n <= 0) return;
    // where the subtiles j - 1 .. j + 3 lie, which go round
    unsigned before = 3 * F::kSlot, here = 4 * F::kSlot, next = 0, then = F::kSlot, asked = 2 * F::kSlot;
    request(0, next);
    if (n > 1) request(1, then);
    int j = -1;
    auto turn = [&]() __attribute__((always_inline)) {
        // (fewer loads than this are on their way in the last turns: all of them are waited for)
        if (j + 2 >= n || !loads) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * F::Loads::L + 1) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (j + 3 < n) request(j + 3, asked);
    };
    auto turned = [&]() __attribute__((always_inline)) {
        const unsigned last = before;
        before = here;
        here = next;
        next = then;
        then = asked;
        asked = last;
        ++j;
    };
    // every wavefront meets the others at n + 2 barriers; what it does between them differs at its ends alone, so that its sums stay where they are
    if (from < to) {
        while (j < from - 1) {
            turn();
            turned();
        }
        turn();
        scores(next);
        turned();
        weights(std::false_type{}, j, before, here, next, turn);
        turned();
        while (j < to) {
            weights(std::true_type{}, j, before, here, next, turn);
            turned();
        }
        sums(before);
        lds_reads_done();
        turn();
        turned();
    }
    while (j <= n) {
        turn();
        turned();
    }
}

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 64 ? 1 : 2) void k_key_grads(Call A)
{
    typedef bf16_t E;
    typedef Backward<D, WAVES> F;
    typedef typename F::S S;
    typedef typename F::G G;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.tiles * A.splits);
    const int tile = place.inner % A.tiles, split = place.inner / A.tiles;      // those of a causal mask's long columns first
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d / 8;

    // rows begin .. end - 1 see this lane's key
    const int first_key = tile * F::kMine, key = first_key + 32 * wave + c, end = seq.nq * A.G;
    auto begin_of = [&](int j) { return seq.causal ? min(max(j - seq.off, 0), seq.nq) * A.G : 0; };
    const bool live = key < seq.nk;
    const int begin = live ? begin_of(key) : end;
    const int wave_key = first_key + 32 * wave, least = begin_of(wave_key), most = wave_key + 31 < seq.nk ? begin_of(wave_key + 31) : end;
    const int front = begin_of(first_key) / 32, all = first_key < seq.nk ? max((end + 31) / 32 - front, 0) : 0, share = (all + A.splits - 1) / A.splits;
    const int first = front + split * share, n = min(all, (split + 1) * share) - split * share, row0 = 32 * first;

    typename S::Columns x, g;
    const int some = live ? key : 0;
    S::template load<E>(A.K.p + b * A.K.batch + some * A.K.token + hk * A.K.head, live, pieces, h, x);
    S::template load<E>(A.V.p + b * A.V.batch + some * A.V.token + hk * A.V.head, live, pieces, h, g);
    S::arrived(x);
    S::arrived(g);

    const unsigned at = lds_address(lds);
    const char *q = A.Q.p + b * A.Q.batch + hk * A.G * A.Q.head, *o = A.dO.p + b * A.dO.batch + hk * A.G * A.dO.head;
    auto query_at = [&](int r) __attribute__((always_inline)) { const int i = row_query(A, r); return q + i * A.Q.token + (r - i * A.G) * A.Q.head; };
    auto grad_at = [&](int r) __attribute__((always_inline)) { const int i = row_query(A, r); return o + i * A.dO.token + (r - i * A.G) * A.dO.head; };
    // 32 rows on are as many heads and whole tokens on, where they are whole tokens
    const long tokens = 32 % A.G == 0 ? 32 / A.G : 0;
    typename F::Loads queries(query_at, tokens * A.Q.token, row0, end, pieces, threadIdx.x), grads(grad_at, tokens * A.dO.token, row0, end, pieces, threadIdx.x);
    const float *row_sums = (h ? A.row_delta : A.row_lse) + (long)hb * A.rows;

    const Reader<G> reader(lane);
    Pipe<G> pipe;
    clear(pipe.sum[0]);
    clear(pipe.sum[1]);
    const bool loads = wave < F::Loads::kLoaders, steady = queries.whole && queries.step && grads.step;
    take_turns<F>(
        n, max(least / 32 - first, 0), wave_key < seq.nk ? n : 0, loads,
        [&](unsigned next) __attribute__((always_inline)) { pipe.scores(lds + next, lds + next + F::kTile, reader, x, g); },
        [&](auto columns, int j, unsigned before, unsigned here, unsigned next, auto arrive) __attribute__((always_inline)) {
            // (behind the last subtile: what is there, whose scores nobody uses)
            const float *mine = (const float *)(lds + here + 2 * F::kTile) + 4 * h;
            f32x4 l[4], d[2];
            unrolled<4>([&](auto q) __attribute__((always_inline)) { l[q] = *(const f32x4 *)(mine + 8 * q); });
            d[0] = *(const f32x4 *)(mine + 32);
            // rows that do not see this lane's key have no weight: masks change these numbers, not the products' results, which would move between registers for it
            const int r0 = row0 + 32 * j;
            if (r0 < most || r0 + 32 > end) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = r0 + result_row(r, h);
                    l[r / 4][r % 4] = i >= begin && i < end ? l[r / 4][r % 4] : INFINITY;
                }
            }
            pipe.template step<decltype(columns)::value>(
                lds + before, lds + before + F::kTile, lds + here, lds + here + F::kTile, lds + next, lds + next + F::kTile, reader, x, g, A.c,
                [&](auto r, float &ml, float &dl) __attribute__((always_inline)) {
                    if constexpr (r % 4 == 0 && r < 12) d[(r / 4 + 1) % 2] = *(const f32x4 *)(mine + 2 * r + 40);
                    ml = -l[r / 4][r % 4];
                    dl = d[r / 4 % 2][r % 4];
                },
                arrive);
        },
        [&](unsigned before) __attribute__((always_inline)) { pipe.sums(lds + before, lds + before + F::kTile, reader); },
        [&](int j, unsigned to) __attribute__((always_inline)) {
            if (!loads) return;
            load4_to_lds_untracked(row_sums + min(row0 + 32 * j + c, A.rows - 1), at + to + 2 * F::kTile);
            if (steady && row0 + 32 * j + 32 <= end) {
                queries.request_whole(at + to);
                grads.request_whole(at + to + F::kTile);
            } else {
                queries.request(at + to, pieces, threadIdx.x, query_at);
                grads.request(at + to + F::kTile, pieces, threadIdx.x, grad_at);
            }
        });
    if (key >= A.Nk) return;
    if (!live) {
        clear(pipe.sum[0]);
        clear(pipe.sum[1]);
    }
    if (A.splits > 1) {
        float *part = A.part + ((((long)hb * A.splits + split) * A.Nk + key) * 2) * D;
        store_columns<float, G>((char *)part, pipe.sum[1], A.scale, A.d, h);
        store_columns<float, G>((char *)(part + D), pipe.sum[0], 1.f, A.d, h);
    } else {
        store_columns<E, G>(A.dK.p + b * A.dK.batch + key * A.dK.token + hk * A.dK.head, pipe.sum[1], A.scale, A.d, h);
        store_columns<E, G>(A.dV.p + b * A.dV.batch + key * A.dV.token + hk * A.dV.head, pipe.sum[0], 1.f, A.d, h);
    }
}

// float32: subtiles of 32 rows, the next of which is on its way.  4 x 1000 tokens of 8 heads of 64: 99 us of
// 190 for all gradients; 2 x 1295 of 8 / 2 heads of 72, causal and of different lengths, 72 of 144: matrix cores 37 %, one workgroup to a compute unit.
template <int D, int WAVES>
struct BackwardF32 {
    static constexpr int T = 3, kThreads = 64 * WAVES, kMine = 32 * WAVES;
    typedef Geometry<bf16_t, D> G;
    static constexpr int kPlane = 32 * G::kPitch, kTile = T * kPlane, kSlot = 2 * kTile + 256, kLds = 2 * kSlot;     // Q, dO, lse and delta
    typedef Slots<G, T, kPlane> S;
    typedef Walk<G, T, 32, kThreads> Loads;
};

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 32 ? 1 : 2) void k_key_grads_f32(Call A)
{
    typedef float E;
    typedef BackwardF32<D, WAVES> F;
    typedef typename F::S S;
    typedef typename F::G G;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.tiles * A.splits);
    const int tile = place.inner % A.tiles, split = place.inner / A.tiles;      // those of a causal mask's long columns first
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d / 8;

    // rows begin .. end - 1 see this lane's key
    const int first_key = tile * F::kMine, key = first_key + 32 * wave + c, end = seq.nq * A.G;
    auto begin_of = [&](int j) { return seq.causal ? min(max(j - seq.off, 0), seq.nq) * A.G : 0; };
    const bool live = key < seq.nk;
    const int begin = live ? begin_of(key) : end;
    const int wave_key = first_key + 32 * wave, least = begin_of(wave_key), most = wave_key + 31 < seq.nk ? begin_of(wave_key + 31) : end;
    const int front = begin_of(first_key) / 32, all = first_key < seq.nk ? max((end + 31) / 32 - front, 0) : 0, share = (all + A.splits - 1) / A.splits;
    const int first = front + min(all, split * share), last = front + min(all, (split + 1) * share);

    const unsigned at = lds_address(lds);
    typename F::Loads queries(row_source<G>(A, A.pQ, hb), 32 * first, threadIdx.x), grads(row_source<G>(A, A.pG, hb), 32 * first, threadIdx.x);
    const float *row_sums = (h ? A.row_delta : A.row_lse) + (long)hb * A.rows;
    auto request = [&](int t, int slot) __attribute__((always_inline)) {
        queries.request(at + slot, threadIdx.x);
        grads.request(at + slot + F::kTile, threadIdx.x);
        if (wave == 0) load4_to_lds_untracked(row_sums + min(32 * t + c, A.rows - 1), at + slot + 2 * F::kTile);
    };
    if (first < last) request(first, 0);
    typename S::Columns x, g;
    const int some = live ? key : 0;
    S::template load<E>(A.K.p + b * A.K.batch + some * A.K.token + hk * A.K.head, live, pieces, h, x);
    S::template load<E>(A.V.p + b * A.V.batch + some * A.V.token + hk * A.V.head, live, pieces, h, g);
    S::arrived(x);
    S::arrived(g);

    const Reader<G> reader(lane);
    f32x16 sum[2][G::NT];           // dV and dK
    clear(sum[0]);
    clear(sum[1]);
    auto body = [&](auto B, int t) __attribute__((always_inline)) {
        constexpr int kMine = decltype(B)::value * F::kSlot, kOther = F::kSlot - kMine;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < last) request(t + 1, kOther);
        const int r0 = 32 * t;
        if (r0 + 32 <= least || wave_key >= seq.nk) return;
        const char *qt = lds + kMine, *gt = qt + F::kTile;
        const float *ls = (const float *)(gt + F::kTile) + 4 * h;
        f32x16 s{}, d{};
        unrolled<2 * S::kRows>([&](auto f) __attribute__((always_inline)) {
            if (S::kLeaves && f / 2 == S::kRows - 1 && 16 * (f / 2) >= A.d) return;
            typename S::Operand o;
            S::read_rows(o, f % 2 ? gt : qt, reader, f / 2);
            S::template rows<true>(f % 2 ? d : s, o, f % 2 ? g : x, f / 2);
        });
        if (r0 < most || r0 + 32 > end) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = r0 + result_row(r, h);
                const bool see = i >= begin && i < end;
                s[r] = see ? s[r] : -INFINITY;
                d[r] = see ? d[r] : 0.f;
            }
        }
        typename S::Weights p, ds;
        unrolled<4>([&](auto q) __attribute__((always_inline)) {
            const f32x4 l4 = *(const f32x4 *)(ls + 8 * q), d4 = *(const f32x4 *)(ls + 32 + 8 * q);
            unrolled<4>([&](auto e) __attribute__((always_inline)) {
                constexpr int i = e, r = 4 * decltype(q)::value + i;
                s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], A.c, -l4[i]));
                d[r] = s[r] * (d[r] - d4[i]);
                if constexpr (r % 2) {
                    S::keep(p, s, r);
                    S::keep(ds, d, r);
                }
            });
        });
        unrolled<2 * S::kColumns>([&](auto f) __attribute__((always_inline)) {
            typename S::Operand o;
            S::read_columns(o, f % 2 ? qt : gt, reader, f / 2);
            S::columns(sum[f % 2], o, f % 2 ? ds : p, f / 2);
        });
    };
    for (int t = first; t < last; t += 2) {
        body(std::integral_constant<int, 0>{}, t);
        if (t + 1 < last) body(std::integral_constant<int, 1>{}, t + 1);
    }
    if (key >= A.Nk) return;
    if (!live) {
        clear(sum[0]);
        clear(sum[1]);
    }
    if (A.splits > 1) {
        float *part = A.part + ((((long)hb * A.splits + split) * A.Nk + key) * 2) * D;
        store_columns<float, G>((char *)part, sum[1], A.scale, A.d, h);
        store_columns<float, G>((char *)(part + D), sum[0], 1.f, A.d, h);
    } else {
        store_columns<E, G>(A.dK.p + b * A.dK.batch + key * A.dK.token + hk * A.dK.head, sum[1], A.scale, A.d, h);
        store_columns<E, G>(A.dV.p + b * A.dV.batch + key * A.dV.token + hk * A.dV.head, sum[0], 1.f, A.d, h);
    }
}

// Both in one launch where a head has up to R rows and R keys: everything is in LDS once, in float32 as terms formed on the way there; half of the wavefronts
// have the query side, half the key side, 32 or 64 rows (keys) each.  Bound by the chain from the loads through the products to the stores: 64 x 49 tokens of
// 16 heads of 32 12 us (float32 22), 8 x 197 of 12 heads of 64 23 us.
template <class E, int D, int R>
struct Short {
    static constexpr int T = sizeof(E) == 4 ? 3 : 1, kGroups = R / 32, kSide = kGroups < 4 ? kGroups : 4, kThreads = 128 * kSide;
    typedef Geometry<bf16_t, D> G;
    static constexpr int kPlane = R * G::kPitch, kTile = T * kPlane, kSub = 32 * G::kPitch, kLds = 4 * kTile + 2 * R * 4;        // K, V, Q, dO, lse, delta
    typedef Slots<G, T, kPlane> S;
};

template <class E, int D, int R>
__global__ __launch_bounds__((Short<E, D, R>::kThreads), D > 64 && R < 128 ? 1 : 2) void k_short_grads(Call A)
{
    typedef Short<E, D, R> F;
    typedef typename F::S S;
    typedef typename F::G G;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const int hb = (int)(A.first + blockIdx.x), b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d / 8, end = seq.nq * A.G;
    char *kt = lds, *vt = kt + F::kTile, *qt = vt + F::kTile, *gt = qt + F::kTile;
    float *sums = (float *)(gt + F::kTile);
    {
        const char *k = A.K.p + b * A.K.batch + hk * A.K.head, *v = A.V.p + b * A.V.batch + hk * A.V.head;
        const char *q = A.Q.p + b * A.Q.batch + hk * A.G * A.Q.head, *o = A.dO.p + b * A.dO.batch + hk * A.G * A.dO.head;
        load_short<E, F>(kt, seq.nk, pieces, [&](int r) __attribute__((always_inline)) { return k + r * A.K.token; });
        load_short<E, F>(vt, seq.nk, pieces, [&](int r) __attribute__((always_inline)) { return v + r * A.V.token; });
        load_short<E, F>(qt, end, pieces, [&](int r) __attribute__((always_inline)) { const int i = row_query(A, r); return q + i * A.Q.token + (r - i * A.G) * A.Q.head; });
        load_short<E, F>(gt, end, pieces, [&](int r) __attribute__((always_inline)) { const int i = row_query(A, r); return o + i * A.dO.token + (r - i * A.G) * A.dO.head; });
    }
    // lse log2 e and delta of every row: two lanes to a row
    for (int row = 32 * wave + c; row < R; row += F::kThreads / 2) {
        const int some = min(row, A.rows - 1), query = row_query(A, some), head = hk * A.G + some - query * A.G;
        const bool there = row < end;
        const float delta = pair_sum(row_product<E, G::kSteps>(A.dO.p + b * A.dO.batch + query * A.dO.token + head * A.dO.head, A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head, there, pieces, h));
        float lse = there ? A.lse_in[((long)b * A.Hk * A.G + head) * A.Nq + query] : 0.f;
        lse = lse == -INFINITY ? INFINITY : lse * kLog2e;       // (no weight at all)
        if (h == 0) {
            sums[row] = lse;
            sums[R + row] = delta;
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    const Reader<G> reader(lane);
    // a subtile's rows as what the wavefront keeps
    auto keep = [&](typename S::Columns &x, const char *tile) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < F::T; ++t)
#pragma unroll
            for (int ks = 0; ks < G::kSteps; ++ks) x.v[t][ks] = *(const bf16x8 *)(tile + t * F::kPlane + reader.row[ks]);
    };
    auto scores = [&](auto mirror, f32x16 &s, f32x16 &d, const char *t0, const char *t1, const typename S::Columns &x, const typename S::Columns &g) __attribute__((always_inline)) {
        s = d = f32x16{};
        unrolled<2 * S::kRows>([&](auto f) __attribute__((always_inline)) {
            if (S::kLeaves && f / 2 == S::kRows - 1 && 16 * (f / 2) >= A.d) return;
            typename S::Operand o;
            S::read_rows(o, f % 2 ? t1 : t0, reader, f / 2);
            S::template rows<decltype(mirror)::value>(f % 2 ? d : s, o, f % 2 ? g : x, f / 2);
        });
    };
    typename S::Columns x, g;
    f32x16 s, d;
    if (seq.nk == 1) {              // (as in k_query_grads: the key side subtracts its dO V from itself)
        for (int group = wave; wave < F::kSide && group < F::kGroups; group += F::kSide) {
            const int row = 32 * group + c, limit = row < A.rows ? seq.limit(row_query(A, row)) : 0;
            keep(x, qt + group * F::kSub);
            keep(g, gt + group * F::kSub);
            scores(std::false_type{}, s, d, kt, vt, x, g);
            if (limit == 1 && h == 0 && all_weight(s[0], A.c, sums[row])) sums[R + row] = d[0];
        }
        __syncthreads();
    }
    if (wave < F::kSide) {
        for (int group = wave;; group += F::kSide) {
            const int row = 32 * group + c, some = min(row, A.rows - 1), query = row_query(A, some), head = hk * A.G + some - query * A.G;
            if (32 * group >= A.rows) return;
            const int limit = row < A.rows ? seq.limit(query) : 0, most = columns_max(limit);
            const float delta = sums[R + row];
            float lse = sums[row];
            keep(x, qt + group * F::kSub);
            keep(g, gt + group * F::kSub);
            f32x16 acc[G::NT];
            clear(acc);
            for (int i = 0; 32 * i < most; ++i) {
                scores(std::false_type{}, s, d, kt + i * F::kSub, vt + i * F::kSub, x, g);
                if (i == 0 && limit == 1 && all_weight(s[0], A.c, lse)) lse = INFINITY;
                typename S::Weights w;
                unrolled<16>([&](auto e) __attribute__((always_inline)) {
                    constexpr int r = e;
                    const float p = 32 * i + result_row(r, h) < limit ? __builtin_amdgcn_exp2f(fmaf(s[r], A.c, -lse)) : 0.f;
                    d[r] = p * (d[r] - delta);
                    if constexpr (r % 2) S::keep(w, d, r);
                });
                unrolled<S::kColumns>([&](auto f) __attribute__((always_inline)) {
                    typename S::Operand o;
                    S::read_columns(o, kt + i * F::kSub, reader, f);
                    S::columns(acc, o, w, f);
                });
            }
            if (limit == 0) clear(acc);
            if (row < A.rows) store_columns<E, G>(A.dQ.p + b * A.dQ.batch + query * A.dQ.token + head * A.dQ.head, acc, A.scale, A.d, h);
            if (F::kGroups == F::kSide || group + F::kSide >= F::kGroups) return;
        }
    }
    for (int group = wave - F::kSide;; group += F::kSide) {
        const int key = 32 * group + c;
        if (32 * group >= A.Nk) return;
        const bool live = key < seq.nk;
        const int begin = !live ? end : seq.causal ? min(max(key - seq.off, 0), seq.nq) * A.G : 0;
        keep(x, kt + group * F::kSub);
        keep(g, vt + group * F::kSub);
        f32x16 dk[G::NT], dv[G::NT];
        clear(dk);
        clear(dv);
        for (int i = columns_min(begin) / 32; 32 * i < end; ++i) {
            scores(std::true_type{}, s, d, qt + i * F::kSub, gt + i * F::kSub, x, g);
            const float *mine = sums + 32 * i + 4 * h;
            typename S::Weights p, ds;
            unrolled<4>([&](auto q) __attribute__((always_inline)) {
                const f32x4 l4 = *(const f32x4 *)(mine + 8 * q), d4 = *(const f32x4 *)(mine + R + 8 * q);
                unrolled<4>([&](auto e) __attribute__((always_inline)) {
                    constexpr int j = e, r = 4 * decltype(q)::value + j;
                    const int at_row = 32 * i + result_row(r, h);
                    const bool see = at_row >= begin && at_row < end;
                    s[r] = see ? __builtin_amdgcn_exp2f(fmaf(s[r], A.c, -l4[j])) : 0.f;
                    d[r] = see ? s[r] * (d[r] - d4[j]) : 0.f;
                    if constexpr (r % 2) {
                        S::keep(p, s, r);
                        S::keep(ds, d, r);
                    }
                });
            });
            unrolled<2 * S::kColumns>([&](auto f) __attribute__((always_inline)) {
                typename S::Operand o;
                S::read_columns(o, (f % 2 ? qt : gt) + i * F::kSub, reader, f / 2);
                S::columns(f % 2 ? dk : dv, o, f % 2 ? ds : p, f / 2);
            });
        }
        if (!live) {
            clear(dk);
            clear(dv);
        }
        if (key < A.Nk) {
            store_columns<E, G>(A.dK.p + b * A.dK.batch + key * A.dK.token + hk * A.dK.head, dk, A.scale, A.d, h);
            store_columns<E, G>(A.dV.p + b * A.dV.batch + key * A.dV.token + hk * A.dV.head, dv, 1.f, A.d, h);
        }
        if (F::kGroups == F::kSide || group + F::kSide >= F::kGroups) return;
    }
}

// What k_grads_join puts together: dQ, [heads][splits][rows][D], and dK and dV, [heads][splits][Nk][2][D], whichever have splits.
struct Joins {
    const float *query, *key;
    int query_splits, key_splits;
    long query_pieces, key_pieces;              // of 8 channels of a result; 0 where there are no splits
};

// The splits' sums put together, in their order: memory (8192 tokens of 16 / 4 heads of 128 in two splits 14 us).
template <class E, int D>
__global__ __launch_bounds__(256) void k_grads_join(Call A, Joins J, long first)
{
    constexpr int CH = D / 8;
    long i = (first + blockIdx.x) * 256 + threadIdx.x;
    const bool keys = i >= J.query_pieces;
    if (keys) i -= J.query_pieces;
    if (keys && i >= J.key_pieces) return;
    const int ch = 8 * (int)(i % CH), splits = keys ? J.key_splits : J.query_splits, W = keys ? 2 : 1;
    if (ch >= A.d) return;
    const long r = i / CH, each = keys ? A.Nk : A.rows;
    const int which = keys ? (int)(r & 1) : 0, row = (int)((keys ? r >> 1 : r) % each), hb = (int)((keys ? r >> 1 : r) / each), b = hb / A.Hk, hk = hb % A.Hk;
    const float *p = (keys ? J.key : J.query) + (((long)hb * splits * each + row) * W + which) * D + ch;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s, p += each * W * D) {
        const f32x4 v0 = *(const f32x4 *)p, v1 = *(const f32x4 *)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] += v0[e];
            v[4 + e] += v1[e];
        }
    }
    if (keys) {
        const Rows &R = which ? A.dV : A.dK;
        store8<E>(R.p + b * R.batch + row * R.token + hk * R.head + ch * sizeof(E), v);
    } else {
        const int query = row_query(A, row), head = hk * A.G + row - query * A.G;
        store8<E>(A.dQ.p + b * A.dQ.batch + query * A.dQ.token + head * A.dQ.head + ch * sizeof(E), v);
    }
}

// Wavefronts of a workgroup, of 32 rows (keys) each.
int waves_of(long mine) { return mine <= 64 ? 2 : 4; }

// Shares of the keys (of the rows) that workgroups walk over, where there are few of them, or a causal mask makes them of different lengths.
int splits_of(const Sizes &S, bool keys)
{
    const long mine = keys ? S.Nk : S.rows(), walked = keys ? S.rows() : S.Nk;
    const long each = 32 * waves_of(mine), blocks = (mine + each - 1) / each * S.B * S.Hk, tiles = (walked + 63) / 64;
    if (blocks == 0) return 1;
    // (us with 256 / 384 / 512 / 768 / 1024 workgroups at least: causal, 8192 of 16 / 4 heads of 128 1685 / 1682 / 1146 / 1347 / 1170, 2048 of them 156 / 152 / 149 / 171 /
    // 177, 4096 of 8 heads of 64 179 / 179 / 138 / 127 / 129, 3 x 2048 of lengths from a third on of 4 / 2 heads of 128 151 / 124 / 126 / 132 / 158; not causal, 1024 of
    // 12 heads of 64 48 / 50 / 49 / 58 / 58; float32, 2 x 1295 causal of lengths from a half on of 8 / 2 heads of 72 245 / 168 / 152 / 155 / 168)
    const long want = 512;
    return (int)std::max(1L, std::min({want / blocks, tiles / 2, 16L}));
}
size_t part_bytes(const Sizes &S, bool keys)
{
    const size_t n = splits_of(S, keys), row = sizeof(float) * S.width() * S.B * S.Hk;
    return n > 1 ? align256(n * (keys ? 2 * (size_t)S.Nk : S.rows()) * row) : 0;
}

template <class E, int D>
int join(const Call &A, const Joins &J, hipStream_t st)
{
    const long blocks = (J.query_pieces + J.key_pieces + 255) / 256;
    for (long first = 0; first < blocks; first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_JOIN);
        k_grads_join<E, D><<<(unsigned)std::min(kMaxBlocks, blocks - first), 256, 0, st>>>(A, J, first);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D, int WAVES>
int query_grads(const Sizes &S, Call A, long heads, hipStream_t st)
{
    typedef Queries<E, D, WAVES> F;
    const int rc = allow_lds<k_query_grads<E, D, WAVES>>(F::kLds);
    if (rc != BRA_OK) return rc;
    set_grid(A, heads, (A.rows + F::kMine - 1) / F::kMine, splits_of(S, false));
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_QUERY_GRADS);
        k_query_grads<E, D, WAVES><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D, int WAVES>
int key_grads(const Sizes &S, Call A, long heads, hipStream_t st)
{
    constexpr bool f32 = sizeof(E) == 4;
    typedef typename std::conditional<f32, BackwardF32<D, WAVES>, Backward<D, WAVES>>::type F;
    int rc;
    if constexpr (f32) rc = allow_lds<k_key_grads_f32<D, WAVES>>(F::kLds);
    else rc = allow_lds<k_key_grads<D, WAVES>>(F::kLds);
    if (rc != BRA_OK) return rc;
    set_grid(A, heads, (A.Nk + F::kMine - 1) / F::kMine, splits_of(S, true));
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_KEY_GRADS);
        const unsigned n = (unsigned)std::min(kMaxBlocks, A.blocks - A.first);
        if constexpr (f32) k_key_grads_f32<D, WAVES><<<n, F::kThreads, F::kLds, st>>>(A);
        else k_key_grads<D, WAVES><<<n, F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

// Rows and keys that a call of k_short_grads takes, 0 where it is not the one.
int short_side(const Sizes &S)
{
    const long most = std::max(S.rows(), (long)S.Nk);
    const int fits = S.f32 ? (S.width() <= 32 ? 128 : S.width() <= 64 ? 64 : 32) : S.width() <= 64 ? 256 : 128;      // in LDS
    for (int side = 32; side <= fits; side *= 2)
        if (most <= side) return S.f32 || side >= 64 ? side : 64;
    return 0;
}

template <class E, int D, int R>
int short_grads(Call A, long heads, hipStream_t st)
{
    typedef Short<E, D, R> F;
    const int rc = allow_lds<k_short_grads<E, D, R>>(F::kLds);
    if (rc != BRA_OK) return rc;
    for (A.first = 0; A.first < heads; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_SHORT_GRADS);
        k_short_grads<E, D, R><<<(unsigned)std::min(kMaxBlocks, heads - A.first), F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D>
int run(const Sizes &S, const Call &A, hipStream_t st)
{
    const long heads = (long)S.B * S.Hk;
    constexpr bool f32 = sizeof(E) == 4;
    switch (short_side(S)) {
    case 32:
        if constexpr (f32) return short_grads<E, D, 32>(A, heads, st);
        break;
    case 64:
        if constexpr (!f32 || D <= 64) return short_grads<E, D, 64>(A, heads, st);
        break;
    case 128:
        if constexpr (!f32 || D <= 32) return short_grads<E, D, 128>(A, heads, st);
        break;
    case 256:
        if constexpr (!f32 && D <= 64) return short_grads<E, D, 256>(A, heads, st);
        break;
    }
    Call Q = A, K = A;
    K.part = A.part + part_bytes(S, false) / sizeof(float);
    int rc = waves_of(S.rows()) == 2 ? query_grads<E, D, 2>(S, Q, heads, st) : query_grads<E, D, 4>(S, Q, heads, st);
    if (rc == BRA_OK) rc = waves_of(S.Nk) == 2 ? key_grads<E, D, 2>(S, K, heads, st) : key_grads<E, D, 4>(S, K, heads, st);
    if (rc != BRA_OK) return rc;
    Joins J{Q.part, K.part, splits_of(S, false), splits_of(S, true), 0, 0};
    if (J.query_splits > 1) J.query_pieces = heads * A.rows * (D / 8);
    if (J.key_splits > 1) J.key_pieces = heads * A.Nk * 2 * (D / 8);
    return join<E, D>(A, J, st);
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

size_t attention_backward_workspace_bytes(const Sizes &S) { return short_side(S) ? 0 : 2 * align256(sizeof(float) * S.rows() * S.B * S.Hk) + part_bytes(S, false) + part_bytes(S, true) + (S.f32 ? terms_bytes(S, true) : 0); }

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
    if (S.f32 && !short_side(S)) {
        const int rc = make_terms(S, A, true, (char *)A.part + part_bytes(S, false) + part_bytes(S, true), st);
        if (rc != BRA_OK) return rc;
    }
    return S.f32 ? run<float>(S, A, st) : run<bf16_t>(S, A, st);
}

}  // namespace bra
