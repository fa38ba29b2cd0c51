// Attention between whole sequences, forward:
//     S = scale Q K^T, P = exp(S - max) masked, O = P V / sum P, lse = max + log sum P
// in one pass over keys and values with the running maximum and sum of each query.  A wavefront has 32 rows (queries of the heads that share
// a key head) in its lanes; tiles of keys and values come to LDS by direct loads while the tile before is worked on.  Few rows: the
// wavefronts of a workgroup have the same rows and share the keys out.  Where workgroups are few, the keys are shared out to several, whose sums
// k_attention_join puts together.
#include "bra_attention_dev.h"

#include <algorithm>

namespace bra {
namespace att {
namespace {

// Few rows, as when a token is added to a sequence: up to 32 rows of a key head in the lanes, tiles of 32 keys, each wavefront with its own share and its own ring of two
// tiles.  Bound by reading keys and values: 8 caches of 32768 keys of 8 heads of 128, 4 query heads each, 188 us, 5.7 TB/s (6.3 is what the card
// reads); lengths from an eighth on 118, 5.3 TB/s in this kernel.  Workgroups dealt out to the sequences by length read no faster (113 us for 115), and working out
// whose share it is cost 3 to 4 us of the short ones.  One sequence of 197 keys of 12 heads of 64: 6 us, a launch and two round trips to memory.
template <class E, int D, int WAVES>
struct Few {
    typedef Geometry<E, D> G;
    static constexpr int KT = 32, kThreads = 64 * WAVES, kRows = 32;
    static constexpr int kTile = KT * G::kPitch, kBuffer = 2 * kTile, kRings = 2 * kBuffer * WAVES;
    static constexpr int kColumn = D + 4;       // floats of a column's sums: the lanes of a wavefront begin in different banks
    static constexpr int kJoin = WAVES * 32 * (kColumn + 2) * 4;
    static constexpr int kLds = kRings > kJoin ? kRings : kJoin;
    typedef Stage<G, KT, 64> Loads;
};

// O (or its share before the division) and the statistics of one row.
template <class E, class G>
__device__ __forceinline__ void finish(const Call &A, int b, int hk, int split, int row, int h, f32x16 (&acc)[G::NT], float m, float l)
{
    if (l == 0.f) clear(acc);               // no weight: zeros, also where the values that others see are not finite
    const int query = row_query(A, row), head = hk * A.G + row - query * A.G;
    if (A.splits > 1) {
        const long at = ((long)(b * A.Hk + hk) * A.splits + split) * A.rows + row;
        store_columns<float, G>((char *)(A.part + at * G::D), acc, 1.f, A.d, h);
        if (h == 0) {
            A.part_ml[2 * at] = m;
            A.part_ml[2 * at + 1] = l;
        }
        return;
    }
    store_columns<E, G>(A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head, acc, l == 0.f ? 0.f : 1.f / l, A.d, h);
    if (A.lse && h == 0) A.lse[((long)b * A.Hk * A.G + head) * A.Nq + query] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <class E, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 64 ? 1 : 2) void k_attention_few(Call A)
{
    typedef Few<E, D, WAVES> F;
    typedef typename F::G G;
    constexpr int KT = F::KT;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.splits);
    const int split = place.inner, hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int pieces = A.d * (int)sizeof(E) / 16;

    const int row = c;
    const bool valid = row < A.rows;
    const int query = row_query(A, min(row, A.rows - 1)), limit = valid ? seq.limit(query) : 0, least = columns_min(limit);
    // keys that any row sees
    const int end = columns_max(limit), all = (end + KT - 1) / KT, share = (all + A.splits - 1) / A.splits, last = min(all, (split + 1) * share);

    typename G::Piece x[G::kSteps];
    {
        const int head = hk * A.G + min(row, A.rows - 1) - query * A.G;
        load_columns<G>(A.Q.p + b * A.Q.batch + query * A.Q.token + head * A.Q.head, limit > 0, pieces, h, x);
    }
    const char *keys = A.K.p + b * A.K.batch + hk * A.K.head, *values = A.V.p + b * A.V.batch + hk * A.V.head;
    char *ring = lds + wave * 2 * F::kBuffer;
    const unsigned ring_at = lds_address(ring);
    auto request = [&](bool value, int t, int buffer) {
        const long token = value ? A.V.token : A.K.token;
        const int k0 = t * KT;
        const char *from = (value ? values : keys) + k0 * token;
        F::Loads::request([&](int r) { return from + r * token; }, seq.nk - k0, pieces, ring_at + buffer * F::kBuffer + (value ? F::kTile : 0), lane);
    };

    f32x16 acc[G::NT];
    clear(acc);
    Running run(limit > 0);
    // Each wavefront for itself, two tiles ahead: keys (values) are asked for as soon as those two tiles before them have been read (8 caches of up to 32768
    // keys of 8 heads of 128 one tile ahead 126 us, two 122).
    constexpr int L = F::Loads::L;
    int t = split * share + wave;
    for (int n = 0; n < 2; ++n)
        if (t + n * WAVES < last) {
            request(false, t + n * WAVES, n);
            request(true, t + n * WAVES, n);
        }
    arrived<G>(x);
    for (int buffer = 0; t < last; t += WAVES, buffer ^= 1) {
        const bool one = t + WAVES < last, two = t + 2 * WAVES < last;
        const char *kt = ring + buffer * F::kBuffer, *vt = kt + F::kTile;
        const int k0 = t * KT;
        if (one) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * L) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" : : "n"(L) : "memory");
        f32x16 s{};
        multiply_rows<G>(s, kt, 0, x, lane);
        if (k0 + KT > least) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = k0 + result_row(r, h) < limit ? s[r] : -INFINITY;
        }
        lds_reads_done();
        if (two) request(false, t + 2 * WAVES, buffer);
        run.weights(s, A.c, acc);
        if (two) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * L) : "memory");
        else if (one) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * L) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        multiply_columns<G>(acc, vt, 0, s, lane);
        lds_reads_done();
        if (two) request(true, t + 2 * WAVES, buffer);
    }

    // the wavefronts' shares: [wave][column][kColumn] sums, then [wave][column] m and l; every wavefront puts some of the channels together
    const float share_l = pair_sum(run.l);
    float *sums = (float *)lds, *ml = sums + WAVES * 32 * F::kColumn;
    __syncthreads();
    if (limit > 0) store_columns<float, G>((char *)(sums + (wave * 32 + c) * F::kColumn), acc, 1.f, D, h);
    if (h == 0) {
        ml[2 * (32 * wave + c)] = run.m;
        ml[2 * (32 * wave + c) + 1] = share_l;
    }
    __syncthreads();
    if (!valid) return;
    float m = -INFINITY, l = 0.f, factor[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[2 * (32 * w + c)]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float mw = ml[2 * (32 * w + c)];
        factor[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - m);
        l = fmaf(factor[w], ml[2 * (32 * w + c) + 1], l);
    }
    const int head = hk * A.G + row - query * A.G;
    const long at = (long)(hb * (long)A.splits + split) * A.rows + row;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int piece = 2 * wave + h; piece < D / 8; piece += 2 * WAVES) {
        if (8 * piece >= A.d) break;
        float v[8] = {};
        if (l != 0.f)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float *from = sums + (w * 32 + c) * F::kColumn + 8 * piece;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(factor[w], from[e], v[e]);
            }
        if (A.splits > 1) store8<float>((char *)(A.part + at * D + 8 * piece), v);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= inv;
            store8<E>(A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head + 8 * piece * (int)sizeof(E), v);
        }
    }
    if (wave || h) return;
    if (A.splits > 1) {
        A.part_ml[2 * at] = m;
        A.part_ml[2 * at + 1] = l;
    } else if (A.lse) A.lse[((long)b * A.Hk * A.G + head) * A.Nq + query] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Many rows: the wavefronts of a workgroup have 32 rows each and share tiles of KT keys and values, the next of which is on its way.  Heads of 128 are bound by
// the matrix cores at the clock that the card's power leaves them (1.8 GHz): 8192 causal tokens of 32 / 8 heads 520 to 555 us, 0.99 to 1.06 PFLOP/s by the card, where a large
// product of the library reaches 1.15.  Heads of 64 by the vector instructions, 16 exponentials of 16 cycles and 40 others of 4 to 256 cycles of products:
// 32 x 1024 tokens of 12 heads 130 us, 2 x 8192 of 16 heads 563 us, 0.98 PFLOP/s.  float32: six products for one, 8 x 1000 of 8 heads of 64 98 us with the
// terms, 168 TFLOP/s (the float32 instruction has 154 at most).
template <class E, int D, int WAVES>
struct Main {
    static constexpr int T = sizeof(E) == 4 ? 3 : 1, kThreads = 64 * WAVES, kRows = 32 * WAVES, KT = T == 3 ? 32 : 64;
    typedef Geometry<bf16_t, D> G;
    static constexpr int kPlane = KT * G::kPitch, kTile = T * kPlane, kSub = 32 * G::kPitch, kLds = 4 * kTile;       // K, V, K, V
    typedef Slots<G, T, kPlane> S;
    typedef Walk<G, T, KT, kThreads> Loads;
};

template <class E, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, sizeof(E) == 4 && D > 64 ? 1 : sizeof(E) == 2 && D <= 64 ? 3 : 2) void k_attention_rows(Call A)
{
    typedef Main<E, D, WAVES> F;
    typedef typename F::G G;
    typedef typename F::S S;
    constexpr int KT = F::KT;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.tiles * A.splits);
    const int tile = A.tiles - 1 - place.inner % A.tiles, split = place.inner / A.tiles;     // those of a causal mask's long rows first
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);

    const int first_row = tile * F::kRows, row = first_row + 32 * wave + c;
    const bool valid = row < A.rows;
    const int query = row_query(A, min(row, A.rows - 1)), limit = valid ? seq.limit(query) : 0;
    const int least = columns_min(limit), most = columns_max(limit);
    // keys that any row of the workgroup sees
    int end = 0;
    if (row_query(A, first_row) < seq.nq) end = seq.limit(min(row_query(A, min(first_row + F::kRows, A.rows) - 1), seq.nq - 1));
    const int all = (end + KT - 1) / KT, share = (all + A.splits - 1) / A.splits, first = split * share, last = min(all, first + share);

    const unsigned at = lds_address(lds);
    typename F::Loads keys(key_source<G, F::T>(A, A.K, A.pK, b, hb, seq.nk), first * KT, threadIdx.x), values(key_source<G, F::T>(A, A.V, A.pV, b, hb, seq.nk), first * KT, threadIdx.x);
    typename S::Columns x;
    {
        const int head = hk * A.G + min(row, A.rows - 1) - query * A.G;
        S::template load<E>(A.Q.p + b * A.Q.batch + query * A.Q.token + head * A.Q.head, limit > 0, A.d / 8, h, x);
    }
    if (first < last) {
        keys.request(at, threadIdx.x);
        values.request(at + F::kTile, threadIdx.x);
    }
    S::arrived(x);

    const Reader<G> reader(lane);
    f32x16 acc[G::NT];
    clear(acc);
    Running run(limit > 0);
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
        f32x16 s[KT / 32];
        unrolled<KT / 32>([&](auto i) __attribute__((always_inline)) {
            s[i] = f32x16{};
            unrolled<S::kRows>([&](auto f) __attribute__((always_inline)) {
                if (S::kLeaves && f == S::kRows - 1 && 16 * f >= A.d) return;
                typename S::Operand o;
                S::read_rows(o, lds + kMine + i * F::kSub, reader, f);
                S::rows(s[i], o, x, f);
            });
        });
        if (k0 + KT > least) {
#pragma unroll
            for (int i = 0; i < KT / 32; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[i][r] = k0 + 32 * i + result_row(r, h) < limit ? s[i][r] : -INFINITY;
        }
        unrolled<KT / 32>([&](auto i) __attribute__((always_inline)) {
            run.weights(s[i], A.c, acc);
            typename S::Weights p;
            unrolled<8>([&](auto r) __attribute__((always_inline)) { S::keep(p, s[i], 2 * r + 1); });
            unrolled<S::kColumns>([&](auto f) __attribute__((always_inline)) {
                typename S::Operand o;
                S::read_columns(o, lds + kMine + F::kTile + i * F::kSub, reader, f);
                S::columns(acc, o, p, f);
            });
        });
    };
    for (int t = first; t < last; t += 2) {
        body(std::integral_constant<int, 0>{}, t);
        if (t + 1 < last) body(std::integral_constant<int, 1>{}, t + 1);
    }
    if (valid) finish<E, G>(A, b, hk, split, row, h, acc, run.m, pair_sum(run.l));
}

// float32 and up to R keys, which lie in LDS at once as terms that are formed on the way there: no planes of terms in memory, no launch for them (8 x 100 tokens of 8
// heads of 64 15.8 -> 10.8 us).
template <int D, int R, int WAVES>
struct ShortKeys {
    static constexpr int T = 3, kThreads = 64 * WAVES, kRows = 32 * WAVES;
    typedef Geometry<bf16_t, D> G;
    static constexpr int kPlane = R * G::kPitch, kTile = T * kPlane, kSub = 32 * G::kPitch, kLds = 2 * kTile;
    typedef Slots<G, T, kPlane> S;
};

template <int D, int R, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 64 ? 1 : 2) void k_attention_short_f32(Call A)
{
    typedef float E;
    typedef ShortKeys<D, R, WAVES> F;
    typedef typename F::G G;
    typedef typename F::S S;
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 32, c = lane % 32;
    const Place place(A, A.first + blockIdx.x, A.tiles);
    const int hb = place.head, b = hb / A.Hk, hk = hb % A.Hk;
    const Sequence seq(A, b);
    const int row = place.inner * F::kRows + 32 * wave + c;
    const bool valid = row < A.rows;
    const int query = row_query(A, min(row, A.rows - 1)), head = hk * A.G + min(row, A.rows - 1) - query * A.G, limit = valid ? seq.limit(query) : 0, pieces = A.d / 8;
    char *kt = lds, *vt = kt + F::kTile;
    {
        const char *k = A.K.p + b * A.K.batch + hk * A.K.head, *v = A.V.p + b * A.V.batch + hk * A.V.head;
        load_short<E, F>(kt, seq.nk, pieces, [&](int r) __attribute__((always_inline)) { return k + r * A.K.token; });
        load_short<E, F>(vt, seq.nk, pieces, [&](int r) __attribute__((always_inline)) { return v + r * A.V.token; });
    }
    typename S::Columns x;
    S::template load<E>(A.Q.p + b * A.Q.batch + query * A.Q.token + head * A.Q.head, limit > 0, pieces, h, x);
    __syncthreads();

    const Reader<G> reader(lane);
    const int most = columns_max(limit);
    f32x16 acc[G::NT];
    clear(acc);
    Running run(limit > 0);
    for (int i = 0; 32 * i < most; ++i) {
        f32x16 s{};
        unrolled<S::kRows>([&](auto f) __attribute__((always_inline)) {
            if (S::kLeaves && f == S::kRows - 1 && 16 * f >= A.d) return;
            typename S::Operand o;
            S::read_rows(o, kt + i * F::kSub, reader, f);
            S::rows(s, o, x, f);
        });
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 32 * i + result_row(r, h) < limit ? s[r] : -INFINITY;
        run.weights(s, A.c, acc);
        typename S::Weights p;
        unrolled<8>([&](auto r) __attribute__((always_inline)) { S::keep(p, s, 2 * r + 1); });
        unrolled<S::kColumns>([&](auto f) __attribute__((always_inline)) {
            typename S::Operand o;
            S::read_columns(o, vt + i * F::kSub, reader, f);
            S::columns(acc, o, p, f);
        });
    }
    if (valid) finish<E, G>(A, b, hk, 0, row, h, acc, run.m, pair_sum(run.l));
}

// What a thread of k_attention_join has: 8 channels from ch on of row `slot` of a workgroup's, every groups-th split from `group` on.  Pieces and groups that do not divide 256
// leave threads over, which have no row; the first group takes the others' sums from LDS rows thread + CH, thread + 2 CH ...
struct JoinPlace {
    int per, ch, group, slot;
    constexpr JoinPlace(int thread, int CH, int groups) : per(256 / (CH * groups)), ch(8 * (thread % CH)), group(thread / CH % groups), slot(thread / (CH * groups)) {}
    constexpr bool has_row() const { return slot < per; }
};
constexpr bool join_stays_in_lds(int CH)
{
    for (int groups = 1; CH * groups <= 256; groups *= 2)
        for (int t = 0; t < 256; ++t) {
            const JoinPlace P(t, CH, groups);
            if (P.has_row() && P.group == 0 && t + (groups - 1) * CH >= 256) return false;
        }
    return true;
}

// The splits' sums put together.  A thread has 8 channels of a row and every `groups`-th of its splits (one after another they took 26 us for
// 32 splits of 256 rows, this way 6); the groups meet in LDS.
template <class E, int D>
__global__ __launch_bounds__(256) void k_attention_join(Call A, int groups)
{
    constexpr int CH = D / 8;
    __shared__ float lds[256][11];
    static_assert(join_stays_in_lds(CH), "rows of lds");
    const JoinPlace P(threadIdx.x, CH, groups);
    const int ch = P.ch, group = P.group;
    const long r = (A.first + blockIdx.x) * P.per + P.slot, rows = A.blocks * A.rows;           // here blocks: sequences x key heads
    const bool valid = P.has_row() && r < rows;
    const int row = valid ? (int)(r % A.rows) : 0, hb = valid ? (int)(r / A.rows) : 0, b = hb / A.Hk, hk = hb % A.Hk;
    const long at = (long)hb * A.splits * A.rows + row;
    float top = -INFINITY, l = 0.f, o[8] = {};
    auto add = [&](float m, float sum, const float (&v)[8]) {
        const float next = fmaxf(top, m), old = next == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next), factor = next == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - next);
        top = next;
        l = fmaf(factor, sum, l * old);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(factor, v[e], o[e] * old);
    };
    if (valid && ch < A.d)
#pragma unroll 4
        for (int s = group; s < A.splits; s += groups) {
            const long p = at + (long)s * A.rows;
            if (A.part_ml[2 * p + 1] == 0.f) continue;          // (not the maximum: sums that are NaN have none)
            const f32x4 v0 = *(const f32x4 *)(A.part + p * D + ch), v1 = *(const f32x4 *)(A.part + p * D + ch + 4);
            const f32x2 ml = *(const f32x2 *)(A.part_ml + 2 * p);
            const float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            add(ml[0], ml[1], v);
        }
    if (groups > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) lds[threadIdx.x][e] = o[e];
        lds[threadIdx.x][8] = top;
        lds[threadIdx.x][9] = l;
        __syncthreads();
        if (group || !valid) return;        // (threads without a row have none in lds behind them either)
        for (int g = 1; g < groups; ++g) {
            const float *from = lds[threadIdx.x + g * CH];
            const float v[8] = {from[0], from[1], from[2], from[3], from[4], from[5], from[6], from[7]};
            add(from[8], from[9], v);
        }
    }
    if (!valid) return;
    const int query = row_query(A, row), head = hk * A.G + row - query * A.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= inv;
    if (ch < A.d) store8<E>(A.O.p + b * A.O.batch + query * A.O.token + head * A.O.head + ch * sizeof(E), o);
    if (A.lse && ch == 0) A.lse[((long)b * A.Hk * A.G + head) * A.Nq + query] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

bool few(const Sizes &S) { return S.rows() <= 32; }
int key_tile(const Sizes &S) { return few(S) || S.f32 ? 32 : 64; }
int waves(const Sizes &S) { return few(S) ? (S.f32 && S.width() > 64 ? 2 : 4) : S.rows() <= 64 ? 2 : 4; }
long row_tiles(const Sizes &S)
{
    const int rows = few(S) ? 32 : 32 * waves(S);
    return (S.rows() + rows - 1) / rows;
}
// Keys that k_attention_short_f32 has in LDS, 0 where it is not the one.
int short_keys(const Sizes &S)
{
    const int fits = S.width() <= 32 ? 256 : S.width() <= 64 ? 128 : 64;
    return !S.f32 || few(S) || S.Nk > fits ? 0 : S.Nk > fits / 2 || fits == 64 ? fits : fits / 2;
}
int splits_of(const Sizes &S)
{
    if (short_keys(S)) return 1;
    const long blocks = row_tiles(S) * S.B * S.Hk, tiles = (S.Nk + key_tile(S) - 1) / key_tile(S);
    if (blocks == 0) return 1;
    // A split is worth its join (5 us and more) where enough tiles are left to it (us without / with: 1024 tokens of 12 heads of 64 16.7 / 17.8, 2 x 512 of 8
    // heads 13.0 / 15.1; 2048 causal of 16 / 4 heads of 128 46.8 / 44.5; float32 3 x 667 of 6 heads of 40 37.7 / 30.4).
    // Workgroups at least (single tokens, us with 512 / 1024 / 2048: 8 caches of up to 32768 keys of 8 heads of 128 119 / 119 / 134, 4 of up to 16384 46 / 54 / 75, 32 of
    // up to 4096 69 / 66 / 84, float32, 4 of 8192 of 12 heads of 64 62 / 78 / 83).
    const long want = 512, least = few(S) ? 2 * waves(S) : S.f32 ? 5 : 12;
    return (int)std::max(1L, std::min({want / blocks, tiles / least, 64L}));
}

template <class E, int D, int WAVES>
int launch_few(Call A, hipStream_t st)
{
    typedef Few<E, D, WAVES> F;
    const int rc = allow_lds<k_attention_few<E, D, WAVES>>(F::kLds);
    if (rc != BRA_OK) return rc;
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION);
        k_attention_few<E, D, WAVES><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D, int WAVES>
int launch_rows(Call A, hipStream_t st)
{
    typedef Main<E, D, WAVES> F;
    const int rc = allow_lds<k_attention_rows<E, D, WAVES>>(F::kLds);
    if (rc != BRA_OK) return rc;
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION);
        k_attention_rows<E, D, WAVES><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D>
int join(Call A, long heads, hipStream_t st)
{
    constexpr int CH = D / 8;
    A.blocks = heads;
    int groups = 1;
    while (2 * groups * CH <= 256 && 2 * groups <= A.splits) groups *= 2;
    const long per = 256 / (CH * groups), blocks = (heads * A.rows + per - 1) / per;
    for (A.first = 0; A.first < blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION_JOIN);
        k_attention_join<E, D><<<(unsigned)std::min(kMaxBlocks, blocks - A.first), 256, 0, st>>>(A, groups);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <int D, int R, int WAVES>
int launch_short(Call A, hipStream_t st)
{
    typedef ShortKeys<D, R, WAVES> F;
    const int rc = allow_lds<k_attention_short_f32<D, R, WAVES>>(F::kLds);
    if (rc != BRA_OK) return rc;
    for (A.first = 0; A.first < A.blocks; A.first += kMaxBlocks) {
        const ProfScope scope(st, K_ATTENTION);
        k_attention_short_f32<D, R, WAVES><<<(unsigned)std::min(kMaxBlocks, A.blocks - A.first), F::kThreads, F::kLds, st>>>(A);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
    }
    return BRA_OK;
}

template <class E, int D>
int run(const Sizes &S, const Call &A, hipStream_t st)
{
    constexpr bool f32 = sizeof(E) == 4;
    constexpr int kFits = D <= 32 ? 256 : D <= 64 ? 128 : 64;
    int rc;
    if constexpr (f32) {
        const int keys = short_keys(S);
        if (keys == kFits) return waves(S) == 2 ? launch_short<D, kFits, 2>(A, st) : launch_short<D, kFits, 4>(A, st);
        if constexpr (D <= 64) {
            if (keys) return waves(S) == 2 ? launch_short<D, kFits / 2, 2>(A, st) : launch_short<D, kFits / 2, 4>(A, st);
        }
    }
    if (few(S)) rc = launch_few<E, D, (f32 && D > 64 ? 2 : 4)>(A, st);
    else rc = waves(S) == 2 ? launch_rows<E, D, 2>(A, st) : launch_rows<E, D, 4>(A, st);
    if (rc == BRA_OK && A.splits > 1) rc = join<E, D>(A, (long)S.B * S.Hk, st);
    return rc;
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

Call make_call(const Sizes &S)
{
    Call A{};
    A.q_lens = S.q_lens;
    A.k_lens = S.k_lens;
    A.Nq = S.Nq;
    A.Nk = S.Nk;
    A.G = S.group();
    A.Hk = S.Hk;
    A.d = S.d;
    A.magic = A.G > 1 ? (unsigned)((1ull << 32) / A.G + 1) : 0;
    A.rows = (int)S.rows();
    A.causal = S.causal;
    A.scale = S.scale;
    A.c = S.scale * kLog2e;
    A.splits = 1;
    return A;
}

}  // namespace att

using namespace att;

size_t attention_workspace_bytes(const Sizes &S)
{
    const long splits = splits_of(S), rows = S.rows() * S.B * S.Hk;
    return (S.f32 && !few(S) && !short_keys(S) ? terms_bytes(S, false) : 0) + (splits > 1 ? align256(sizeof(float) * splits * rows * S.width()) + align256(2 * sizeof(float) * splits * rows) : 0);
}

int attention_forward(const Sizes &S, const Rows &Q, const Rows &K, const Rows &V, const Rows &O, float *lse, void *ws, hipStream_t st)
{
    Call A = make_call(S);
    A.Q = Q;
    A.K = K;
    A.V = V;
    A.O = O;
    A.lse = lse;
    set_grid(A, (long)S.B * S.Hk, row_tiles(S), splits_of(S));
    if (S.f32 && !few(S) && !short_keys(S)) {
        const int rc = make_terms(S, A, false, ws, st);
        if (rc != BRA_OK) return rc;
        ws = (char *)ws + terms_bytes(S, false);
    }
    if (A.splits > 1) {
        A.part = (float *)ws;
        A.part_ml = (float *)((char *)ws + align256(sizeof(float) * A.splits * S.rows() * S.B * S.Hk * S.width()));
    }
    return S.f32 ? run<float>(S, A, st) : run<bf16_t>(S, A, st);
}

}  // namespace bra
