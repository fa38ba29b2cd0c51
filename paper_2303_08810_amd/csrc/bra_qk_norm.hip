// Norms of queries and keys for each head, and the rotation of their channels by position, in one pass over both:
//     u = x / sqrt(mean of squares + eps) gamma,   (a, b) -> (a cos - b sin, b cos + a sin) for each pair of the first `turned` channels
// and backwards g = R^T dy, dgamma = sum g x / rms, dx = (g gamma - x / rms mean(g gamma x / rms)) / rms.
// A team of lanes has a row (a head of a token) in registers, each lane two chunks of V channels that hold whole pairs, and works on RPT heads
// of a token, which share the angles.  A workgroup has queries or keys alone: one gamma and one set of its gradient's sums.  Bound by memory.
#include "bra_mfma_dev.h"
#include "bra_qk_norm.h"

#include <algorithm>

namespace bra {

using namespace mfma;

namespace {

constexpr int kThreads = 256;

// Queries or keys.
struct Part {
    att::Rows x, g, o;          // what goes in, what comes back (backward), what is written
    const float *gamma;         // or NULL: no norm
    unsigned groups, items;     // a token's heads go to `groups` teams; tokens x groups
    int heads;
};

struct Work {
    Part part[2];
    const float *cos, *sin;
    const int *positions;
    unsigned N;
    int d, turned, table_rows, team;
    float eps, d_inv;
    bool halves;
    unsigned query_blocks;      // workgroups of the queries, the others are the keys'
    float *sums;                // [workgroups][d]
};

template <class E, int V>
__device__ __forceinline__ void load(const char *p, float (&x)[V])
{
    if constexpr (sizeof(E) == 4) {
        typedef float vec __attribute__((ext_vector_type(V)));
        if constexpr (V == 1) x[0] = *(const float *)p;
        else {
            const vec v = *(const vec *)p;
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = v[e];
        }
    } else if constexpr (V == 1) x[0] = bf16_to_f32(*(const bf16_t *)p);
    else {
        typedef unsigned vec __attribute__((ext_vector_type(V / 2)));
        if constexpr (V == 2) {
            const unsigned v = *(const unsigned *)p;
            x[0] = bf16_lo(v);
            x[1] = bf16_hi(v);
        } else {
            const vec v = *(const vec *)p;
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = e % 2 ? bf16_hi(v[e / 2]) : bf16_lo(v[e / 2]);
        }
    }
}

template <class E, int V>
__device__ __forceinline__ void store(char *p, const float (&x)[V])
{
    if constexpr (V == 1) store_from_f32((E *)p, x[0]);
    else if constexpr (sizeof(E) == 4) {
        typedef float vec __attribute__((ext_vector_type(V)));
        vec v;
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = x[e];
        *(vec *)p = v;
    } else if constexpr (V == 2) *(unsigned *)p = pack_bf16(x[0], x[1]);
    else {
        typedef unsigned vec __attribute__((ext_vector_type(V / 2)));
        vec v;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) v[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
        *(vec *)p = v;
    }
}

// Values of a float32 vector whose alignment is that of its elements.
template <int V>
__device__ __forceinline__ void load_vector(const float *p, float (&x)[V])
{
    if (V % 4 == 0 && (uintptr_t)p % 16 == 0) {
#pragma unroll
        for (int e = 0; e < V / 4; ++e) {
            const f32x4 v = *(const f32x4 *)(p + 4 * e);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * e + i] = v[i];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = p[e];
}

__device__ __forceinline__ float team_sum(float v, int team)
{
    if (team > 1) v = dpp_fadd<0xB1>(v);        // lane ^ 1
    if (team > 2) v = dpp_fadd<0x4E>(v);        // lane ^ 2
    if (team > 4) v = dpp_fadd<0x141>(v);       // mirrored halves of 8
    if (team > 8) v = dpp_fadd<0x140>(v);       // mirrored rows of 16
    if (team > 16) v += __shfl_xor(v, 16);
    if (team > 32) v += __shfl_xor(v, 32);
    return v;
}

// The pairs of chunks a, b rotated.  halves: pairs are a[i], b[i], else neighbours within them.
template <int V>
__device__ __forceinline__ void turn(float (&a)[V], float (&b)[V], const float (&cos)[V], const float (&sin)[V], bool halves)
{
    if (halves || V == 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = a[e], v = b[e];
            a[e] = u * cos[e] - v * sin[e];
            b[e] = v * cos[e] + u * sin[e];
        }
        return;
    }
    if constexpr (V > 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float (&x)[V] = e < V / 2 ? a : b;
            const int i = 2 * (e % (V / 2));
            const float u = x[i], v = x[i + 1];
            x[i] = u * cos[e] - v * sin[e];
            x[i + 1] = v * cos[e] + u * sin[e];
        }
    }
}

// Bound by memory, near what a copy reaches (5.1 TB/s): 32 x 1024 tokens of 12 + 12 heads of 64 41 to 44 us, 4.6 to 4.9 TB/s; backward 2 x 8192 of 32 + 8 heads of 128 114 us,
// 4.4 TB/s (its sums keep it at two workgroups to a compute unit).  Backward in float32, 6475 tokens of 6 + 6 heads of 40: 13 us where the bytes take 7: the 512 workgroups take three
// turns for 2.37 turns' rows, and three of a team's eight lanes have no channels.  One token: 6 us, the call on the host; the kernel 2.8.
template <class E, int V, int RPT, bool BACK>
__global__ __launch_bounds__(kThreads) void k_qk_norm(Work W)
{
    const bool keys = blockIdx.x >= W.query_blocks;
    const Part &P = W.part[keys];
    const unsigned block = blockIdx.x - (keys ? W.query_blocks : 0), blocks = keys ? gridDim.x - W.query_blocks : W.query_blocks;
    const int lane = threadIdx.x % W.team, teams = kThreads / W.team;
    const bool active = 2 * V * lane < W.d, turned = 2 * V * lane < W.turned;
    const int unit = active ? lane : 0, ca = turned && W.halves ? V * unit : 2 * V * unit, cb = turned && W.halves ? W.turned / 2 + V * unit : ca + V;
    const bool norm = P.gamma != nullptr;
    float ga[V], gb[V], suma[V], sumb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        ga[e] = gb[e] = 1.f;
        suma[e] = sumb[e] = 0.f;
    }
    if (norm) {
        load_vector<V>(P.gamma + ca, ga);
        load_vector<V>(P.gamma + cb, gb);
    }
    for (unsigned item = block * (unsigned)teams + threadIdx.x / W.team; item < P.items; item += blocks * (unsigned)teams) {
        const unsigned token = item / P.groups, group = item - token * P.groups, b = token / W.N, n = token - b * W.N;
        float xa[RPT][V], xb[RPT][V], ya[BACK ? RPT : 1][V], yb[BACK ? RPT : 1][V], cos[V], sin[V];
        // rows that do not exist are read in another's place and not written
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int head = min((int)(group + i * P.groups), P.heads - 1);
            if (!BACK || norm) {
                const char *p = P.x.p + b * P.x.batch + n * P.x.token + head * P.x.head;
                load<E, V>(p + ca * sizeof(E), xa[i]);
                load<E, V>(p + cb * sizeof(E), xb[i]);
            }
            if constexpr (BACK) {
                const char *p = P.g.p + b * P.g.batch + n * P.g.token + head * P.g.head;
                load<E, V>(p + ca * sizeof(E), ya[i]);
                load<E, V>(p + cb * sizeof(E), yb[i]);
            }
        }
        if (turned) {
            const int at = W.positions ? min(max(W.positions[token], 0), W.table_rows - 1) : (int)n;
            const long pair = (long)at * (W.turned / 2) + V * unit;
            load_vector<V>(W.cos + pair, cos);
            load_vector<V>(W.sin + pair, sin);
            if (BACK) {
#pragma unroll
                for (int e = 0; e < V; ++e) sin[e] = -sin[e];
            }
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int head = (int)(group + i * P.groups);
            const bool live = active && head < P.heads;
            float inv = 1.f;
            if (norm) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) s = fmaf(xa[i][e], xa[i][e], fmaf(xb[i][e], xb[i][e], s));
                inv = 1.0f / sqrtf(fmaf(team_sum(active ? s : 0.f, W.team), W.d_inv, W.eps));
            }
            float oa[V], ob[V];
            if constexpr (!BACK) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    oa[e] = norm ? xa[i][e] * inv * ga[e] : xa[i][e];
                    ob[e] = norm ? xb[i][e] * inv * gb[e] : xb[i][e];
                }
                if (turned) turn<V>(oa, ob, cos, sin, W.halves);
            } else {
                if (turned) turn<V>(ya[i], yb[i], cos, sin, W.halves);
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    oa[e] = ya[i][e];
                    ob[e] = yb[i][e];
                    if (!norm) continue;
                    xa[i][e] *= inv;
                    xb[i][e] *= inv;
                    suma[e] += live ? oa[e] * xa[i][e] : 0.f;
                    sumb[e] += live ? ob[e] * xb[i][e] : 0.f;
                    oa[e] *= ga[e];
                    ob[e] *= gb[e];
                    dot = fmaf(oa[e], xa[i][e], fmaf(ob[e], xb[i][e], dot));
                }
                if (norm) {
                    const float mean = team_sum(active ? dot : 0.f, W.team) * W.d_inv;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        oa[e] = inv * (oa[e] - xa[i][e] * mean);
                        ob[e] = inv * (ob[e] - xb[i][e] * mean);
                    }
                }
            }
            if (live) {
                char *p = P.o.p + b * P.o.batch + n * P.o.token + head * P.o.head;
                store<E, V>(p + ca * sizeof(E), oa);
                store<E, V>(p + cb * sizeof(E), ob);
            }
        }
    }
    if constexpr (BACK) {
        if (!norm) return;
        // the workgroup's sums: teams of a wavefront first, then its four wavefronts
        __shared__ float lds[kThreads / 64][128];
        for (int o = W.team; o < 64; o *= 2)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                suma[e] += __shfl_xor(suma[e], o);
                sumb[e] += __shfl_xor(sumb[e], o);
            }
        if (threadIdx.x % 64 < W.team && active)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                lds[threadIdx.x / 64][ca + e] = suma[e];
                lds[threadIdx.x / 64][cb + e] = sumb[e];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < W.d; c += kThreads) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) v += lds[w][c];
            W.sums[(long)blockIdx.x * W.d + c] = v;
        }
    }
}

// Sums of the workgroups' sums: 8 columns to a workgroup, 32 shares of the rows; the queries' rows, then the keys'.  A chain of reads: 512 rows of 128 4.7 us.
__global__ __launch_bounds__(256) void k_qk_norm_sums(const float *sums, int query_rows, int rows, int d, float *dq, float *dk)
{
    __shared__ float lds[32][9];
    const int each = d / 8, keys = blockIdx.x / each, col = threadIdx.x % 8, share = threadIdx.x / 8, c = blockIdx.x % each * 8 + col;
    const int first = keys ? query_rows : 0, end = keys ? rows : query_rows;
    float v = 0.f;
#pragma unroll 8
    for (int r = first + share; r < end; r += 32) v += sums[(long)r * d + c];
    lds[share][col] = v;
    __syncthreads();
    if (share) return;
    v = 0.f;
#pragma unroll
    for (int s = 0; s < 32; ++s) v += lds[s][col];
    float *out = keys ? dk : dq;
    if (out) out[c] = v;
}

// Channels of a chunk: whole pairs of the rotated part to a lane, chunks of up to 16 bytes.
int chunk(const QkNormSizes &S)
{
    int V = S.f32 ? 4 : 8;
    while (S.turned % (2 * V) || S.d % (2 * V)) V /= 2;
    return V;
}
int team_of(const QkNormSizes &S, int V)
{
    int t = 1;
    while (2 * V * t < S.d) t *= 2;
    return t;
}
// Heads of a token to a team: several share the angles and are on their way at once; of few rows each goes to a team of its own.
int rows_per_team(const QkNormSizes &S)
{
    if (S.tokens * (S.heads + S.kv_heads) < 16384) return 1;
    auto fits = [&](int r) {
        auto waste = [&](int heads) { return 4 * ((heads + r - 1) / r * r) > 5 * heads; };
        return !waste(S.heads) && !(S.kv_heads && waste(S.kv_heads));
    };
    return fits(4) ? 4 : fits(2) ? 2 : 1;
}
// Workgroups of the queries and of the keys.
struct Blocks {
    long query, key;
    Blocks(const QkNormSizes &S, bool back)
    {
        const int rpt = rows_per_team(S), teams = kThreads / team_of(S, chunk(S));
        auto all = [&](int heads) { return (S.tokens * ((heads + rpt - 1) / rpt) + teams - 1) / teams; };
        query = all(S.heads);
        key = all(S.kv_heads);
        const long most = back ? 512L : 1L << 20;
        if (query + key > most) {
            const long sum = query + key;
            query = std::max(1L, query * most / sum);
            key = key ? std::max(1L, key * most / sum) : 0;
        }
    }
};

template <class E, int V, bool BACK>
int launch(const QkNormSizes &S, const Work &W, int rpt, hipStream_t st)
{
    const ProfScope scope(st, BACK ? K_QK_NORM_BACKWARD : K_QK_NORM);
    const Blocks n(S, BACK);
    const unsigned blocks = (unsigned)(n.query + n.key);
    if (rpt == 4) k_qk_norm<E, V, 4, BACK><<<blocks, kThreads, 0, st>>>(W);
    else if (rpt == 2) k_qk_norm<E, V, 2, BACK><<<blocks, kThreads, 0, st>>>(W);
    else k_qk_norm<E, V, 1, BACK><<<blocks, kThreads, 0, st>>>(W);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <class E, bool BACK>
int pick(const QkNormSizes &S, const Work &W, int rpt, hipStream_t st)
{
    switch (chunk(S)) {
    case 8:
        if constexpr (sizeof(E) == 2) return launch<E, 8, BACK>(S, W, rpt, st);
        [[fallthrough]];
    case 4: return launch<E, 4, BACK>(S, W, rpt, st);
    case 2: return launch<E, 2, BACK>(S, W, rpt, st);
    default: return launch<E, 1, BACK>(S, W, rpt, st);
    }
}

Work make_work(const QkNormSizes &S, const QkNormIn &I, int rpt, bool back)
{
    Work W{};
    for (int k = 0; k < 2; ++k) {
        Part &P = W.part[k];
        P.x = k ? I.K : I.Q;
        P.gamma = k ? I.k_gamma : I.q_gamma;
        P.heads = k ? S.kv_heads : S.heads;
        P.groups = (unsigned)((P.heads + rpt - 1) / rpt);
        P.items = (unsigned)(S.tokens * P.groups);
    }
    W.cos = I.cos;
    W.sin = I.sin;
    W.positions = I.positions;
    W.N = (unsigned)S.N;
    W.d = S.d;
    W.turned = S.turned;
    W.table_rows = S.table_rows;
    W.team = team_of(S, chunk(S));
    W.eps = S.eps;
    W.d_inv = 1.0f / (float)S.d;
    W.halves = S.halves;
    W.query_blocks = (unsigned)Blocks(S, back).query;
    return W;
}

}  // namespace

int qk_norm_forward(const QkNormSizes &S, const QkNormIn &I, const att::Rows &Qout, const att::Rows &Kout, hipStream_t st)
{
    if (S.tokens == 0) return BRA_OK;
    const int rpt = rows_per_team(S);
    Work W = make_work(S, I, rpt, false);
    W.part[0].o = Qout;
    W.part[1].o = Kout;
    return S.f32 ? pick<float, false>(S, W, rpt, st) : pick<bf16_t, false>(S, W, rpt, st);
}

size_t qk_norm_backward_workspace_bytes(const QkNormSizes &S)
{
    const Blocks n(S, true);
    return align256(sizeof(float) * S.d * std::max(n.query + n.key, 1L));
}

int qk_norm_backward(const QkNormSizes &S, const QkNormIn &I, const att::Rows &gQ, const att::Rows &gK, const att::Rows &dQ, const att::Rows &dK, float *dq_gamma,
                     float *dk_gamma, void *ws, hipStream_t st)
{
    const int rpt = rows_per_team(S);
    Work W = make_work(S, I, rpt, true);
    W.part[0].g = gQ;
    W.part[1].g = gK;
    W.part[0].o = dQ;
    W.part[1].o = dK;
    W.sums = (float *)ws;
    if (S.tokens > 0) {
        const int rc = S.f32 ? pick<float, true>(S, W, rpt, st) : pick<bf16_t, true>(S, W, rpt, st);
        if (rc != BRA_OK) return rc;
    }
    if (!I.q_gamma || (!dq_gamma && !dk_gamma)) return BRA_OK;
    const ProfScope scope(st, K_QK_NORM_SUMS);
    const Blocks n(S, true);
    k_qk_norm_sums<<<2 * S.d / 8, 256, 0, st>>>(W.sums, (int)n.query, (int)(n.query + n.key), S.d, dq_gamma, dk_gamma);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

}  // namespace bra
