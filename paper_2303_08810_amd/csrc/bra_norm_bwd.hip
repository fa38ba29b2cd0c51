// Gradients of the norms around a residual sum, R = X + scale * gate[group] * Z, Z = post(Y) = yu post_gamma + post_beta,
// N = norm(R) gamma + beta = u gamma + beta.  With g = dN gamma and means over the row's channels:
//     D  = dR + (g - [mean g] - u mean(g u)) / sigma(R)           dX = D;  the bracket with LayerNorm only
//     t  = D scale gate post_gamma,  dY = (t - [mean t] - yu mean(t yu)) / sigma(Y);   without the post norm dY = D scale gate
//     dgamma = sum dN u,  dbeta = sum dN                            over the rows
//     Q = sum D yu,  S = sum D                                      over the rows of a group (Q = sum D Y without the post norm)
//     T = post_gamma Q + post_beta S:  dgate = scale T,  dscale = sum over groups of gate T,
//     dpost_gamma = scale sum gate Q,  dpost_beta = scale sum gate S
// so that a row adds to four sums per channel, whatever is asked for.  One pass over the maps; a row stays in registers.  No atomic
// adds: a thread's sums go through LDS to its workgroup's, those through memory to k_norm_sums, in a fixed order.
#include "bra_norm_dev.h"

namespace bra {

using namespace norm;

namespace {

constexpr int kSums = 5;            // dgamma, dbeta, and where groups are finished in this kernel dscale, dpost_gamma, dpost_beta
// Wavefronts per SIMD, with `values` channels per thread: three where the registers allow it, or nearly (33 spilled at most;
// 32768 x 768 115 -> 97 us), two where they do not (6475 x 192 in float32 19 us, with three and their spills 24).
constexpr int waves(int values, bool f32, bool finish) { return values == 16 || (values == 12 && (f32 || finish)) ? 2 : 3; }

// Lines of LDS in which teams meet.
__host__ __device__ constexpr int meeting_lines(int teams) { return teams > 1 ? teams : 0; }

struct BackArgs {
    NormIn I;
    const void *dN, *dR;
    void *dX, *dY, *dgate;
    float *part, *units;            // [workgroup][kSums or 2][C]; [unit][Q, S][C]
    long rows, groups;
    unsigned per_group;
    int C, tpr, parts;
    float eps;
    bool vec;                       // rows are whole 16-byte pieces
    float *out[kSums];              // where a single workgroup finishes everything: the results
    int whole;                      // FINISH: a workgroup has a whole group at a time, otherwise each of its teams has one
};

// How rows are shared out.
struct Split {
    Team T;
    int parts;
    bool finish, whole;
    long units;
    unsigned blocks;
    Split(const NormSizes &S) : T(S.C, S.vec)
    {
        const int teams = T.teams(), kTarget = 256 * waves(T.V * T.nch, S.f32, false);        // workgroups that run at once
        // Many groups of fewer rows than half of a workgroup's teams: each team takes whole groups.  Otherwise a workgroup takes a group, or,
        // where groups are few, a part of one
        const bool by_team = S.per_group <= teams / 2 && S.groups > kTarget;
        parts = 1;
        if (!by_team) parts = (int)std::max(1L, std::min<long>((kTarget + S.groups - 1) / S.groups, (S.per_group + 2 * teams - 1) / (2 * teams)));
        finish = parts == 1;
        whole = !by_team;
        units = (long)S.groups * parts;
        blocks = (unsigned)std::max(1L, std::min<long>(kTarget, by_team ? (units + teams - 1) / teams : units));
    }
    int sums() const { return finish ? kSums : 2; }
};

// 32768 x 768, LayerNorm twice, gate and scale: 88 us (90 in a trace) for 302 MB, 3.4 TB/s: three wavefronts per SIMD, each with one row's loads in flight, do not cover the
// memory's latency.  6475 x 192 in float32: 12.5 us.
template <typename E, bool LAYER, bool POST, int V, int NCH, bool FULL, bool FINISH>
__global__ __launch_bounds__(kMaxTeam, waves(V * NCH, sizeof(E) == 4, FINISH)) void k_norm_backward(BackArgs A)
{
    extern __shared__ __attribute__((aligned(16))) float smem[];
    const int C = A.C, tpr = A.tpr, team = threadIdx.x / tpr, teams = blockDim.x / tpr, t = threadIdx.x % tpr, width = V * NCH * tpr;
    const bool vec = A.vec;
    float *meet = smem;                                     // [teams][width]
    float *vectors = meet + meeting_lines(teams) * width;   // gamma, scale, post_gamma, post_beta: [4][width]
    float *lds = vectors + 4 * width;                       // of team_sums
    const float c_inv = 1.0f / (float)C;
    int n[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) n[k] = C - V * (t + k * tpr);
    for (int c = threadIdx.x; c < width; c += blockDim.x) {
        const bool in = c < C;
        vectors[c] = in && A.I.gamma ? A.I.gamma[c] : 0.f;
        vectors[width + c] = !in ? 0.f : A.I.scale ? A.I.scale[c] : 1.f;
        vectors[2 * width + c] = !in ? 0.f : POST ? A.I.post_gamma[c] : 1.f;
        vectors[3 * width + c] = in && POST && A.I.post_beta ? A.I.post_beta[c] : 0.f;
    }
    __syncthreads();
    int own = V * t;
    auto vector = [&](int which, int k, float (&v)[V]) {
        const f32x4 *p = (const f32x4 *)(vectors + which * width + own + V * k * tpr);
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const f32x4 a = p[q];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = a[e];
        }
    };
    auto gate_of = [&](long group, int k) { return load<FULL, E, V>((const E *)A.I.gate + (size_t)group * C + V * (t + k * tpr), n[k], vec); };

    float sums[FINISH ? kSums : 2][NCH][V], Q[NCH][V], S[POST ? NCH : 1][V];
#pragma unroll
    for (int s = 0; s < (FINISH ? kSums : 2); ++s)
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[s][k][e] = 0.f;
    auto clear = [&]() {
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) { Q[k][e] = 0.f; if (POST) S[k][e] = 0.f; }
    };

    // one row per team; the next one is on its way while one is worked on
    Raw<E, V> rx[NCH], ry[NCH], rn[NCH], rd[NCH];
    auto fetch = [&](long r) {
        const size_t at = (size_t)r * C + V * t;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            rx[k] = load<FULL, E, V>((const E *)A.I.X + at + V * k * tpr, n[k], vec);
            if (A.I.Y) ry[k] = load<FULL, E, V>((const E *)A.I.Y + at + V * k * tpr, n[k], vec);
            if (A.dN) rn[k] = load<FULL, E, V>((const E *)A.dN + at + V * k * tpr, n[k], vec);
            if (A.dR) rd[k] = load<FULL, E, V>((const E *)A.dR + at + V * k * tpr, n[k], vec);
        }
    };
    // row r, which has been fetched; then row `next` (-1: none).  Teams without a row (`mine` unset) go along with another's and add nothing: both factors
    // are 0, for where dX or dY lies in R's, dN's or Y's place that row may have been overwritten by its own team, and 0 times what is there now
    // may be NaN
    auto row = [&](long r, long next, long group, bool mine) {
        // the vectors stay in LDS: kept in registers over the rows, they cost a wavefront per SIMD
        asm volatile("" : "+v"(own));
        const size_t at = (size_t)r * C + V * t;
        float x[NCH][V], y[NCH][V], dn[NCH][V], d[NCH][V];
        Raw<E, V> gate[NCH];
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[k][e] = value(rx[k], e);
                y[k][e] = A.I.Y ? value(ry[k], e) : 0.f;
                dn[k][e] = A.dN ? value(rn[k], e) : 0.f;
                d[k][e] = A.dR ? value(rd[k], e) : 0.f;
            }
            if (A.I.gate) gate[k] = gate_of(group, k);
        }
        if (next >= 0) fetch(next);
        if (LAYER) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NCH; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) { m[0] += x[k][e]; if (POST) m[1] += y[k][e]; }
            team_sums(m, tpr, lds);
#pragma unroll
            for (int k = 0; k < NCH; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    x[k][e] = FULL || e < n[k] ? x[k][e] - m[0] * c_inv : 0.f;
                    if (POST) y[k][e] = FULL || e < n[k] ? y[k][e] - m[1] * c_inv : 0.f;
                }
        }
        float v[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) { v[0] = fmaf(x[k][e], x[k][e], v[0]); if (POST) v[1] = fmaf(y[k][e], y[k][e], v[1]); }
        team_sums(v, tpr, lds);
        const float inv = 1.0f / sqrtf(fmaf(v[0], c_inv, A.eps)), yinv = POST ? 1.0f / sqrtf(fmaf(v[1], c_inv, A.eps)) : 1.f;
        if (A.dN) {
            float p[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NCH; ++k) {
                float gamma[V];
                vector(0, k, gamma);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    x[k][e] *= inv;
                    const float w = mine ? dn[k][e] : 0.f;
                    sums[0][k][e] = fmaf(w, mine ? x[k][e] : 0.f, sums[0][k][e]);
                    sums[1][k][e] += w;
                    dn[k][e] *= gamma[e];
                    p[0] += dn[k][e];
                    p[1] = fmaf(dn[k][e], x[k][e], p[1]);
                }
            }
            team_sums(p, tpr, lds);
            const float m1 = LAYER ? p[0] * c_inv : 0.f, m2 = p[1] * c_inv;
#pragma unroll
            for (int k = 0; k < NCH; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float g = fmaf(-x[k][e], m2, dn[k][e] - m1);
                    d[k][e] = FULL || e < n[k] ? fmaf(g, inv, d[k][e]) : 0.f;
                }
        }
        if (mine)
#pragma unroll
            for (int k = 0; k < NCH; ++k) store<FULL>((E *)A.dX + at + V * k * tpr, d[k], n[k], vec);
        if (!A.I.Y) return;
        float p[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            float scale[V], pg[V];
            vector(1, k, scale);
            if (POST) vector(2, k, pg);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (POST) y[k][e] *= yinv;
                const float w = mine ? d[k][e] : 0.f;
                Q[k][e] = fmaf(w, mine ? y[k][e] : 0.f, Q[k][e]);
                if (POST) S[k][e] += w;
                d[k][e] *= A.I.gate ? scale[e] * value(gate[k], e) : scale[e];
                if (POST) {
                    d[k][e] *= pg[e];
                    p[0] += d[k][e];
                    p[1] = fmaf(d[k][e], y[k][e], p[1]);
                }
            }
        }
        if constexpr (POST) {
            team_sums(p, tpr, lds);
            const float m1 = LAYER ? p[0] * c_inv : 0.f, m2 = p[1] * c_inv;
#pragma unroll
            for (int k = 0; k < NCH; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) d[k][e] = yinv * fmaf(-y[k][e], m2, d[k][e] - m1);
        }
        if (mine)
#pragma unroll
            for (int k = 0; k < NCH; ++k) store<FULL>((E *)A.dY + at + V * k * tpr, d[k], n[k], vec);
    };

    // the sum over the teams of what each of their threads holds, for every thread; the whole workgroup calls it
    auto over_teams = [&](float (&v)[NCH][V]) {
        if (teams == 1) return;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; e += 4) *(f32x4 *)(meet + team * width + V * (t + k * tpr) + e) = f32x4{v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3]};
        __syncthreads();
        for (int c = threadIdx.x; c < width; c += blockDim.x) {
            float s = 0.f;
            for (int j = 0; j < teams; ++j) s += meet[j * width + c];
            meet[c] = s;        // column c of team 0's line is read by this thread alone
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const f32x4 s = *(const f32x4 *)(meet + V * (t + k * tpr) + e);
                v[k][e] = s[0]; v[k][e + 1] = s[1]; v[k][e + 2] = s[2]; v[k][e + 3] = s[3];
            }
    };
    // a group's sums are complete: its gate's gradient, and its part of the others
    auto finish = [&](long group) {
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            float scale[V], pg[V], pb[V], T[V];
            vector(1, k, scale);
            vector(2, k, pg);
            vector(3, k, pb);
            Raw<E, V> gate;
            if (A.I.gate) gate = gate_of(group, k);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = A.I.gate ? value(gate, e) : 1.f;
                T[e] = POST ? fmaf(pg[e], Q[k][e], pb[e] * S[POST ? k : 0][e]) : Q[k][e];
                if constexpr (FINISH) {
                    sums[2][k][e] = fmaf(g, T[e], sums[2][k][e]);
                    if (POST) {
                        sums[3][k][e] = fmaf(scale[e] * g, Q[k][e], sums[3][k][e]);
                        sums[4][k][e] = fmaf(scale[e] * g, S[POST ? k : 0][e], sums[4][k][e]);
                    }
                }
                T[e] *= scale[e];
            }
            if (A.dgate) store<FULL>((E *)A.dgate + (size_t)group * C + V * (t + k * tpr), T, n[k], vec);
        }
    };

    if (FINISH && !A.whole) {
        for (long g0 = (long)blockIdx.x * teams; g0 < A.groups; g0 += (long)gridDim.x * teams) {
            const bool mine = g0 + team < A.groups;
            const long g = mine ? g0 + team : A.groups - 1;
            clear();
            fetch(g * A.per_group);
            for (unsigned i = 0; i < A.per_group; ++i) row(g * A.per_group + i, i + 1 < A.per_group ? g * A.per_group + i + 1 : -1, g, mine);
            if (mine && A.I.Y) finish(g);
        }
    } else {
        for (long u = blockIdx.x; u < A.groups * A.parts; u += gridDim.x) {
            const long g = u / A.parts, part = u % A.parts, begin = A.per_group * part / A.parts, end = A.per_group * (part + 1) / A.parts, base = g * A.per_group;
            clear();
            fetch(base + min(begin + team, end - 1));
            for (long i = begin; i < end; i += teams) row(base + min(i + team, end - 1), i + teams < end ? base + min(i + teams + team, end - 1) : -1, g, i + team < end);
            if (!A.I.Y) continue;
            over_teams(Q);
            if constexpr (POST) over_teams(S);
            if (team != 0) continue;
            if (FINISH) finish(g);
            else
#pragma unroll
                for (int k = 0; k < NCH; ++k) {
                    float *to = A.units + (size_t)u * 2 * C + V * (t + k * tpr);
                    store<FULL>(to, Q[k], n[k], vec);
                    if constexpr (POST) store<FULL>(to + C, S[k], n[k], vec);
                }
        }
    }
#pragma unroll
    for (int s = 0; s < (FINISH ? kSums : 2); ++s) {
        if (s < 2 ? !A.dN : !A.I.Y || (s > 2 && !POST)) continue;
        over_teams(sums[s]);
        if (team != 0) continue;
        if (FINISH && gridDim.x == 1) {
            if (A.out[s])
#pragma unroll
                for (int k = 0; k < NCH; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (FULL || e < n[k]) A.out[s][V * (t + k * tpr) + e] = sums[s][k][e];
        } else
#pragma unroll
            for (int k = 0; k < NCH; ++k) store<FULL>(A.part + ((size_t)blockIdx.x * (FINISH ? kSums : 2) + s) * C + V * (t + k * tpr), sums[s][k], n[k], vec);
    }
}

struct SumArgs {
    const float *part, *units;
    const void *gate;
    const float *scale, *post_gamma, *post_beta;
    float *out[kSums];          // dgamma, dbeta, dscale, dpost_gamma, dpost_beta; NULL where not asked for
    void *dgate;
    int C, blocks, sums, parts, column_blocks;
    long groups;
    bool post;
};

// Columns in workgroups of 16, 64 threads to a column: dgamma, dbeta, and what the groups give (one workgroup each: blockIdx.y); behind
// them, where groups came in parts, their gates' gradients.  A chain of reads that cross the chip: 13 us for 768 workgroups' sums of 768
// channels (deeper unrolling changed nothing), 4 us for 203 of 192.
template <typename E>
__global__ __launch_bounds__(1024) void k_norm_sums(SumArgs A)
{
    __shared__ float meet[64][17];
    const int y = blockIdx.y;
    if ((int)blockIdx.x >= A.column_blocks) {
        const long count = A.groups * A.C, step = (long)(gridDim.x - A.column_blocks) * gridDim.y * 1024;
        for (long i = ((long)(blockIdx.x - A.column_blocks) * gridDim.y + y) * 1024 + threadIdx.x; i < count; i += step) {
            const long g = i / A.C;
            const int c = (int)(i % A.C);
            float q = 0.f, s = 0.f;
#pragma unroll 4
            for (int p = 0; p < (A.blocks ? A.parts : 0); ++p) {
                const float *u = A.units + (size_t)(g * A.parts + p) * 2 * A.C + c;
                q += u[0];
                if (A.post) s += u[A.C];
            }
            // (0 without rows, whatever scale is)
            const float t = A.post ? fmaf(A.post_gamma[c], q, (A.post_beta ? A.post_beta[c] : 0.f) * s) : q;
            store_from_f32((E *)A.dgate + i, A.blocks ? (A.scale ? A.scale[c] : 1.f) * t : 0.f);
        }
        return;
    }
    const int x = threadIdx.x % 16, slot = threadIdx.x / 16, c = blockIdx.x * 16 + x;
    const bool in = c < A.C;
    auto total = [&](float v) {
        __syncthreads();
        meet[slot][x] = v;
        __syncthreads();
        for (int half = 32; half; half /= 2) {
            if (slot < half) meet[slot][x] += meet[slot + half][x];
            __syncthreads();
        }
        return meet[0][x];
    };
    for (int s = y; s < A.sums; s += 3) {
        if (!A.out[s]) continue;
        float v = 0.f;
        if (in)
#pragma unroll 4
            for (int b = slot; b < A.blocks; b += 64) v += A.part[((size_t)b * A.sums + s) * A.C + c];
        v = total(v);
        if (in && slot == 0) A.out[s][c] = v;
    }
    if (y != 2 || A.parts == 1 || !(A.out[2] || A.out[3] || A.out[4])) return;
    float q = 0.f, s = 0.f;
    if (in)
#pragma unroll 4
        for (int u = slot; u < (int)A.groups * A.parts; u += 64) {
            const float gate = A.gate ? load_f32((const E *)A.gate + (size_t)((unsigned)u / (unsigned)A.parts) * A.C + c) : 1.f;
            q = fmaf(gate, A.units[(size_t)u * 2 * A.C + c], q);
            if (A.post) s = fmaf(gate, A.units[((size_t)u * 2 + 1) * A.C + c], s);
        }
    q = total(q);
    if (A.post) s = total(s);
    if (!in || slot != 0) return;
    const float scale = A.scale ? A.scale[c] : 1.f;
    if (A.out[2]) A.out[2][c] = A.post ? fmaf(A.post_gamma[c], q, (A.post_beta ? A.post_beta[c] : 0.f) * s) : q;
    if (A.out[3]) A.out[3][c] = scale * q;
    if (A.out[4]) A.out[4][c] = scale * s;
}

size_t part_floats(const NormSizes &S, const Split &P) { return align256((size_t)P.blocks * P.sums() * S.C * 4) / 4; }
size_t unit_floats(const NormSizes &S, const Split &P) { return P.finish ? 0 : (size_t)P.units * 2 * S.C; }

template <typename E, bool LAYER, bool POST, int V, int NCH, bool FULL>
int launch(const BackArgs &A, const Split &P, hipStream_t st)
{
    const int width = V * NCH * P.T.tpr, threads = P.T.threads();
    const size_t bytes = ((size_t)(meeting_lines(P.T.teams()) + 4) * width + 2 * (threads / 64)) * 4;
    if ((P.finish ? allow_lds<k_norm_backward<E, LAYER, POST, V, NCH, FULL, true>>(kMaxLds) : allow_lds<k_norm_backward<E, LAYER, POST, V, NCH, FULL, false>>(kMaxLds)) != BRA_OK)
        return BRA_ERR_LAUNCH;
    if (P.finish) k_norm_backward<E, LAYER, POST, V, NCH, FULL, true><<<P.blocks, threads, bytes, st>>>(A);
    else k_norm_backward<E, LAYER, POST, V, NCH, FULL, false><<<P.blocks, threads, bytes, st>>>(A);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <typename E, bool LAYER, bool POST>
int pick(const BackArgs &A, const Split &P, hipStream_t st)
{
    if (P.T.nch == 3) return launch<E, LAYER, POST, 4, 3, true>(A, P, st);
    if (P.T.nch == 1) return P.T.full ? launch<E, LAYER, POST, 8, 1, true>(A, P, st) : launch<E, LAYER, POST, 8, 1, false>(A, P, st);
    return P.T.full ? launch<E, LAYER, POST, 8, 2, true>(A, P, st) : launch<E, LAYER, POST, 8, 2, false>(A, P, st);
}

}  // namespace

size_t norm_backward_workspace_bytes(const NormSizes &S)
{
    if (S.rows == 0) return 0;
    const Split P(S);
    return (part_floats(S, P) + unit_floats(S, P)) * 4;
}

int norm_backward(const NormSizes &S, const NormIn &I, const void *dN, const void *dR, const NormGrads &G, void *ws, hipStream_t st)
{
    // no rows: whatever is asked for is zero
    const bool none = S.rows == 0, y = I.Y || none, post = none || S.post;
    float *outs[kSums] = {dN || none ? G.dgamma : nullptr, dN || none ? G.dbeta : nullptr, y ? G.dscale : nullptr, y && post ? G.dpost_gamma : nullptr,
                          y && post ? G.dpost_beta : nullptr};
    SumArgs F{};
    F.gate = I.gate; F.scale = I.scale; F.post_gamma = I.post_gamma; F.post_beta = I.post_beta;
    for (int s = 0; s < kSums; ++s) F.out[s] = outs[s];
    F.C = S.C; F.sums = kSums; F.parts = 1; F.column_blocks = (S.C + 15) / 16; F.post = S.post && !none;
    // (more than these only where there are no rows: 2^32 threads cannot be launched)
    auto gates = [&] { return (unsigned)std::min(((long)S.groups * S.C + 3 * 1024 - 1) / (3 * 1024), 1L << 16); };
    unsigned gate_blocks = 0;
    if (S.rows > 0) {
        const Split P(S);
        F.part = (const float *)ws; F.units = (const float *)ws + part_floats(S, P);
        F.blocks = (int)P.blocks; F.sums = P.sums(); F.parts = P.parts; F.groups = S.groups;
        BackArgs A{I, dN, dR, G.dX, G.dY, P.finish ? G.dgate : nullptr, (float *)ws, (float *)ws + part_floats(S, P), S.rows, S.groups, (unsigned)S.per_group, S.C, P.T.tpr,
                         P.parts, S.eps, S.vec, {}, P.whole};
        for (int s = 0; s < kSums; ++s) A.out[s] = outs[s];
        {
            ProfScope prof(st, K_NORM_BACKWARD);
            int rc;
            if (S.f32) {
                if (S.layer) rc = S.post ? pick<float, true, true>(A, P, st) : pick<float, true, false>(A, P, st);
                else rc = S.post ? pick<float, false, true>(A, P, st) : pick<float, false, false>(A, P, st);
            } else {
                if (S.layer) rc = S.post ? pick<bf16_t, true, true>(A, P, st) : pick<bf16_t, true, false>(A, P, st);
                else rc = S.post ? pick<bf16_t, false, true>(A, P, st) : pick<bf16_t, false, false>(A, P, st);
            }
            if (rc != BRA_OK || (P.finish && P.blocks == 1)) return rc;
        }
        if (!P.finish && I.Y && G.dgate) {
            F.dgate = G.dgate;
            gate_blocks = gates();
        }
    } else if (G.dgate) {
        F.dgate = G.dgate; F.groups = S.groups;
        gate_blocks = gates();
    }
    bool any = gate_blocks > 0;
    for (int s = 0; s < kSums; ++s) any = any || outs[s];
    if (!any) return BRA_OK;
    ProfScope prof(st, K_NORM_SUMS);
    if (S.f32) k_norm_sums<float><<<dim3(F.column_blocks + gate_blocks, 3), 1024, 0, st>>>(F);
    else k_norm_sums<bf16_t><<<dim3(F.column_blocks + gate_blocks, 3), 1024, 0, st>>>(F);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

}  // namespace bra
