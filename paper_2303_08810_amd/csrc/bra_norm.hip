// Norms before and after a block with its gate and residual scale:
//     R = X + scale * gate[group] * post(Y),   N = norm(R) gamma + beta
// norm and post are LayerNorm or RMSNorm over a row's C channels.  One pass: X and Y are read once, R and N written once; the row
// stays in registers from the loads to the stores, its statistics are those of the float32 sum.  The next row is on its way while
// one is worked on.  Bound by memory.
#include "bra_norm_dev.h"

namespace bra {

using namespace norm;

namespace {

// (x - mean) / sqrt(var + eps) or x / sqrt(mean of squares + eps), in place; n[k]: channels of chunk k that exist.
template <bool LAYER, bool FULL, int V, int NCH>
__device__ __forceinline__ void normalise(float (&v)[NCH][V], const int (&n)[NCH], float c_inv, float eps, int tpr, float *lds)
{
    float s[1] = {0.f};
    if (LAYER) {
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += v[k][e];
        team_sums(s, tpr, lds);
        const float mean = s[0] * c_inv;
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) v[k][e] = FULL || e < n[k] ? v[k][e] - mean : 0.f;
        s[0] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) s[0] = fmaf(v[k][e], v[k][e], s[0]);
    team_sums(s, tpr, lds);
    const float inv = 1.0f / sqrtf(fmaf(s[0], c_inv, eps));
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) v[k][e] *= inv;
}

// 200704 x 64, LayerNorm twice, gate and scale: 22.3 us among other calls for 103 MB, 4.6 TB/s (24 in a trace, 4.2); one row of 768 2.8 us.
template <typename E, bool LAYER, bool POST, int V, int NCH, bool FULL>
__global__ __launch_bounds__(kMaxTeam) void k_norm(NormIn I, E *R, E *N, long rows, unsigned per_group, int C, int tpr, float eps, bool vec)
{
    __shared__ float lds[kMaxTeam / 64];
    const int team = threadIdx.x / tpr, teams = blockDim.x / tpr, t = threadIdx.x % tpr;
    const float c_inv = 1.0f / (float)C;
    int n[NCH];
    float scale[NCH][V], gamma[NCH][V], beta[NCH][V], pg[POST ? NCH : 1][V], pb[POST ? NCH : 1][V];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
        const int c0 = V * (t + k * tpr);
        n[k] = C - c0;
        load_vector(I.scale, c0, n[k], 1.f, scale[k]);
        load_vector(I.gamma, c0, n[k], 0.f, gamma[k]);
        load_vector(I.beta, c0, n[k], 0.f, beta[k]);
        if constexpr (POST) {
            load_vector(I.post_gamma, c0, n[k], 0.f, pg[k]);
            load_vector(I.post_beta, c0, n[k], 0.f, pb[k]);
        }
    }
    Raw<E, V> x0[NCH], y0[NCH], g0[NCH];
    auto fetch = [&](long first) {
        const long row = min(first + team, rows - 1);
        const size_t at = (size_t)row * C + V * t;
#pragma unroll
        for (int k = 0; k < NCH; ++k) x0[k] = load<FULL, E, V>((const E *)I.X + at + V * k * tpr, n[k], vec);
        if (!I.Y) return;
#pragma unroll
        for (int k = 0; k < NCH; ++k) y0[k] = load<FULL, E, V>((const E *)I.Y + at + V * k * tpr, n[k], vec);
        if (!I.gate) return;
        const size_t group = (unsigned)row / per_group;
#pragma unroll
        for (int k = 0; k < NCH; ++k) g0[k] = load<FULL, E, V>((const E *)I.gate + group * C + V * (t + k * tpr), n[k], vec);
    };
    // every workgroup walks the same number of rows for all its teams: they meet in team_sums()
    const long step = (long)gridDim.x * teams;
    long first = (long)blockIdx.x * teams;
    if (first >= rows) return;
    fetch(first);
    for (;;) {
        const bool mine = first + team < rows, more = first + step < rows;
        const size_t at = (size_t)(first + team) * C + V * t;
        float x[NCH][V], y[NCH][V], f[NCH][V];
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[k][e] = value(x0[k], e);
                if (I.Y) y[k][e] = value(y0[k], e);
                f[k][e] = I.Y && I.gate ? scale[k][e] * value(g0[k], e) : scale[k][e];
            }
        if (more) fetch(first + step);
        if (I.Y) {
            if constexpr (POST) {
                normalise<LAYER, FULL>(y, n, c_inv, eps, tpr, lds);
#pragma unroll
                for (int k = 0; k < NCH; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) y[k][e] = fmaf(y[k][e], pg[k][e], pb[k][e]);
            }
#pragma unroll
            for (int k = 0; k < NCH; ++k) {
#pragma unroll
                for (int e = 0; e < V; ++e) x[k][e] = fmaf(f[k][e], y[k][e], x[k][e]);
                if (mine) store<FULL>(R + at + V * k * tpr, x[k], n[k], vec);
            }
        }
        if (N) {
            normalise<LAYER, FULL>(x, n, c_inv, eps, tpr, lds);
#pragma unroll
            for (int k = 0; k < NCH; ++k) {
#pragma unroll
                for (int e = 0; e < V; ++e) x[k][e] = fmaf(x[k][e], gamma[k][e], beta[k][e]);
                if (mine) store<FULL>(N + at + V * k * tpr, x[k], n[k], vec);
            }
        }
        if (!more) return;
        first += step;
    }
}

template <typename E, bool LAYER, bool POST, int V, int NCH, bool FULL>
int launch(const NormSizes &S, const NormIn &I, void *R, void *N, const Team &T, hipStream_t st)
{
    // one round of workgroups, all with as many rows
    const long steps = (S.rows + T.teams() - 1) / T.teams(), at_once = V * NCH == 8 ? 1280 : 768, each = (steps + at_once - 1) / at_once;
    const unsigned blocks = (unsigned)((steps + each - 1) / each);
    k_norm<E, LAYER, POST, V, NCH, FULL><<<blocks, T.threads(), 0, st>>>(I, (E *)R, (E *)N, S.rows, (unsigned)S.per_group, S.C, T.tpr, S.eps, S.vec);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <typename E, bool LAYER, bool POST>
int pick(const NormSizes &S, const NormIn &I, void *R, void *N, hipStream_t st)
{
    const Team T(S.C, S.vec);
    if (T.nch == 3) return launch<E, LAYER, POST, 4, 3, true>(S, I, R, N, T, st);
    if (T.nch == 1) return T.full ? launch<E, LAYER, POST, 8, 1, true>(S, I, R, N, T, st) : launch<E, LAYER, POST, 8, 1, false>(S, I, R, N, T, st);
    return T.full ? launch<E, LAYER, POST, 8, 2, true>(S, I, R, N, T, st) : launch<E, LAYER, POST, 8, 2, false>(S, I, R, N, T, st);
}

}  // namespace

int norm_forward(const NormSizes &S, const NormIn &I, void *R, void *N, hipStream_t st)
{
    if (S.rows == 0) return BRA_OK;
    ProfScope prof(st, K_NORM);
    if (S.f32) {
        if (S.layer) return S.post ? pick<float, true, true>(S, I, R, N, st) : pick<float, true, false>(S, I, R, N, st);
        return S.post ? pick<float, false, true>(S, I, R, N, st) : pick<float, false, false>(S, I, R, N, st);
    }
    if (S.layer) return S.post ? pick<bf16_t, true, true>(S, I, R, N, st) : pick<bf16_t, true, false>(S, I, R, N, st);
    return S.post ? pick<bf16_t, false, true>(S, I, R, N, st) : pick<bf16_t, false, false>(S, I, R, N, st);
}

}  // namespace bra
