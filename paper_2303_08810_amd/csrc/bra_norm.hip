// Norms before and after a block with its gate and residual scale:
//     R = X + scale * gate[group] * post(Y),   N = norm(R) gamma + beta
// norm and post are LayerNorm or RMSNorm over a row's C channels.  One pass: X and Y are read once, R and N written once; the row
// stays in registers from the loads to the stores, its statistics are those of the float32 sum.  Bound by memory.
#include "bra_norm_dev.h"

namespace bra {

using namespace norm;

namespace {

// (x - mean) / sqrt(var + eps) or x / sqrt(mean of squares + eps), in place; n[k]: channels of chunk k that exist.
template <bool LAYER, int NCH>
__device__ __forceinline__ void normalise(float (&v)[NCH][8], const int (&n)[NCH], float c_inv, float eps, int tpr, float *lds)
{
    float s[1] = {0.f};
    if (LAYER) {
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += v[k][e];
        team_sums(s, tpr, lds);
        const float mean = s[0] * c_inv;
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = e < n[k] ? v[k][e] - mean : 0.f;
        s[0] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = fmaf(v[k][e], v[k][e], s[0]);
    team_sums(s, tpr, lds);
    const float inv = 1.0f / sqrtf(fmaf(s[0], c_inv, eps));
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[k][e] *= inv;
}

template <typename E, bool LAYER, bool POST, int NCH, bool VEC>
__global__ __launch_bounds__(kMaxTeam) void k_norm(NormIn I, E *R, E *N, long rows, unsigned per_group, int C, int tpr, float eps)
{
    __shared__ float lds[kMaxTeam / 64];
    const int team = threadIdx.x / tpr, teams = blockDim.x / tpr, t = threadIdx.x % tpr;
    const float c_inv = 1.0f / (float)C;
    int n[NCH];
    float scale[NCH][8], gamma[NCH][8], beta[NCH][8], pg[POST ? NCH : 1][8], pb[POST ? NCH : 1][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
        const int c0 = 8 * (t + k * tpr);
        n[k] = VEC ? (c0 < C ? 8 : 0) : C - c0;
        load_vector(I.scale, c0, n[k], 1.f, scale[k]);
        load_vector(I.gamma, c0, n[k], 0.f, gamma[k]);
        load_vector(I.beta, c0, n[k], 0.f, beta[k]);
        if constexpr (POST) {
            load_vector(I.post_gamma, c0, n[k], 0.f, pg[k]);
            load_vector(I.post_beta, c0, n[k], 0.f, pb[k]);
        }
    }
    // every workgroup walks the same number of rows for all its teams: they meet in team_sums()
    for (long first = (long)blockIdx.x * teams; first < rows; first += (long)gridDim.x * teams) {
        const bool mine = first + team < rows;
        const long row = mine ? first + team : rows - 1;
        const size_t at = (size_t)row * C + 8 * t;
        float x[NCH][8];
#pragma unroll
        for (int k = 0; k < NCH; ++k) load8<VEC>((const E *)I.X + at + 8 * k * tpr, n[k], x[k]);
        if (I.Y) {
            float y[NCH][8], g[NCH][8];
#pragma unroll
            for (int k = 0; k < NCH; ++k) load8<VEC>((const E *)I.Y + at + 8 * k * tpr, n[k], y[k]);
            if (I.gate) {
                const size_t group = (unsigned)row / per_group;
#pragma unroll
                for (int k = 0; k < NCH; ++k) load8<VEC>((const E *)I.gate + group * C + 8 * (t + k * tpr), n[k], g[k]);
            }
            if constexpr (POST) {
                normalise<LAYER, NCH>(y, n, c_inv, eps, tpr, lds);
#pragma unroll
                for (int k = 0; k < NCH; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[k][e] = fmaf(y[k][e], pg[k][e], pb[k][e]);
            }
#pragma unroll
            for (int k = 0; k < NCH; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[k][e] = fmaf(I.gate ? scale[k][e] * g[k][e] : scale[k][e], y[k][e], x[k][e]);
                if (mine) store8<VEC>(R + at + 8 * k * tpr, n[k], x[k]);
            }
        }
        if (!N) continue;
        normalise<LAYER, NCH>(x, n, c_inv, eps, tpr, lds);
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = fmaf(x[k][e], gamma[k][e], beta[k][e]);
            if (mine) store8<VEC>(N + at + 8 * k * tpr, n[k], x[k]);
        }
    }
}

template <typename E, bool LAYER, bool POST, int NCH>
int launch(const NormSizes &S, const NormIn &I, void *R, void *N, int tpr, hipStream_t st)
{
    const int threads = std::max(kThreads, tpr), teams = threads / tpr;
    const unsigned blocks = (unsigned)std::min((S.rows + teams - 1) / teams, 2048L);
    if (S.vec) k_norm<E, LAYER, POST, NCH, true><<<blocks, threads, 0, st>>>(I, (E *)R, (E *)N, S.rows, (unsigned)S.per_group, S.C, tpr, S.eps);
    else k_norm<E, LAYER, POST, NCH, false><<<blocks, threads, 0, st>>>(I, (E *)R, (E *)N, S.rows, (unsigned)S.per_group, S.C, tpr, S.eps);
    return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
}

template <typename E, bool LAYER, bool POST>
int pick(const NormSizes &S, const NormIn &I, void *R, void *N, hipStream_t st)
{
    const int tpr = team_size(S.C, 1);
    return tpr <= 64 ? launch<E, LAYER, POST, 1>(S, I, R, N, tpr, st) : launch<E, LAYER, POST, 2>(S, I, R, N, tpr / 2, st);
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
