// What the kernels of the norms share (internal).
//
// A row is shared by a team of `tpr` threads (a power of two), thread t of it owning the 8-channel chunks t, t + tpr, .. (NCH of
// them).  Teams of up to a wavefront add their partial sums by lane exchanges, larger ones (C > 512 NCH) by way of LDS too.
// VEC: rows are whole 16-byte pieces; otherwise they are read by elements.
#pragma once

#include "bra_mfma_dev.h"
#include "bra_norm.h"

namespace bra {
namespace norm {

using namespace mfma;

constexpr int kThreads = 256;           // of a workgroup, unless a team is larger
constexpr int kMaxTeam = 512;

template <bool VEC>
__device__ __forceinline__ void load8(const bf16_t *p, int n, float (&v)[8])
{
    if (VEC) {
        const u32x4 t = n > 0 ? *(const u32x4 *)p : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(t[e]); v[2 * e + 1] = bf16_hi(t[e]); }
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? bf16_to_f32(p[e]) : 0.f;
}
template <bool VEC>
__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8])
{
    if (VEC) {
        const f32x4 z = {0.f, 0.f, 0.f, 0.f}, a = n > 0 ? *(const f32x4 *)p : z, b = n > 0 ? *(const f32x4 *)(p + 4) : z;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
}
template <bool VEC>
__device__ __forceinline__ void store8(bf16_t *p, int n, const float (&v)[8])
{
    if (VEC) {
        if (n > 0) *(u32x4 *)p = __builtin_bit_cast(u32x4, pack8(v));
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = f32_to_bf16(v[e]);
}
template <bool VEC>
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8])
{
    if (VEC) {
        if (n > 0) {
            *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = v[e];
}

// 8 values of a float32 vector (aligned to its elements only), `fill` where there is none and beyond its end.
__device__ __forceinline__ void load_vector(const float *p, int c0, int n, float fill, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p && e < n ? p[c0 + e] : fill;
}

// Sums of K values over a team's threads, for every thread of it.  lds: K floats for each wavefront of the workgroup; the whole workgroup
// calls it where a team is larger than a wavefront.
template <int K>
__device__ __forceinline__ void team_sums(float (&v)[K], int tpr, float *lds)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (tpr > 1) v[k] = dpp_fadd<0xB1>(v[k]);       // lane ^ 1
        if (tpr > 2) v[k] = dpp_fadd<0x4E>(v[k]);       // lane ^ 2
        if (tpr > 4) v[k] = dpp_fadd<0x141>(v[k]);      // mirrored halves of 8: the other 4
        if (tpr > 8) v[k] = dpp_fadd<0x140>(v[k]);      // mirrored rows of 16: the other 8
        if (tpr > 16) v[k] += __shfl_xor(v[k], 16);
        if (tpr > 32) v[k] += __shfl_xor(v[k], 32);
    }
    if (tpr <= 64) return;
    const int wave = threadIdx.x / 64, waves = tpr / 64, first = wave / waves * waves;
    __syncthreads();                                    // the last sums have been read
    if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[wave * K + k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = 0.f;
        for (int w = 0; w < waves; ++w) s += lds[(first + w) * K + k];
        v[k] = s;
    }
}

// Threads of a team with at most `most` chunks per thread.
inline int team_size(int C, int most)
{
    const int chunks = (C + 7) / 8;
    int t = 1;
    while (t * most < chunks) t *= 2;
    return t;
}

}  // namespace norm
}  // namespace bra
