// What the kernels of the norms share (internal).
//
// A row is shared by a team of `tpr` threads (a power of two), thread t of it owning the chunks t, t + tpr, .. of V channels (NCH of
// them).  Teams of up to a wavefront add their partial sums by lane exchanges, larger ones by way of LDS too.
// Rows of 3 2^k channels go in three chunks of 4 per thread, others in one or two of 8, so that few lanes are idle.
// FULL: C = V NCH tpr and rows aligned to whole chunks, nothing to be masked.
#pragma once

#include "bra_mfma_dev.h"
#include "bra_norm.h"

#include <algorithm>

namespace bra {
namespace norm {

using namespace mfma;

constexpr int kThreads = 256;           // of a workgroup, unless a team is larger
constexpr int kMaxTeam = 512;

// A chunk of V values as it comes from memory.
template <typename E, int V>
struct Raw {
    static constexpr int kWords = V * (int)sizeof(E) / 4;
    unsigned w[kWords];
};

// vec: whole chunks, aligned; n: values that exist (others read as 0).
template <bool FULL, typename E, int V>
__device__ __forceinline__ Raw<E, V> load(const E *p, int n, bool vec)
{
    Raw<E, V> r;
    constexpr int W = Raw<E, V>::kWords;
    if (FULL || vec) {
        if (FULL || n > 0) {
            if constexpr (W == 2) {
                const u32x2 t = *(const u32x2 *)p;
                r.w[0] = t[0]; r.w[1] = t[1];
            } else
#pragma unroll
                for (int q = 0; q < W; q += 4) {
                    const u32x4 t = *(const u32x4 *)((const unsigned *)p + q);
#pragma unroll
                    for (int e = 0; e < 4; ++e) r.w[q + e] = t[e];
                }
        } else
#pragma unroll
            for (int q = 0; q < W; ++q) r.w[q] = 0;
        return r;
    }
#pragma unroll
    for (int q = 0; q < W; ++q) r.w[q] = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        if (e >= n) continue;
        if constexpr (sizeof(E) == 4) r.w[e] = __builtin_bit_cast(unsigned, p[e]);
        else r.w[e / 2] |= (unsigned)p[e] << (16 * (e % 2));
    }
    return r;
}

template <typename E, int V>
__device__ __forceinline__ float value(const Raw<E, V> &r, int e)
{
    if constexpr (sizeof(E) == 4) return __builtin_bit_cast(float, r.w[e]);
    else return e % 2 ? bf16_hi(r.w[e / 2]) : bf16_lo(r.w[e / 2]);
}

template <bool FULL, typename E, int V>
__device__ __forceinline__ void store(E *p, const float (&v)[V], int n, bool vec)
{
    if (FULL || vec) {
        if (!FULL && n <= 0) return;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int q = 0; q < V; q += 4) *(f32x4 *)(p + q) = f32x4{v[q], v[q + 1], v[q + 2], v[q + 3]};
        } else if constexpr (V == 4) *(u32x2 *)p = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else *(u32x4 *)p = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < n) store_from_f32(p + e, v[e]);
}

// V values of a float32 vector, `fill` where there is none and beyond its end.  Whole pieces where the vector is aligned: a lane's V reads of one
// element each, 4 V bytes apart from the next lane's, took longer than a few rows do (12544 x 256 24.2 us, in pieces 10.4; 200704 x 64 30 and 24).
template <int V>
__device__ __forceinline__ void load_vector(const float *p, int c0, int n, float fill, float (&v)[V])
{
    if (p && (uintptr_t)p % 16 == 0 && n >= V) {
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const f32x4 t = *(const f32x4 *)(p + c0 + q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[q + e] = t[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = p && e < n ? p[c0 + e] : fill;
}

// x + x of the lane 16 (32) further on, and before.
__device__ __forceinline__ float add_16(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float add_32(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Sums of K values over a team's threads, for every thread of it.  lds: K floats for each wavefront of the workgroup; the whole workgroup
// calls it where a team is larger than a wavefront.
template <int K>
__device__ __forceinline__ void team_sums(float (&v)[K], int tpr, float *lds)
{
    auto add = [&](auto f) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = f(v[k]);
    };
    if (tpr > 1) add([](float x) { return dpp_fadd<0xB1>(x); });        // lane ^ 1
    if (tpr > 2) add([](float x) { return dpp_fadd<0x4E>(x); });        // lane ^ 2
    if (tpr > 4) add([](float x) { return dpp_fadd<0x141>(x); });       // mirrored halves of 8: the other 4
    if (tpr > 8) add([](float x) { return dpp_fadd<0x140>(x); });       // mirrored rows of 16: the other 8
    if (tpr > 16) add(add_16);
    if (tpr > 32) add(add_32);
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

// How a row of C channels goes to a team; `whole`: rows and pointers are aligned to 16 bytes.
struct Team {
    int V, nch, tpr;
    bool full;
    Team(int C, bool whole)
    {
        for (int t = 1; whole && t <= 64; t *= 2)
            if (C == 12 * t) {
                V = 4; nch = 3; tpr = t; full = true;
                return;
            }
        V = 8;
        int t = 1;
        while (8 * t < C) t *= 2;
        nch = t <= 64 ? 1 : 2;
        tpr = t / nch;
        full = whole && C == V * nch * tpr;
    }
    int threads() const { return std::max(kThreads, tpr); }
    int teams() const { return threads() / tpr; }
};

}  // namespace norm
}  // namespace bra
