// AdamW, many tensors in one launch (kPerLaunch of them; the table travels in the kernel's arguments, so that a captured graph
// holds it and nothing has to be copied first).
//     m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
//     p = p (1 - lr decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
// One pass, bound by memory: p, m, v read and written once, g read once.  A workgroup has kChunk consecutive values of one tensor, a
// thread 8 of them.  Sums and products are rounded one by one (no contraction), as the formula reads.
//
// States in 8 bits: e4m3 codes with one power of two per 32 values (4 threads), the smallest with which the largest value is at most 448.
// The second moment is kept as its root, which halves the range that the codes have to span; a root that is not zero takes the smallest
// code at least, so that a small first moment is never divided by eps alone.
#include "bra_adamw.h"
#include "bra_mfma_dev.h"

#include <math.h>

#include <algorithm>
#include <vector>

namespace bra {

using namespace mfma;

namespace {

constexpr int kPerLaunch = 72;
constexpr int kChunk = 2048;
constexpr int kBlock = BRA_ADAMW_BLOCK;

struct Entry {
    void *param;
    const void *grad;
    bf16_t *copy;
    long n;
    unsigned place;         // in blocks of the state
    unsigned first;         // workgroup
    float keep;             // 1 - lr * decay
    unsigned kinds;         // bit 0: param is bf16, 1: grad is bf16, 2: whole 16-byte pieces
};
struct Table {
    Entry e[kPerLaunch];
    int count;
};

__device__ __forceinline__ void get8(const void *base, long at, bool bf16, bool vec, int n, float (&v)[8])
{
    if (vec && n >= 8) {
        if (bf16) {
            const u32x4 t = *(const u32x4 *)((const bf16_t *)base + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[2 * e] = bf16_lo(t[e]); v[2 * e + 1] = bf16_hi(t[e]); }
        } else {
            const f32x4 a = *(const f32x4 *)((const float *)base + at), b = *(const f32x4 *)((const float *)base + at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e >= n ? 0.f : bf16 ? bf16_to_f32(((const bf16_t *)base)[at + e]) : ((const float *)base)[at + e];
}

__device__ __forceinline__ void put8(void *base, long at, bool bf16, bool vec, int n, const float (&v)[8])
{
    if (vec && n >= 8) {
        if (bf16) *(u32x4 *)((bf16_t *)base + at) = __builtin_bit_cast(u32x4, pack8(v));
        else {
            *(f32x4 *)((float *)base + at) = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4 *)((float *)base + at + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e >= n) continue;
        if (bf16) ((bf16_t *)base)[at + e] = f32_to_bf16(v[e]);
        else ((float *)base)[at + e] = v[e];
    }
}

// What a state holds is code * 2^(scale - 127), exact, as the scale's own conversion to float32 has it: here, on the CPU, and with any math library.
__device__ __forceinline__ float power_of_two(unsigned scale) { return __builtin_bit_cast(float, scale ? scale << 23 : 0x400000u); }

// Codes are formed with powers of two as torch.ldexp has them on this GPU, by powf, which is a unit of float32 low for 41 of 254 exponents (2^16 to 2^20 among
// them): a value half way between two codes goes to the lower one there, not to the even one, 5 codes in 10000.  A state that a program forms
// with torch.ldexp then has the step's codes.  A workgroup forms the powers once, a thread one of them, while its loads are on their way.
constexpr int kPowers = 256;

__device__ __forceinline__ void decode8(u32x2 codes, unsigned scale, float (&v)[8])
{
    const float by = power_of_two(scale);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[w], true);
        v[4 * w] = a[0] * by; v[4 * w + 1] = a[1] * by; v[4 * w + 2] = b[0] * by; v[4 * w + 3] = b[1] * by;
    }
}

// The codes of this thread's 8 values and the scale of the 32 that 4 threads hold.
template <bool ROOT>
__device__ __forceinline__ u32x2 encode8(const float (&v)[8], const float *powers, unsigned &scale)
{
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
    most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, most), 0xB1, 0xf, 0xf, true)));
    most = fmaxf(most, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, most), 0x4E, 0xf, 0xf, true)));
    const unsigned bits = __builtin_bit_cast(unsigned, most);
    const int e2 = max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u), -126);       // at most 120
    scale = (unsigned)(e2 + 127);
    const float by = powers[127 - e2];
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        q[e] = v[e] * by;
        if (ROOT && q[e] > 0.f) q[e] = fmaxf(q[e], 0x1p-9f);
    }
    u32x2 codes;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w], q[4 * w + 1], 0, false);
        codes[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * w + 2], q[4 * w + 3], c, true);
    }
    return codes;
}

// 57 million values with 8-bit states, float32 weights and bf16 copies: 190 us for 0.92 GB, 4.8 TB/s, as a large copy reaches; 11 tensors of 43136 values
// together 4.4 us.
template <int BITS>
__global__ __launch_bounds__(256) void k_adamw(Table T, AdamwSteps A, void *__restrict__ moments, void *__restrict__ squares, unsigned char *__restrict__ scales,
                                               unsigned char *__restrict__ root_scales)
{
#pragma clang fp contract(off)
    int lo = 0, hi = T.count - 1;           // the last entry that begins at or before this workgroup
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (T.e[mid].first <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const Entry &E = T.e[lo];
    __shared__ float powers[BITS == 8 ? kPowers : 1];
    const long i = (long)(blockIdx.x - E.first) * kChunk + 8 * threadIdx.x;
    const bool live = i < (E.n + kBlock - 1) / kBlock * kBlock;     // whole blocks: 4 threads go on or stay behind together
    const int n = (int)max(0L, min(E.n - i, 8L));
    const bool pb = E.kinds & 1, gb = E.kinds & 2, vec = E.kinds & 4;
    float p[8], g[8], m[8], v[8];
    const long at = (long)E.place * kBlock + i;
    u32x2 mc = {0u, 0u}, vc = {0u, 0u};
    unsigned ms = 0, vs = 0;
    if (live) {
        get8(E.param, i, pb, vec, n, p);
        get8(E.grad, i, gb, vec, n, g);
        if (BITS == 32) {
            get8(moments, at, false, true, 8, m);
            get8(squares, at, false, true, 8, v);
        } else {
            mc = *(const u32x2 *)((const unsigned char *)moments + at);
            vc = *(const u32x2 *)((const unsigned char *)squares + at);
            ms = scales[at / kBlock];
            vs = root_scales[at / kBlock];
        }
    }
    if constexpr (BITS == 8) {
        powers[threadIdx.x] = powf(2.0f, (float)((int)threadIdx.x - 127));
        __syncthreads();
    }
    if (!live) return;
    if (BITS == 8) {
        decode8(mc, ms, m);
        decode8(vc, vs, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * v[e];
    }
    const float away = A.scalars ? A.scalars[0] : A.away, bias = A.scalars ? A.scalars[1] : A.root;
    if (A.grad_scale) {
        const float s = *A.grad_scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = e < n ? g[e] * s : 0.f;       // (what lies behind a tensor's end stays 0 whatever s is)
    }
    float root[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        m[e] = A.beta1 * m[e] + A.rest1 * g[e];
        v[e] = A.beta2 * v[e] + A.rest2 * (g[e] * g[e]);
        root[e] = sqrtf(v[e]);
        p[e] = p[e] * E.keep - away * (m[e] / (root[e] * bias + A.eps));
    }
    put8(E.param, i, pb, vec, n, p);
    if (E.copy) put8(E.copy, i, true, vec, n, p);
    if (BITS == 32) {
        put8(moments, at, false, true, 8, m);
        put8(squares, at, false, true, 8, v);
    } else {
        unsigned s;
        *(u32x2 *)((unsigned char *)moments + at) = encode8<false>(m, powers, s);
        if (threadIdx.x % 4 == 0) scales[at / kBlock] = (unsigned char)s;
        *(u32x2 *)((unsigned char *)squares + at) = encode8<true>(root, powers, s);
        if (threadIdx.x % 4 == 0) root_scales[at / kBlock] = (unsigned char)s;
    }
}

__global__ void k_adamw_scalars(const int32_t *step, double lr, double beta1, double beta2, float *out)
{
    const double t = (double)*step;
    out[0] = (float)(lr / (1.0 - pow(beta1, t)));
    out[1] = (float)(1.0 / sqrt(1.0 - pow(beta2, t)));
}

}  // namespace

int adamw_step(const bra_adamw_tensor *tensors, int count, const bra_adamw_args &A, hipStream_t st)
{
    AdamwSteps S{(float)A.beta1, (float)(1.0 - A.beta1), (float)A.beta2, (float)(1.0 - A.beta2), (float)A.eps, 0.f, 0.f, nullptr, A.grad_scale};
    ProfScope prof(st, K_ADAMW);
    if (A.step_device) {
        k_adamw_scalars<<<1, 1, 0, st>>>(A.step_device, A.lr, A.beta1, A.beta2, A.scalars);
        if (hipGetLastError() != hipSuccess) return BRA_ERR_LAUNCH;
        S.scalars = A.scalars;
    } else {
        S.away = (float)(A.lr / (1.0 - pow(A.beta1, (double)A.step)));
        S.root = (float)(1.0 / sqrt(1.0 - pow(A.beta2, (double)A.step)));
    }
    Table T;
    T.count = 0;
    unsigned blocks = 0;
    unsigned long place = 0;
    auto launch = [&]() -> int {
        if (!T.count) return BRA_OK;
        if (A.bits == 32) k_adamw<32><<<blocks, 256, 0, st>>>(T, S, A.exp_avg, A.exp_avg_sq, nullptr, nullptr);
        else k_adamw<8><<<blocks, 256, 0, st>>>(T, S, A.exp_avg, A.exp_avg_sq, (unsigned char *)A.exp_avg_scale, (unsigned char *)A.exp_avg_sq_scale);
        T.count = 0;
        blocks = 0;
        return hipGetLastError() == hipSuccess ? BRA_OK : BRA_ERR_LAUNCH;
    };
    for (int i = 0; i < count; ++i) {
        const bra_adamw_tensor &t = tensors[i];
        const unsigned long here = place;
        place += (unsigned long)((t.n + kBlock - 1) / kBlock);
        if (!t.n || !t.grad) continue;
        const unsigned long chunks = (unsigned long)((t.n + kChunk - 1) / kChunk);
        if (T.count == kPerLaunch || blocks + chunks > 0xffffffu) {        // (2^32 threads and more cannot be launched)
            const int rc = launch();
            if (rc != BRA_OK) return rc;
        }
        const bool vec = ((uintptr_t)t.param | (uintptr_t)t.grad | (uintptr_t)t.copy) % 16 == 0;
        T.e[T.count++] = Entry{t.param, t.grad, (bf16_t *)t.copy, t.n, (unsigned)here, blocks, (float)(1.0 - A.lr * (double)t.weight_decay),
                               (unsigned)(t.param_dtype == BRA_BF16) | (unsigned)(t.grad_dtype == BRA_BF16) << 1 | (unsigned)vec << 2};
        blocks += (unsigned)chunks;
    }
    return launch();
}

}  // namespace bra
