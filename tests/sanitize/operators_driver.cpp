// The host side of bra_ffn_*, bra_norm_* and bra_adamw_step as api_driver.cpp has it for the layer: size queries over the whole range of shapes, and calls
// that must be refused before anything is enqueued, in a build whose host code runs under AddressSanitizer and UndefinedBehaviorSanitizer.  No
// GPU is needed: no call here reaches a launch.  Exit status 0 means every code was as expected and no report was raised.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "../../include/bra.h"

static int failures = 0;
#define EXPECT(expr, code)                                                            \
    do {                                                                              \
        const int rc_ = (expr);                                                       \
        if (rc_ != (code)) { std::printf("%s -> %d, expected %d\n", #expr, rc_, (int)(code)); ++failures; } \
    } while (0)

static void gated_block()
{
    void *fake = (void *)4096;
    float *vec = (float *)fake;
    size_t n = 0;
    const int64_t tokens[] = {0, 1, 8, 33, 128, 129, 700, 2001, 12544, 65535, 1 << 20, (1 << 30) - 1, 1 << 30};
    const int32_t widths[] = {1, 7, 8, 64, 99, 256, 771, 1024, 4096, 1 << 17, 1 << 20};
    for (int dtype : {BRA_F32, BRA_BF16})
        for (int64_t M : tokens)
            for (int32_t C : widths)
                for (int32_t h : widths) {
                    const bra_ffn_shape s = {M, C, h, dtype, BRA_GELU};
                    for (int backward = 0; backward < 2; ++backward) {
                        EXPECT(backward ? bra_ffn_backward_workspace_bytes(&s, &n) : bra_ffn_workspace_bytes(&s, &n), BRA_OK);
                        if (n % 256) ++failures;
                        // a byte less is refused (no tokens: nothing to do in the forward)
                        if (n == 0 || (!backward && M == 0) || (backward && M == 1 << 30)) continue;
                        EXPECT(backward ? bra_ffn_backward(&s, fake, fake, vec, fake, nullptr, fake, fake, fake, fake, fake, fake, BRA_F32, fake, n - 1, nullptr)
                                        : bra_ffn_forward(&s, fake, fake, vec, fake, vec, fake, fake, fake, n - 1, nullptr), BRA_ERR_WORKSPACE);
                    }
                }
    bra_ffn_shape s = {64, 64, 128, BRA_BF16, BRA_SILU};
    EXPECT(bra_ffn_workspace_bytes(nullptr, &n), BRA_ERR_NULL);
    EXPECT(bra_ffn_workspace_bytes(&s, nullptr), BRA_ERR_NULL);
    EXPECT(bra_ffn_forward(&s, fake, nullptr, nullptr, fake, nullptr, fake, nullptr, fake, SIZE_MAX, nullptr), BRA_ERR_NULL);
    EXPECT(bra_ffn_forward(&s, (char *)fake + 2, fake, nullptr, fake, nullptr, fake, nullptr, fake, SIZE_MAX, nullptr), BRA_ERR_ALIGN);
    for (bra_ffn_shape bad : {bra_ffn_shape{-1, 64, 128, 1, 0}, bra_ffn_shape{INT64_MAX, 64, 128, 1, 0}, bra_ffn_shape{64, INT32_MAX, 128, 1, 0}, bra_ffn_shape{64, 64, INT32_MIN, 1, 0}}) {
        EXPECT(bra_ffn_workspace_bytes(&bad, &n), BRA_ERR_SHAPE);
        EXPECT(bra_ffn_backward_workspace_bytes(&bad, &n), BRA_ERR_SHAPE);
    }
}

static void norms()
{
    void *fake = (void *)4096;
    size_t n = 0;
    for (int dtype : {BRA_F32, BRA_BF16})
        for (int64_t per : {0, 1, 2, 17, 1000, 1 << 20})
            for (int32_t groups : {1, 3, 700, 1 << 10, INT32_MAX})
                for (int32_t C : {1, 8, 24, 64, 99, 768, 1000, 8192}) {
                    const bra_norm_shape s = {per * groups, groups, C, dtype, BRA_RMSNORM, 1e-6f};
                    const bool ok = s.rows <= 1 << 30;
                    EXPECT(bra_norm_backward_workspace_bytes(&s, 1, &n), ok ? BRA_OK : BRA_ERR_SHAPE);
                    if (!ok || !per) continue;
                    const bra_norm_params p = {(const float *)fake, nullptr, (const float *)fake, nullptr, nullptr, fake};
                    bra_norm_grads g = {fake, fake, fake, nullptr, nullptr, nullptr, nullptr, nullptr};
                    EXPECT(bra_norm_backward(&s, fake, fake, &p, fake, nullptr, &g, fake, 0, nullptr), BRA_ERR_WORKSPACE);
                    g.dY = nullptr;
                    EXPECT(bra_norm_backward(&s, fake, fake, &p, fake, nullptr, &g, fake, SIZE_MAX, nullptr), BRA_ERR_NULL);
                }
    for (bra_norm_shape bad : {bra_norm_shape{INT64_MAX, 1, 64, 1, 0, 0.f}, bra_norm_shape{10, 3, 64, 1, 0, 0.f}, bra_norm_shape{10, 0, 64, 1, 0, 0.f}, bra_norm_shape{10, INT32_MIN, 64, 1, 0, 0.f},
                               bra_norm_shape{10, 1, 64, 1, 0, NAN}})
        EXPECT(bra_norm_backward_workspace_bytes(&bad, 0, &n), BRA_ERR_SHAPE);
}

static void adamw()
{
    char *fake = (char *)4096;
    bra_adamw_args a = {};
    a.lr = 1e-3; a.beta1 = 0.9; a.beta2 = 0.999; a.eps = 1e-8; a.step = INT64_MAX; a.bits = 8;
    a.exp_avg = a.exp_avg_sq = a.exp_avg_scale = a.exp_avg_sq_scale = fake;
    // many tensors next to each other, the last of them over the first
    std::vector<bra_adamw_tensor> t;
    for (int i = 0; i < 1000; ++i) t.push_back({fake + 4096 * (1000 - i), fake, i % 2 ? fake + (1 << 28) + 2048 * i : nullptr, 1024, 0.1f, BRA_F32, BRA_BF16});
    t.push_back({fake + 4096 + 4092, fake, nullptr, 1, 0.f, BRA_F32, BRA_F32});
    EXPECT(bra_adamw_step(t.data(), (int32_t)t.size(), &a, nullptr), BRA_ERR_OVERLAP);
    t.back().n = INT64_MAX;
    EXPECT(bra_adamw_step(t.data(), (int32_t)t.size(), &a, nullptr), BRA_ERR_SHAPE);
    for (auto &e : t) { e.n = 1LL << 34; e.grad = nullptr; }
    EXPECT(bra_adamw_step(t.data(), 5, &a, nullptr), BRA_ERR_SHAPE);            // 5 x 2^29 blocks
    EXPECT(bra_adamw_step(t.data(), 4, &a, nullptr), BRA_OK);                   // nothing to do
    a.step = 0;
    EXPECT(bra_adamw_step(t.data(), 4, &a, nullptr), BRA_ERR_SHAPE);
    EXPECT(bra_adamw_step(nullptr, INT32_MIN, &a, nullptr), BRA_ERR_SHAPE);
}

int main()
{
    gated_block();
    norms();
    adamw();
    std::printf("%d unexpected results\n", failures);
    return failures ? 1 : 0;
}
