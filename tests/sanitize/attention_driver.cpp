// The host side of bra_attention_* and bra_qk_norm_* as api_driver.cpp has it for the layer: size queries over the whole range of shapes, and calls that must be refused before
// anything is enqueued, in a build whose host code runs under AddressSanitizer and UndefinedBehaviorSanitizer.  No GPU is needed: no call here reaches a launch.  Exit
// status 0 means every code was as expected and no report was raised.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "../../include/bra.h"

static int failures = 0;
#define EXPECT(expr, code)                                                            \
    do {                                                                              \
        const int rc_ = (expr);                                                       \
        if (rc_ != (code)) { std::printf("%s -> %d, expected %d\n", #expr, rc_, (int)(code)); ++failures; } \
    } while (0)

static char *const kFake = (char *)(1ull << 40);
static bra_rows rows(int i, int64_t N, int64_t heads, int64_t d)
{
    return bra_rows{kFake + ((long)i << 50), N * heads * d, heads * d, d};
}

static void attention()
{
    size_t n = 0;
    const int32_t batches[] = {0, 1, 3, 64, 4099, 1 << 20, 1 << 28}, lengths[] = {0, 1, 31, 32, 33, 64, 100, 197, 256, 257, 1295, 8192, 65537, 1 << 20, 1 << 28};
    const int32_t heads[][2] = {{1, 1}, {12, 12}, {7, 1}, {32, 8}, {48, 3}, {65536, 1}, {65536, 65536}};
    long taken = 0, refused = 0;
    for (int dtype : {BRA_F32, BRA_BF16})
        for (int32_t B : batches)
            for (int32_t Nq : lengths)
                for (int32_t Nk : lengths)
                    for (auto &h : heads)
                        for (int32_t d : {8, 40, 64, 72, 96, 128}) {
                            const bra_attention_shape s = {B, Nq, Nk, h[0], h[1], d, dtype, (B + d) % 2, 0.f};
                            const bool ok = (int64_t)B * h[0] <= 1 << 30 && (int64_t)Nq * h[0] <= 1 << 30 && (int64_t)B * h[0] <= (1LL << 40) / (Nq > Nk ? (Nq ? Nq : 1) : (Nk ? Nk : 1));
                            ++(ok ? taken : refused);
                            const bra_rows q = rows(1, Nq, h[0], d), k = rows(2, Nk, h[1], d), v = rows(3, Nk, h[1], d), o = rows(4, Nq, h[0], d), g = rows(5, Nq, h[0], d), dq = rows(6, Nq, h[0], d),
                                           dk = rows(7, Nk, h[1], d), dv = rows(8, Nk, h[1], d);
                            float *lse = (float *)(kFake + (9l << 50));
                            for (int backward = 0; backward < 2; ++backward) {
                                n = 0;
                                EXPECT(backward ? bra_attention_backward_workspace_bytes(&s, &n) : bra_attention_workspace_bytes(&s, &n), ok ? BRA_OK : BRA_ERR_SHAPE);
                                if (n % 256) ++failures;
                                if (!ok || B == 0 || Nq == 0) continue;
                                // a byte less is refused; with enough of it, gradients (an output) where an input lies
                                if (n) EXPECT(backward ? bra_attention_backward(&s, &q, &k, &v, &o, lse, &g, nullptr, nullptr, &dq, &dk, &dv, kFake, n - 1, nullptr)
                                                       : bra_attention_forward(&s, &q, &k, &v, nullptr, nullptr, &o, lse, kFake, n - 1, nullptr), BRA_ERR_WORKSPACE);
                                EXPECT(backward ? bra_attention_backward(&s, &q, &k, &v, &o, lse, &g, nullptr, nullptr, &q, &dk, &dv, kFake, SIZE_MAX, nullptr)
                                                : bra_attention_forward(&s, &q, &k, &v, nullptr, nullptr, &q, lse, kFake, SIZE_MAX, nullptr), BRA_ERR_OVERLAP);
                            }
                        }
    if (taken < 10000 || refused < 1000) ++failures;
    const bra_attention_shape s = {2, 40, 50, 4, 2, 64, BRA_BF16, 0, 0.f};
    EXPECT(bra_attention_workspace_bytes(nullptr, &n), BRA_ERR_NULL);
    EXPECT(bra_attention_backward_workspace_bytes(&s, nullptr), BRA_ERR_NULL);
    for (bra_attention_shape bad : {bra_attention_shape{INT32_MIN, 1, 1, 1, 1, 8, 1, 0, 0.f}, bra_attention_shape{1, INT32_MAX, 1, 1, 1, 8, 1, 0, 0.f}, bra_attention_shape{1, 1, 1, INT32_MAX, 1, 8, 1, 0, 0.f},
                                    bra_attention_shape{1, 1, 1, 1, INT32_MIN, 8, 1, 0, 0.f}, bra_attention_shape{1, 1, 1, 1, 1, INT32_MIN, 1, 0, 0.f}, bra_attention_shape{1, 1, 1, 1, 1, 8, 1, 0, NAN},
                                    bra_attention_shape{1, 1, 1, 1, 1, 8, 1, 0, INFINITY}}) {
        EXPECT(bra_attention_workspace_bytes(&bad, &n), BRA_ERR_SHAPE);
        EXPECT(bra_attention_backward_workspace_bytes(&bad, &n), BRA_ERR_SHAPE);
    }
    const bra_rows fine = rows(1, 50, 4, 64);
    for (int64_t far : {INT64_MAX, INT64_MIN, (int64_t)1 << 60, (int64_t)-16})
        for (int which = 0; which < 3; ++which) {
            bra_rows bad = fine;
            (which == 0 ? bad.batch : which == 1 ? bad.token : bad.head) = far;
            EXPECT(bra_attention_forward(&s, &fine, &bad, &fine, nullptr, nullptr, &fine, nullptr, kFake, SIZE_MAX, nullptr), BRA_ERR_SHAPE);
            EXPECT(bra_attention_backward(&s, &fine, &fine, &fine, &fine, (float *)kFake, &fine, nullptr, nullptr, &fine, &bad, &fine, kFake, SIZE_MAX, nullptr), BRA_ERR_SHAPE);
        }
}

static void norms_and_rotation()
{
    size_t n = 0;
    const float *vec = (const float *)(kFake + (20l << 50));
    for (int dtype : {BRA_F32, BRA_BF16})
        for (int32_t B : {0, 1, 5, 1 << 14, 1 << 30, INT32_MAX})
            for (int32_t N : {0, 1, 7, 1295, 65536, 1 << 30, INT32_MAX})
                for (int32_t H : {1, 6, 32, 65536, INT32_MAX})
                    for (int32_t Hk : {0, 1, 8, INT32_MAX})
                        for (int32_t d : {8, 40, 64, 128})
                            for (int32_t turned : {0, 2, 6, d}) {
                                const bra_qk_norm_shape s = {B, N, H, Hk, d, turned, N ? N : 1, turned % 4 / 2, dtype, 1e-6f};
                                const int64_t most = 1 << 30, tokens = (int64_t)B * N, all = (int64_t)H + Hk;
                                const bool ok = tokens <= most && all <= most && tokens * all <= most;
                                EXPECT(bra_qk_norm_backward_workspace_bytes(&s, &n), ok ? BRA_OK : BRA_ERR_SHAPE);
                                if (!ok || !tokens) continue;
                                if (n % 256) ++failures;
                                const bra_rows q = rows(1, N, H, d), k = rows(2, N, Hk, d), gq = rows(3, N, H, d), gk = rows(4, N, Hk, d), dq = rows(5, N, H, d), dk = rows(6, N, Hk, d);
                                const bra_qk_norm_params p = {vec, Hk ? vec : nullptr, vec, vec, nullptr};
                                EXPECT(bra_qk_norm_backward(&s, &q, &k, &p, &gq, &gk, &dq, &dk, nullptr, nullptr, kFake, n - 1, nullptr), BRA_ERR_WORKSPACE);
                                EXPECT(bra_qk_norm_backward(&s, &q, &k, &p, &gq, &gk, &dq, &dk, (float *)vec, nullptr, kFake, SIZE_MAX, nullptr), BRA_ERR_OVERLAP);
                                bra_rows on = q;
                                on.data = (char *)q.data + 16;
                                if (tokens * H * d * (dtype == BRA_F32 ? 4 : 2) == 16) continue;         // all that there is lies before it
                                EXPECT(bra_qk_norm_forward(&s, &q, &k, &p, &on, &dk, nullptr), BRA_ERR_OVERLAP);
                            }
    EXPECT(bra_qk_norm_backward_workspace_bytes(nullptr, &n), BRA_ERR_NULL);
    for (bra_qk_norm_shape bad : {bra_qk_norm_shape{1, 1, INT32_MIN, 1, 8, 0, 1, 0, 1, 0.f}, bra_qk_norm_shape{1, 1, 1, INT32_MIN, 8, 0, 1, 0, 1, 0.f}, bra_qk_norm_shape{1, 1, 1, 1, 8, INT32_MIN, 1, 0, 1, 0.f},
                                  bra_qk_norm_shape{1, 1, 1, 1, INT32_MAX, INT32_MAX, 1, 0, 1, 0.f}, bra_qk_norm_shape{1, 1, 1, 1, 8, 0, 1, 0, 1, NAN}})
        EXPECT(bra_qk_norm_backward_workspace_bytes(&bad, &n), BRA_ERR_SHAPE);
}

int main()
{
    attention();
    norms_and_rotation();
    std::printf("%d unexpected results\n", failures);
    return failures ? 1 : 0;
}
