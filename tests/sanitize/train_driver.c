/* Sanitizer driver for the host side of the training entry points (test
 * infrastructure): every size and stride at the ends of its range, refused or
 * taken; the launches behind it do nothing.  Built and run by
 * tests/test_sanitizers_train.py against host code that carries AddressSanitizer and
 * UndefinedBehaviorSanitizer. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/reqat.h"

static int fails = 0;
#define EXPECT(call, ok)                                                              \
    do {                                                                              \
        reqat_status got_ = (call);                                                   \
        if ((got_ == REQAT_OK) != (ok)) {                                             \
            printf("line %d: %s -> %d, i %d\n", __LINE__, #call, (int)got_, i);       \
            ++fails;                                                                  \
        }                                                                             \
    } while (0)

#define P ((void *)(uintptr_t)(1u << 20)) /* addresses that nothing reads */
#define FAR ((void *)(uintptr_t)(INT64_C(1) << 62))
#define BIG (INT64_C(1) << 62)

static const int64_t ends[] = {INT64_MIN, -BIG, -1, 0, 1, 7, 8, 9, 32768, 32769, INT64_C(1) << 22, (INT64_C(1) << 22) + 1, INT64_C(1) << 23,
                               (INT64_C(1) << 23) + 1, INT64_C(1) << 30, (INT64_C(1) << 30) + 1, INT64_C(0x7FFFFFFF), INT64_C(0x80000000),
                               INT64_C(1) << 37, INT64_C(1) << 40, INT64_C(1) << 59, BIG, INT64_MAX};

static reqat_status policy(int64_t T, int64_t V, int64_t ld, void *grad, int64_t ldg, float temp)
{
    return reqat_policy_loss(P, REQAT_DT_F32, T, V, ld, P, P, P, P, P, 0.2f, 0.2f, 0.1f, temp, P, P, grad, ldg, P, 0);
}
static reqat_status policy_back(int64_t T, int64_t V, int64_t ld, int64_t ldg)
{
    return reqat_policy_loss_backward(P, REQAT_DT_BF16, T, V, ld, P, P, 1.0f, 0, FAR, ldg, 0);
}
static reqat_status norm(int64_t rows, int64_t cols, int64_t ldx, int64_t ldy)
{
    return reqat_layer_norm(P, REQAT_DT_F32, rows, cols, ldx, P, P, REQAT_DT_BF16, 1e-6f, 1, FAR, ldy, P, 0);
}
static reqat_status norm_back(int64_t rows, int64_t cols, int64_t lddy, int64_t ldx, int64_t lddx)
{
    return reqat_layer_norm_backward(P, lddy, P, ldx, REQAT_DT_F32, rows, cols, P, REQAT_DT_F32, P, 1, FAR, lddx, P, P, P, 0);
}
static reqat_status embed(int64_t T, int64_t V, int64_t D, int64_t ldt, int64_t ldo)
{
    return reqat_embedding(P, T, P, REQAT_DT_F32, V, D, ldt, 1.0f, FAR, ldo, 0);
}
static reqat_status embed_back(int64_t T, int64_t V, int64_t D, int64_t lddy, int64_t ldt, int add)
{
    return reqat_embedding_backward(P, REQAT_DT_F32, lddy, P, T, V, D, 1.0f, FAR, REQAT_DT_F32, ldt, add, P, 0);
}

int main(void)
{
    const int n = (int)(sizeof ends / sizeof *ends);
    const int64_t M22 = INT64_C(1) << 22, M30 = INT64_C(1) << 30, M59 = INT64_C(1) << 59;
    int i, j;
    for (i = 0; i < n; ++i) {
        const int64_t e = ends[i];
        /* sizes, rows as far apart as their limit allows */
        EXPECT(policy(e, 100, 100, 0, 0, 1.0f), e >= 0 && e <= M22);
        EXPECT(policy(4, e, M30, 0, 0, 1.0f), e > 0 && e <= M30);
        EXPECT(policy(e, 100, M59 >> 22, FAR, M59 >> 22, 1.0f), e >= 0 && e <= M22);
        EXPECT(policy_back(e, 100, 100, 100), e >= 0 && e <= M22);
        EXPECT(policy_back(4, e, M30, M30), e > 0 && e <= M30);
        EXPECT(norm(e, 64, 64, 64), e >= 0 && e <= INT64_C(1) << 40);
        EXPECT(norm(3, e, 32768, 32768), e > 0 && e <= 32768);
        EXPECT(norm_back(e, 64, 64, 64, 64), e >= 0 && e <= INT64_C(1) << 40);
        EXPECT(norm_back(3, e, 32768, 32768, 32768), e > 0 && e <= 32768);
        EXPECT(embed(e, 100, 64, 64, 64), e >= 0 && e <= M22);
        EXPECT(embed(5, e, 64, 64, 64), e >= 0 && e <= INT64_C(1) << 23);
        EXPECT(embed(5, 100, e, M30, M30), e > 0 && e <= 1 << 20);
        EXPECT(embed_back(e, 100, 64, 64, 64, 0), e >= 0 && e <= M22);
        EXPECT(embed_back(5, e, 64, 64, 64, 1), e >= 0 && e <= INT64_C(1) << 23);
        EXPECT(embed_back(5, 100, e, M30, M30, 0), e > 0 && e <= 1 << 20);
        /* strides: one row, several, none (whose stride says nothing but is no smaller than a row) */
        for (j = 0; j < 3; ++j) {
            const int64_t rows = j == 0 ? 0 : (j == 1 ? 1 : 4), most = rows == 0 ? INT64_MAX : M59 / rows;
            const int ok = e >= 64 && e <= most;
            EXPECT(policy(rows, 64, e, 0, 0, 1.0f), ok);
            EXPECT(policy(rows, 64, 64, FAR, e, 1.0f), ok);
            EXPECT(policy_back(rows, 64, e, 64), ok);
            EXPECT(policy_back(rows, 64, 64, e), ok);
            EXPECT(norm(rows, 64, e, 64), ok);
            EXPECT(norm(rows, 64, 64, e), ok);
            EXPECT(norm_back(rows, 64, e, 64, 64), ok);
            EXPECT(norm_back(rows, 64, 64, e, 64), ok);
            EXPECT(norm_back(rows, 64, 64, 64, e), ok);
            EXPECT(embed(5, rows, 64, e, 64), ok);
            EXPECT(embed(rows, 100, 64, 64, e), ok);
            EXPECT(embed_back(rows, 100, 64, e, 64, 0), ok);
            EXPECT(embed_back(rows, 100, 64, e, 64, 1), ok);
            EXPECT(embed_back(5, rows, 64, 64, e, 0), ok);
        }
        /* workspace queries take anything */
        for (j = 0; j < n; ++j) {
            (void)reqat_policy_loss_workspace_bytes(REQAT_DT_BF16, e, ends[j]);
            (void)reqat_policy_loss_workspace_bytes(REQAT_DT_F32, e, ends[j]);
            (void)reqat_layer_norm_workspace_bytes(REQAT_DT_F32, e, ends[j], 1);
            (void)reqat_layer_norm_workspace_bytes(REQAT_DT_BF16, e, ends[j], 0);
            (void)reqat_embedding_workspace_bytes(e, ends[j], 64);
            (void)reqat_embedding_workspace_bytes(e, 64, ends[j]);
        }
        {
            reqat_adamw_tensor t[2] = {{P, P, P, P, P, P, P, 10}, {P, P, P, P, P, P, P, 10}};
            reqat_adamw_hyper h = {1e-3, 0.9, 0.999, 1e-8, 0.01, 1};
            t[1].n = e;
            EXPECT(reqat_adamw_step(t, 2, REQAT_DT_F32, REQAT_DT_BF16, 8, &h, P, 0, 0), e >= 0 && e <= INT64_C(1) << 34);
            t[1].n = 10;
            EXPECT(reqat_adamw_step(t, 2, REQAT_DT_F32, REQAT_DT_F32, (int)(e & 0xFFFF), &h, P, P, 0), (e & 0xFFFF) == 8);
            h.step = e;
            EXPECT(reqat_adamw_step(t, 2, REQAT_DT_BF16, REQAT_DT_F32, 32, &h, 0, 0, 0), e >= 1);
            EXPECT(reqat_adamw_step(t, 2, REQAT_DT_BF16, REQAT_DT_F32, 32, &h, 0, P, 0), 1);
            EXPECT(reqat_adamw_coefficients(&h, 0, P, P, 0), 1);
            EXPECT(reqat_adamw_moments(P, P, P, P, e, P, P, 0), e >= 0 && e <= INT64_C(1) << 33);
        }
    }
    i = 0;
    {
        const double bad[] = {NAN, INFINITY, -INFINITY, -1.0, 1.0, 1e308, 1e-308};
        for (i = 0; i < 7; ++i) {
            reqat_adamw_tensor t = {P, P, P, P, P, P, 0, 10};
            reqat_adamw_hyper h = {bad[i], 0.9, 0.999, 1e-8, 0.01, 1};
            EXPECT(reqat_adamw_step(&t, 1, REQAT_DT_F32, REQAT_DT_F32, 32, &h, 0, 0, 0), i >= 3);
            h.lr = 1e-3;
            h.beta1 = bad[i];
            EXPECT(reqat_adamw_step(&t, 1, REQAT_DT_F32, REQAT_DT_F32, 32, &h, 0, 0, 0), i == 6);
            h.beta1 = 0.0;
            h.beta2 = bad[i];
            EXPECT(reqat_adamw_step(&t, 1, REQAT_DT_F32, REQAT_DT_F32, 32, &h, 0, 0, 0), i == 6);
            h.beta2 = 0.0;
            h.eps = bad[i];
            EXPECT(reqat_adamw_step(&t, 1, REQAT_DT_F32, REQAT_DT_F32, 32, &h, 0, 0, 0), i >= 4);
            EXPECT(policy(4, 100, 100, 0, 0, (float)bad[i]), i == 4);
        }
    }
    if (!fails) printf("train driver ok\n");
    return fails != 0;
}
