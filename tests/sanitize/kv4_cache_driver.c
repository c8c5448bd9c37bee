/* Sanitizer driver for the host side of the paged KV4 cache's entry points
 * (test infrastructure): arguments that validation must reject before any HIP
 * call, sizes at the ends of their ranges among them, and the workspace query.
 * Built and run by tests/test_sanitizers_kv4_cache.py against host code that carries
 * AddressSanitizer and UndefinedBehaviorSanitizer. */
#include <stdint.h>
#include <stdio.h>

#include "../../include/reqat.h"

static int fails = 0;
#define EXPECT(call, st)                                                                        \
    do {                                                                                        \
        reqat_status got_ = (call);                                                             \
        if (got_ != (st)) {                                                                     \
            printf("line %d: %s -> %d, expected %d\n", __LINE__, #call, (int)got_, (int)(st)); \
            ++fails;                                                                            \
        }                                                                                       \
    } while (0)

#define P ((void *)(uintptr_t)(1u << 20)) /* never dereferenced: validation rejects before any use */
#define FAR ((void *)(uintptr_t)(1u << 28))
#define BIG (INT64_C(1) << 62)

static reqat_kv4_cache cache(void)
{
    reqat_kv4_cache c = {P, P, P, P, P, P, 0, 4, 16, 2, 128};
    return c;
}

static reqat_status append(const reqat_kv4_cache *c, int64_t T, void *q, int64_t ldq, int64_t heads, void *q_out,
                           int64_t ldq_out, int64_t ldk)
{
    return reqat_kv4_append(c, T, P, P, ldk, P, 256, q, ldq, heads, q_out, ldq_out, P, P, P, 9, 0);
}

static reqat_status attend(const reqat_kv4_cache *c, int64_t B, int64_t T, int64_t ldq, int64_t heads, void *q_start,
                           int64_t ldt, int64_t cols, int64_t max_q, int64_t max_kv, float scale, void *out, int64_t ldo,
                           void *ws)
{
    return reqat_kv4_attention(c, B, T, P, ldq, heads, q_start, P, P, ldt, cols, max_q, max_kv, 1, scale, out, ldo, 0, ws, 0);
}

int main(void)
{
    const int64_t ends[] = {INT64_MIN, -BIG, -1, 0, 1, 255, 65535, 65536, INT64_C(0x7FFFFFFF), INT64_C(0x80000000), BIG, INT64_MAX};
    const int n = (int)(sizeof ends / sizeof *ends);
    reqat_kv4_cache c = cache();
    int i, j, k, l;
    EXPECT(append(0, 4, P, 1024, 8, FAR, 1024, 256), REQAT_E_NULL);
    EXPECT(reqat_kv4_gather(0, 4, P, P, 256, P, 256, 0, 0), REQAT_E_NULL);
    EXPECT(attend(0, 2, 2, 1024, 8, 0, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_E_NULL);
    for (i = 0; i < n; ++i) {
        /* sizes of the cache: four pages of 16 tokens of 2 heads of 128 hold, the ends of the ranges do not */
        c = cache();
        c.page_size = ends[i];
        EXPECT(reqat_kv4_gather(&c, 4, P, P, 256, P, 256, 0, 0), ends[i] == 65536 ? REQAT_E_UNSUPPORTED : REQAT_E_SHAPE);
        c = cache();
        c.head_dim = ends[i];
        EXPECT(reqat_kv4_gather(&c, 4, P, P, 256, P, 256, 0, 0), REQAT_E_UNSUPPORTED);
        c = cache();
        c.num_pages = ends[i];
        if (ends[i] < 0 || ends[i] >= BIG) EXPECT(reqat_kv4_gather(&c, 4, P, P, 256, P, 256, 0, 0), REQAT_E_SHAPE);
        c = cache();
        c.kv_heads = ends[i];
        if (ends[i] <= 0 || ends[i] > 65535) EXPECT(reqat_kv4_gather(&c, 4, P, P, 256, P, 256, 0, 0), REQAT_E_SHAPE);
        c = cache();
        /* counts and strides of the calls */
        if (ends[i] < 0 || ends[i] > INT64_C(0x7FFFFFFF)) {
            EXPECT(append(&c, ends[i], P, 1024, 8, FAR, 1024, 256), REQAT_E_SHAPE);
            EXPECT(reqat_kv4_gather(&c, ends[i], P, P, 256, P, 256, 0, 0), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, ends[i], 1024, 8, P, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, 2, 1024, 8, 0, INT64_MAX, ends[i], 1, 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, 2, 1024, 8, 0, 4, 4, ends[i], 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, 2, 1024, 8, 0, 4, 4, 1, ends[i], 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
        }
        if (ends[i] < 0 || ends[i] > 65535) {
            EXPECT(append(&c, 4, P, 1024, ends[i], FAR, 1024, 256), REQAT_E_SHAPE);
            EXPECT(attend(&c, ends[i], 2, 1024, 8, P, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, 2, 1024, ends[i], 0, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
        }
        if (ends[i] < 256) {
            EXPECT(append(&c, 4, P, 1024, 8, FAR, 1024, ends[i]), REQAT_E_SHAPE);
            EXPECT(reqat_kv4_gather(&c, 4, P, P, ends[i], FAR, 256, 0, 0), REQAT_E_SHAPE);
            EXPECT(attend(&c, 2, 2, ends[i], 8, 0, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_E_SHAPE);
        }
    }
    /* outputs over inputs, near and with strides whose products pass 64 bits */
    EXPECT(append(&c, 4, FAR, 1024, 8, (char *)FAR + 64, 1024, 256), REQAT_E_UNSUPPORTED);
    EXPECT(append(&c, 4, FAR, 1024, 8, P, 1024, 256), REQAT_E_UNSUPPORTED);
    EXPECT(append(&c, 0x7FFFFFFF, FAR, BIG, 8, (char *)FAR + 64, BIG, 256), REQAT_E_UNSUPPORTED);
    EXPECT(append(&c, 0x7FFFFFFF, P, BIG, 8, FAR, 1024, BIG - 8), REQAT_E_UNSUPPORTED);
    EXPECT(reqat_kv4_gather(&c, 4, P, P, 256, (char *)P + 16, 256, 0, 0), REQAT_E_UNSUPPORTED);
    EXPECT(reqat_kv4_gather(&c, 0x7FFFFFFF, P, P, BIG, (char *)P + 16, BIG + 8, 0, 0), REQAT_E_UNSUPPORTED);
    EXPECT(attend(&c, 2, 2, 1024, 8, 0, 4, 4, 1, 64, 0.1f, (char *)P + 512, 1024, P), REQAT_E_UNSUPPORTED);
    EXPECT(attend(&c, 2, 0x7FFFFFFF, BIG, 8, P, 4, 4, 1, 64, 0.1f, (char *)P + 512, BIG, P), REQAT_E_UNSUPPORTED);
    EXPECT(attend(&c, 65535, 0x7FFFFFFF, 65536 * 128, 65534, P, 4, 4, 0x7FFFFFFF, 1 << 30, 0.1f, FAR, 65536 * 128, P),
           REQAT_E_SHAPE);
    EXPECT(attend(&c, 1, 1, 1024, 8, 0, 4, 4, 1, 1 << 20, 0.1f, FAR, 1024, 0), REQAT_E_NULL);
    EXPECT(attend(&c, 2, 2, 1024, 8, 0, 4, 4, 1, 64, 0.0f, FAR, 1024, P), REQAT_E_UNSUPPORTED);
    EXPECT(attend(&c, 0, 0, 1024, 8, 0, 4, 4, 1, 64, 0.1f, FAR, 1024, P), REQAT_OK);
    for (i = 0; i < n; ++i)
        for (j = 0; j < n; ++j)
            for (k = 0; k < n; ++k)
                for (l = 0; l < n; ++l)
                    if (reqat_kv4_attention_workspace_bytes(ends[i], ends[j], ends[j], ends[k], ends[l], 1, 128) > 8192u * 32u * 528u)
                        ++fails;
    if (fails) return 1;
    printf("kv4 cache driver ok\n");
    return 0;
}
