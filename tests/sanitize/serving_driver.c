/*
 * Host checks of the serving calls (kv_cache_append, attn_decode_paged,
 * gemm_bf16_epilogue and their plans and workspace sizes), built with
 * AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_serving_plan.py:
 * validation with fake addresses and the largest sizes (nothing passes, so nothing
 * is launched), and the plans over many sizes.
 */
#include <stdint.h>
#include <stdio.h>

#include "tileattn.h"

static int failures = 0;
#define EXPECT(cond, ...)                                        \
    do {                                                         \
        if (!(cond)) {                                           \
            fprintf(stderr, "FAIL line %d: ", __LINE__);         \
            fprintf(stderr, __VA_ARGS__);                        \
            fputc('\n', stderr);                                 \
            ++failures;                                          \
        }                                                        \
    } while (0)

#define P(x) ((void *)(uintptr_t)(x))
#define BIG 2147483647

static int append(int T, int B, int Hkv, int D, int pages, int page, int per, int64_t stride, const void *seq, uintptr_t vc)
{
    return kv_cache_append(P(0x10000000), P(0x20000000), stride, stride, seq, P(0x30000000), P(0x100000000000), P(vc), 0, NULL,
                           NULL, P(0x50000000), T, B, Hkv, D, pages, page, per, NULL);
}

static int attn(int B, int Hq, int Hkv, int D, int pages, int page, int per, int64_t stride, int parts, size_t ws, uintptr_t o)
{
    return attn_decode_paged(P(0x10000000), stride, P(0x100000000000), P(0x200000000000), 0, NULL, NULL, P(0x300000000000),
                             P(0x400000000000), P(o), 0, P(0x600000000000), B, Hq, Hkv, D, pages, page, per, 0.1f, parts,
                             P(0x700000000000), ws, NULL);
}

static int product(int act, int M, int N, int K, int sp, size_t ws)
{
    return gemm_bf16_epilogue(P(0x100000000000), P(0x200000000000), P(0x300000000000), P(0x400000000000), P(0x500000000000), 1,
                              act, M, N, K, sp, P(0x600000000000), ws, NULL);
}

int main(void)
{
    const uintptr_t VC = 0x200000000000, O = 0x500000000000;
    /* every size at its largest and smallest */
    const int odd[] = {BIG, BIG - 1, 1 << 30, -1, 0, -BIG - 1};
    for (unsigned i = 0; i < sizeof odd / sizeof *odd; ++i) {
        const int x = odd[i];
        EXPECT(append(x, 4, 8, 128, 100, 64, 20, 1024, P(0x40000000), VC) != TA_OK, "T %d", x);
        EXPECT(append(5, 4, x, 128, 100, 64, 20, 1024, P(0x40000000), VC) != TA_OK, "Hkv %d", x);
        EXPECT(append(5, 4, 8, x, 100, 64, 20, 1024, P(0x40000000), VC) != TA_OK, "D %d", x);
        EXPECT(append(5, 4, 8, 128, x, 64, 20, 1024, P(0x40000000), VC) != TA_OK, "pages %d", x);
        EXPECT(append(5, 4, 8, 128, 100, x, 20, 1024, P(0x40000000), VC) != TA_OK, "page %d", x);
        EXPECT(append(5, 4, 8, 128, 100, 64, x, 1024, P(0x40000000), VC) != TA_OK, "per %d", x);
        EXPECT(attn(x, 32, 8, 128, 100, 64, 20, 4096, 64, SIZE_MAX, O) != TA_OK, "B %d", x);
        EXPECT(attn(4, x, 8, 128, 100, 64, 20, 4096, 64, SIZE_MAX, O) != TA_OK, "Hq %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, x, 4096, 64, SIZE_MAX, O) != TA_OK, "per %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, 20, x, 64, SIZE_MAX, O) != TA_OK, "stride %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, 20, 4096, x ? x : -1, SIZE_MAX, O) != TA_OK, "parts %d", x);
        EXPECT(product(0, x, 64, 64, 1, 0) != TA_OK, "M %d", x);
        EXPECT(product(0, 64, x & ~7, 64, 1, 0) != TA_OK, "N %d", x);
        EXPECT(product(0, 64, 64, x & ~7, 1, 0) != TA_OK, "K %d", x);
        EXPECT(product(x ? x : 9, 64, 64, 64, 1, 0) != TA_OK, "act %d", x);
        EXPECT(product(0, 64, 64, 64, x, SIZE_MAX) != TA_OK, "splits %d", x);
        int n;
        size_t b;
        EXPECT(attn_paged_plan(x, 32, 8, 128, 64, 20, &n) != TA_OK || x > 0, "plan %d", x);
        EXPECT(attn_paged_plan(4, 32, 8, 128, x, x, &n) != TA_OK || x > 0, "plan %d", x);
        EXPECT(attn_paged_workspace_bytes(x, 8, 128, 64, &b) != TA_OK, "bytes %d", x);
        EXPECT(gemm_epilogue_plan(x, 64, 64, &n) != TA_OK, "plan %d", x);
        EXPECT(gemm_epilogue_workspace_bytes(64, x & ~7, 64, 2, &b) != TA_OK, "bytes %d", x);
    }
    /* the largest caches and products that the checks let through overlap something */
    EXPECT(append(5, 4, 1 << 16, 128, 1 << 28, 16, 20, 1 << 23, P(0x40000000), VC) == TA_ERR_ALIASING, "largest pool");
    EXPECT(attn(4, 1 << 16, 1 << 16, 128, 1 << 28, 16, 20, 1 << 23, 0, 0, O) == TA_ERR_ALIASING, "largest pool");
    EXPECT(attn(4, 32, 8, 128, 100, 64, 20, 4096, 4096, 1, O) == TA_ERR_WORKSPACE, "small workspace");
    EXPECT(product(4, 1 << 20, (1 << 15) - 8, 8, 2, SIZE_MAX) == TA_ERR_ALIASING || product(4, 1 << 20, 1 << 15, 8, 2, 0) != TA_OK,
           "largest product");
    EXPECT(gemm_epilogue_plan(1, 8, 8, NULL) == TA_ERR_NULL_POINTER && attn_paged_plan(1, 1, 1, 64, 16, 1, NULL) == TA_ERR_NULL_POINTER,
           "null");

    const int sizes[] = {8, 16, 64, 128, 136, 1000, 4096, 4104, 8200, 65536, (1 << 22) - 8, (1 << 24) - 8};
    for (int M = 1; M <= 1 << 20; M = M < 70 ? M + 1 : M * 2 + 3)
        for (unsigned i = 0; i < sizeof sizes / sizeof *sizes; ++i)
            for (unsigned j = 0; j < sizeof sizes / sizeof *sizes; ++j) {
                int n = 0;
                const int rc = gemm_epilogue_plan(M, sizes[i], sizes[j], &n);
                if (rc != TA_OK) {
                    EXPECT(rc == TA_ERR_INVALID_SHAPE, "plan %d %d %d", M, sizes[i], sizes[j]);
                    continue;
                }
                EXPECT(n >= 1 && n <= 64, "plan %d %d %d: %d", M, sizes[i], sizes[j], n);
                for (int sp = 1; sp <= 64; sp *= 4) {
                    size_t b = 1;
                    EXPECT(gemm_epilogue_workspace_bytes(M, sizes[i], sizes[j], sp, &b) == TA_OK && b % 16 == 0 &&
                               (sp > 1 || b == 0) && b <= (size_t)(M <= 64 ? 8 : 1) * 64 * M * (sizes[i] + 128) * 4,
                           "bytes %d %d %d %d: %zu", M, sizes[i], sizes[j], sp, b);
                }
            }
    for (int g = 1; g <= 1 << 16; g = g * 3 + 1)
        for (int parts = 0; parts <= 4096; parts = parts * 5 + 1) {
            size_t b = 1;
            EXPECT(attn_paged_workspace_bytes(g, 1, 128, parts, &b) == TA_OK && b % 16 == 0 && (b == 0) == (parts == 0), "bytes %d", g);
        }
    if (failures)
        return 1;
    puts("all checks passed");
    return 0;
}
