/*
 * Host checks of the serving calls on 4-bit numbers and of the next token's choice
 * (qk_norm_rope_append, attn_decode_paged_mxfp4, gemm_mxfp4_epilogue, sample_logits and
 * their plans and workspace sizes), built with AddressSanitizer and
 * UndefinedBehaviorSanitizer by tests/test_more_serving_plan.py: validation with fake
 * addresses and the largest sizes (nothing passes, so nothing is launched), and the plans
 * and workspaces over many sizes.
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

/* (V_cache lies where the K cache's last bytes do, for pools that pass all other checks) */
static int rope(int type, int T, int B, int Hq, int Hkv, int D, int pages, int page, int per, int64_t stride, int positions, int rot,
                float eps)
{
    return qk_norm_rope_append(P(0x10000000), P(0x20000000), P(0x30000000), stride, stride, stride, P(0x40000000), P(0x40001000), eps,
                               P(0x50000000), positions, rot, 0, P(0x60000000), P(0x70000000), P(0x300000000000), P(0x100000000000),
                               P(0x100000000010), type, type ? P(0x200000000000) : NULL, type ? P(0x280000000000) : NULL, P(0x80000000),
                               T, B, Hq, Hkv, D, pages, page, per, NULL);
}

static int attn(int B, int Hq, int Hkv, int D, int pages, int page, int per, int64_t stride, int parts, size_t ws)
{
    return attn_decode_paged_mxfp4(P(0x10000000), stride, P(0x100000000000), P(0x200000000000), P(0x300000000000), P(0x380000000000),
                                   P(0x400000000000), P(0x500000000000), P(0x600000000000), 0, P(0x600000000000), B, Hq, Hkv, D, pages,
                                   page, per, 0.1f, parts, P(0x700000000000), ws, NULL);
}

static int product(int act, int M, int N, int K, int parts, size_t ws)
{
    return gemm_mxfp4_epilogue(P(0x100000000000), P(0x200000000000), P(0x300000000000), P(0x400000000000), P(0x500000000000),
                               P(0x500000000010), 1, act, M, N, K, parts, P(0x600000000000), ws, NULL);
}

static int sample(int64_t stride, int bf16, int B, int V, size_t ws)
{
    return sample_logits(P(0x100000000000), stride, bf16, P(0x10000000), P(0x20000000), P(0x30000000), P(0x40000000), P(0x50000000),
                         P(0x60000000), P(0x60000000), B, V, P(0x200000000000), ws, NULL);
}

int main(void)
{
    /* every size at its largest and smallest */
    const int odd[] = {BIG, BIG - 1, 1 << 30, 1 << 24, -1, 0, -BIG - 1};
    for (unsigned i = 0; i < sizeof odd / sizeof *odd; ++i) {
        const int x = odd[i];
        for (int type = 0; type < 3; ++type) {
            EXPECT(rope(type, x, 4, 32, 8, 128, 100, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "T %d", x);
            EXPECT(rope(type, 5, x, 32, 8, 128, 100, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "B %d", x);
            EXPECT(rope(type, 5, 4, x, 8, 128, 100, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "Hq %d", x);
            EXPECT(rope(type, 5, 4, 32, x, 128, 100, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "Hkv %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, x, 100, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "D %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, x, 64, 20, 4096, 99, 128, 1e-6f) != TA_OK, "pages %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, 100, x, 20, 4096, 99, 128, 1e-6f) != TA_OK, "page %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, 100, 64, x, 4096, 99, 128, 1e-6f) != TA_OK, "per %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, 100, 64, 20, x, 99, 128, 1e-6f) != TA_OK, "stride %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, 100, 64, 20, 4096, x, 128, 1e-6f) != TA_OK, "positions %d", x);
            EXPECT(rope(type, 5, 4, 32, 8, 128, 100, 64, 20, 4096, 99, x, 1e-6f) != TA_OK, "rot %d", x);
        }
        EXPECT(attn(x, 32, 8, 128, 100, 64, 20, 4096, 64, SIZE_MAX) != TA_OK, "B %d", x);
        EXPECT(attn(4, x, 8, 128, 100, 64, 20, 4096, 64, SIZE_MAX) != TA_OK, "Hq %d", x);
        EXPECT(attn(4, 32, 8, 128, x, 64, 20, 4096, 64, SIZE_MAX) != TA_OK, "pages %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, x, 4096, 64, SIZE_MAX) != TA_OK, "per %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, 20, x, 64, SIZE_MAX) != TA_OK, "stride %d", x);
        EXPECT(attn(4, 32, 8, 128, 100, 64, 20, 4096, x, SIZE_MAX) != TA_OK, "parts %d", x);
        EXPECT(product(0, x, 64, 64, 1, SIZE_MAX) != TA_OK, "M %d", x);
        EXPECT(product(0, 64, x & ~7, 64, 1, SIZE_MAX) != TA_OK, "N %d", x);
        EXPECT(product(0, 64, 64, x & ~31, 1, SIZE_MAX) != TA_OK, "K %d", x);
        EXPECT(product(x ? x : 9, 64, 64, 64, 1, SIZE_MAX) != TA_OK, "act %d", x);
        EXPECT(product(0, 64, 64, 64, x, SIZE_MAX) != TA_OK, "parts %d", x);
        EXPECT(sample(50000, i & 1, x, 50000, SIZE_MAX) != TA_OK, "B %d", x);
        EXPECT(sample(50000, i & 1, 3, x, SIZE_MAX) != TA_OK, "V %d", x);
        EXPECT(sample(x, i & 1, 3, 50000, SIZE_MAX) != TA_OK, "stride %d", x);
        int n;
        size_t b;
        EXPECT(attn_paged_mxfp4_plan(x, 32, 8, 128, 64, 20, &n) != TA_OK || x > 0, "plan %d", x);
        EXPECT(attn_paged_mxfp4_plan(4, 32, 8, 128, x, x, &n) != TA_OK || x > 0, "plan %d", x);
        EXPECT(gemm_mxfp4_plan(x, 64, 64, &n) != TA_OK, "plan %d", x);
        EXPECT(gemm_mxfp4_plan(64, x & ~7, 64, &n) != TA_OK, "plan %d", x);
        EXPECT(gemm_mxfp4_plan(64, 64, x & ~31, &n) != TA_OK, "plan %d", x);
        EXPECT(gemm_mxfp4_workspace_bytes(64, x & ~7, 64, 2, &b) != TA_OK, "bytes %d", x);
        EXPECT(gemm_mxfp4_workspace_bytes(64, 64, 64, x, &b) != TA_OK || x == 0, "bytes %d", x);
        EXPECT(sample_logits_workspace_bytes(x, 100, 1, &b) != TA_OK && sample_workspace_bytes(100, x, &b) != TA_OK, "bytes %d", x);
    }
    /* the largest that the checks let through overlap something, or lack a workspace */
    for (int type = 0; type < 3; ++type)
        EXPECT(rope(type, (1 << 24) - 1, 4, 1 << 16, 1 << 16, 128, 1 << 28, 16, 20, 1 << 23, BIG, 128, 0.f) == TA_ERR_ALIASING, "pool");
    EXPECT(attn(4, 1 << 16, 1 << 16, 128, 1 << 28, 16, 20, 1 << 23, 0, 0) == TA_ERR_ALIASING, "largest pool");
    EXPECT(product(4, 1 << 20, (1 << 15) - 8, 32, 4096, SIZE_MAX) == TA_ERR_ALIASING, "largest product");
    EXPECT(sample(1 << 30, 0, 1 << 16, 1 << 20, SIZE_MAX) == TA_ERR_ALIASING, "largest rows");
    EXPECT(gemm_mxfp4_plan(1, 8, 32, NULL) == TA_ERR_NULL_POINTER && attn_paged_mxfp4_plan(1, 1, 1, 64, 16, 1, NULL) == TA_ERR_NULL_POINTER &&
               gemm_mxfp4_workspace_bytes(1, 8, 32, 1, NULL) == TA_ERR_NULL_POINTER && sample_workspace_bytes(1, 1, NULL) == TA_ERR_NULL_POINTER &&
               sample_logits_workspace_bytes(1, 1, 1, NULL) == TA_ERR_NULL_POINTER,
           "null");

    const int rows[] = {8, 16, 64, 128, 136, 1000, 6144, 6152, 10240, 65536, (1 << 22) - 8, (1 << 24) - 8};
    const int cols[] = {32, 64, 128, 160, 1024, 2048, 4128, 8224, 65536, (1 << 18), (1 << 22) - 32};
    for (int M = 1; M <= 1 << 20; M = M < 70 ? M + 1 : M * 2 + 3)
        for (unsigned i = 0; i < sizeof rows / sizeof *rows; ++i)
            for (unsigned j = 0; j < sizeof cols / sizeof *cols; ++j) {
                const int N = rows[i], K = cols[j];
                int n = -1;
                const int rc = gemm_mxfp4_plan(M, N, K, &n);
                if (rc != TA_OK) {
                    EXPECT(rc == TA_ERR_INVALID_SHAPE, "plan %d %d %d", M, N, K);
                    continue;
                }
                EXPECT(n >= 0 && n <= 256, "plan %d %d %d: %d", M, N, K, n);
                for (int parts = 0; parts <= 4096; parts = parts * 4 + 1) {
                    size_t b = 1;
                    /* two records a part, of a strip of 64 columns or a tile of 128 x 256 at most */
                    EXPECT(gemm_mxfp4_workspace_bytes(M, N, K, parts, &b) == TA_OK && b % 16 == 0 && (parts || b == 0) &&
                               b <= (size_t)parts * 2 * (M <= 64 ? M * 64 : 128 * 256) * 4,
                           "bytes %d %d %d %d: %zu", M, N, K, parts, b);
                }
            }
    for (int B = 1; B <= 1 << 16; B = B < 140 ? B + 1 : B * 2 + 1)
        for (int V = 1; V <= 1 << 20; V += 1 + V / 7) {
            size_t b[3] = {1, 1, 1};
            EXPECT(sample_logits_workspace_bytes(B, V, 0, b) == TA_OK && sample_logits_workspace_bytes(B, V, 1, b + 1) == TA_OK &&
                       sample_workspace_bytes(B, V, b + 2) == TA_OK && b[0] % 16 == 0 && b[1] % 16 == 0 && b[1] <= b[0] && b[2] == b[0],
                   "bytes %d %d", B, V);
            /* at most 32 slices, of which each has 2048 sums and counts */
            EXPECT(b[0] <= (size_t)B * (1024 * 8 + 32 * (2048 * 12 + 32)), "bytes %d %d: %zu", B, V, b[0]);
        }
    if (failures)
        return 1;
    puts("all checks passed");
    return 0;
}
