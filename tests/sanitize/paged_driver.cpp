/*
 * Host checks of the paged cache's integer logic (csrc/paged_plan.h), built with
 * AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_serving_plan.py:
 * the parts cover every tile once, in order and evenly, and each tile's part is
 * found again, also for lengths outside the table and the largest counts; a walk
 * over the parts as the kernels make it writes every result once.
 */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <vector>
#include "paged_plan.h"

using namespace tileattn_detail;

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

static void check_parts(uint32_t n, uint32_t parts)
{
    const uint32_t used = paged_parts_used(n, parts);
    EXPECT(used >= 1 && used <= parts && used <= n / 2 + n % 2, "used %u", used);
    EXPECT(even_begin(n, used, 0) == 0 && even_begin(n, used, used) == n, "ends of %u in %u", n, used);
    for (uint32_t p = 0; p < used; ++p) {
        const uint32_t b = even_begin(n, used, p), e = even_begin(n, used, p + 1);
        EXPECT(e > b && e - b <= n / used + 1 && e - b >= n / used, "part %u: %u..%u of %u in %u", p, b, e, n, used);
        EXPECT(even_part_of(n, used, b) == p && even_part_of(n, used, e - 1) == p, "part of %u, %u", b, e - 1);
    }
}

/* the kernels' walk: which part writes what of every head */
static void walk(const int *lens, int B, int cap, uint32_t HR, uint32_t parts)
{
    uint32_t n = 0;
    for (int b = 0; b < B; ++b)
        n += paged_tiles(lens[b], cap);
    n *= HR;
    const uint32_t used = paged_parts_used(n, parts);
    const size_t heads = (size_t)B * HR;
    std::vector<int> whole(heads), tiles(heads), record(2 * used, -1);   /* the head of each record */
    for (uint32_t p = 0; p < used; ++p) {
        uint32_t at = even_begin(n, used, p), left = even_begin(n, used, p + 1) - at, b = 0, first = 0;
        while (first + HR * paged_tiles(lens[b], cap) <= at)
            first += HR * paged_tiles(lens[b++], cap);
        uint32_t per = paged_tiles(lens[b], cap), hr = (at - first) / per, t = (at - first) % per;
        for (;;) {
            EXPECT(b < (uint32_t)B && hr < HR, "past the last head");
            per = paged_tiles(lens[b], cap);
            const uint32_t take = left < per - t ? left : per - t;
            const size_t head = (size_t)b * HR + hr;
            tiles[head] += (int)take;
            if (t == 0 && t + take == per) {
                ++whole[head];
            } else {
                EXPECT(record[2 * p + (t == 0)] == -1, "a record written twice");
                record[2 * p + (t == 0)] = (int)head;
            }
            left -= take;
            if (left == 0)
                break;
            t = 0;
            if (++hr == HR)
                hr = 0, ++b;
        }
    }
    uint32_t t0 = 0;
    for (size_t head = 0; head < heads; ++head) {       /* the merge */
        const uint32_t per = paged_tiles(lens[head / HR], cap);
        EXPECT(tiles[head] == (int)per, "head %zu: %d tiles of %u", head, tiles[head], per);
        const uint32_t p0 = even_part_of(n, used, t0), p1 = even_part_of(n, used, t0 + per - 1);
        EXPECT(whole[head] == (p0 == p1), "head %zu whole", head);
        if (p0 != p1)
            for (uint32_t p = p0; p <= p1; ++p)
                EXPECT(record[2 * p + (p == p0)] == (int)head, "head %zu, record of part %u", head, p);
        t0 += per;
    }
}

int main(void)
{
    const uint32_t ns[] = {1, 2, 3, 7, 63, 64, 65, 511, 512, 513, 1000, 4095, 4096, 4097, 123457, 2147483647};
    const uint32_t ps[] = {1, 2, 3, 5, 64, 100, 511, 512, 4096};
    for (size_t i = 0; i < sizeof ns / sizeof *ns; ++i)
        for (size_t j = 0; j < sizeof ps / sizeof *ps; ++j)
            check_parts(ns[i], ps[j]);
    const int T = PAGED_TILE, H = PAGED_HEAD;
    EXPECT(paged_tiles(0, 100) == (uint32_t)H && paged_tiles(-5, 100) == (uint32_t)H && paged_tiles(101, 100) == (uint32_t)H, "no keys");
    EXPECT(paged_tiles(1, 999) == (uint32_t)H + 1 && paged_tiles(T, 999) == (uint32_t)H + 1 && paged_tiles(T + 1, 999) == (uint32_t)H + 2, "tiles");
    EXPECT(paged_tiles(1 << 30, 1 << 30) == (1u << 30) / T + H && paged_tiles(INT32_MIN, 1 << 30) == (uint32_t)H, "largest");
    EXPECT(paged_key(0) == 0 && paged_key(H) == 0 && paged_key(H + 1) == T && paged_key(H + 5) == 5 * T, "keys");
    for (int len : {1, 2, T - 1, T, T + 1, 1000, (1 << 30) - 1, 1 << 30})
        EXPECT(paged_key(paged_tiles(len, 1 << 30)) >= len && paged_key(paged_tiles(len, 1 << 30) - 1) < len, "last tile of %d", len);
    EXPECT(paged_checked(0, 1) == 0 && paged_checked(1, 1) == -1 && paged_checked(-1, 1) == -1 &&
               paged_checked(INT32_MIN, 1) == -1 && paged_checked(INT32_MAX, 1 << 28) == -1, "pages");
    for (int g = 1; g <= 300; ++g) {
        const int rb = paged_row_blocks(g), rows = paged_block_rows(g);
        EXPECT(rows <= PAGED_MAX_ROWS && rb * rows >= g && (rb - 1) * rows < g, "rows of %d", g);
        EXPECT(paged_record(rows, 128) % 4 == 0 && paged_record(rows, 128) >= (uint64_t)rows * 130, "record");
    }
    srand(1);
    for (int c = 0; c < 2000; ++c) {
        int lens[80];
        const int B = 1 + rand() % 80, cap = 1 + rand() % 3000;
        for (int b = 0; b < B; ++b)
            lens[b] = rand() % 4 == 0 ? rand() % 3 - 1 : rand() % (cap + 2);
        walk(lens, B, cap, 1 + (uint32_t)(rand() % 9), 1 + (uint32_t)(rand() % 600));
    }
    if (failures)
        return 1;
    puts("all checks passed");
    return 0;
}
