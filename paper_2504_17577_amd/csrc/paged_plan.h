// Integer logic of the paged cache's kernels: where a position lies, and how the
// cached positions of a batch are divided over workgroups.  No HIP: the kernels
// and host code (its tests too) share it.
#pragma once

#include "even_parts.h"

#define PAGED_FN EVEN_FN

namespace tileattn_detail {

constexpr int PAGED_NW = 4;            // waves of an attention workgroup
constexpr int PAGED_MAX_PARTS = 4096;
constexpr int PAGED_MAX_ROWS = 32;     // query heads of a group that one workgroup takes

// Keys of a tile, the unit that the batch is divided in: a 16-key block per wave,
// the least that a wave reads, so that shares are even to within it.
constexpr int PAGED_TILE = 16 * PAGED_NW;

// What a head costs besides its keys, in tiles: looking it up, the first loads'
// way, the meeting of the waves.  Short sequences would make the longest shares
// without it.  These tiles come first and hold no keys.
constexpr int PAGED_HEAD = 2;

// Tiles of one sequence's head (a length outside 0..cap counts as none: its
// results are written too)
PAGED_FN uint32_t paged_tiles(int len, int cap)
{
    return PAGED_HEAD + (len <= 0 || len > cap ? 0u : (uint32_t)(len - 1) / (uint32_t)PAGED_TILE + 1u);
}

// The first key of tile t of a head
PAGED_FN int paged_key(uint32_t t) { return t > PAGED_HEAD ? (int)(t - PAGED_HEAD) * PAGED_TILE : 0; }

// The parts that n tiles are cut into where `parts` workgroups run: two tiles each
// at least (a small batch of long rows in 64-key parts joined 15 % slower)
PAGED_FN uint32_t paged_parts_used(uint32_t n, uint32_t parts)
{
    const uint32_t most = n / 2 + n % 2;
    return most < parts ? most : parts;
}

// A page index of the table, or -1 for one outside the pool
PAGED_FN int paged_checked(int page, int num_pages) { return page >= 0 && page < num_pages ? page : -1; }

// Row blocks of a group of `group` query heads, and the heads in each
PAGED_FN int paged_row_blocks(int group) { return (group + PAGED_MAX_ROWS - 1) / PAGED_MAX_ROWS; }
PAGED_FN int paged_block_rows(int group)
{
    const int rb = paged_row_blocks(group);
    return (group + rb - 1) / rb;
}

// Partial results: part p has two records, 2 p for what it does of a head that an
// earlier part began and 2 p + 1 for one that it begins and a later part goes on
// with.  A record is [rows][D] sums, [rows] maxima and [rows] weights in fp32,
// rows rounded up to four (16-byte records).
PAGED_FN uint64_t paged_record(int rows, int D) { return (uint64_t)((rows + 3) & ~3) * (uint64_t)(D + 2); }

}  // namespace tileattn_detail
