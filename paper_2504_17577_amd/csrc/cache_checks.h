// What the entry points of the paged cache check alike.  Host code, internal to
// libtileattn.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "tileattn.h"

namespace tileattn_detail {

inline bool misaligned(const void *p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

struct Span {
    const void *p;
    size_t n;
};

inline bool overlaps(Span a, Span b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.n && y < x + a.n;
}

// the sizes and types of a cache; `scaled`: scales are given
inline ta_status check_cache(int B, int Hkv, int D, int num_pages, int page_size, int max_pages, int type, bool scaled)
{
    if (B < 1 || Hkv < 1 || D < 1 || num_pages < 1 || page_size < 1 || max_pages < 1)
        return TA_ERR_INVALID_SHAPE;
    if ((D != 64 && D != 128) || page_size < 16 || (page_size & (page_size - 1)))
        return TA_ERR_UNSUPPORTED;
    if (type == TA_CACHE_BF16 && scaled)
        return TA_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * page_size > 1ll << 30 || num_pages > 1 << 28 || Hkv > 1 << 16 ||
        (int64_t)Hkv * page_size > 1ll << 30)
        return TA_ERR_INVALID_SHAPE;
    return TA_OK;
}

// bytes of a cache whose rows take `row`: below 2^28 2^30 2^8 = 2^66 by the checks
// alone, so in 128 bits
inline size_t cache_bytes(int Hkv, int num_pages, int page_size, int row)
{
    const unsigned __int128 n = (unsigned __int128)num_pages * Hkv * page_size * row;
    return n > (1ull << 62) ? (size_t)1 << 62 : (size_t)n;
}

inline int cache_row_bytes(int D, int type) { return type == TA_CACHE_BF16 ? 2 * D : type == TA_CACHE_E4M3 ? D : D / 2; }

// bytes of a vector or tensor of scales
inline size_t scale_bytes(int Hkv, int D, int num_pages, int page_size, int type)
{
    return type == TA_CACHE_MXFP4 ? cache_bytes(Hkv, num_pages, page_size, D / 32) : (size_t)Hkv * 4;
}

inline bool heads_ok(int B, int Hq, int Hkv)
{
    return B >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && Hq <= 1 << 16 && (int64_t)B * Hq < 1ll << 24;
}

}  // namespace tileattn_detail
