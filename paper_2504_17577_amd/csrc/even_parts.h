// n units of work in `parts` parts, as even as they go, in order: the first n %
// parts parts have one unit more.  No HIP: kernels and host code share it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define EVEN_FN __host__ __device__ inline
#else
#define EVEN_FN inline
#endif

namespace tileattn_detail {

EVEN_FN uint32_t even_begin(uint32_t n, uint32_t parts, uint32_t p)
{
    const uint32_t r = n % parts;
    return n / parts * p + (p < r ? p : r);
}

// the part that unit t is in (parts <= n)
EVEN_FN uint32_t even_part_of(uint32_t n, uint32_t parts, uint32_t t)
{
    const uint32_t q = n / parts, r = n % parts, big = r * (q + 1);
    return t < big ? t / (q + 1) : r + (t - big) / q;
}

}  // namespace tileattn_detail
