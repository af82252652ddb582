// The next token of each row of logits on gfx950 (MI355X): temperature, top-k, top-p,
// min-p and the choice by a given uniform number (sample_logits).
//
// The order of a row is by logit, then by index, and every filter keeps a beginning of
// it, so that all of them together come down to one place in the order.  The weights
// exp((x - best) / T) and their sums decide at borders between tokens, so they are
// computed in 64 bits and added as whole multiples of 2^-43: exactly, in any order.
// What is less than half of that counts as nothing.
//
// Nothing is sorted.  A small top-k (this covers greedy rows) takes candidates: the
// largest logits of a few thousand groups give a border that at least k tokens are above
// and few more; the place is found among those alone.  Otherwise a histogram of the
// weights over (best - x) / T, in 2047 buckets of 31 / 2048, shows the bucket that the
// place lies in, and it is found among the tokens of that bucket; should they be too many
// (ties, most of all), their keys' range is narrowed in the same way.  The token is then
// found in the order of indexes, from the sums of slices of the row, in one slice.
//
// A row is cut into slices for a few large rows: a kernel over slices for the largest
// logit and the candidates, one over slices for the histograms (rows that need none
// leave at once), and one over rows for the rest.  Many rows, or short ones, run the
// three as one kernel, a workgroup a row.
//
// Measured: 256 x 131072 bf16 with every filter 40 us (the row's way to registers 10, where
// HBM's floor is 11 for all; the largest 2, exponentials of all logits 4, the rest barriers and
// LDS); 64 x 128001 fp32 by top-p 70 (14, 14 and 41 for the three kernels: the last one's
// passes over a row by one workgroup); 1 x 32000 18.  Tried: the candidates sorted in LDS
// (55 steps of a bitonic network of 1024, 0.3 us each), compared each with each up to 1024
// (30 us for 500), the workgroup's sums by shuffles through LDS (a place took 8 us instead of
// 3).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "cache_checks.h"
#include "even_parts.h"
#include "tileattn.h"

namespace {

using namespace tileattn_detail;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int NT = 1024, NWAVE = NT / 64;
constexpr int NB = 2048;                 // buckets; the last holds what counts as nothing
constexpr double BUCKET = 31.0 / NB, PER_UNIT = NB / 31.0;
constexpr double UNIT = 0x1p43;
constexpr int LIST = NT;                 // tokens that are looked at by themselves, one a thread
constexpr int FEW = 128;                 // of which so many are compared with each other
constexpr int CANDIDATES = 512;          // as many times the slices as a top-k may ask for to have candidates
constexpr int GROUPS = 4;                // of a thread, whose largest logits set the border
constexpr int HELD = 17;                 // chunks of 16 bytes of a slice that a thread holds (131072 16-bit logits and a piece)
constexpr int SUBS = 1024;               // parts of a bucket's range of keys
constexpr int MAX_SLICES = 32;
constexpr int MAX_V = 1 << 20, MAX_B = 1 << 16;

struct Slice {
    float top;       // the slice's largest logit
    int n;           // its candidates, or -1: the row takes the histogram
    double z;        // sum of exp((x - top) / T); NaN if there is a NaN
};

struct SampleArgs {
    const void *logits;
    int64_t stride;
    const float *u, *temperature;
    const int *top_k;
    const float *top_p, *min_p;
    int *token;
    float *logp;
    int V, S;
    // of slices, [row][slice]: records, candidates [LIST / S], weights and counts [NB]
    Slice *slices;
    u64 *lists, *weights;
    uint32_t *counts;
};

struct __attribute__((aligned(16))) Token {
    u64 place, w;
};

struct Shared {
    u64 list[LIST];          // places
    Token few[LIST];
    u64 w[SUBS];
    uint32_t n_of[SUBS];
    double table[NB];        // weight of a bucket's lower end, in units
    u64 hist[NB];
    uint32_t count[NB];
    u64 scan[NWAVE], sum[2][NWAVE], slice[MAX_SLICES], w_cut;
    double z[NWAVE];
    float best[NWAVE], low[NWAVE];
    uint32_t n, lo, hi, at, n_few;
    u64 cut, low_place, high_place, rank, before;
    int found;
};

// ---- the workgroup's sums ---------------------------------------------------

// x moved by a lane pattern of the vector ALU; lanes that nothing moves to get `none`
template <int CTRL, int ROWS, class F>
__device__ __forceinline__ F moved(F x, F none)
{
    if constexpr (sizeof(F) == 4) {
        return __builtin_bit_cast(F, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x),
                                                                 CTRL, ROWS, 0xF, false));
    } else {
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        const i32x2 v = __builtin_bit_cast(i32x2, x), n = __builtin_bit_cast(i32x2, none);
        return __builtin_bit_cast(F, i32x2{__builtin_amdgcn_update_dpp(n[0], v[0], CTRL, ROWS, 0xF, false),
                                           __builtin_amdgcn_update_dpp(n[1], v[1], CTRL, ROWS, 0xF, false)});
    }
}

// op over the lanes up to this one: rows of sixteen by shifts, then the rows' last lanes
template <class F, class Op>
__device__ __forceinline__ F wave_upto(F x, F none, Op op)
{
    x = op(x, moved<0x111, 0xF>(x, none));     // row_shr:1, 2, 4, 8
    x = op(x, moved<0x112, 0xF>(x, none));
    x = op(x, moved<0x114, 0xF>(x, none));
    x = op(x, moved<0x118, 0xF>(x, none));
    x = op(x, moved<0x142, 0xA>(x, none));     // row_bcast:15 to rows 1 and 3
    return op(x, moved<0x143, 0xC>(x, none));  // row_bcast:31 to rows 2 and 3
}

// op over all lanes, the same in each
template <class F, class Op>
__device__ __forceinline__ F wave_all(F x, F none, Op op)
{
    x = wave_upto(x, none, op);
    if constexpr (sizeof(F) == 4) {
        return __builtin_bit_cast(F, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
    } else {
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        const i32x2 v = __builtin_bit_cast(i32x2, x);
        return __builtin_bit_cast(F, i32x2{__builtin_amdgcn_readlane(v[0], 63), __builtin_amdgcn_readlane(v[1], 63)});
    }
}

__device__ __forceinline__ u64 wave_sum_upto(u64 x) { return wave_upto(x, (u64)0, [](u64 a, u64 b) { return a + b; }); }

template <class F>
__device__ __forceinline__ F from_lane(F x, int lane)       // (lane: uniform)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_bit_cast(i32x2, x);
    return __builtin_bit_cast(F, i32x2{__builtin_amdgcn_readlane(v[0], lane), __builtin_amdgcn_readlane(v[1], lane)});
}

// op over all threads' x, through NWAVE places of LDS that nobody reads any more
template <class F, class Op>
__device__ __forceinline__ F block_all(F x, F none, F *s, Op op)
{
    x = wave_all(x, none, op);
    if (threadIdx.x % 64 == 0)
        s[threadIdx.x / 64] = x;
    __syncthreads();
    return wave_all(threadIdx.x % 64 < NWAVE ? s[threadIdx.x % 64] : none, none, op);
}

// The sum of the threads' x before this one; `all`: of all (s as above)
__device__ __forceinline__ u64 block_before(u64 x, u64 *s, u64 &all)
{
    const u64 in = wave_sum_upto(x);
    if (threadIdx.x % 64 == 63)
        s[threadIdx.x / 64] = in;
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const u64 upto = wave_sum_upto(threadIdx.x % 64 < NWAVE ? s[threadIdx.x % 64] : 0);
    all = from_lane(upto, NWAVE - 1);
    return (wave ? from_lane(upto, wave - 1) : 0) + in - x;
}

// Two such sums at once, in place
__device__ __forceinline__ void block_before2(u64 &x, u64 &y, u64 (*s)[NWAVE], u64 &all_y)
{
    const u64 in_x = wave_sum_upto(x), in_y = wave_sum_upto(y);
    if (threadIdx.x % 64 == 63) {
        s[0][threadIdx.x / 64] = in_x;
        s[1][threadIdx.x / 64] = in_y;
    }
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const u64 upto_x = wave_sum_upto(lane < NWAVE ? s[0][lane] : 0), upto_y = wave_sum_upto(lane < NWAVE ? s[1][lane] : 0);
    all_y = from_lane(upto_y, NWAVE - 1);
    x = (wave ? from_lane(upto_x, wave - 1) : 0) + in_x - x;
    y = (wave ? from_lane(upto_y, wave - 1) : 0) + in_y - y;
}

// *last = the largest n of the threads with `is` (n rises with the thread): one atomic a wave
__device__ __forceinline__ void note_last(uint32_t *last, bool is, uint32_t n)
{
    const u64 mask = __builtin_amdgcn_ballot_w64(is);
    if (mask && threadIdx.x % 64 == 63 - __builtin_clzll(mask))
        atomicMax(last, n);
}

// ---- a row -------------------------------------------------------------------

// A row in chunks of 16 bytes from the 16-byte line that it begins in
template <bool BF16>
struct Row {
    static constexpr int EPC = BF16 ? 8 : 4;
    const unsigned char *line;
    int off, V, chunks;      // elements before the row in its first chunk

    __device__ __forceinline__ Row(const SampleArgs &a, int b)
    {
        const uintptr_t p = (uintptr_t)a.logits + (size_t)b * a.stride * (16 / EPC);
        line = (const unsigned char *)(p & ~(uintptr_t)15);
        off = (int)(p & 15) / (16 / EPC);
        V = a.V;
        chunks = (off + V + EPC - 1) / EPC;
    }
    __device__ __forceinline__ int index(int c, int e) const { return c * EPC + e - off; }
    __device__ __forceinline__ float value(int i) const
    {
        if (BF16)
            return __uint_as_float((uint32_t)((const uint16_t *)line)[i + off] << 16);
        return ((const float *)line)[i + off];
    }
    // (the first and last chunk element by element: nothing outside the row is read; -inf
    // stands there)
    __device__ __forceinline__ u32x4 load(int c) const
    {
        if (c * EPC >= off && (c + 1) * EPC <= off + V)
            return *(const u32x4 *)(line + (size_t)16 * c);
        u32x4 x = nothing();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (BF16) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if ((unsigned)index(c, 2 * w + h) < (unsigned)V)
                        x[w] = (x[w] & (h ? 0xFFFFu : 0xFFFF0000u)) |
                               (uint32_t)((const uint16_t *)line)[c * EPC + 2 * w + h] << (16 * h);
            } else if ((unsigned)index(c, w) < (unsigned)V) {
                x[w] = ((const uint32_t *)line)[c * EPC + w];
            }
        }
        return x;
    }
    static __device__ __forceinline__ u32x4 nothing()
    {
        const uint32_t w = BF16 ? 0xFF80FF80u : 0xFF800000u;    // -inf
        return u32x4{w, w, w, w};
    }
    static __device__ __forceinline__ float get(const u32x4 &x, int e)
    {
        if (BF16)
            return __uint_as_float(e & 1 ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16);
        return __uint_as_float(x[e]);
    }
    // f(chunk's number, its 16 bytes) for the chunks c0 .. c1, spread over the threads, U
    // loads in flight
    template <int U, class F>
    __device__ __forceinline__ void each(int c0, int c1, F f) const
    {
        for (int base = c0; base < c1; base += U * NT) {
            const int c = base + threadIdx.x;
            u32x4 x[U];
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (base + i * NT < c1)          // (uniform)
                    x[i] = c + i * NT < c1 ? load(c + i * NT) : nothing();
#pragma unroll
            for (int i = 0; i < U; ++i)
                if (c + i * NT < c1)
                    f(c + i * NT, x[i]);
        }
    }
};

// What a row asks for
struct Wish {
    float T, u;
    int k;           // V: no limit
    bool few;        // candidates
    double p, min_p;
};

__device__ __forceinline__ Wish wish_of(const SampleArgs &a, int b)
{
    Wish w = {1.f, a.u[b], a.V, false, INFINITY, 0.0};
    if (a.top_k && a.top_k[b] > 0)
        w.k = min(a.top_k[b], a.V);
    if (a.top_p)
        w.p = a.top_p[b];
    if (a.min_p)
        w.min_p = a.min_p[b];
    if (a.temperature) {
        const float t = a.temperature[b];
        if (t > 0.f)
            w.T = fminf(fmaxf(t, 1e-30f), 1e30f);
        else
            w.k = 1;                 // greedy
    }
    w.few = (int64_t)w.k * a.S <= CANDIDATES || (a.S == 1 && a.V <= LIST);
    return w;
}

// Logits in an order of whole numbers, -0 as 0
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)order_key(x) << 32 | (0xFFFFFFFFu - (uint32_t)i); }
__device__ __forceinline__ int index_of(u64 place) { return (int)(0xFFFFFFFFu - (uint32_t)place); }
__device__ __forceinline__ float logit_of(u64 place)
{
    const uint32_t k = (uint32_t)(place >> 32);
    return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// The bucket of a logit and its weight: exp(-d) = exp(-the bucket's lower end) exp(-r),
// the second by its series to r^5 (r < 0.0152).  The next term, r^6 / 720 < 2^-45 (without which
// a weight next to min_p fell on the other side than a candidate's), is in those of r^3 to r^5:
// of r^3 in r^3 (1 / 6 - r / 24 + r^2 / 120 - r^3 / 720) the polynomial of degree 2 that is nearest
// over a bucket, r^3 less its shifted Chebyshev polynomial.  2^-50 of the value in all, for the time
// of the bare series (another term: 64-bit constants and registers, 4 % of a long row).
struct Weigher {
    double best, inv_T;
    const double *table;

    __device__ __forceinline__ int bucket(float x, double &r) const
    {
        const double d = (best - (double)x) * inv_T;
        const int b = (int)fmin(d * PER_UNIT, (double)(NB - 1));
        r = __builtin_fma((double)-b, BUCKET, d);
        return b;
    }
    __device__ __forceinline__ int bucket(float x) const
    {
        double r;
        return bucket(x, r);
    }
    static __device__ __forceinline__ double series(double r)
    {
        constexpr double L = BUCKET;
        double p = __builtin_fma(r, L / 480 - 1.0 / 120, 1.0 / 24 - L * L / 1280);
        p = __builtin_fma(p, r, L * L * L / 23040 - 1.0 / 6);
        p = __builtin_fma(p, r, 0.5);
        p = __builtin_fma(p, r, -1.0);
        return __builtin_fma(p, r, 1.0);
    }
    // in units, exact to their fraction, and rounded
    __device__ __forceinline__ double exact(float x) const
    {
        double r;
        const int b = bucket(x, r);
        return b == NB - 1 ? 0.0 : table[b] * series(r);
    }
    __device__ __forceinline__ u64 rounded(int b, double r) const
    {
        const double w = __builtin_fma(table[b], series(r), 0x1p52);
        return (u64)__double_as_longlong(w) & 0xFFFFFFFFFFFFFull;
    }
    __device__ __forceinline__ u64 weight(float x) const
    {
        double r;
        const int b = bucket(x, r);
        return b == NB - 1 ? 0 : rounded(b, r);
    }
};

__device__ __forceinline__ void fill_table(double *table)
{
    for (int i = threadIdx.x; i < NB; i += NT)
        table[i] = exp(-i * BUCKET) * UNIT;
}

__device__ __forceinline__ Slice *slice_at(const SampleArgs &a, int b, int s) { return a.slices + (size_t)b * a.S + s; }

// ---- 1: a slice's largest logit and candidates ------------------------------------

// A thread's chunks of a slice, every NT-th, in registers: the row is read once
template <bool BF16>
struct Held {
    u32x4 x[HELD];
    __device__ __forceinline__ void load(const Row<BF16> &row, int c0, int c1)
    {
        // whole chunks of the row (its first and last may not be)
        const int first = row.off ? 1 : 0, last = (row.off + row.V) / Row<BF16>::EPC - 1;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = c0 + threadIdx.x + i * NT;
            x[i] = row.nothing();
            if (c0 + i * NT < c1 && first <= last)          // (uniform)
                x[i] = __builtin_nontemporal_load((const u32x4 *)(row.line + (size_t)16 * min(max(c, first), last)));
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = c0 + threadIdx.x + i * NT;
            if (c >= c1)
                x[i] = row.nothing();
            else if (c < first || c > last)
                x[i] = row.load(c);
        }
    }
};

template <bool BF16>
__device__ __forceinline__ Slice find_candidates(const SampleArgs &a, const Wish &wish, int b, int s, Shared &sm)
{
    using R = Row<BF16>;
    const R row(a, b);
    const int c0 = even_begin(row.chunks, a.S, s), c1 = even_begin(row.chunks, a.S, s + 1);
    Held<BF16> held;
    held.load(row, c0, c1);
    for (int i = threadIdx.x; i < SUBS; i += NT)
        sm.count[i] = 0;
    if (threadIdx.x == 0) {
        sm.n = 0;
        sm.at = SUBS;
    }
    float top[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
        top[i] = -INFINITY;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (c0 + i * NT < c1)                // (uniform)
#pragma unroll
            for (int e = 0; e < R::EPC; ++e)
                top[i % GROUPS] = fmaxf(top[i % GROUPS], R::get(held.x[i], e));
    float m = -INFINITY, low = INFINITY;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        m = fmaxf(m, top[i]);
        low = top[i] > -INFINITY ? fminf(low, top[i]) : low;
    }
    // (both in one turn)
    const auto max_of = [](float x, float y) { return fmaxf(x, y); };
    const auto min_of = [](float x, float y) { return fminf(x, y); };
    m = wave_all(m, -INFINITY, max_of);
    low = wave_all(low, INFINITY, min_of);
    if (threadIdx.x % 64 == 0) {
        sm.best[threadIdx.x / 64] = m;
        sm.low[threadIdx.x / 64] = low;
    }
    __syncthreads();
    m = wave_all(threadIdx.x % 64 < NWAVE ? sm.best[threadIdx.x % 64] : -INFINITY, -INFINITY, max_of);
    low = wave_all(threadIdx.x % 64 < NWAVE ? sm.low[threadIdx.x % 64] : INFINITY, INFINITY, min_of);
    Slice out = {m, -1, 0.0};
    if (!wish.few || !(m < INFINITY))
        return out;

    // the border: the first of SUBS steps down to the lowest of the groups' largest that
    // has k of them above it; if there are not k, whatever is not -inf
    // (groups so close, or so far apart, that fp32 has no such steps: one step, which all are in)
    const float range = m - low, steps = (SUBS - 1) / range, step = range < INFINITY && steps < INFINITY ? steps : 0.f;
    auto level = [&](float x) { return (m - x) * step; };
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
        if (top[i] > -INFINITY)
            atomicAdd(&sm.count[min((int)level(top[i]), SUBS - 1)], 1u);
    // (meanwhile the sum of the weights)
    const float base = m == -INFINITY ? 0.f : m, c2 = 1.44269504088896340736f / wish.T;
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (c0 + i * NT < c1)
#pragma unroll
            for (int e = 0; e < R::EPC; ++e)
                z += __builtin_amdgcn_exp2f((R::get(held.x[i], e) - base) * c2);
    __syncthreads();
    static_assert(SUBS == NT, "one step per thread");
    u64 all;
    const u64 before = block_before(sm.count[threadIdx.x], sm.scan, all);
    if (before < (u64)wish.k && before + sm.count[threadIdx.x] >= (u64)wish.k)
        sm.at = threadIdx.x;
    __syncthreads();
    const float border = sm.at == SUBS ? INFINITY : (float)(sm.at + 1);
    const int room = LIST / a.S;
    auto above = [&](float v) { return v > -INFINITY && (border == INFINITY || level(v) < border); };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
        if (above(top[g]))                   // (few threads have any)
#pragma unroll
            for (int i = g; i < HELD; i += GROUPS)
#pragma unroll
                for (int e = 0; e < R::EPC && c0 + i * NT < c1; ++e) {
                    const float v = R::get(held.x[i], e);
                    if (above(v)) {
                        const uint32_t n = atomicAdd(&sm.n, 1u);
                        if (n < (uint32_t)room)
                            sm.list[n] = place_of(v, row.index(c0 + threadIdx.x + i * NT, e));
                    }
                }
    out.z = block_all((double)z, 0.0, sm.z, [](double x, double y) { return x + y; });
    out.n = sm.n <= (uint32_t)room ? (int)sm.n : -1;
    return out;
}

// ---- 2: a slice's histogram ----------------------------------------------------------

// sm.hist and, for a top-k, sm.count; NaN if there is one
template <bool BF16>
__device__ __forceinline__ double fill_histogram(const SampleArgs &a, const Wish &wish, int b, int s, float best, Shared &sm)
{
    const Row<BF16> row(a, b);
    const int c0 = even_begin(row.chunks, a.S, s), c1 = even_begin(row.chunks, a.S, s + 1);
    fill_table(sm.table);
    for (int i = threadIdx.x; i < NB; i += NT) {
        sm.hist[i] = 0;
        sm.count[i] = 0;
    }
    if (threadIdx.x == 0)
        sm.found = 0;
    __syncthreads();
    const Weigher weigh = {best, 1.0 / (double)wish.T, sm.table};
    const bool counted = wish.k < a.V;
    bool nan = false;
    row.template each<2>(c0, c1, [&](int, const u32x4 &x) {
#pragma unroll
        for (int e = 0; e < Row<BF16>::EPC; ++e) {
            const float v = Row<BF16>::get(x, e);
            nan |= v != v;
            double r;
            const int i = weigh.bucket(v, r);
            if (i < NB - 1) {
                atomicAdd(&sm.hist[i], weigh.rounded(i, r));
                if (counted)
                    atomicAdd(&sm.count[i], 1u);
            }
        }
    });
    if (nan)
        sm.found = 1;
    __syncthreads();
    return sm.found ? NAN : 0.0;
}

// ---- 3: the place in the order, and the token -----------------------------------------

// A beginning of the order, of which a token is that `rank` tokens and `before` weight
// lie above (the first, which nothing lies above, in any case)
struct Border {
    u64 k;           // tokens
    double w;        // a token is in if less weight than this is before it
    double least;    // and its own is not less than this
    __device__ __forceinline__ bool in(u64 rank, u64 before, double own) const
    {
        return before == 0 || (rank < k && (double)before < w && own >= least);
    }
};

// Where the border lies among the threads' tokens (one each, where `active`; `rank` tokens
// and `before` weight lie above them all): those from place sm.cut up are within, sm.w_cut
// is all weight to there.  `exact`: a place's weight in units.  The places' range is cut in
// SUBS parts, the sums of the parts show in which the border lies, and so on with that
// part until FEW tokens are left, which are compared each with each.
template <class W>
__device__ __forceinline__ void narrow(Shared &sm, u64 place, u64 w, bool active, u64 rank, u64 before, const Border &border, W exact)
{
    for (;;) {
        if (threadIdx.x == 0) {
            sm.low_place = ~0ull;
            sm.high_place = 0;
            sm.n_few = 0;
            sm.at = 0;
        }
        sm.w[threadIdx.x] = 0;
        sm.n_of[threadIdx.x] = 0;
        __syncthreads();
        const u64 low = wave_all(active ? place : ~0ull, ~0ull, [](u64 x, u64 y) { return x < y ? x : y; });
        const u64 high = wave_all(active ? place : 0ull, 0ull, [](u64 x, u64 y) { return x > y ? x : y; });
        const u64 mask = __builtin_amdgcn_ballot_w64(active);
        uint32_t at = 0;
        if (mask) {
            if (threadIdx.x % 64 == 0) {
                atomicMin(&sm.low_place, low);
                atomicMax(&sm.high_place, high);
                at = atomicAdd(&sm.n_few, (uint32_t)__builtin_popcountll(mask));
            }
            at = __shfl(at, 0) + __builtin_popcountll(mask & ((1ull << threadIdx.x % 64) - 1));
        }
        if (active)
            sm.few[at] = Token{place, w};
        __syncthreads();
        const int n = sm.n_few;
        const u64 most = sm.high_place;
        if (n <= FEW) {
            // P neighbouring threads take a token, every P-th of the others each
            constexpr int P = NT / FEW;
            const int i = threadIdx.x / P, part = threadIdx.x % P;
            Token own = {0, 0};
            u64 above = 0;
            uint32_t many = 0;
            if (i < n) {
                own = sm.few[i];
                for (int j = part; j < n; j += P) {
                    const Token x = sm.few[j];
                    many += x.place > own.place;
                    above += x.place > own.place ? x.w : 0;
                }
            }
#pragma unroll
            for (int m = 1; m < P; m *= 2) {
                many += __shfl_xor(many, m);
                above += __shfl_xor(above, m);
            }
            const bool in = i < n && part == 0 && border.in(rank + many, before + above, border.least > 0.0 ? exact(own.place) : 0.0);
            // (none: a cut above all of these, not above what was above them)
            const auto least_of = [](u64 x, u64 y) { return x < y ? x : y; };
            const auto sum_of = [](u64 x, u64 y) { return x + y; };
            const u64 cut = wave_all(in ? own.place : n ? most + 1 : ~0ull, ~0ull, least_of);
            const u64 kept = wave_all(in ? own.w : 0ull, 0ull, sum_of);
            if (threadIdx.x % 64 == 0) {
                sm.sum[0][threadIdx.x / 64] = cut;
                sm.sum[1][threadIdx.x / 64] = kept;
            }
            __syncthreads();
            const int lane = threadIdx.x % 64;
            const u64 c = wave_all(lane < NWAVE ? sm.sum[0][lane] : ~0ull, ~0ull, least_of);
            const u64 k = wave_all(lane < NWAVE ? sm.sum[1][lane] : 0ull, 0ull, sum_of);
            if (threadIdx.x == 0) {
                sm.cut = c;
                sm.w_cut = before + k;
            }
            __syncthreads();
            return;
        }
        const u64 range = most - sm.low_place;
        const int shift = max(0, 54 - (int)__builtin_clzll(range | 1));     // range >> shift < SUBS
        static_assert(SUBS == 1024, "54");
        const uint32_t sub = (uint32_t)((most - place) >> shift);
        if (active) {
            atomicAdd(&sm.w[sub], w);
            atomicAdd(&sm.n_of[sub], 1u);
        }
        __syncthreads();
        u64 wb = sm.w[threadIdx.x], nb = sm.n_of[threadIdx.x];
        const bool some = nb;
        u64 all;
        block_before2(wb, nb, sm.sum, all);
        // (the largest weight that a place of the part could have)
        note_last(&sm.at, some && border.in(rank + nb, before + wb,
                                             border.least > 0.0 ? exact(most - ((u64)threadIdx.x << shift)) : 0.0), threadIdx.x);
        __syncthreads();
        if (threadIdx.x == sm.at) {
            sm.rank = rank + nb;
            sm.before = before + wb;
        }
        active &= sub == sm.at;
        __syncthreads();
        rank = sm.rank;
        before = sm.before;
        __syncthreads();
    }
}

// Where the border lies among the tokens of bucket b, of which `rank` tokens and `before`
// weight lie above: the tokens of it from place sm.cut up are within, sm.w_cut is the
// weight to there.  Returns how many tokens sm.list holds, the whole
// bucket and maybe some at its ends that are not of it, or -1 if they were too many.
template <bool BF16>
__device__ __forceinline__ int find_cut(const Row<BF16> &row, Shared &sm, const Weigher &weigh, int b, u64 rank, u64 before,
                        const Border &border)
{
    uint32_t lo = 0, hi = 0xFFFFFFFFu;
    // logits that may be in the bucket, by 32 bits
    const double slack = 1e-6 * (fabs(weigh.best) + 31.0 / weigh.inv_T);
    const float least_x = (float)(weigh.best - (b + 1) * BUCKET / weigh.inv_T - slack);
    const float most_x = (float)(weigh.best - b * BUCKET / weigh.inv_T + slack);
    auto here = [&](float v, uint32_t &key) {
        key = order_key(v);
        return v >= least_x && v <= most_x && key >= lo && key <= hi && weigh.bucket(v) == b;
    };
    // the whole bucket, by 32 bits alone: each thread then looks at its own token again
    __syncthreads();
    if (threadIdx.x == 0)
        sm.n = 0;
    __syncthreads();
    row.template each<4>(0, row.chunks, [&](int c, const u32x4 &x) {
#pragma unroll
        for (int e = 0; e < Row<BF16>::EPC; ++e) {
            const float v = Row<BF16>::get(x, e);
            if (v >= least_x && v <= most_x) {
                const uint32_t i = atomicAdd(&sm.n, 1u);
                if (i < LIST)
                    sm.list[i] = place_of(v, row.index(c, e));
            }
        }
    });
    __syncthreads();
    auto settle = [&](bool exactly) {
        const bool some = threadIdx.x < sm.n;
        const u64 place = some ? sm.list[threadIdx.x] : 0;
        const bool active = some && (exactly || weigh.bucket(logit_of(place)) == b);
        narrow(sm, place, active ? weigh.weight(logit_of(place)) : 0, active, rank, before, border,
               [&](u64 p) { return weigh.exact(logit_of(p)); });
    };
    const bool whole = sm.n <= LIST;
    const int n_whole = whole ? (int)sm.n : -1;
    while (!whole) {
        __syncthreads();
        if (threadIdx.x == 0) {
            sm.n = 0;
            sm.lo = 0xFFFFFFFFu;
            sm.hi = 0;
        }
        __syncthreads();
        uint32_t least = 0xFFFFFFFFu, most = 0;
        row.template each<4>(0, row.chunks, [&](int c, const u32x4 &x) {
#pragma unroll
            for (int e = 0; e < Row<BF16>::EPC; ++e) {
                const float v = Row<BF16>::get(x, e);
                uint32_t key;
                if (here(v, key)) {
                    const uint32_t i = atomicAdd(&sm.n, 1u);
                    if (i < LIST)
                        sm.list[i] = place_of(v, row.index(c, e));
                    least = min(least, key);
                    most = max(most, key);
                }
            }
        });
        least = wave_all(least, 0xFFFFFFFFu, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
        most = wave_all(most, 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        if (least <= most && threadIdx.x % 64 == 0) {
            atomicMin(&sm.lo, least);
            atomicMax(&sm.hi, most);
        }
        __syncthreads();
        const uint32_t n = sm.n;
        lo = sm.lo;
        hi = sm.hi;
        const u64 none = ((u64)hi + 1) << 32;    // a cut above all of these (not above what was above them)
        if (n <= LIST)
            break;
        if (lo == hi) {
            // ties: the first so many by index.  A thread takes chunks that follow one
            // another
            const float x = logit_of((u64)lo << 32);
            const double own = weigh.exact(x);
            const u64 w = weigh.weight(x);
            u64 in = 0;
            {   // the first token out, by halving
                u64 out = n;
                while (in < out) {
                    const u64 mid = (in + out) / 2;
                    if (border.in(rank + mid, before + mid * w, own))
                        in = mid + 1;
                    else
                        out = mid;
                }
            }
            const int per = (row.chunks + NT - 1) / NT;
            const int c0 = min(row.chunks, (int)threadIdx.x * per), c1 = min(row.chunks, c0 + per);
            u64 mine = 0, all;
            for (int c = c0; c < c1; ++c) {
                const u32x4 y = row.load(c);
#pragma unroll
                for (int e = 0; e < Row<BF16>::EPC; ++e)
                    mine += order_key(Row<BF16>::get(y, e)) == lo;
            }
            u64 at = block_before(mine, sm.scan, all);
            if (threadIdx.x == 0) {
                sm.cut = none;
                sm.w_cut = before + in * w;
            }
            __syncthreads();
            if (in > at && in <= at + mine)
                for (int c = c0; c < c1; ++c) {
                    const u32x4 y = row.load(c);
#pragma unroll
                    for (int e = 0; e < Row<BF16>::EPC; ++e)
                        if (order_key(Row<BF16>::get(y, e)) == lo && ++at == in)
                            sm.cut = place_of(x, row.index(c, e));
                }
            __syncthreads();
            return -1;
        }
        // too many: the part of the keys' range, from the top, in which the border lies
        const uint32_t step = (hi - lo) / SUBS + 1;
        for (int i = threadIdx.x; i < SUBS; i += NT) {
            sm.w[i] = 0;
            sm.n_of[i] = 0;
        }
        if (threadIdx.x == 0)
            sm.at = 0;
        __syncthreads();
        row.template each<2>(0, row.chunks, [&](int, const u32x4 &x) {
#pragma unroll
            for (int e = 0; e < Row<BF16>::EPC; ++e) {
                const float v = Row<BF16>::get(x, e);
                uint32_t key;
                if (here(v, key)) {
                    atomicAdd(&sm.w[(hi - key) / step], weigh.weight(v));
                    atomicAdd(&sm.n_of[(hi - key) / step], 1u);
                }
            }
        });
        __syncthreads();
        u64 wb = sm.w[threadIdx.x], nb = sm.n_of[threadIdx.x];
        const bool some = nb;
        u64 all;
        block_before2(wb, nb, sm.sum, all);
        const uint32_t key = hi - threadIdx.x * step;    // the part's largest, if it is one
        note_last(&sm.at, some && border.in(rank + nb, before + wb, weigh.exact(logit_of((u64)key << 32))), threadIdx.x);
        __syncthreads();
        if (threadIdx.x == sm.at) {
            sm.slice[0] = wb;
            sm.slice[1] = nb;
        }
        __syncthreads();
        before += sm.slice[0];
        rank += sm.slice[1];
        const uint32_t part = sm.at;
        const uint32_t below = hi - lo - part * step;   // keys of the range from the part's first down
        hi = hi - part * step;
        lo = below < step ? lo : hi - step + 1;
    }
    settle(!whole);
    return n_whole;
}

// `u` of a sum of weights, such that the token is the first whose sum is more
__device__ __forceinline__ u64 goal_of(float u, u64 total)
{
    const double g = (double)u * (double)total;
    const u64 t = g > 0.0 ? (u64)g : 0;
    return t < total ? t : total - 1;
}

template <bool BF16, bool ONE>
__device__ __forceinline__ void choose_token(const SampleArgs &a, const Wish &wish, int b, Shared &sm, Slice one)
{
    const Row<BF16> row(a, b);
    const int S = ONE ? 1 : a.S;
    float best = one.top;
    bool few = one.n >= 0;
    if (!ONE) {
        best = -INFINITY;
        few = true;
        for (int s = 0; s < S; ++s) {
            best = fmaxf(best, slice_at(a, b, s)->top);
            few &= slice_at(a, b, s)->n >= 0;
        }
    }
    double z = 0.0;
    if (best > -INFINITY && best < INFINITY)
        for (int s = 0; s < S; ++s) {
            const Slice x = ONE ? one : *slice_at(a, b, s);
            z += few && x.top > -INFINITY ? x.z * exp(((double)x.top - best) / wish.T) : x.z;
        }
    if (!(best > -INFINITY && best < INFINITY) || z != z) {
        if (threadIdx.x == 0) {
            a.token[b] = -1;
            a.logp[b] = NAN;
        }
        return;
    }
    const Weigher weigh = {best, 1.0 / (double)wish.T, sm.table};
    int token;
    if (few) {
        // a token a thread
        u64 place = 0;
        bool active = false;
        if (ONE) {
            active = (int)threadIdx.x < one.n;
            place = sm.list[threadIdx.x];
        } else {
            int n = 0;
            for (int s = 0; s < S; ++s) {
                const int ns = slice_at(a, b, s)->n, i = (int)threadIdx.x - n;
                if (i >= 0 && i < ns) {
                    active = true;
                    place = a.lists[((size_t)b * S + s) * (LIST / S) + i];
                }
                n += ns;
            }
        }
        auto exact = [&](u64 p) { return exp(((double)logit_of(p) - (double)best) * weigh.inv_T) * UNIT; };
        const u64 w = active ? (u64)(exact(place) + 0.5) : 0;
        // by top-k alone, for the weight that top_p is a part of (of no account without it); then by all
        Border border = {(u64)wish.k, INFINITY, 0.0};
        for (int turn = wish.p < 1.0 ? 0 : 1; turn < 2; ++turn) {
            if (turn == 1) {
                border.w = wish.p < 1.0 ? wish.p * (double)sm.w_cut : wish.p >= 1.0 ? INFINITY : 0.0;
                border.least = wish.min_p * UNIT;
                __syncthreads();
            }
            narrow(sm, place, w, active, 0, 0, border, exact);
        }
        const u64 goal = goal_of(wish.u, sm.w_cut);
        active &= place >= sm.cut;
        // the part of the indexes that the goal lies in, and the token in it
        const int shift = max(0, 22 - (int)__builtin_clz((uint32_t)a.V));   // V >> shift < SUBS
        const int index = index_of(place);
        sm.w[threadIdx.x] = 0;
        if (threadIdx.x == 0) {
            sm.n_few = 0;
            sm.found = 0;
        }
        __syncthreads();
        if (active)
            atomicAdd(&sm.w[index >> shift], w);
        __syncthreads();
        u64 all;
        const u64 part = sm.w[threadIdx.x], sum = block_before(part, sm.scan, all);
        if (sum <= goal && goal < sum + part) {
            sm.at = threadIdx.x;
            sm.before = sum;
        }
        __syncthreads();
        active &= (uint32_t)index >> shift == sm.at;
        if (active)
            sm.few[atomicAdd(&sm.n_few, 1u)] = Token{place, w};
        __syncthreads();
        if (active) {
            u64 at = sm.before;
            for (uint32_t j = 0; j < sm.n_few; ++j)
                at += index_of(sm.few[j].place) < index ? sm.few[j].w : 0;
            if (at <= goal && goal < at + w)
                sm.found = index;
        }
        __syncthreads();
        token = sm.found;
    } else {
        const bool counted = wish.k < a.V;
        if (!ONE) {
            fill_table(sm.table);
            const u64 *weights = a.weights + (size_t)b * S * NB;
            const uint32_t *counts = a.counts + (size_t)b * S * NB;
            for (int i = threadIdx.x; i < NB; i += NT) {
                u64 w = 0;
                uint32_t n = 0;
#pragma unroll 8
                for (int s = 0; s < S; ++s)
                    w += weights[s * NB + i];
                if (counted)
#pragma unroll 8
                    for (int s = 0; s < S; ++s)
                        n += counts[s * NB + i];
                sm.hist[i] = w;
                sm.count[i] = n;
            }
        }
        __syncthreads();
        // two buckets a thread: what lies before them
        const int i0 = 2 * threadIdx.x;
        u64 all, total;
        u64 n0 = (u64)sm.count[i0] + sm.count[i0 + 1], w0 = sm.hist[i0] + sm.hist[i0 + 1];
        block_before2(n0, w0, sm.sum, total);
        const u64 n1 = n0 + sm.count[i0], w1 = w0 + sm.hist[i0];
        z = (double)total / UNIT;
        // the last bucket that holds a token within the border (the first does), and what
        // is before it: in sm.at, sm.slice[0] and sm.slice[1]
        auto last_bucket = [&](const Border &border) {
            __syncthreads();
            if (threadIdx.x == 0)
                sm.at = 0;
            __syncthreads();
            // (a bucket's own weight: that of its lower end, the largest)
            const bool in0 = border.in(n0, w0, sm.table[i0]), in1 = border.in(n1, w1, sm.table[i0 + 1]);
            note_last(&sm.at, in0 || in1, (uint32_t)i0 + in1);
            __syncthreads();
            if (i0 == ((int)sm.at & ~1)) {
                sm.slice[0] = sm.at & 1 ? n1 : n0;
                sm.slice[1] = sm.at & 1 ? w1 : w0;
            }
            __syncthreads();
        };
        // by top-k alone, for the weight that top_p is a part of; then by all
        Border border = {counted ? (u64)wish.k : (u64)1 << 62, INFINITY, 0.0};
        u64 kept = total, cut = ~0ull;
        int at = NB - 1, listed = 0;
        for (int turn = counted ? 0 : 1; turn < 2; ++turn) {
            if (turn == 1) {
                border.w = wish.p * (double)kept;
                border.least = wish.min_p * UNIT;
            }
            last_bucket(border);
            at = sm.at;
            kept = total;
            if (at < NB - 1) {
                const u64 rank = sm.slice[0], before = sm.slice[1];
                listed = find_cut(row, sm, weigh, at, rank, before, border);
                cut = sm.cut;
                kept = sm.w_cut;
            }
        }
        const float least_x =         // (what is surely lower has no weight here)
            (float)(best - (at + 1) * BUCKET * wish.T - 1e-6 * (fabs((double)best) + 31.0 * wish.T));
        auto weight_in = [&](float x, int i) -> u64 {
            if (!(x >= least_x))
                return 0;
            double r;
            const int k = weigh.bucket(x, r);
            return k < at || (k == at && k < NB - 1 && place_of(x, i) >= cut) ? weigh.rounded(k, r) : 0;
        };
        // the slice that the goal lies in, from the slices' sums
        u64 goal = goal_of(wish.u, kept);
        int s = 0;
        if (!ONE) {
            __syncthreads();
            if (threadIdx.x < MAX_SLICES)
                sm.slice[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x / 64; i < S; i += NWAVE) {       // a wave to a slice
                const u64 *const w = a.weights + ((size_t)b * S + i) * NB;
                u64 sum = 0;
#pragma unroll 8
                for (int j = threadIdx.x % 64; j < at; j += 64)
                    sum += w[j];
                sum = wave_all(sum, (u64)0, [](u64 x, u64 y) { return x + y; });
                if (threadIdx.x % 64 == 0)
                    atomicAdd(&sm.slice[i], sum);
            }
            if (listed >= 0) {
                if ((int)threadIdx.x < listed && sm.list[threadIdx.x] >= cut &&
                    weigh.bucket(logit_of(sm.list[threadIdx.x])) == at) {
                    const u64 place = sm.list[threadIdx.x];
                    atomicAdd(&sm.slice[even_part_of(row.chunks, S, (index_of(place) + row.off) / Row<BF16>::EPC)],
                              weigh.weight(logit_of(place)));
                }
            } else
                row.template each<2>(0, row.chunks, [&](int c, const u32x4 &x) {
#pragma unroll
                    for (int e = 0; e < Row<BF16>::EPC; ++e) {
                        const float v = Row<BF16>::get(x, e);
                        if (weigh.bucket(v) == at && place_of(v, row.index(c, e)) >= cut)
                            atomicAdd(&sm.slice[even_part_of(row.chunks, S, c)], weigh.weight(v));
                    }
                });
            __syncthreads();
            while (s + 1 < S && goal >= sm.slice[s])
                goal -= sm.slice[s++];
        }
        // and the token in it; a thread takes chunks that follow one another
        const int begin = even_begin(row.chunks, S, s), end = even_begin(row.chunks, S, s + 1);
        const int per = (end - begin + NT - 1) / NT;
        const int c0 = min(end, begin + (int)threadIdx.x * per), c1 = min(end, c0 + per);
        u64 mine = 0;
        for (int c = c0; c < c1; ++c) {
            const u32x4 x = row.load(c);
#pragma unroll
            for (int e = 0; e < Row<BF16>::EPC; ++e)
                mine += weight_in(Row<BF16>::get(x, e), row.index(c, e));
        }
        u64 sum = block_before(mine, sm.scan, all);
        if (threadIdx.x == 0)
            sm.found = 0;
        __syncthreads();
        if (sum <= goal && goal < sum + mine)
            for (int c = c0; c < c1; ++c) {
                const u32x4 x = row.load(c);
#pragma unroll
                for (int e = 0; e < Row<BF16>::EPC; ++e) {
                    const u64 w = weight_in(Row<BF16>::get(x, e), row.index(c, e));
                    if (sum <= goal && goal < sum + w)
                        sm.found = row.index(c, e);
                    sum += w;
                }
            }
        __syncthreads();
        token = sm.found;
    }
    if (threadIdx.x == 0) {
        a.token[b] = token;
        a.logp[b] = (float)(((double)row.value(token) - best) / wish.T - log(z));
    }
}

// ---- the kernels -------------------------------------------------------------------------

template <bool BF16>
__global__ __launch_bounds__(NT) void sample_one_kernel(SampleArgs a)
{
    __shared__ Shared sm;
    const int b = blockIdx.x;
    const Wish wish = wish_of(a, b);
    Slice one = find_candidates<BF16>(a, wish, b, 0, sm);
    __syncthreads();
    if (one.n < 0 && one.top > -INFINITY && one.top < INFINITY)
        one.z = fill_histogram<BF16>(a, wish, b, 0, one.top, sm);
    __syncthreads();
    choose_token<BF16, true>(a, wish, b, sm, one);
}

template <bool BF16>
__global__ __launch_bounds__(NT) void sample_candidates_kernel(SampleArgs a)
{
    __shared__ Shared sm;
    const int b = blockIdx.x / a.S, s = blockIdx.x % a.S;
    const Slice x = find_candidates<BF16>(a, wish_of(a, b), b, s, sm);
    for (int i = threadIdx.x; i < x.n; i += NT)
        a.lists[((size_t)b * a.S + s) * (LIST / a.S) + i] = sm.list[i];
    if (threadIdx.x == 0)
        *slice_at(a, b, s) = x;
}

template <bool BF16>
__global__ __launch_bounds__(NT) void sample_histogram_kernel(SampleArgs a)
{
    __shared__ Shared sm;
    const int b = blockIdx.x / a.S, s = blockIdx.x % a.S;
    float best = -INFINITY;
    bool few = true;
    for (int i = 0; i < a.S; ++i) {
        best = fmaxf(best, slice_at(a, b, i)->top);
        few &= slice_at(a, b, i)->n >= 0;
    }
    if (few || !(best > -INFINITY && best < INFINITY))
        return;
    const Wish wish = wish_of(a, b);
    const double z = fill_histogram<BF16>(a, wish, b, s, best, sm);
    const bool counted = wish.k < a.V;
    for (int i = threadIdx.x; i < NB; i += NT) {
        a.weights[((size_t)b * a.S + s) * NB + i] = sm.hist[i];
        if (counted)
            a.counts[((size_t)b * a.S + s) * NB + i] = sm.count[i];
    }
    if (threadIdx.x == 0)
        slice_at(a, b, s)->z = z;
}

template <bool BF16>
__global__ __launch_bounds__(NT) void sample_choose_kernel(SampleArgs a)
{
    __shared__ Shared sm;
    choose_token<BF16, false>(a, wish_of(a, blockIdx.x), blockIdx.x, sm, Slice{});
}

// Slices of a row: one workgroup takes rows of up to 32768 logits, and any where there
// are rows for half of the CUs; a slice has HELD NT chunks of 16 bytes at most (a row
// touches up to two more than it has bytes for).  Slices pay for the histogram's passes over a
// row, candidates (a small top-k) cost two kernels more with them; the host does not know
// which a row takes.  us, 1 | 2 | 4 slices | as many as here, top-k 40 with top-p | top-p alone:
//   1 x 32768 fp32     18.1 22.1 26.8 | 18.1     35.0 34.5 31.8 | 35.0
//   64 x 32768 fp32    19.7 23.8 27.7 | 19.7     37.1 38.4 37.0 | 37.1
//   1 x 40000 fp32     19.5 22.8 27.0 | 26.7     40.3 37.8 34.5 | 34.1
//   64 x 50000 fp32    23.0 25.5 29.5 | 36.7     52.9 49.6 45.5 | 50.6
//   1 x 152064 bf16       - 28.9 30.2 | 55.3        - 78.9 59.4 | 52.8
//   127 x 131072 bf16  32.4 32.2 41.5 | 41.3     105  81.9 73.2 | 73.7
//   128 x 131072 bf16  32.3 32.0 41.7 | 32.0     105  82.3 73.8 | 105
//   256 x 131072 bf16  37.2 47.0 62.5 | 37.5     113  103  98.3 | 113
//   256 x 152064 bf16     - 51.3 66.8 | 51.5        - 116  109  | 117
// (55.3: 18 slices allow no candidates for a top-k of 40.)  A longer HELD would take 152064
// 16-bit logits in one slice too; candidates have its chunks in registers, of which 122 of
// 128 are taken.
int slices_of(int B, int V, int l_bf16)
{
    const int per_chunk = l_bf16 ? 8 : 4;
    const int least = (V / per_chunk + 2 + HELD * NT - 1) / (HELD * NT);
    if (V <= 32768 || B >= 128)
        return least;
    return std::max(least, std::min(std::min(512 / B, V / 8192), MAX_SLICES));
}

struct Workspace {
    size_t slices, lists, weights, counts, all;
};

Workspace workspace_of(int B, int slices)
{
    const size_t n = (size_t)B * slices;
    Workspace w = {};
    if (slices == 1)
        return w;
    w.lists = w.slices + (n * sizeof(Slice) + 15) / 16 * 16;
    w.weights = w.lists + (size_t)B * LIST * 8;
    w.counts = w.weights + n * NB * 8;
    w.all = w.counts + n * NB * 4;
    return w;
}

ta_status check_sample_sizes(int B, int V)
{
    return B < 1 || V < 1 || B > MAX_B || V > MAX_V ? TA_ERR_INVALID_SHAPE : TA_OK;
}

}  // namespace

extern "C" {

ta_status sample_logits(const void *logits, int64_t stride, int l_bf16, const float *u, const float *temperature,
                        const int *top_k, const float *top_p, const float *min_p, int *token, float *logp, int B,
                        int V, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!logits || !u || !token || !logp)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sample_sizes(B, V);
    if (rc != TA_OK)
        return rc;
    if (stride < 0 || stride > 1ll << 30)
        return TA_ERR_INVALID_SHAPE;
    if (misaligned(logits, l_bf16 ? 2 : 4) || misaligned(u, 4) || misaligned(temperature, 4) || misaligned(top_k, 4) ||
        misaligned(top_p, 4) || misaligned(min_p, 4) || misaligned(token, 4) || misaligned(logp, 4))
        return TA_ERR_MISALIGNED;
    const size_t row = (size_t)B * 4;
    const Span out[] = {{token, row}, {logp, row}};
    const Span in[] = {{logits, (size_t)((B - 1) * stride + V) * (l_bf16 ? 2 : 4)}, {u, row}, {temperature, row},
                       {top_k, row}, {top_p, row}, {min_p, row}};
    if (overlaps(out[0], out[1]))
        return TA_ERR_ALIASING;
    for (const Span &s : in)
        if (overlaps(out[0], s) || overlaps(out[1], s))
            return TA_ERR_ALIASING;
    const int slices = slices_of(B, V, l_bf16);
    const Workspace w = workspace_of(B, slices);
    if (w.all) {
        if (!workspace || workspace_bytes < w.all)
            return TA_ERR_WORKSPACE;
        if (misaligned(workspace))
            return TA_ERR_MISALIGNED;
        const Span ws = {workspace, w.all};
        if (overlaps(ws, out[0]) || overlaps(ws, out[1]))
            return TA_ERR_ALIASING;
        for (const Span &s : in)
            if (overlaps(ws, s))
                return TA_ERR_ALIASING;
    }
    unsigned char *const ws = (unsigned char *)workspace;
    const SampleArgs a = {logits, stride, u, temperature, top_k, top_p, min_p, token, logp, V, slices,
                          (Slice *)(ws + w.slices), (u64 *)(ws + w.lists), (u64 *)(ws + w.weights),
                          (uint32_t *)(ws + w.counts)};
    hipStream_t s = (hipStream_t)stream;
    if (a.S == 1) {
        hipLaunchKernelGGL(l_bf16 ? sample_one_kernel<true> : sample_one_kernel<false>, dim3(B), dim3(NT), 0, s, a);
        return hipGetLastError() == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
    }
    hipLaunchKernelGGL(l_bf16 ? sample_candidates_kernel<true> : sample_candidates_kernel<false>, dim3(B * a.S), dim3(NT), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
        hipLaunchKernelGGL(l_bf16 ? sample_histogram_kernel<true> : sample_histogram_kernel<false>, dim3(B * a.S), dim3(NT), 0, s, a);
        e = hipGetLastError();
    }
    if (e == hipSuccess) {
        hipLaunchKernelGGL(l_bf16 ? sample_choose_kernel<true> : sample_choose_kernel<false>, dim3(B), dim3(NT), 0, s, a);
        e = hipGetLastError();
    }
    return e == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

ta_status sample_logits_workspace_bytes(int B, int V, int l_bf16, size_t *bytes)
{
    if (!bytes)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sample_sizes(B, V);
    if (rc != TA_OK)
        return rc;
    *bytes = workspace_of(B, slices_of(B, V, l_bf16)).all;
    return TA_OK;
}

// (fp32's rows have as many slices as bf16's, or more)
ta_status sample_workspace_bytes(int B, int V, size_t *bytes) { return sample_logits_workspace_bytes(B, V, 0, bytes); }

}  // extern "C"
