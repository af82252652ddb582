// Paged key/value cache for gfx950 (MI355X): new tokens' K and V into the
// pages (kv_cache_append), and attention of one new token per sequence over
// them (attn_decode_paged).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tileattn.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float E4M3_MAX = 448.f;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

struct AppendArgs {
    const uint16_t *K, *V;
    int64_t k_stride, v_stride;
    const int *seq, *pos;
    void *Kc, *Vc;
    const float *ks, *vs;
    const int *table;
    int T, B, Hkv, num_pages, page_shift, max_pages;
};

// x / s in the range of e4m3, NaN as it is (the conversion rounds to nearest even)
__device__ __forceinline__ float e4m3_arg(float x, float s)
{
    const float y = x / s;
    return y != y ? y : fminf(fmaxf(y, -E4M3_MAX), E4M3_MAX);
}

// One thread moves 8 elements (16 bytes) of a token's K or V row: thread i of
// a token takes chunk i of its 2 Hkv D / 8, K first.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    const int per = a.Hkv * (D / 8);               // chunks of a token's K
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int t = (int)(i / (2 * per));
    if (t >= a.T)
        return;
    int c = (int)(i % (2 * per));
    const bool is_v = c >= per;
    c -= is_v ? per : 0;
    const int h = c / (D / 8), ch = c % (D / 8);
    const int sq = a.seq ? a.seq[t] : t, pos = a.pos[t];
    const int pg = pos >> a.page_shift;
    if (sq < 0 || sq >= a.B || pos < 0 || pg >= a.max_pages)
        return;
    const int page = a.table[(size_t)sq * a.max_pages + pg];
    if (page < 0 || page >= a.num_pages)
        return;
    const u32x4 x = *(const u32x4 *)(is_v ? a.V + t * a.v_stride + 8 * c : a.K + t * a.k_stride + 8 * c);
    const size_t row = ((((size_t)page * a.Hkv + h) << a.page_shift) + (pos & ((1 << a.page_shift) - 1)));
    void *const to = is_v ? a.Vc : a.Kc;
    if (E4M3) {
        const float *sc = is_v ? a.vs : a.ks;
        const float s = sc ? sc[h] : 1.f;
        u32x2 y;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(bf16_lo(x[2 * j]), s),
                                                    e4m3_arg(bf16_hi(x[2 * j]), s), 0, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_arg(bf16_lo(x[2 * j + 1]), s),
                                                e4m3_arg(bf16_hi(x[2 * j + 1]), s), w, true);
            y[j] = (uint32_t)w;
        }
        *(u32x2 *)((uint8_t *)to + row * D + 8 * ch) = y;
    } else {
        *(u32x4 *)((uint16_t *)to + row * D + 8 * ch) = x;
    }
}

struct PagedArgs {
    const uint16_t *Q;
    int64_t q_stride;
    const void *K, *V;
    const float *ks, *vs;
    const int *table, *lens;
    void *O;
    float *LSE;
    int B, Hq, Hkv, num_pages, page_shift, max_pages;
    float scale;
};

template <int D, bool E4M3>
__device__ __forceinline__ float cache_at(const void *c, size_t row, int d)
{
    if (E4M3)
        return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)c)[row * D + d], 0);
    return __uint_as_float((uint32_t)((const uint16_t *)c)[row * D + d] << 16);
}

// One wave per query row: the lanes share a key's dims, one key after the other.
template <int D, bool E4M3, bool OBF16>
__global__ __launch_bounds__(64) void attn_paged_kernel(PagedArgs a)
{
    constexpr int PL = D / 64;
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, h = hq / (a.Hq / a.Hkv);
    const int lane = threadIdx.x;
    const int len = a.lens[b];
    const float ks = (a.ks ? a.ks[h] : 1.f) * a.scale, vs = a.vs ? a.vs[h] : 1.f;
    float q[PL], acc[PL], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        q[i] = __uint_as_float((uint32_t)a.Q[b * a.q_stride + (size_t)hq * D + lane * PL + i] << 16);
        acc[i] = 0.f;
    }
    bool bad = len < 0 || len > (int64_t)a.max_pages << a.page_shift;
    for (int t = 0; !bad && t < len; ++t) {
        const int page = a.table[(size_t)b * a.max_pages + (t >> a.page_shift)];
        if (page < 0 || page >= a.num_pages) {
            bad = true;
            break;
        }
        const size_t row = (((size_t)page * a.Hkv + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PL; ++i)
            s += q[i] * cache_at<D, E4M3>(a.K, row, lane * PL + i);
#pragma unroll
        for (int o = 32; o; o >>= 1)
            s += __shfl_xor(s, o);
        s *= ks;
        const float mn = fmaxf(m, s);
        const float al = m == mn ? 1.f : __expf(m - mn), p = s == mn ? 1.f : __expf(s - mn);
        m = mn;
        l = l * al + p;
#pragma unroll
        for (int i = 0; i < PL; ++i)
            acc[i] = acc[i] * al + p * cache_at<D, E4M3>(a.V, row, lane * PL + i);
    }
    const size_t r = (size_t)b * a.Hq + hq;
    const float inv = bad ? NAN : len == 0 ? 0.f : vs / l;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        const float o = acc[i] * inv;
        if (OBF16)
            ((uint16_t *)a.O)[r * D + lane * PL + i] = (uint16_t)pack_bf16(o, 0.f);
        else
            ((float *)a.O)[r * D + lane * PL + i] = o;
    }
    if (lane == 0)
        a.LSE[r] = bad ? NAN : len == 0 ? -INFINITY : m + logf(l);
}

bool misaligned(const void *p, uintptr_t to = 16) { return ((uintptr_t)p & (to - 1)) != 0; }

struct Span {
    const void *p;
    size_t n;
};

bool overlaps(Span a, Span b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.n && y < x + a.n;
}

// the sizes and types that both entry points check alike
ta_status check_cache(int B, int Hkv, int D, int num_pages, int page_size, int max_pages, int cache_e4m3,
                      const float *k_scale, const float *v_scale)
{
    if (B < 1 || Hkv < 1 || D < 1 || num_pages < 1 || page_size < 1 || max_pages < 1)
        return TA_ERR_INVALID_SHAPE;
    if ((D != 64 && D != 128) || page_size < 16 || (page_size & (page_size - 1)))
        return TA_ERR_UNSUPPORTED;
    if (!cache_e4m3 && (k_scale || v_scale))
        return TA_ERR_UNSUPPORTED;
    if ((int64_t)max_pages * page_size > 1ll << 30 || num_pages > 1 << 28 || Hkv > 1 << 16 ||
        (int64_t)Hkv * page_size > 1ll << 30)
        return TA_ERR_INVALID_SHAPE;
    return TA_OK;
}

// elements of a cache: below 2^28 2^30 2^7 = 2^65 by the checks alone, so in 128 bits
size_t cache_bytes(int Hkv, int D, int num_pages, int page_size, int cache_e4m3)
{
    const unsigned __int128 n = (unsigned __int128)num_pages * Hkv * page_size * D * (cache_e4m3 ? 1 : 2);
    return n > (1ull << 62) ? (size_t)1 << 62 : (size_t)n;
}

}  // namespace

extern "C" {

ta_status kv_cache_append(const void *K, const void *V, int64_t k_stride, int64_t v_stride,
                          const int *seq, const int *pos, void *K_cache, void *V_cache,
                          int cache_e4m3, const float *k_scale, const float *v_scale,
                          const int *page_table, int T, int B, int Hkv, int D, int num_pages,
                          int page_size, int max_pages, void *stream)
{
    if (!K || !V || !pos || !K_cache || !V_cache || !page_table)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_cache(B, Hkv, D, num_pages, page_size, max_pages, cache_e4m3, k_scale, v_scale);
    if (rc != TA_OK)
        return rc;
    const int64_t row = (int64_t)Hkv * D;
    const int64_t wg = T < 1 ? 0 : ((int64_t)T * (row / 4) + 255) / 256;
    if (T < 1 || (!seq && T > B) || k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8 ||
        k_stride > 1ll << 30 || v_stride > 1ll << 30 || wg >= 1ll << 24)
        return TA_ERR_INVALID_SHAPE;
    if (misaligned(K) || misaligned(V) || misaligned(K_cache) || misaligned(V_cache) || misaligned(seq, 4) ||
        misaligned(pos, 4) || misaligned(page_table, 4) || misaligned(k_scale, 4) || misaligned(v_scale, 4))
        return TA_ERR_MISALIGNED;
    const size_t cb = cache_bytes(Hkv, D, num_pages, page_size, cache_e4m3);
    const Span kc = {K_cache, cb}, vc = {V_cache, cb};
    const Span in[] = {{K, (size_t)((T - 1) * k_stride + row) * 2}, {V, (size_t)((T - 1) * v_stride + row) * 2},
                       {seq, (size_t)T * 4}, {pos, (size_t)T * 4}, {page_table, (size_t)B * max_pages * 4},
                       {k_scale, (size_t)Hkv * 4}, {v_scale, (size_t)Hkv * 4}};
    if (overlaps(kc, vc))
        return TA_ERR_ALIASING;
    for (const Span &s : in)
        if (overlaps(kc, s) || overlaps(vc, s))
            return TA_ERR_ALIASING;
    const AppendArgs a = {(const uint16_t *)K, (const uint16_t *)V, k_stride, v_stride, seq, pos, K_cache, V_cache,
                          k_scale, v_scale, page_table, T, B, Hkv, num_pages, __builtin_ctz(page_size), max_pages};
    const dim3 grid((unsigned)wg), block(256);
    hipStream_t s = (hipStream_t)stream;
    const auto kernel = D == 64 ? (cache_e4m3 ? append_kernel<64, true> : append_kernel<64, false>)
                                : (cache_e4m3 ? append_kernel<128, true> : append_kernel<128, false>);
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
    return hipGetLastError() == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

ta_status attn_decode_paged(const void *Q, int64_t q_stride, const void *K_cache,
                            const void *V_cache, int cache_e4m3, const float *k_scale,
                            const float *v_scale, const int *page_table, const int *seq_lens,
                            void *O, int o_bf16, float *LSE, int B, int Hq, int Hkv, int D,
                            int num_pages, int page_size, int max_pages, float scale,
                            void *stream)
{
    if (!Q || !K_cache || !V_cache || !page_table || !seq_lens || !O || !LSE)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_cache(B, Hkv, D, num_pages, page_size, max_pages, cache_e4m3, k_scale, v_scale);
    if (rc != TA_OK)
        return rc;
    const int64_t row = (int64_t)Hq * D;
    if (Hq < 1 || Hq % Hkv || q_stride < row || q_stride % 8 || q_stride > 1ll << 30 || Hq > 1 << 16 ||
        (int64_t)B * Hq >= 1ll << 24)
        return TA_ERR_INVALID_SHAPE;
    if (misaligned(Q) || misaligned(K_cache) || misaligned(V_cache) || misaligned(O) || misaligned(LSE) ||
        misaligned(page_table, 4) || misaligned(seq_lens, 4) || misaligned(k_scale, 4) || misaligned(v_scale, 4))
        return TA_ERR_MISALIGNED;
    if (!(scale >= 0.f) || !(scale <= 3.402823466e+38f))
        return TA_ERR_INVALID_SCALE;
    const size_t cb = cache_bytes(Hkv, D, num_pages, page_size, cache_e4m3);
    const Span o = {O, (size_t)B * row * (o_bf16 ? 2 : 4)}, l = {LSE, (size_t)B * Hq * 4};
    const Span in[] = {{Q, (size_t)((B - 1) * q_stride + row) * 2}, {K_cache, cb}, {V_cache, cb},
                       {page_table, (size_t)B * max_pages * 4}, {seq_lens, (size_t)B * 4},
                       {k_scale, (size_t)Hkv * 4}, {v_scale, (size_t)Hkv * 4}};
    if (overlaps(o, l))
        return TA_ERR_ALIASING;
    for (const Span &s : in)
        if (overlaps(o, s) || overlaps(l, s))
            return TA_ERR_ALIASING;
    const PagedArgs a = {(const uint16_t *)Q, q_stride, K_cache, V_cache, k_scale, v_scale, page_table, seq_lens, O,
                         LSE, B, Hq, Hkv, num_pages, __builtin_ctz(page_size), max_pages, scale};
    const dim3 grid((unsigned)(B * Hq)), block(64);
    hipStream_t s = (hipStream_t)stream;
    const auto kernel =
        D == 64 ? (cache_e4m3 ? (o_bf16 ? attn_paged_kernel<64, true, true> : attn_paged_kernel<64, true, false>)
                              : (o_bf16 ? attn_paged_kernel<64, false, true> : attn_paged_kernel<64, false, false>))
                : (cache_e4m3 ? (o_bf16 ? attn_paged_kernel<128, true, true> : attn_paged_kernel<128, true, false>)
                              : (o_bf16 ? attn_paged_kernel<128, false, true> : attn_paged_kernel<128, false, false>));
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
    return hipGetLastError() == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

}  // extern "C"
