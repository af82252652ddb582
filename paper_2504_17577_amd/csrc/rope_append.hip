// New tokens' queries, keys and values from a fused projection to where attention
// reads them, on gfx950 (MI355X): norm of queries and keys per head, position
// rotation, and the append to the paged cache, in one pass (qk_norm_rope_append).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "cache_checks.h"
#include "mxfp4.h"
#include "tileattn.h"

namespace {

using namespace tileattn_detail;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float E4M3_MAX = 448.f;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

struct RopeArgs {
    const uint16_t *Q, *K, *V;
    int64_t q_stride, k_stride, v_stride;
    const uint16_t *qw, *kw;
    const float *turn;            // [positions][rot]: cosines, sines
    const int *seq, *pos;
    uint16_t *Qo;
    void *Kc, *Vc;
    const void *ks, *vs;          // fp32 [Hkv]; the 4-bit caches' scales, written
    const int *table;
    float eps;
    int rot, positions;           // 0 and 0 without a rotation
    int B, Hq, Hkv, num_pages, page_shift, max_pages;
};

// The value of lane l of this lane's head, for 32 and 64 bits
template <int HL>
__device__ __forceinline__ float from_lane(float x, int l) { return __shfl(x, l, HL); }
template <int HL>
__device__ __forceinline__ double from_lane(double x, int l) { return __shfl(x, l, HL); }

// 1 / sqrt(mean(x^2) + eps) where 32 bits do not hold the sum or squares that count in it:
// of x over a power of two, the larger one of x's and of the root of eps
template <int HL>
__device__ __forceinline__ float norm_far(float (&x)[8], float eps)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        top = fmaxf(top, fabsf(x[i]));
#pragma unroll
    for (int m = 1; m < HL; m *= 2)
        top = fmaxf(top, __shfl_xor(top, m, HL));
    int e = __builtin_amdgcn_frexp_expf(top);
    if (eps > 0.f)
        e = max(e, (__builtin_amdgcn_frexp_expf(eps) + 1) / 2);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = ldexpf(x[i], -e);
        sum += x[i] * x[i];
    }
#pragma unroll
    for (int m = 1; m < HL; m *= 2)
        sum += __shfl_xor(sum, m, HL);
    return 1.f / sqrtf(sum * (1.f / (8 * HL)) + ldexpf(eps, -2 * e));
}

// One head's eight numbers of this lane, normed (with a weight) and rotated: F is the
// arithmetic's type.  Pairs of halves: the partner's numbers are those of the lane
// rot / 16 to the right or left; pairs of neighbours: the lane's own.
template <int HL, bool INTER, class F>
__device__ __forceinline__ void normed_rotated(const RopeArgs &a, int ch, const uint16_t *w, const float (&cs)[8],
                                               const float (&sn)[8], F (&x)[8])
{
    if (w) {
        // (loaded here: behind the branch below it made 16384 tokens' 72 us 73.2, in 4 bits 96 us 101)
        const u32x4 wv = *(const u32x4 *)(w + 8 * ch);
        F sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            sum += x[i] * x[i];
#pragma unroll
        for (int m = 1; m < HL; m *= 2)
            sum += __shfl_xor(sum, m, HL);
        const F mean = sum * F(1.0 / (8 * HL)) + F(a.eps);
        F r = F(1) / sqrt(mean);
        if constexpr (sizeof(F) == 4)
            if (!(mean >= 0x1p-100f && mean < INFINITY))   // (the same for all of a head's lanes)
                r = norm_far<HL>(x, a.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = x[2 * i] * r * F(bf16_lo(wv[i]));
            x[2 * i + 1] = x[2 * i + 1] * r * F(bf16_hi(wv[i]));
        }
    }
    if (a.rot == 0)
        return;
    const int half = a.rot / 16;            // lanes of half the rotated dims
    if (INTER) {
        if (ch < 2 * half)
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const F p = x[i], q = x[i + 1];
                x[i] = p * F(cs[i / 2]) - q * F(sn[i / 2]);
                x[i + 1] = q * F(cs[i / 2]) + p * F(sn[i / 2]);
            }
    } else {
        const int other = ch < half ? ch + half : ch < 2 * half ? ch - half : ch;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const F y = from_lane<HL>(x[i], other);
            if (ch < 2 * half)
                x[i] = x[i] * F(cs[i]) + (ch < half ? -y : y) * F(sn[i]);
        }
    }
}

// A workgroup takes some of the heads of one token, a lane 8 elements (16 bytes) of a
// head; a head's lanes are 8 or 16 neighbours, so that the norm's sum and the pairs of
// halves are exchanges within a wave.  A lane's cosines and sines serve all its heads.
// Queries and what a bf16 cache takes are computed in 32 bits.  Keys for 8 and 4 bits
// are computed in 64 and rounded to 32 bits once before they meet the cache's type: a
// key next to the border of two of its numbers (a quarter of the value apart in 4 bits)
// falls where the exact one does.  HBM bounds a prefill into bf16 (16384 tokens of 32 + 8 + 8
// heads of 128 dims, normed, 411 MB read and written: 72 us, 5.7 TB/s; a copy of 2 GiB reaches
// 4.8), the loads one behind the other (seq and pos, the table, then the row) a few tokens (32:
// 3.2 us, 3.7 into 8 and 4 bits).  Keys in 64 bits take 94 registers, five waves a SIMD where bf16
// has eight, and e4m3's a division by the scale each: 16384 tokens into 8 bits 108 us of 80 at the
// copy's rate, 92 without the norm, into 4 bits 95 of 75, 78 without; 2047 tokens 12, 17.8 and
// 15.7 us.  Keys and values alone (kv_cache_append into 4 bits): 16384 tokens 33 us of 18, 2047 6.1.
template <int D, int TYPE, bool INTER>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a)
{
    constexpr int HL = D / 8, PER = 256 / HL;   // lanes of a head, heads at a time
    const int t = blockIdx.x, ch = threadIdx.x % HL;
    const int heads = a.Hq + 2 * a.Hkv;
    const int pos = a.pos[t], sq = a.seq ? a.seq[t] : t;
    // a token whose position has no angles: NaN in its queries, nothing in the cache
    const bool turned = a.rot == 0 || pos < a.positions;
    const int pg = pos >> a.page_shift;
    int page = -1;
    if (turned && sq >= 0 && sq < a.B && pos >= 0 && pg < a.max_pages)
        page = a.table[(size_t)sq * a.max_pages + pg];
    const bool held = page >= 0 && page < a.num_pages;

    float cs[8], sn[8];
    if (a.rot && pos >= 0 && turned && 8 * ch < a.rot) {
        const float *c = a.turn + (size_t)pos * a.rot;
        const int j = INTER ? 4 * ch : 8 * ch % (a.rot / 2);
#pragma unroll
        for (int i = 0; i < (INTER ? 4 : 8); i += 4) {
            const f32x4 x = *(const f32x4 *)(c + j + i), y = *(const f32x4 *)(c + a.rot / 2 + j + i);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                cs[i + n] = x[n];
                sn[i + n] = y[n];
            }
        }
    }

    for (int h = blockIdx.y * PER + threadIdx.x / HL; h < heads; h += gridDim.y * PER) {
        const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
        const int hk = is_q ? 0 : is_v ? h - a.Hq - a.Hkv : h - a.Hq;
        if (is_q && (pos < 0 || !turned)) {
            const uint32_t n = pos < 0 ? 0u : 0x7FC07FC0u;
            *(u32x4 *)(a.Qo + ((size_t)t * a.Hq + h) * D + 8 * ch) = u32x4{n, n, n, n};
            continue;
        }
        if (!is_q && !held)
            continue;
        const uint16_t *from = is_q ? a.Q + t * a.q_stride + (size_t)h * D
                               : is_v ? a.V + t * a.v_stride + (size_t)hk * D
                                      : a.K + t * a.k_stride + (size_t)hk * D;
        u32x4 x = __builtin_nontemporal_load((const u32x4 *)(from + 8 * ch));
        const size_t row = (((size_t)max(page, 0) * a.Hkv + hk) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(x[i]);
            f[2 * i + 1] = bf16_hi(x[i]);
        }
        const float s = TYPE == TA_CACHE_E4M3 && !is_q && (is_v ? a.vs : a.ks) ? ((const float *)(is_v ? a.vs : a.ks))[hk] : 1.f;
        if (is_q || (TYPE == TA_CACHE_BF16 && !is_v)) {
            normed_rotated<HL, INTER, float>(a, ch, is_q ? a.qw : a.kw, cs, sn, f);
        } else if (!is_v) {
            double d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                d[i] = f[i];
            normed_rotated<HL, INTER, double>(a, ch, a.kw, cs, sn, d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = (float)(TYPE == TA_CACHE_E4M3 ? d[i] / (double)s : d[i]);
        } else if (TYPE == TA_CACHE_E4M3) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = f[i] / s;
        }
        if (is_q || TYPE == TA_CACHE_BF16) {
            if (!is_v)
                x = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
            uint16_t *to = is_q ? a.Qo + ((size_t)t * a.Hq + h) * D : (uint16_t *)(is_v ? a.Vc : a.Kc) + row * D;
            __builtin_nontemporal_store(x, (u32x4 *)(to + 8 * ch));
        } else if (TYPE == TA_CACHE_E4M3) {
            u32x2 y;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                f[j] = f[j] != f[j] ? f[j] : fminf(fmaxf(f[j], -E4M3_MAX), E4M3_MAX);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
                y[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], w, true);
            }
            *(u32x2 *)((uint8_t *)(is_v ? a.Vc : a.Kc) + row * D + 8 * ch) = y;
        } else {
            uint32_t top = 0;               // of the group's four lanes (as bits: NaN is the largest)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
            top = max(top, (uint32_t)__shfl_xor((int)top, 1, 4));
            top = max(top, (uint32_t)__shfl_xor((int)top, 2, 4));
            const uint32_t e = tileattn_mx::scale_byte(top);
            *(uint32_t *)((uint8_t *)(is_v ? a.Vc : a.Kc) + row * (D / 2) + 4 * ch) =
                e == 255 ? 0u : tileattn_mx::pack(f, tileattn_mx::scale_of(e));
            if (ch % 4 == 0)
                ((uint8_t *)(is_v ? a.vs : a.ks))[row * (D / 32) + ch / 4] = (uint8_t)e;
        }
    }
}

template <int D, int TYPE>
void launch(const RopeArgs &a, bool inter, dim3 grid, hipStream_t s)
{
    const auto kernel = inter ? rope_append_kernel<D, TYPE, true> : rope_append_kernel<D, TYPE, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
}

}  // namespace

extern "C" {

ta_status qk_norm_rope_append(const void *Q, const void *K, const void *V, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, const void *q_weight, const void *k_weight, float eps,
                              const float *cos_sin, int num_positions, int rot_dim, int interleaved, const int *seq,
                              const int *pos, void *Q_out, void *K_cache, void *V_cache, int cache_type,
                              void *k_scale, void *v_scale, const int *page_table, int T, int B, int Hq, int Hkv,
                              int D, int num_pages, int page_size, int max_pages, void *stream)
{
    if ((!Q && Hq != 0) || !K || !V || !pos || (!Q_out && Hq != 0) || !K_cache || !V_cache || !page_table)
        return TA_ERR_NULL_POINTER;
    if (cache_type < TA_CACHE_BF16 || cache_type > TA_CACHE_MXFP4)
        return TA_ERR_UNSUPPORTED;
    const bool mx = cache_type == TA_CACHE_MXFP4;
    if (mx && (!k_scale || !v_scale))
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_cache(B, Hkv, D, num_pages, page_size, max_pages, cache_type, k_scale || v_scale);
    if (rc != TA_OK)
        return rc;
    const int64_t qrow = (int64_t)Hq * D, row = (int64_t)Hkv * D;
    if (T < 1 || T >= 1 << 24 || (!seq && T > B) || Hq < 0 || Hq > 1 << 16 || k_stride < row || v_stride < row ||
        k_stride % 8 || v_stride % 8 || k_stride > 1ll << 30 || v_stride > 1ll << 30 ||
        (Hq && (q_stride < qrow || q_stride % 8 || q_stride > 1ll << 30)))
        return TA_ERR_INVALID_SHAPE;
    if (cos_sin ? rot_dim < 16 || rot_dim > D || rot_dim % 16 : rot_dim != 0)
        return TA_ERR_UNSUPPORTED;
    if (cos_sin ? num_positions < 1 : num_positions != 0)
        return TA_ERR_INVALID_SHAPE;
    if (!(eps >= 0.f) || !(eps <= 3.402823466e+38f))
        return TA_ERR_INVALID_SCALE;
    if (Hq == 0)
        Q = Q_out = nullptr, q_weight = nullptr, q_stride = 0;
    if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Q_out) || misaligned(K_cache) ||
        misaligned(V_cache) || misaligned(q_weight) || misaligned(k_weight) || misaligned(cos_sin) ||
        misaligned(seq, 4) || misaligned(pos, 4) || misaligned(page_table, 4) || misaligned(k_scale, mx ? 16 : 4) ||
        misaligned(v_scale, mx ? 16 : 4))
        return TA_ERR_MISALIGNED;
    const size_t cb = cache_bytes(Hkv, num_pages, page_size, cache_row_bytes(D, cache_type));
    const size_t sb = scale_bytes(Hkv, D, num_pages, page_size, cache_type);
    const Span out[] = {{Q_out, (size_t)T * qrow * 2}, {K_cache, cb}, {V_cache, cb}, {mx ? k_scale : nullptr, sb},
                        {mx ? v_scale : nullptr, sb}};
    const Span in[] = {{Q, (size_t)((T - 1) * q_stride + qrow) * 2}, {K, (size_t)((T - 1) * k_stride + row) * 2},
                       {V, (size_t)((T - 1) * v_stride + row) * 2}, {q_weight, (size_t)D * 2},
                       {k_weight, (size_t)D * 2}, {cos_sin, (size_t)num_positions * rot_dim * 4}, {seq, (size_t)T * 4},
                       {pos, (size_t)T * 4}, {page_table, (size_t)B * max_pages * 4}, {mx ? nullptr : k_scale, sb},
                       {mx ? nullptr : v_scale, sb}};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlaps(out[i], out[j]))
                return TA_ERR_ALIASING;
        for (const Span &s : in)
            if (overlaps(out[i], s))
                return TA_ERR_ALIASING;
    }
    const RopeArgs a = {(const uint16_t *)Q, (const uint16_t *)K, (const uint16_t *)V, q_stride, k_stride, v_stride,
                        (const uint16_t *)q_weight, (const uint16_t *)k_weight, cos_sin, seq, pos, (uint16_t *)Q_out,
                        K_cache, V_cache, k_scale, v_scale, page_table, eps, cos_sin ? rot_dim : 0, num_positions,
                        B, Hq, Hkv, num_pages, __builtin_ctz(page_size), max_pages};
    // Rounds of the heads that 256 threads take at a time: a workgroup each for few tokens, else one
    // behind the other (a token's angles are loaded once).  us, three workgroups a token | one, 32 + 8 +
    // 8 heads of 128 dims, normed, into bf16, 8 and 4 bits:
    //   T = 32    3.2|4.8, 3.8|5.4, 3.6|5.3       512   5.8|6.7, 7.2|7.5, 6.7|7.1
    //   1023      8.4|8.4, 11.4|9.9, 10.9|9.0     1536  10.8|10.3, 15.3|15.5, 14.6|13.8
    //   2047      13.2|12.1, 19.3|17.8, 18.3|15.7 16384 84|73, 132|108, 126|95
    const int rounds = (Hq + 2 * Hkv + 2048 / D - 1) / (2048 / D);
    const dim3 grid((unsigned)T, (unsigned)(T < 1024 ? rounds : 1));
    hipStream_t s = (hipStream_t)stream;
    const bool inter = interleaved != 0;
    if (D == 64)
        cache_type == TA_CACHE_BF16   ? launch<64, TA_CACHE_BF16>(a, inter, grid, s)
        : cache_type == TA_CACHE_E4M3 ? launch<64, TA_CACHE_E4M3>(a, inter, grid, s)
                                      : launch<64, TA_CACHE_MXFP4>(a, inter, grid, s);
    else
        cache_type == TA_CACHE_BF16   ? launch<128, TA_CACHE_BF16>(a, inter, grid, s)
        : cache_type == TA_CACHE_E4M3 ? launch<128, TA_CACHE_E4M3>(a, inter, grid, s)
                                      : launch<128, TA_CACHE_MXFP4>(a, inter, grid, s);
    return hipGetLastError() == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

}  // extern "C"
