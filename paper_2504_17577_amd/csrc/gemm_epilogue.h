// What the matrix products with an epilogue (gemm_epilogue.hip, gemm_mxfp4.hip) do
// alike: act(x + bias) + residual of finished sums, the join of ranges of K, checks.
// Internal to libtileattn.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "gemm_tile.h"
#include "tileattn.h"

namespace {

using namespace tileattn_gemm;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// 1 / (1 + exp(-t)) by the hardware's exponential and reciprocal (1 ulp each) instead
// of the library's (half an ulp, several times the instructions: 10 us of a 4096 x
// 8192 x 8192 product's 480).  The exponent u = -t log2(e) is rounded, and so the value
// off by up to 2^-21 + 1.25 2^-24 |t| of itself (4e-6 at -87; below that the reciprocal
// is less than the smallest normal number, and 0).  A bf16 result, rounded by 2^-8,
// takes it so.
// FINE, for an fp32 result: within 2^-21 + 2^-22 |t| / 87 of the value down to 2^-128,
// then 0.  What the rounding left out of the exponent, d = -t - u ln 2 (ln 2 as one fp32
// number is the second term), goes into the exponential as 1 + d, and the reciprocal is
// taken of a fourth of the sum.  4096 x 8192 x 1024, silu, fp32 C: 82.4 us without, 84.0
// with; in the kernels of a bf16 C, 75 without and 80 with.
template <bool FINE>
__device__ __forceinline__ float sigmoid(float t)
{
    const float u = t * -1.44269504088896340736f;
    float e = __builtin_amdgcn_exp2f(u);
    if (!FINE)
        return __builtin_amdgcn_rcpf(1.f + e);
    const float d = __builtin_fmaf(u, -0.69314718055994530942f, -t);
    e = fabsf(u) < 128.f ? __builtin_fmaf(e, d, e) : e;   // (0 and infinity as they are)
    return 0.25f * __builtin_amdgcn_rcpf(__builtin_fmaf(e, 0.25f, 0.25f));
}

// The two gelus and silu as x times a sigmoid-like factor in (0, 1): no
// difference of nearly equal numbers for negative x.  One branch for U quads.
template <bool FINE, int U>
__device__ __forceinline__ void activate(int act, f32x4 (&x)[U])
{
    auto all = [&](auto f) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[u][i] = f(x[u][i]);
    };
    switch (act) {
    case TA_ACT_RELU:
        all([](float v) { return v < 0.f ? 0.f : v; });
        break;
    case TA_ACT_GELU:
        all([](float v) { return 0.5f * v * erfcf(v * -0.70710678118654752440f); });
        break;
    case TA_ACT_GELU_TANH:
        all([](float v) { return v * sigmoid<FINE>(1.59576912160573071176f * (v + 0.044715f * v * v * v)); });
        break;
    case TA_ACT_SILU:
        all([](float v) { return v * sigmoid<FINE>(v); });
        break;
    }
}

// A, B, M, N and K with the tiled kernel's arguments; C is the workspace [n_split]
// [M][N - n_begin] there where K is split, `out` the result in any case
template <bool CBF16>
struct EArgs : GArgs {
    int n_begin;     // the first column of a launch
    const uint16_t *bias;
    const void *R;
    void *out;
    int act;
    static constexpr bool EDGE = true;

    // The residual of four columns from n (a multiple of 4) of rows m, m + step, ..,
    // as it is in memory (nothing for what lies past M or N)
    template <int U>
    struct Added {
        u32x4 w[U];
        __device__ __forceinline__ void load(const EArgs &a, int m, int step, int n)
        {
            size_t e = (size_t)m * a.N + n;
#pragma unroll
            for (int u = 0; u < U; ++u, e += (size_t)step * a.N) {
                w[u] = u32x4{0, 0, 0, 0};
                if (a.R && m + u * step < a.M && n < a.N) {
                    if constexpr (CBF16) {
                        const u32x2 h = *(const u32x2 *)((const uint16_t *)a.R + e);
                        w[u][0] = h[0];
                        w[u][1] = h[1];
                    } else {
                        w[u] = *(const u32x4 *)((const float *)a.R + e);
                    }
                }
            }
        }
    };

    // These columns and rows of the result from their fp32 sums
    template <int U>
    __device__ __forceinline__ void store(int m, int step, int n, f32x4 (&x)[U], const Added<U> &r) const
    {
        if (n >= N)
            return;
        if (bias) {
            const u32x2 w = *(const u32x2 *)(bias + n);
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] += f32x4{bf16_lo(w[0]), bf16_hi(w[0]), bf16_lo(w[1]), bf16_hi(w[1])};
        }
        activate<!CBF16>(act, x);
        size_t e = (size_t)m * N + n;
        if constexpr (CBF16) {
            if (R)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    x[u] += f32x4{bf16_lo(r.w[u][0]), bf16_hi(r.w[u][0]), bf16_lo(r.w[u][1]), bf16_hi(r.w[u][1])};
#pragma unroll
            for (int u = 0; u < U; ++u, e += (size_t)step * N)
                if (m + u * step < M)
                    *(u32x2 *)((uint16_t *)out + e) = u32x2{pack_bf16(x[u][0], x[u][1]), pack_bf16(x[u][2], x[u][3])};
        } else {
            if (R)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    x[u] += __builtin_bit_cast(f32x4, r.w[u]);
#pragma unroll
            for (int u = 0; u < U; ++u, e += (size_t)step * N)
                if (m + u * step < M)
                    *(f32x4 *)((float *)out + e) = x[u];
        }
    }

    __device__ __forceinline__ void store(int m, int n, f32x4 x) const
    {
        f32x4 xx[1] = {x};
        Added<1> r;
        r.load(*this, m, 0, n);
        store<1>(m, 0, n, xx, r);
    }
};

// The ranges' products added in range order, and the epilogue: four columns per
// thread, up to eight ranges' loads in flight.
template <bool CBF16>
__global__ __launch_bounds__(256) void gemm_join_kernel(EArgs<CBF16> a)
{
    const uint32_t width = a.N - a.n_begin;
    const size_t e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4, mn = (size_t)a.M * width;
    if (e >= mn)
        return;
    const float *const w = (const float *)a.C;
    f32x4 sum = *(const f32x4 *)(w + e);
    for (int s = 1; s < a.n_split; s += 8) {
        f32x4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = s + u < a.n_split ? *(const f32x4 *)(w + (s + u) * mn + e) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s + u < a.n_split)
                sum += v[u];
    }
    a.store((int)(e / width), a.n_begin + (int)(e % width), sum);
}

constexpr int MAX_SPLITS = 64;

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

bool overlaps(const void *p, size_t pn, const void *q, size_t qn)
{
    const uintptr_t x = (uintptr_t)p, y = (uintptr_t)q;
    return p && q && x < y + qn && y < x + pn;
}

}  // namespace
