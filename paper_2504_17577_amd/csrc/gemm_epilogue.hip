// C = act(A B + bias) + residual for bf16 A [M, K] and B [K, N] on gfx950
// (MI355X), any M, N and K multiples of 8.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tileattn.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

__device__ __forceinline__ float bf16_f32(uint16_t w) { return __uint_as_float((uint32_t)w << 16); }

struct EArgs {
    const uint16_t *A, *B, *bias;
    const void *R;
    void *C;
    int M, N, K;
};

// The two gelus and silu as x times a sigmoid-like factor in (0, 1): no
// difference of nearly equal numbers for negative x.
template <int ACT>
__device__ __forceinline__ float activated(float x)
{
    if (ACT == TA_ACT_RELU)
        return x < 0.f ? 0.f : x;
    if (ACT == TA_ACT_GELU)
        return 0.5f * x * erfcf(x * -0.70710678118654752440f);
    if (ACT == TA_ACT_GELU_TANH)
        return x / (1.f + expf(-1.59576912160573071176f * (x + 0.044715f * x * x * x)));
    if (ACT == TA_ACT_SILU)
        return x / (1.f + expf(-x));
    return x;
}

// A thread per element of C, 16 x 16 of them sharing their operands in LDS.
template <int ACT, bool CBF16>
__global__ __launch_bounds__(256) void gemm_epilogue_kernel(EArgs a)
{
    __shared__ float as[16][17], bs[16][17];
    const int x = threadIdx.x % 16, y = threadIdx.x / 16;
    const int m = blockIdx.y * 16 + y, n = blockIdx.x * 16 + x;
    float sum = 0.f;
    for (int k0 = 0; k0 < a.K; k0 += 16) {
        as[y][x] = m < a.M && k0 + x < a.K ? bf16_f32(a.A[(size_t)m * a.K + k0 + x]) : 0.f;
        bs[y][x] = n < a.N && k0 + y < a.K ? bf16_f32(a.B[(size_t)(k0 + y) * a.N + n]) : 0.f;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
            sum = __builtin_fmaf(as[y][k], bs[k][x], sum);
        __syncthreads();
    }
    if (m >= a.M || n >= a.N)
        return;
    const size_t e = (size_t)m * a.N + n;
    if (a.bias)
        sum += bf16_f32(a.bias[n]);
    sum = activated<ACT>(sum);
    if (a.R)
        sum += CBF16 ? bf16_f32(((const uint16_t *)a.R)[e]) : ((const float *)a.R)[e];
    if (CBF16)
        ((uint16_t *)a.C)[e] = (uint16_t)pack_bf16(sum, 0.f);
    else
        ((float *)a.C)[e] = sum;
}

template <int ACT>
hipError_t launch(const EArgs &a, bool c_bf16, hipStream_t s)
{
    const dim3 grid((a.N + 15) / 16, (a.M + 15) / 16);
    if (c_bf16)
        hipLaunchKernelGGL((gemm_epilogue_kernel<ACT, true>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((gemm_epilogue_kernel<ACT, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

bool overlaps(const void *p, size_t pn, const void *q, size_t qn)
{
    const uintptr_t x = (uintptr_t)p, y = (uintptr_t)q;
    return p && q && x < y + qn && y < x + pn;
}

}  // namespace

extern "C" {

ta_status gemm_bf16_epilogue(const void *A, const void *B, const void *bias, const void *residual,
                             void *C, int c_bf16, int activation, int M, int N, int K,
                             void *stream)
{
    if (!A || !B || !C)
        return TA_ERR_NULL_POINTER;
    if (M < 1 || N < 1 || K < 1)
        return TA_ERR_INVALID_SHAPE;
    if (N % 8 || K % 8 || activation < TA_ACT_NONE || activation > TA_ACT_SILU)
        return TA_ERR_UNSUPPORTED;
    if (N >= 1 << 24 || K >= 1 << 22 || M > 1 << 20 || (int64_t)M * N >= 1ll << 40 || (int64_t)M * K >= 1ll << 40)
        return TA_ERR_INVALID_SHAPE;
    if (misaligned(A) || misaligned(B) || misaligned(C) || misaligned(bias) || misaligned(residual))
        return TA_ERR_MISALIGNED;
    const size_t c_bytes = (size_t)M * N * (c_bf16 ? 2 : 4);
    if (overlaps(C, c_bytes, A, (size_t)M * K * 2) || overlaps(C, c_bytes, B, (size_t)K * N * 2) ||
        overlaps(C, c_bytes, bias, (size_t)N * 2) || (residual != C && overlaps(C, c_bytes, residual, c_bytes)))
        return TA_ERR_ALIASING;
    const EArgs a = {(const uint16_t *)A, (const uint16_t *)B, (const uint16_t *)bias, residual, C, M, N, K};
    hipStream_t s = (hipStream_t)stream;
    const bool cb = c_bf16 != 0;
    const hipError_t e = activation == TA_ACT_NONE        ? launch<TA_ACT_NONE>(a, cb, s)
                         : activation == TA_ACT_RELU      ? launch<TA_ACT_RELU>(a, cb, s)
                         : activation == TA_ACT_GELU      ? launch<TA_ACT_GELU>(a, cb, s)
                         : activation == TA_ACT_GELU_TANH ? launch<TA_ACT_GELU_TANH>(a, cb, s)
                                                          : launch<TA_ACT_SILU>(a, cb, s);
    return e == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

}  // extern "C"
