// C = act(A B + bias) + residual for bf16 A [M, K] and B [K, N] on gfx950
// (MI355X), any M, N and K multiples of 8.  Up to 64 rows run the kernel below that
// streams B through registers; more rows the tiled kernel of gemm_tile.h, in 256 x
// 256 tiles for as many columns as fill whole rounds of one workgroup per CU and in
// 128 x 128 tiles, with K split if they are few, for the others.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "even_parts.h"
#include "gemm_epilogue.h"
#include "gemm_tile.h"
#include "tileattn.h"

namespace {

using namespace tileattn_gemm;
using tileattn_detail::even_begin;
using tileattn_detail::even_part_of;

// ---- few rows: up to 64, a decode step's tokens ---------------------------
// HBM bounds it: every weight is read once and meets a few tokens.  A wave takes
// a strip of 128 columns and a range of K: a lane loads the same 8 columns of 8
// rows (16 bytes each, four whole 256-byte row pieces an instruction) and
// transposes the 8 x 8 block with byte permutes into the operands of
// v_mfma_f32_16x16x32_bf16, of which operand j is columns 8 c16 + j: nothing of B
// goes through LDS.  A's operands are 16 bytes of a row as they are, from L2.
// C^T = B^T A^T, so that a lane ends up with 32 consecutive columns of a token.
// The waves of a workgroup take every eighth step, so that two of them read the
// halves of A's lines at about the same time, and add up in LDS, in wave order.  A
// workgroup has a strip to itself or, where strips do not come in whole rounds of
// one per CU, an even share of all strips' steps (parts); strips that a share's ends
// cut leave partial sums for gemm_few_join_kernel.
// Measured, weights from HBM (us, with the join): 1 x 4096 x 4096 12, 24 x 14336 x
// 4096 28 (4.2 TB/s; the kernel alone 24), 1 x 28672 x 8192 80 (5.9 TB/s), 64 x 28672
// x 8192 106 (A, which every strip reads from L2, is half of B's bytes there).
constexpr int SK_WAVES = 8;
constexpr int SK_COLS = 128;

__device__ __forceinline__ uint32_t high16(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302); }
__device__ __forceinline__ uint32_t low16(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x05040100); }

template <bool NONTEMP>
__device__ __forceinline__ u32x4 ld_b(const void *p)
{
    if (NONTEMP)
        return __builtin_nontemporal_load((const u32x4 *)p);
    return *(const u32x4 *)p;
}

// MT: blocks of 16 rows.  parts: 0, or the workgroups that share the steps
template <bool CBF16, int MT, bool NONTEMP>
__global__ __launch_bounds__(64 * SK_WAVES, MT == 1 ? 4 : 2) void gemm_few_kernel(EArgs<CBF16> a, int parts)
{
    __shared__ __attribute__((aligned(16))) float red[SK_WAVES][16][SK_COLS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;

    // this workgroup's steps of 32 rows of B: from step `at` of a strip, `left` of them
    const uint32_t all = (a.K + 31) / 32;
    uint32_t strip = blockIdx.x, at = 0, left = all;
    if (parts) {
        const uint32_t n = (a.N + SK_COLS - 1) / SK_COLS * all, begin = even_begin(n, parts, blockIdx.x);
        left = even_begin(n, parts, blockIdx.x + 1) - begin;
        strip = begin / all;
        at = begin % all;
    }

    for (;;) {
        const uint32_t take = min(left, all - at);
        const int n0 = strip * SK_COLS;
        const int s0 = at + wave, s1 = at + take;   // (every eighth step)

        // Bytes of this lane's columns in a row of B, and of its rows of A (columns past N
        // read the last eight, rows past M the last: never stored)
        const uint32_t bo = 2 * min(n0 + 8 * c16, a.N - 8);
        uint32_t ao[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t)
            ao[t] = 2 * (uint32_t)min(16 * t + c16, a.M - 1) * a.K;

        f32x4 acc[MT][8];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        struct Step {
            u32x4 b[8], x[MT];
        };
        auto load = [&](int s, Step &st) {
            // (a last step of fewer rows: the lanes behind them read the last eight,
            // and take zeros below)
            const uint32_t k = min(8 * g, a.K - 8 - 32 * s);
            const unsigned char *bs = (const unsigned char *)(a.B + (size_t)(32 * s) * a.N);
            const unsigned char *as = (const unsigned char *)(a.A + 32 * s);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                st.b[i] = ld_b<NONTEMP>(bs + (size_t)i * a.N * 2 + (k * 2 * a.N + bo));
#pragma unroll
            for (int t = 0; t < MT; ++t)
                st.x[t] = *(const u32x4 *)(as + (ao[t] + 2 * k));
        };
        auto compute = [&](int s, Step &st) {
            if (32 * s + 32 > a.K) {
                const bool in = 32 * s + 8 * g < a.K;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        st.b[i][w] = in ? st.b[i][w] : 0u;
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        st.x[t][w] = in ? st.x[t][w] : 0u;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                u32x4 v;
#pragma unroll
                for (int p = 0; p < 4; ++p)
                    v[p] = j & 1 ? high16(st.b[2 * p][j >> 1], st.b[2 * p + 1][j >> 1])
                                 : low16(st.b[2 * p][j >> 1], st.b[2 * p + 1][j >> 1]);
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t][j] = mfma(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, st.x[t]), acc[t][j]);
            }
        };
        Step st[2];
        if (s0 < s1)
            load(s0, st[0]);
        for (int s = s0; s < s1; s += 2 * SK_WAVES) {
            if (s + SK_WAVES < s1)
                load(s + SK_WAVES, st[1]);
            compute(s, st[0]);
            if (s + 2 * SK_WAVES < s1)
                load(s + 2 * SK_WAVES, st[0]);
            if (s + SK_WAVES < s1)
                compute(s + SK_WAVES, st[1]);
        }

        // lane: row c16 of the block, columns 32 g + 8 r + j; 16-byte chunk ch of row x
        // at ch ^ x
        const bool whole = take == all;
        float *const rec = (float *)a.C + (2 * (size_t)blockIdx.x + (at == 0)) * a.M * SK_COLS;
        // (the thread's number anew, so that no address below occupies a register while
        // the steps run)
        int te = threadIdx.x;
        asm volatile("" : "+v"(te));
        const int ce = te & 15, ge = (te & 63) >> 4;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            __syncthreads();   // (what was there has been read)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *(f32x4 *)&red[wave][ce][4 * ((8 * ge + 2 * r + q) ^ ce)] =
                        f32x4{acc[t][4 * q][r], acc[t][4 * q + 1][r], acc[t][4 * q + 2][r], acc[t][4 * q + 3][r]};
            __syncthreads();
            static_assert(16 * SK_COLS / 4 == 64 * SK_WAVES, "four columns of a row per thread");
            const int x = te / (SK_COLS / 4), ch = te % (SK_COLS / 4);
            const int m = 16 * t + x, n = n0 + 4 * ch;
            if (m < a.M && n < a.N) {
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < SK_WAVES; ++w)
                    sum += *(const f32x4 *)&red[w][x][4 * (ch ^ x)];
                if (whole)
                    a.store(m, n, sum);
                else
                    *(f32x4 *)(rec + m * SK_COLS + 4 * ch) = sum;
            }
        }
        left -= take;
        if (left == 0)
            return;
        ++strip;
        at = 0;
    }
}

// The partial sums of the strips that were cut, added in order of K, and the
// epilogue: four columns per thread, up to eight records' loads in flight.  Part
// p's record 2 p is of the strip that an earlier part began, 2 p + 1 of one that it
// began itself and a later part goes on with.
template <bool CBF16>
__global__ __launch_bounds__(256) void gemm_few_join_kernel(EArgs<CBF16> a, int parts)
{
    const uint32_t all = (a.K + 31) / 32, n = (a.N + SK_COLS - 1) / SK_COLS * all, strip = blockIdx.x;
    const uint32_t p0 = even_part_of(n, parts, strip * all), p1 = even_part_of(n, parts, strip * all + all - 1);
    const int e = blockIdx.y * 256 + threadIdx.x, m = e / (SK_COLS / 4), col = e % (SK_COLS / 4) * 4;
    if (p0 == p1 || m >= a.M || (int)(strip * SK_COLS) + col >= a.N)
        return;
    const size_t rec = (size_t)a.M * SK_COLS;
    const float *const w = (const float *)a.C + m * SK_COLS + col;
    f32x4 sum = *(const f32x4 *)(w + (2 * (size_t)p0 + 1) * rec);
    for (uint32_t p = p0 + 1; p <= p1; p += 8) {
        f32x4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = p + u <= p1 ? *(const f32x4 *)(w + 2 * (size_t)(p + u) * rec) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (p + u <= p1)
                sum += v[u];
    }
    a.store(m, strip * SK_COLS + col, sum);
}

constexpr int FEW_MAX_PARTS = 4096;

bool few(int M) { return M <= 64; }

// The workgroups that share the steps of all strips where num_splits is more than
// one: about num_splits for each strip, in whole rounds of one per CU, with a step
// for every wave at least; 0 for a workgroup per strip.
int few_parts(int N, int K, int num_splits)
{
    if (num_splits == 1)
        return 0;
    const int64_t strips = (N + SK_COLS - 1) / SK_COLS, most = (strips * ((K + 31) / 32) + SK_WAVES - 1) / SK_WAVES;
    int64_t parts = strips * num_splits;
    if (parts > 256)
        parts -= parts % 256;
    parts = std::min(std::min(parts, most), (int64_t)FEW_MAX_PARTS);
    return parts <= strips ? 0 : (int)parts;
}

template <int MT, bool CBF16>
hipError_t launch_few(const EArgs<CBF16> &a, bool nt, hipStream_t s)
{
    const int strips = (a.N + SK_COLS - 1) / SK_COLS, parts = few_parts(a.N, a.K, a.n_split);
    const auto kernel = nt ? gemm_few_kernel<CBF16, MT, true> : gemm_few_kernel<CBF16, MT, false>;
    hipLaunchKernelGGL(kernel, dim3(parts ? parts : strips), dim3(64 * SK_WAVES), 0, s, a, parts);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && parts) {
        hipLaunchKernelGGL(gemm_few_join_kernel<CBF16>, dim3(strips, (a.M * (SK_COLS / 4) + 255) / 256), dim3(256), 0, s, a, parts);
        e = hipGetLastError();
    }
    return e;
}

// The tiled kernel (gemm_tile.h) on the columns up to n_end
template <int BM, int BN, int ST, int KS, bool CBF16>
hipError_t launch_tiles(EArgs<CBF16> a, int n_end, hipStream_t s)
{
    constexpr int MF = (BK / 32) % KS == 0 ? 16 : 32;
    a.tiles_n = (n_end - a.n_begin + BN - 1) / BN;
    a.n_tiles = (a.M + BM - 1) / BM * a.tiles_n;
    a.n_wg = a.n_tiles * a.n_split;
    auto kernel = gemm_kernel<BM, BN, ST, KS, MF, false, false, EArgs<CBF16>>;
    if constexpr (BM == 128)
        if (a.n_split > 1)
            kernel = gemm_kernel<BM, BN, ST, KS, MF, false, true, EArgs<CBF16>>;
    hipLaunchKernelGGL(kernel, dim3(a.n_wg), dim3(NT), 0, s, a);
    return hipGetLastError();
}

// Estimates of the tiled kernels' times in us, for the choices below: fitted to
// products whose B comes from HBM (a model's other weights have passed through
// the caches since), where a tile of few others to cover its loads costs 0.7 us a
// step, and two per CU 1.25 together.  kt: steps of 64 rows of B.
double time_256(int kt, int rounds) { return rounds * (kt * 1.65 + 15); }

double time_128(int M, int N, int kt, int sp)
{
    const int64_t wg = (int64_t)((M + 127) / 128) * ((N + 127) / 128) * sp;
    const int steps = (kt + sp - 1) / sp;
    const double step = wg <= 256 ? 0.7 : wg <= 512 ? 0.8 + 0.45 * (wg - 256) / 256 : 1.25 * (double)((wg + 511) / 512);
    const double hbm = (double)kt * 128 * N / 5e6;
    const double t = 6 + (steps * step > hbm ? steps * step : hbm);
    return sp == 1 ? t : t + 4 + 8.0 * M * N * sp / 4.5e6;
}

// How a product of more than 64 rows runs: 256 x 256 tiles on its first columns,
// in whole rounds of one workgroup per CU, and 128 x 128 tiles on the others, with K
// split in n_split there.  (In 256 x 256 tiles alone 4000 x 8200 x 8200, 528 of
// them, took three rounds.)
struct Choice {
    int n_256;       // columns of the 256 x 256 tiles
    double time;
};

Choice choose(int M, int N, int K, int sp)
{
    const int kt = (K + BK - 1) / BK, rows = (M + 255) / 256, cols = (N + 255) / 256;
    const int64_t tiles = (int64_t)rows * cols;
    Choice best = {0, time_128(M, N, kt, sp)};
    // the last rounds that are nearly whole, and all tiles
    const int full = (int)(tiles / 256), all = (int)((tiles + 255) / 256);
    for (int r = full > 1 ? full - 1 : 1; r <= all; ++r) {
        const int64_t n1 = (int64_t)r * 256 / rows * 256;
        if (n1 == 0)
            continue;
        const Choice c = n1 >= N ? Choice{N, time_256(kt, r)}
                                 : Choice{(int)n1, time_256(kt, r) + time_128(M, N - (int)n1, kt, sp)};
        if (c.time < best.time)
            best = c;
    }
    return best;
}

// ranges are whole steps
int ranges(int K, int num_splits) { return std::min(num_splits, (K + BK - 1) / BK); }

size_t workspace_need(int M, int N, int K, int num_splits)
{
    if (few(M))
        return (size_t)few_parts(N, K, num_splits) * 2 * M * SK_COLS * 4;
    const int sp = ranges(K, num_splits);
    return sp > 1 ? (size_t)sp * M * (N - choose(M, N, K, sp).n_256) * 4 : 0;
}

template <bool CBF16>
hipError_t launch(EArgs<CBF16> a, hipStream_t s)
{
    if (few(a.M)) {
        // Weights that the 256 MB Infinity Cache cannot hold: non-temporal.  us, ordinary |
        // non-temporal: 470 MB (1 x 28672 x 8192) 81.4 | 74.7, 1 GB (24 x 65536 x 8192) 185 | 169;
        // 117 MB (24 x 14336 x 4096) read again by every call 22.9 | 24.9, from HBM 27.4 | 26.2
        const bool nt = (size_t)a.K * a.N * 2 > ((size_t)256 << 20);
        return a.M <= 16   ? launch_few<1>(a, nt, s)
               : a.M <= 32 ? launch_few<2>(a, nt, s)
               : a.M <= 48 ? launch_few<3>(a, nt, s)
                           : launch_few<4>(a, nt, s);
    }
    hipError_t e = hipSuccess;
    a.n_split = ranges(a.K, a.n_split);
    const Choice c = choose(a.M, a.N, a.K, a.n_split);
    if (c.n_256) {
        EArgs<CBF16> first = a;
        first.n_split = 1;
        e = launch_tiles<256, 256, 2, 1>(first, c.n_256, s);
        if (c.n_256 == a.N)
            return e;
    }
    a.n_begin = c.n_256;
    const int64_t wg = (int64_t)((a.M + 127) / 128) * ((a.N - a.n_begin + 127) / 128) * a.n_split;
    if (e == hipSuccess)
        e = wg <= 256 ? launch_tiles<128, 128, 4, 4>(a, a.N, s) : launch_tiles<128, 128, 2, 2>(a, a.N, s);
    if (e != hipSuccess || a.n_split == 1)
        return e;
    const size_t threads = (size_t)a.M * (a.N - a.n_begin) / 4;
    hipLaunchKernelGGL(gemm_join_kernel<CBF16>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

// the sizes that every entry point checks alike
ta_status check_sizes(int M, int N, int K)
{
    if (M < 1 || N < 1 || K < 1)
        return TA_ERR_INVALID_SHAPE;
    if (N % 8 || K % 8)
        return TA_ERR_UNSUPPORTED;
    if (N >= 1 << 24 || K >= 1 << 22 || M > 1 << 20 || (int64_t)M * N >= 1ll << 35 || (int64_t)M * K >= 1ll << 40 ||
        (int64_t)N * K >= 1ll << 40)
        return TA_ERR_INVALID_SHAPE;
    return TA_OK;
}

}  // namespace

extern "C" {

ta_status gemm_bf16_epilogue(const void *A, const void *B, const void *bias, const void *residual,
                             void *C, int c_bf16, int activation, int M, int N, int K,
                             int num_splits, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!A || !B || !C)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_splits < 1 || num_splits > MAX_SPLITS)
        return TA_ERR_INVALID_SHAPE;
    if (activation < TA_ACT_NONE || activation > TA_ACT_SILU)
        return TA_ERR_UNSUPPORTED;
    if (misaligned(A) || misaligned(B) || misaligned(C) || misaligned(bias) || misaligned(residual))
        return TA_ERR_MISALIGNED;
    const size_t a_bytes = (size_t)M * K * 2, b_bytes = (size_t)K * N * 2;
    const size_t c_bytes = (size_t)M * N * (c_bf16 ? 2 : 4);
    if (overlaps(C, c_bytes, A, a_bytes) || overlaps(C, c_bytes, B, b_bytes) ||
        overlaps(C, c_bytes, bias, (size_t)N * 2) || (residual != C && overlaps(C, c_bytes, residual, c_bytes)))
        return TA_ERR_ALIASING;
    const size_t w_bytes = workspace_need(M, N, K, num_splits);
    if (w_bytes) {
        if (!workspace || workspace_bytes < w_bytes)
            return TA_ERR_WORKSPACE;
        if (misaligned(workspace))
            return TA_ERR_MISALIGNED;
        if (overlaps(workspace, w_bytes, A, a_bytes) || overlaps(workspace, w_bytes, B, b_bytes) ||
            overlaps(workspace, w_bytes, C, c_bytes) || overlaps(workspace, w_bytes, bias, (size_t)N * 2) ||
            overlaps(workspace, w_bytes, residual, c_bytes))
            return TA_ERR_ALIASING;
    }
    GArgs p = {};
    p.A = (const uint16_t *)A;
    p.B = (const uint16_t *)B;
    p.C = workspace;
    p.M = M;
    p.N = N;
    p.K = K;
    p.n_split = num_splits;
    const auto run = [&](auto a) {
        a.bias = (const uint16_t *)bias;
        a.R = residual;
        a.out = C;
        a.act = activation;
        return launch(a, (hipStream_t)stream);
    };
    return (c_bf16 ? run(EArgs<true>{p}) : run(EArgs<false>{p})) == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

ta_status gemm_epilogue_workspace_bytes(int M, int N, int K, int num_splits, size_t *bytes)
{
    if (!bytes)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_splits < 1 || num_splits > MAX_SPLITS)
        return TA_ERR_INVALID_SHAPE;
    *bytes = workspace_need(M, N, K, num_splits);
    return TA_OK;
}

ta_status gemm_epilogue_plan(int M, int N, int K, int *num_splits)
{
    if (!num_splits)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (!few(M)) {
        double best = choose(M, N, K, 1).time;
        *num_splits = 1;
        for (int sp = 2; sp <= 32 && sp <= (K + BK - 1) / BK; ++sp)
            if (choose(M, N, K, sp).time < best) {
                best = choose(M, N, K, sp).time;
                *num_splits = sp;
            }
        return TA_OK;
    }
    // One workgroup per strip where they fill three quarters of their rounds of one
    // per CU, else several per strip if those do (24 x 14336 x 4096, 112 strips: 38 us
    // with one, 28 with two, 31 as 256 shares), else even shares of all strips (8 x
    // 40000 x 4096, 313 strips: 65 us with one each, 57 as 512 shares).  Up to four
    // steps a wave the second kernel costs what it saves (8 x 1000 x 1000: 7.0 us
    // with one, 6.8 with four; x 2048: 10.9 and, with eight, 7.1)
    const int strips = (N + SK_COLS - 1) / SK_COLS, steps = (K + 31) / 32;
    const auto fills = [](int wg) { return 4 * (int64_t)wg >= 3 * 256 * (int64_t)((wg + 255) / 256); };
    int sp = 1;
    if (!fills(strips) && steps > 4 * SK_WAVES) {
        sp = std::max(1, 256 / strips);
        if (!fills(strips * sp))
            ++sp;
    }
    *num_splits = std::max(1, std::min(sp, std::min(steps / SK_WAVES, MAX_SPLITS)));
    return TA_OK;
}

ta_status gemm_epilogue_route(int M, int N, int K, int num_splits, int *large_columns)
{
    if (!large_columns)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_splits < 1 || num_splits > MAX_SPLITS)
        return TA_ERR_INVALID_SHAPE;
    *large_columns = few(M) ? 0 : choose(M, N, K, ranges(K, num_splits)).n_256;
    return TA_OK;
}

}  // extern "C"
