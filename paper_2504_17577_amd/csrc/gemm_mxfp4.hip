// C = act(A W^T + bias) + residual for bf16 A [M, K] and W [N, K] in 4 bits (MXFP4) on
// gfx950 (MI355X), any M, N a multiple of 8 and K of 32.  The codes become bf16 in
// registers, two by one instruction, scale included and exactly, on their way into
// bf16 matrix instructions: the products are those of the numbers that they stand for.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gemm_epilogue.h"
#include "lds_dma.h"
#include "mxfp4.h"
#include "tileattn.h"

namespace {

// (B of EArgs is not used)
template <bool CBF16>
struct MxArgs : EArgs<CBF16> {
    const uint8_t *W, *S;      // codes [N, K / 2], scales [N, K / 32]
};

// ---- few rows: up to 64, a decode step's tokens ---------------------------
// HBM bounds it: every weight is read once and meets a few tokens.  A wave takes a
// strip of 16 NB rows of W and every eighth step of 128 columns of K: a lane's 16 bytes
// of a row are 32 numbers, one group, and so four operands of
// v_mfma_f32_16x16x32_bf16 with one scale; A's operands are taken from the same places
// of K, 16 bytes of a row, from L2.  C^T = W A^T, so that a lane ends up with four
// consecutive columns of a token.  The waves add up in LDS, in wave order.
constexpr int FW = 8;

template <bool CBF16, int NB, int MT, bool SPLIT>
__global__ __launch_bounds__(64 * FW, 2) void gemm_mx_few_kernel(MxArgs<CBF16> a)
{
    constexpr int CH = 4 * NB;                 // 16-byte chunks of a strip's row of C
    __shared__ __attribute__((aligned(16))) float red[FW][16 * MT][16 * NB];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * (16 * NB);
    const int all = (a.K + 127) / 128;
    int lo = 0, hi = all;
    if (SPLIT) {
        lo = (int)((uint32_t)all * blockIdx.y / a.n_split);
        hi = (int)((uint32_t)all * (blockIdx.y + 1) / a.n_split);
    }

    // Bytes of this lane's rows of W, of their scales and of its rows of A (rows past the
    // last read the last: never stored)
    size_t wo[NB], so[NB];
    uint32_t ao[MT];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const size_t n = min(n0 + 16 * b + c16, a.N - 1);
        wo[b] = n * (a.K / 2);
        so[b] = n * (a.K / 32);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
        ao[t] = (uint32_t)min(16 * t + c16, a.M - 1) * a.K * 2;

    f32x4 acc[MT][NB];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};

    struct Step {
        u32x4 w[NB], x[MT][4];
        uint32_t e[NB];
    };
    auto load = [&](int s, Step &st) {
        const int k = min(128 * s + 32 * g, a.K - 32);   // (lanes past K read the last group, and take zeros below)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            st.w[b] = __builtin_nontemporal_load((const u32x4 *)(a.W + wo[b] + k / 2));
            st.e[b] = a.S[so[b] + k / 32];
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                st.x[t][kk] = *(const u32x4 *)((const unsigned char *)a.A + ao[t] + (uint32_t)(2 * k + 16 * kk));
    };
    auto compute = [&](int s, Step &st) {
        if (128 * s + 128 > a.K) {
            const bool in = 128 * s + 32 * g < a.K;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                st.w[b] = in ? st.w[b] : u32x4{0, 0, 0, 0};
                st.e[b] = in ? st.e[b] : 127u;
            }
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    st.x[t][kk] = in ? st.x[t][kk] : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const bf16x8 w = tileattn_mx::eight(st.w[b][kk], tileattn_mx::scale_of(st.e[b]));
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t][b] = mfma(w, __builtin_bit_cast(bf16x8, st.x[t][kk]), acc[t][b]);
            }
    };
    Step st[2];
    const int s0 = lo + wave;
    if (s0 < hi)
        load(s0, st[0]);
    for (int s = s0; s < hi; s += 2 * FW) {
        if (s + FW < hi)
            load(s + FW, st[1]);
        compute(s, st[0]);
        if (s + 2 * FW < hi)
            load(s + 2 * FW, st[0]);
        if (s + FW < hi)
            compute(s + FW, st[1]);
    }

    // lane: row 16 t + c16, columns 16 b + 4 g .. + 3; chunk ch of row x at ch ^ x
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            *(f32x4 *)&red[wave][16 * t + c16][4 * ((4 * b + g) ^ (c16 % CH))] = acc[t][b];
    __syncthreads();
    for (int e = tid; e < 16 * MT * CH; e += 64 * FW) {
        const int x = e / CH, ch = e % CH, n = n0 + 4 * ch;
        if (x >= a.M || n >= a.N)
            continue;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < FW; ++w)
            sum += *(const f32x4 *)&red[w][x][4 * (ch ^ (x % CH))];
        if (SPLIT)
            *(f32x4 *)((float *)a.C + ((size_t)blockIdx.y * a.M + x) * a.N + n) = sum;
        else
            a.store(x, n, sum);
    }
}

// ---- more rows: tiles of 128 x 128 -----------------------------------------
// A workgroup of eight waves computes 128 rows by 128 columns in stages of 128 of K,
// a ring of ST of them in LDS: A's rows (32 KB), W's codes (8 KB) and the scales' bytes,
// one a dword (2 KB), all by DMA.  Two groups of four waves take half of a stage's K
// each and 64 x 64 of the tile a wave, in v_mfma_f32_32x32x16_bf16: a lane's 16 bytes
// of a row of W are the 32 numbers of a group, four operands, with one scale, and A's
// operands come from the same places of K.  W stays in 4 bits up to the registers, so
// that LDS holds and gives a quarter of a bf16 tile's bytes for it.
constexpr int TM = 128, TN = 128, TK = 128, TST = 3;
constexpr int A_STAGE = TM * TK * 2, W_STAGE = TN * TK / 2, S_STAGE = TN * TK / 32 * 4;
constexpr int STAGE = A_STAGE + W_STAGE + S_STAGE;
constexpr int A_DMA = A_STAGE / 16 / NT, DMAS = A_DMA + 2;   // of a thread and stage
static_assert(W_STAGE / 16 == NT && S_STAGE / 4 == NT, "one each of W's chunks and scales per thread");

// One byte at byte `voff` of the buffer per lane, as a dword at LDS `lds` + 4 lane
__device__ __forceinline__ void dma_byte(uint32_t lds, uint32_t voff, uint32_t soff, u32x4s rsrc)
{
    asm volatile("s_nop 0\n\t"
                 "buffer_load_ubyte %0, %1, %2 offen lds"
                 :
                 : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

template <bool CBF16, bool SPLIT>
__global__ __launch_bounds__(NT, 2) void gemm_mx_kernel(MxArgs<CBF16> args)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[TST * STAGE];
    static_assert(TST * STAGE >= TM * TN * 4, "the tile's sums");
    const MxArgs<CBF16> &a = args;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int kg = wave >> 2, wm = (wave >> 1 & 1) * 64, wn = (wave & 1) * 64;

    // XCD-contiguous tile index, in groups of four rows of tiles
    const int per = a.n_wg / NXCD, rem = a.n_wg % NXCD;
    const int xcd = blockIdx.x % NXCD;
    const int ts = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / NXCD;
    const uint32_t split = SPLIT ? ts / a.n_tiles : 0;
    const int t = ts - split * a.n_tiles;
    const int grp = t / (GROUP_M * a.tiles_n), w = t % (GROUP_M * a.tiles_n);
    const int rows = min((a.M + TM - 1) / TM - grp * GROUP_M, GROUP_M);
    const int m0 = (grp * GROUP_M + w % rows) * TM, n0 = w / rows * TN;

    const int all = (a.K + TK - 1) / TK;
    int lo = 0, n_kt = all;
    if (SPLIT) {
        lo = (int)((uint32_t)all * split / a.n_split);
        n_kt = (int)((uint32_t)all * (split + 1) / a.n_split) - lo;
    }

    // Where this thread's chunks come from (rows past the last are the last; in a last
    // stage, chunks past K are the last: those are cleared in the operands)
    const int mr = min(TM, a.M - m0), nr = min(TN, a.N - n0);
    const u32x4s ra = tileattn_dma::buffer_rsrc(a.A + (size_t)m0 * a.K, (uint32_t)mr * a.K * 2);
    const u32x4s rw = tileattn_dma::buffer_rsrc(a.W + (size_t)n0 * (a.K / 2), (uint32_t)nr * (a.K / 2));
    const u32x4s rs = tileattn_dma::buffer_rsrc(a.S + (size_t)n0 * (a.K / 32), (uint32_t)nr * (a.K / 32));
    // A: slot s is row s / 16, stored chunk s % 16; W: row s / 4, stored chunk s % 4; scale
    // of slot s: group s / 128 of row s % 128
    auto a_row = [&](int i) { return (i * NT + tid) / 16; };
    auto a_ch = [&](int i) { return (tid % 16) ^ (a_row(i) & 15); };
    const int w_row = tid / 4, w_ch = (tid % 4) ^ ((w_row >> 1) & 3);
    const int s_row = tid % TN, s_grp = tid / TN;
    uint32_t ao[A_DMA];
#pragma unroll
    for (int i = 0; i < A_DMA; ++i)
        ao[i] = (uint32_t)min(a_row(i), mr - 1) * a.K * 2;
    const uint32_t wo = (uint32_t)min(w_row, nr - 1) * (a.K / 2), so = (uint32_t)min(s_row, nr - 1) * (a.K / 32);
    auto dma = [&](int kt, unsigned char *to) {
        const int k0 = (lo + kt) * TK;
        const uint32_t base = tileattn_dma::lds_addr(to);
        const int left = a.K - k0;                    // of K (whole stages: not looked at)
        const bool part = left < TK;
#pragma unroll
        for (int i = 0; i < A_DMA; ++i)
            tileattn_dma::dma16_soff(base + (i * NT + wave * 64) * 16,
                                     ao[i] + 16 * (part ? min(a_ch(i), left / 8 - 1) : a_ch(i)), k0 * 2, ra);
        tileattn_dma::dma16_soff(base + A_STAGE + wave * 64 * 16, wo + 16 * (part ? min(w_ch, left / 32 - 1) : w_ch),
                                 k0 / 2, rw);
        dma_byte(base + A_STAGE + W_STAGE + wave * 64 * 4, so + (part ? min(s_grp, left / 32 - 1) : s_grp), k0 / 32, rs);
    };

    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[i][j][r] = 0.f;

    auto compute = [&](const unsigned char *st, bool in) {
        u32x4 wv[2];
        float sc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = wn + 32 * j + col, q = 2 * kg + half;
            wv[j] = *(const u32x4 *)(st + A_STAGE + n * 64 + 16 * (q ^ ((n >> 1) & 3)));
            sc[j] = tileattn_mx::scale_of(*(const uint32_t *)(st + A_STAGE + W_STAGE + 4 * (q * TN + n)));
            if (!in) {
                wv[j] = u32x4{0, 0, 0, 0};
                sc[j] = 1.f;
            }
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            bf16x8 av[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = wm + 32 * i + col, ch = 8 * kg + 4 * half + kk;
                u32x4 x = *(const u32x4 *)(st + r * 256 + 16 * (ch ^ (r & 15)));
                if (!in)
                    x = u32x4{0, 0, 0, 0};
                av[i] = __builtin_bit_cast(bf16x8, x);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bf16x8 wb = tileattn_mx::eight(wv[j][kk], sc[j]);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    acc[i][j] = mfma(wb, av[i], acc[i][j]);
            }
        }
    };

    // stage kt lives in kt % TST; the loads of up to TST - 2 later ones may stay in flight
    // at its beginning, and the barrier frees the stage before it
#pragma unroll
    for (int s = 0; s < TST - 1; ++s)
        if (s < n_kt)
            dma(s, lds + s * STAGE);
    for (int kt = 0; kt < n_kt; ++kt) {
        if (kt + 1 < n_kt)
            tileattn_dma::wait_vmcnt<DMAS * (TST - 2)>();
        else
            tileattn_dma::wait_vmcnt<0>();
        __syncthreads();
        const int nx = kt + TST - 1;
        if (nx < n_kt)
            dma(nx, lds + nx % TST * STAGE);
        const unsigned char *st = lds + kt % TST * STAGE;
        const int k0 = (lo + kt) * TK;
        if (k0 + TK <= a.K)
            compute(st, true);
        else
            compute(st, k0 + 64 * kg + 32 * half < a.K);
    }

    // The two groups' sums meet in LDS, row by row of C; then all waves store, whole lines.
    // Lane: row wm + 32 i + col, columns wn + 32 j + 8 q + 4 half .. + 3; 16-byte chunk c of
    // row r at c ^ (r % 32).
    float *const sums = (float *)lds;
    auto at = [&](int r, int c) { return (f32x4 *)(sums + r * TN + 4 * (c ^ (r & 31))); };
    __syncthreads();
    if (kg == 1)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *at(wm + 32 * i + col, (wn + 32 * j) / 4 + 2 * q + half) =
                        f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    if (kg == 0)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *at(wm + 32 * i + col, (wn + 32 * j) / 4 + 2 * q + half) +=
                        f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    constexpr int U = 4, RPI = NT / (TN / 4);        // rows at a time, U steps of them
    const int c = tid % (TN / 4), n = n0 + 4 * c;
    if (n >= a.N)
        return;
    typename EArgs<CBF16>::template Added<U> now, next;
    int m = m0 + tid / (TN / 4);
    if (!SPLIT)
        now.load(a, m, RPI, n);
#pragma unroll 1
    for (int s = 0; s < TM; s += U * RPI, m += U * RPI) {
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            x[u] = *at(m - m0 + u * RPI, c);
        if (SPLIT) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (m + u * RPI < a.M)
                    *(f32x4 *)((float *)a.C + ((size_t)split * a.M + m + u * RPI) * a.N + n) = x[u];
        } else {
            if (s + U * RPI < TM)
                next.load(a, m + U * RPI, RPI, n);
            a.store(m, RPI, n, x, now);
            now = next;
        }
    }
}

bool mx_few(int M) { return M <= 64; }

int mx_steps(int K) { return (K + 127) / 128; }

// Blocks of 16 rows of W that a wave takes
int few_blocks(int N) { return N <= 16 * 512 ? 1 : N <= 32 * 512 ? 2 : 4; }

int mx_ranges(int M, int N, int K, int num_splits)
{
    (void)N;
    const int steps = mx_steps(K), most = mx_few(M) ? std::max(1, steps / FW) : steps;
    return std::min(num_splits, most);
}

size_t mx_workspace(int M, int N, int K, int num_splits)
{
    const int sp = mx_ranges(M, N, K, num_splits);
    return sp > 1 ? (size_t)sp * M * N * 4 : 0;
}

template <bool CBF16, int NB, int MT>
void launch_mx_few(const MxArgs<CBF16> &a, hipStream_t s)
{
    const dim3 grid((a.N + 16 * NB - 1) / (16 * NB), a.n_split);
    const auto kernel = a.n_split > 1 ? gemm_mx_few_kernel<CBF16, NB, MT, true> : gemm_mx_few_kernel<CBF16, NB, MT, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * FW), 0, s, a);
}

template <bool CBF16, int MT>
void launch_mx_few(const MxArgs<CBF16> &a, hipStream_t s)
{
    const int nb = few_blocks(a.N);
    nb == 1   ? launch_mx_few<CBF16, 1, MT>(a, s)
    : nb == 2 ? launch_mx_few<CBF16, 2, MT>(a, s)
              : launch_mx_few<CBF16, 4, MT>(a, s);
}

template <bool CBF16>
hipError_t launch_mx(MxArgs<CBF16> a, hipStream_t s)
{
    a.n_split = mx_ranges(a.M, a.N, a.K, a.n_split);
    if (mx_few(a.M)) {
        a.M <= 16   ? launch_mx_few<CBF16, 1>(a, s)
        : a.M <= 32 ? launch_mx_few<CBF16, 2>(a, s)
        : a.M <= 48 ? launch_mx_few<CBF16, 3>(a, s)
                    : launch_mx_few<CBF16, 4>(a, s);
    } else {
        a.tiles_n = (a.N + TN - 1) / TN;
        a.n_tiles = (a.M + TM - 1) / TM * a.tiles_n;
        a.n_wg = a.n_tiles * a.n_split;
        const auto kernel = a.n_split > 1 ? gemm_mx_kernel<CBF16, true> : gemm_mx_kernel<CBF16, false>;
        hipLaunchKernelGGL(kernel, dim3(a.n_wg), dim3(NT), 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_split == 1)
        return e;
    const size_t threads = (size_t)a.M * a.N / 4;
    hipLaunchKernelGGL(gemm_join_kernel<CBF16>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, (EArgs<CBF16>)a);
    return hipGetLastError();
}

ta_status check_mx_sizes(int M, int N, int K)
{
    if (M < 1 || N < 1 || K < 1)
        return TA_ERR_INVALID_SHAPE;
    if (N % 8 || K % 32)
        return TA_ERR_UNSUPPORTED;
    if (N >= 1 << 24 || K >= 1 << 22 || M > 1 << 20 || (int64_t)M * N >= 1ll << 35 || (int64_t)M * K >= 1ll << 40 ||
        (int64_t)N * K >= 1ll << 40)
        return TA_ERR_INVALID_SHAPE;
    return TA_OK;
}

}  // namespace

extern "C" {

ta_status gemm_mxfp4_epilogue(const void *A, const void *W, const void *W_scale, const void *bias, const void *residual,
                              void *C, int c_bf16, int activation, int M, int N, int K, int num_splits,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!A || !W || !W_scale || !C)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_splits < 1 || num_splits > MAX_SPLITS)
        return TA_ERR_INVALID_SHAPE;
    if (activation < TA_ACT_NONE || activation > TA_ACT_SILU)
        return TA_ERR_UNSUPPORTED;
    if (misaligned(A) || misaligned(W) || misaligned(C) || misaligned(bias) || misaligned(residual))
        return TA_ERR_MISALIGNED;
    const size_t a_bytes = (size_t)M * K * 2, w_bytes = (size_t)N * (K / 2), s_bytes = (size_t)N * (K / 32);
    const size_t c_bytes = (size_t)M * N * (c_bf16 ? 2 : 4);
    if (overlaps(C, c_bytes, A, a_bytes) || overlaps(C, c_bytes, W, w_bytes) || overlaps(C, c_bytes, W_scale, s_bytes) ||
        overlaps(C, c_bytes, bias, (size_t)N * 2) || (residual != C && overlaps(C, c_bytes, residual, c_bytes)))
        return TA_ERR_ALIASING;
    const size_t need = mx_workspace(M, N, K, num_splits);
    if (need) {
        if (!workspace || workspace_bytes < need)
            return TA_ERR_WORKSPACE;
        if (misaligned(workspace))
            return TA_ERR_MISALIGNED;
        if (overlaps(workspace, need, A, a_bytes) || overlaps(workspace, need, W, w_bytes) ||
            overlaps(workspace, need, W_scale, s_bytes) || overlaps(workspace, need, C, c_bytes) ||
            overlaps(workspace, need, bias, (size_t)N * 2) || overlaps(workspace, need, residual, c_bytes))
            return TA_ERR_ALIASING;
    }
    const auto run = [&](auto a) {
        a.A = (const uint16_t *)A;
        a.C = workspace;
        a.M = M;
        a.N = N;
        a.K = K;
        a.n_split = num_splits;
        a.bias = (const uint16_t *)bias;
        a.R = residual;
        a.out = C;
        a.act = activation;
        a.W = (const uint8_t *)W;
        a.S = (const uint8_t *)W_scale;
        return launch_mx(a, (hipStream_t)stream);
    };
    return (c_bf16 ? run(MxArgs<true>{}) : run(MxArgs<false>{})) == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

ta_status gemm_mxfp4_workspace_bytes(int M, int N, int K, int num_splits, size_t *bytes)
{
    if (!bytes)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_splits < 1 || num_splits > MAX_SPLITS)
        return TA_ERR_INVALID_SHAPE;
    *bytes = mx_workspace(M, N, K, num_splits);
    return TA_OK;
}

ta_status gemm_mxfp4_plan(int M, int N, int K, int *num_splits)
{
    if (!num_splits)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    *num_splits = 1;
    return TA_OK;
}

}  // extern "C"
