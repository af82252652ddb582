// C = act(A W^T + bias) + residual for bf16 A [M, K] and W [N, K] in 4 bits (MXFP4) on
// gfx950 (MI355X), any M, N a multiple of 8 and K of 32.  The codes become bf16 in
// registers, two by one instruction, scale included and exactly, on their way into
// bf16 matrix instructions: the products are those of the numbers that they stand for.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "even_parts.h"
#include "gemm_epilogue.h"
#include "lds_dma.h"
#include "mxfp4.h"
#include "tileattn.h"

namespace {

using tileattn_detail::even_begin;
using tileattn_detail::even_part_of;

// (B and n_split of EArgs are not used; C is the workspace)
template <bool CBF16>
struct MxArgs : EArgs<CBF16> {
    const uint8_t *W, *S;      // codes [N, K / 2], scales [N, K / 32]
    int parts;                 // 0, or the workgroups that share all strips' or tiles' steps
};

// Steps of K = 128 in order, of one strip or tile after the other: a workgroup takes one
// of them whole or, with parts, an even share of all steps.  Those that a share's ends cut
// leave partial sums for gemm_mx_join_kernel: part p's record 2 p is of one that an earlier
// part began, 2 p + 1 of one that it began itself and a later part goes on with.
struct Share {
    uint32_t unit, at, left;   // from step `at` of a strip or tile, `left` of them
};

__device__ __forceinline__ Share share_of(uint32_t units, uint32_t steps, uint32_t parts, uint32_t p)
{
    if (!parts)
        return {p, 0, steps};
    const uint32_t n = units * steps, begin = even_begin(n, parts, p);
    return {begin / steps, begin % steps, even_begin(n, parts, p + 1) - begin};
}

// ---- up to 16 rows: a decode step's tokens ---------------------------------
// HBM bounds it: every weight is read once and meets a few tokens.  A wave takes a
// strip of 16 NB rows of W and every eighth step of 128 columns of K (its workgroup's
// waves read the same rows side by side): a lane's 16 bytes of a row are 32 numbers, one
// group, and so four operands of v_mfma_f32_16x16x32_bf16 with one scale; A's operands
// are taken from the same places of K, 16 bytes of a row, from L2.  C^T = W A^T, so that a
// lane ends up with four consecutive columns of a token.  The waves add up in LDS, in
// wave order.  1 x 4096 x 4096 5.4 us, 1 x 14336 x 4096 12.8; for 1 x 16384 x 16384 the
// loads of the scales are a quarter of the time (45 us, 34 without them), A's a tenth.
constexpr int FW = 8, TK = 128;

template <bool CBF16, int NB>
__global__ __launch_bounds__(64 * FW, 2) void gemm_mx_few_kernel(MxArgs<CBF16> a)
{
    constexpr int CH = 4 * NB;                 // 16-byte chunks of a strip's row of C
    __shared__ __attribute__((aligned(16))) float red[FW][16][16 * NB];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const uint32_t all = (a.K + TK - 1) / TK;
    Share share = share_of((a.N + 16 * NB - 1) / (16 * NB), all, a.parts, blockIdx.x);

    for (;;) {
        const uint32_t take = min(share.left, all - share.at);
        const int n0 = share.unit * (16 * NB), lo = share.at, hi = share.at + take;

        // This lane's rows of W, their scales, and its row of A (rows past the last are the
        // last: never stored)
        const uint8_t *w[NB], *e[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const size_t n = min(n0 + 16 * b + c16, a.N - 1);
            w[b] = a.W + n * (a.K / 2);
            e[b] = a.S + n * (a.K / 32);
        }
        const uint16_t *const x = a.A + (size_t)min(c16, a.M - 1) * a.K;

        f32x4 acc[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};

        struct Step {
            u32x4 w[NB], x[4];
            uint32_t e[NB];
        };
        auto load = [&](int s, Step &st) {
            // (lanes past K read the last group, and take zeros below)
            const int k = min(TK * s + 32 * g, a.K - 32);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                st.w[b] = __builtin_nontemporal_load((const u32x4 *)(w[b] + k / 2));
                st.e[b] = e[b][k / 32];
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                st.x[kk] = *(const u32x4 *)(x + k + 8 * kk);
        };
        auto compute = [&](int s, Step &st) {
            if (TK * s + TK > a.K) {
                const bool in = TK * s + 32 * g < a.K;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    st.w[b] = in ? st.w[b] : u32x4{0, 0, 0, 0};
                    st.e[b] = in ? st.e[b] : 127u;
                }
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    st.x[kk] = in ? st.x[kk] : u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    acc[b] = mfma(tileattn_mx::eight(st.w[b][kk], tileattn_mx::scale_of(st.e[b])),
                                  __builtin_bit_cast(bf16x8, st.x[kk]), acc[b]);
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

        // lane: row c16, columns 16 b + 4 g .. + 3; chunk ch of row x at ch ^ x
#pragma unroll
        for (int b = 0; b < NB; ++b)
            *(f32x4 *)&red[wave][c16][4 * ((4 * b + g) ^ (c16 % CH))] = acc[b];
        __syncthreads();
        float *const rec = (float *)a.C + (2 * (size_t)blockIdx.x + (lo == 0)) * a.M * (16 * NB);
        const int m = tid / CH, ch = tid % CH, n = n0 + 4 * ch;
        if (m < a.M && n < a.N) {              // (a row has 16 CH <= 128 of the threads)
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < FW; ++v)
                sum += *(const f32x4 *)&red[v][m][4 * (ch ^ (m % CH))];
            if (take == all)
                a.store(m, n, sum);
            else
                *(f32x4 *)(rec + m * (16 * NB) + 4 * ch) = sum;
        }
        share.left -= take;
        if (share.left == 0)
            return;
        ++share.unit;
        share.at = 0;
        __syncthreads();   // (the sums have been read)
    }
}

// One byte at byte `voff` of the buffer per lane, as a dword at LDS `lds` + 4 lane
__device__ __forceinline__ void dma_byte(uint32_t lds, uint32_t voff, uint32_t soff, u32x4s rsrc)
{
    asm volatile("s_nop 0\n\t"
                 "buffer_load_ubyte %0, %1, %2 offen lds"
                 :
                 : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

// ---- up to 64 rows through LDS --------------------------------------------
// The same product where A's operands, which every wave of the kernel above fetches for
// itself, would cost more than W: a workgroup takes all rows (16 MT of them) and 64
// columns in stages of 128 of K, a ring of them in LDS filled by DMA, A's rows, W's codes
// and the scales.  Wave: half of the columns and a quarter of the stage's K, so a lane's
// operand of W is 4 bytes; the quarters add up in LDS in the end.  24 x 14336 x 4096 16 us:
// W's DMA alone 8.8, A's and the scales' with it 13.5, the products hide but for 2.5.
// (Strips of 128 columns, 20 us as 256 parts; twelve stages, one workgroup to a CU, 19;
// workgroups that begin at different stages, so that rows a power of two apart are not read
// at once, 19: A is then not shared in L2.)
template <int MT, bool S4>
struct Skinny {
    static constexpr int TN = 64;
    static constexpr int A_BYTES = 16 * MT * 256, W_BYTES = TN * 64, S_BYTES = TN * (S4 ? 4 : 16);
    static constexpr int STAGE = A_BYTES + W_BYTES + S_BYTES;
    static constexpr int ST = 79 * 1024 / STAGE < 8 ? 79 * 1024 / STAGE : 8;
    static constexpr int SUMS = 4 * 16 * MT * TN * 4;                   // bytes of the quarters' sums
    static constexpr int LDS = ST * STAGE > SUMS ? ST * STAGE : SUMS;
    // DMA instructions of a stage, shared out to the waves in turn
    static constexpr int NA = A_BYTES / 1024, NW = W_BYTES / 1024, NS = S4 ? TN / 64 : TN / 16, ALL = NA + NW + NS;
    static constexpr int MOST = (ALL + 7) / 8, LEAST = ALL / 8;          // of a wave
    static_assert(MOST * (ST - 2) < 64, "vmcnt");
};

// wait until the loads of at most `later` stages of C instructions are in flight
template <int C, int L>
__device__ __forceinline__ void wait_stages(int later)
{
    if constexpr (L == 0)
        tileattn_dma::wait_vmcnt<0>();
    else if (later >= L)
        tileattn_dma::wait_vmcnt<C * L>();
    else
        wait_stages<C, L - 1>(later);
}

// The 4 bytes at byte `voff` of the buffer per lane to LDS `lds` + 4 lane
__device__ __forceinline__ void dma_dword(uint32_t lds, uint32_t voff, uint32_t soff, u32x4s rsrc)
{
    asm volatile("s_nop 0\n\t"
                 "buffer_load_dword %0, %1, %2 offen lds"
                 :
                 : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

// S4: K is a multiple of 128 and the scales' rows are of aligned dwords
template <bool CBF16, int MT, bool S4>
__global__ __launch_bounds__(NT, 2) void gemm_mx_skinny_kernel(MxArgs<CBF16> a)
{
    using Z = Skinny<MT, S4>;
    constexpr int TN = Z::TN, ST = Z::ST, NB = TN / 32, CH = TN / 4;
    __shared__ __attribute__((aligned(16))) unsigned char lds[Z::LDS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int nh = wave & 1, kq = wave >> 1;
    const uint32_t all = (a.K + TK - 1) / TK;
    Share share = share_of((a.N + TN - 1) / TN, all, a.parts, blockIdx.x);
    const u32x4s ra = tileattn_dma::buffer_rsrc(a.A, (uint32_t)a.M * a.K * 2);

    for (;;) {
        const int n_kt = min(share.left, all - share.at), lo = share.at, n0 = share.unit * TN;
        const int nr = min(TN, a.N - n0);
        const u32x4s rw = tileattn_dma::buffer_rsrc(a.W + (size_t)n0 * (a.K / 2), (uint32_t)nr * (a.K / 2));
        const u32x4s rs = tileattn_dma::buffer_rsrc(a.S + (size_t)n0 * (a.K / 32), (uint32_t)nr * (a.K / 32));
        // This wave's instructions: instruction i = 8 j + wave of a stage, its lanes' rows and chunks
        // (rows past the last are the last; never stored)
        uint32_t off[Z::MOST];
        int chunk[Z::MOST];
#pragma unroll
        for (int j = 0; j < Z::MOST; ++j) {
            const int i = 8 * j + wave;
            if (i < Z::NA) {
                const int r = (i * 64 + lane) / 16;
                chunk[j] = (lane % 16) ^ (r & 15);
                off[j] = (uint32_t)min(r, a.M - 1) * a.K * 2;
            } else if (i < Z::NA + Z::NW) {
                const int r = ((i - Z::NA) * 64 + lane) / 4;
                chunk[j] = (lane % 4) ^ ((r >> 2) & 3);
                off[j] = (uint32_t)min(r, nr - 1) * (a.K / 2);
            } else {
                const int r = S4 ? (i - Z::NA - Z::NW) * 64 + lane : ((i - Z::NA - Z::NW) * 64 + lane) / 4;
                chunk[j] = S4 ? 0 : lane % 4;
                off[j] = (uint32_t)min(r, nr - 1) * (a.K / 32);
            }
        }
        auto dma = [&](int kt) {
            const int k0 = (lo + kt) * TK, left = a.K - k0;      // (of a last stage, chunks past K are the last)
            const uint32_t base = tileattn_dma::lds_addr(lds) + kt % ST * Z::STAGE;
#pragma unroll
            for (int j = 0; j < Z::MOST; ++j) {
                const int i = 8 * j + wave;
                if (i < Z::NA)
                    tileattn_dma::dma16_soff(base + i * 1024, off[j] + 16 * (S4 ? chunk[j] : min(chunk[j], left / 8 - 1)),
                                             k0 * 2, ra);
                else if (i < Z::NA + Z::NW)
                    tileattn_dma::dma16_soff<true>(base + i * 1024, off[j] + 16 * (S4 ? chunk[j] : min(chunk[j], left / 32 - 1)),
                                             k0 / 2, rw);
                else if (i < Z::ALL) {
                    const uint32_t to = base + Z::A_BYTES + Z::W_BYTES + (i - Z::NA - Z::NW) * 256;
                    if (S4)
                        dma_dword(to, off[j], k0 / 32, rs);
                    else
                        dma_byte(to, off[j] + min(chunk[j], left / 32 - 1), k0 / 32, rs);
                }
            }
        };

        f32x4 acc[MT][NB];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                acc[t][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto compute = [&](const unsigned char *st) {
            uint32_t w[NB];
            float sc[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int n = nh * (TN / 2) + 16 * b + c16;
                w[b] = *(const uint32_t *)(st + Z::A_BYTES + n * 64 + 16 * (kq ^ ((n >> 2) & 3)) + 4 * g);
                const unsigned char *e = st + Z::A_BYTES + Z::W_BYTES;
                sc[b] = tileattn_mx::scale_of(S4 ? e[n * 4 + kq] : *(const uint32_t *)(e + 4 * (n * 4 + kq)));
            }
            bf16x8 x[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int r = 16 * t + c16;
                x[t] = *(const bf16x8 *)(st + r * 256 + 16 * ((4 * kq + g) ^ (r & 15)));
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bf16x8 wb = tileattn_mx::eight(w[b], sc[b]);
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t][b] = mfma(wb, x[t], acc[t][b]);
            }
        };

#pragma unroll
        for (int s = 0; s < ST - 1; ++s)
            if (s < n_kt)
                dma(s);
        for (int kt = 0; kt < n_kt; ++kt) {
            const int later = min(ST - 2, n_kt - 1 - kt);
            if (Z::MOST == Z::LEAST || wave < Z::ALL % 8)
                wait_stages<Z::MOST, ST - 2>(later);
            else
                wait_stages<Z::LEAST, ST - 2>(later);
            __syncthreads();
            if (kt + ST - 1 < n_kt)
                dma(kt + ST - 1);
            if ((lo + kt) * TK + 32 * kq < a.K)     // (a quarter of a last stage may lie past K)
                compute(lds + kt % ST * Z::STAGE);
        }

        // lane: row 16 t + c16, columns of chunk nh CH / 2 + 4 b + g; chunk c of row x at c ^ (x % 16)
        __syncthreads();
        float *const sums = (float *)lds;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                *(f32x4 *)(sums + (kq * 16 * MT + 16 * t + c16) * TN + 4 * ((nh * (CH / 2) + 4 * b + g) ^ c16)) = acc[t][b];
        __syncthreads();
        float *const rec = (float *)a.C + (2 * (size_t)blockIdx.x + (lo == 0)) * a.M * TN;
        for (int e = tid; e < 16 * MT * CH; e += NT) {
            const int x = e / CH, c = e % CH;
            if (x >= a.M || n0 + 4 * c >= a.N)
                continue;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 4; ++q)
                sum += *(const f32x4 *)(sums + (q * 16 * MT + x) * TN + 4 * (c ^ (x & 15)));
            if ((uint32_t)n_kt == all)
                a.store(x, n0 + 4 * c, sum);
            else
                *(f32x4 *)(rec + x * TN + 4 * c) = sum;
        }
        share.left -= n_kt;
        if (share.left == 0)
            return;
        ++share.unit;
        share.at = 0;
        tileattn_dma::wait_vmcnt<0>();   // (the stores: the next strip's loads are counted by hand)
        __syncthreads();                 // the sums have been read
    }
}

// ---- more rows: tiles of 128 rows by 128 or 256 columns --------------------
// A workgroup of eight waves computes a tile in stages of 128 of K, a ring of three of
// them in LDS: A's rows (32 KB), W's codes (8 or 16 KB) and the scales' bytes, one a
// dword (2 or 4 KB), all by DMA.  Two groups of four waves take half of a stage's K each
// and half of the tile's rows and columns a wave, in v_mfma_f32_32x32x16_bf16: a lane's
// 16 bytes of a row of W are the 32 numbers of a group, four operands, with one scale,
// and A's operands come from the same places of K.  W stays in 4 bits up to the
// registers, so that LDS holds and gives a quarter of a bf16 tile's bytes for it.
// 1021 x 16384 x 16384 448 us (1222 TFLOP/s; a bf16 product of that size by the library 1215),
// 1021 x 4232 x 8224 93: 80 for 256 shares of 136 tiles, 13 for the join.  A stage of 256
// columns takes 1.75 us where its matrix instructions take 0.85 at 2.4 GHz (the clock is at
// 2.0): half of the rest is LDS and its barrier.  Tried: the two groups taking turns, one's
// reads under the other's products (no change with 128 columns, registers spill with 256).
constexpr int TM = 128, TST = 3;
constexpr int A_STAGE = TM * TK * 2, A_DMA = A_STAGE / 16 / NT;

template <int TN>
struct Tile {
    static constexpr int W_STAGE = TN * TK / 2, S_STAGE = TN * TK / 32 * 4;
    static constexpr int STAGE = A_STAGE + W_STAGE + S_STAGE;
    static constexpr int W_DMA = TN * 4 / NT, DMAS = A_DMA + 2 * W_DMA;   // of a thread and stage
    static constexpr int FN = TN / 64;                                    // 32 x 32 blocks of a wave's columns
    static_assert(W_DMA * NT == TN * 4 && TST * STAGE >= TM * TN * 4 && TST * STAGE <= 160 * 1024, "LDS");
};

template <bool CBF16, int TN>
__global__ __launch_bounds__(NT, 2) void gemm_mx_kernel(MxArgs<CBF16> args)
{
    using T = Tile<TN>;
    constexpr int FN = T::FN, STAGE = T::STAGE, W_STAGE = T::W_STAGE;
    __shared__ __attribute__((aligned(16))) unsigned char lds[TST * STAGE];
    const MxArgs<CBF16> &a = args;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int kg = wave >> 2, wm = (wave >> 1 & 1) * 64, wn = (wave & 1) * (TN / 2);

    // shares in XCD-contiguous order; tiles in groups of four rows of tiles
    const int per = a.n_wg / NXCD, rem = a.n_wg % NXCD;
    const int xcd = blockIdx.x % NXCD;
    const uint32_t part = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / NXCD;
    const uint32_t all = (a.K + TK - 1) / TK;
    Share share = share_of(a.n_tiles, all, a.parts, part);
    for (;;) {
        const int t = share.unit, lo = share.at, n_kt = min(share.left, all - share.at);
        const int grp = t / (GROUP_M * a.tiles_n), w = t % (GROUP_M * a.tiles_n);
        const int rows = min((a.M + TM - 1) / TM - grp * GROUP_M, GROUP_M);
        const int m0 = (grp * GROUP_M + w % rows) * TM, n0 = w / rows * TN;

        // Where this thread's chunks come from (rows past the last are the last; in a last
        // stage, chunks past K are the last: those are cleared in the operands)
        const int mr = min(TM, a.M - m0), nr = min(TN, a.N - n0);
        const u32x4s ra = tileattn_dma::buffer_rsrc(a.A + (size_t)m0 * a.K, (uint32_t)mr * a.K * 2);
        const u32x4s rw = tileattn_dma::buffer_rsrc(a.W + (size_t)n0 * (a.K / 2), (uint32_t)nr * (a.K / 2));
        const u32x4s rs = tileattn_dma::buffer_rsrc(a.S + (size_t)n0 * (a.K / 32), (uint32_t)nr * (a.K / 32));
        // A: slot s is row s / 16, stored chunk s % 16; W: row s / 4, stored chunk s % 4; scales:
        // row s / 4, group s % 4
        auto a_row = [&](int i) { return (i * NT + tid) / 16; };
        auto a_ch = [&](int i) { return (tid % 16) ^ (a_row(i) & 15); };
        const int w_ch = (tid % 4) ^ ((tid / 8) & 3), s_grp = tid % 4;   // (row / 2 % 4, for all its rows)
        uint32_t ao[A_DMA];
#pragma unroll
        for (int i = 0; i < A_DMA; ++i)
            ao[i] = (uint32_t)min(a_row(i), mr - 1) * a.K * 2;
        uint32_t wr[T::W_DMA];
#pragma unroll
        for (int i = 0; i < T::W_DMA; ++i)
            wr[i] = (uint32_t)min((i * NT + tid) / 4, nr - 1) * (a.K / 32);
        auto dma = [&](int kt, unsigned char *to) {
            const int k0 = (lo + kt) * TK, left = a.K - k0;
            const uint32_t base = tileattn_dma::lds_addr(to);
            int ac[A_DMA], wc = w_ch, sg = s_grp;
#pragma unroll
            for (int i = 0; i < A_DMA; ++i)
                ac[i] = a_ch(i);
            if (left < TK) {
#pragma unroll
                for (int i = 0; i < A_DMA; ++i)
                    ac[i] = min(ac[i], left / 8 - 1);
                wc = min(wc, left / 32 - 1);
                sg = min(sg, left / 32 - 1);
            }
#pragma unroll
            for (int i = 0; i < A_DMA; ++i)
                tileattn_dma::dma16_soff(base + (i * NT + wave * 64) * 16, ao[i] + 16 * ac[i], k0 * 2, ra);
#pragma unroll
            for (int i = 0; i < T::W_DMA; ++i)
                tileattn_dma::dma16_soff(base + A_STAGE + (i * NT + wave * 64) * 16, 16 * wr[i] + 16 * wc, k0 / 2, rw);
#pragma unroll
            for (int i = 0; i < T::W_DMA; ++i)
                dma_byte(base + A_STAGE + W_STAGE + (i * NT + wave * 64) * 4, wr[i] + sg, k0 / 32, rs);
        };

        f32x16 acc[2][FN];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[i][j][r] = 0.f;

        // `part`: a last stage of less than 128, in which this lane's 32 of K may be past the
        // end (`in`: they are not)
        auto compute = [&](const unsigned char *st, auto part, bool in) {
            u32x4 wv[FN];
            float sc[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int n = wn + 32 * j + col, q = 2 * kg + half;
                wv[j] = *(const u32x4 *)(st + A_STAGE + n * 64 + 16 * (q ^ ((n >> 1) & 3)));
                sc[j] = tileattn_mx::scale_of(*(const uint32_t *)(st + A_STAGE + W_STAGE + 4 * (n * 4 + q)));
                if (part && !in) {
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
                    if (part && !in)
                        x = u32x4{0, 0, 0, 0};
                    av[i] = __builtin_bit_cast(bf16x8, x);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const bf16x8 wb = tileattn_mx::eight(wv[j][kk], sc[j]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        acc[i][j] = mfma(wb, av[i], acc[i][j]);
                }
            }
        };

        // stage kt lives in kt % TST; the loads of up to TST - 2 later ones may stay in flight
        // at its beginning, and the barrier frees the stage before it
        const int n_whole = n_kt - ((lo + n_kt) * TK > a.K);
#pragma unroll
        for (int s = 0; s < TST - 1; ++s)
            if (s < n_kt)
                dma(s, lds + s * STAGE);
        for (int kt = 0; kt < n_whole; ++kt) {
            if (kt + 1 < n_kt)
                tileattn_dma::wait_vmcnt<T::DMAS * (TST - 2)>();
            else
                tileattn_dma::wait_vmcnt<0>();
            __syncthreads();
            const int nx = kt + TST - 1;
            if (nx < n_kt)
                dma(nx, lds + nx % TST * STAGE);
            compute(lds + kt % TST * STAGE, std::false_type{}, true);
        }
        if (n_whole < n_kt) {
            tileattn_dma::wait_vmcnt<0>();
            __syncthreads();
            compute(lds + n_whole % TST * STAGE, std::true_type{}, (lo + n_whole) * TK + 64 * kg + 32 * half < a.K);
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
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *at(wm + 32 * i + col, (wn + 32 * j) / 4 + 2 * q + half) =
                            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        if (kg == 0)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *at(wm + 32 * i + col, (wn + 32 * j) / 4 + 2 * q + half) +=
                            f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        constexpr int U = 4, RPI = NT / (TN / 4);        // rows at a time, U steps of them
        const int c = tid % (TN / 4), n = n0 + 4 * c, r0 = tid / (TN / 4);
        if ((uint32_t)n_kt == all) {
            typename EArgs<CBF16>::template Added<U> now, next;
            now.load(a, m0 + r0, RPI, n);
#pragma unroll 1
            for (int r = r0; r < TM; r += U * RPI) {
                f32x4 x[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    x[u] = *at(r + u * RPI, c);
                if (r + U * RPI < TM)
                    next.load(a, m0 + r + U * RPI, RPI, n);
                a.store(m0 + r, RPI, n, x, now);
                now = next;
            }
        } else {
            float *const rec = (float *)a.C + (2 * (size_t)part + (lo == 0)) * TM * TN;
#pragma unroll 4
            for (int r = r0; r < TM; r += RPI)
                *(f32x4 *)(rec + r * TN + 4 * c) = *at(r, c);
        }
        share.left -= n_kt;
        if (share.left == 0)
            return;
        ++share.unit;
        share.at = 0;
        tileattn_dma::wait_vmcnt<0>();   // (the stores: the next tile's loads are counted by hand)
        __syncthreads();                 // the sums have been read
    }
}

// The partial sums of the strips (of `width` columns, all rows) or tiles that were cut,
// added in order of K, and the epilogue: four columns per thread, up to eight records'
// loads in flight
template <bool CBF16>
__global__ __launch_bounds__(256) void gemm_mx_join_kernel(MxArgs<CBF16> a, int rows, int width)
{
    const uint32_t all = (a.K + 127) / 128, t = blockIdx.x;
    const uint32_t p0 = even_part_of(a.n_tiles * all, a.parts, t * all);
    const uint32_t p1 = even_part_of(a.n_tiles * all, a.parts, t * all + all - 1);
    const int e = blockIdx.y * 256 + threadIdx.x, r = e / (width / 4), col = e % (width / 4) * 4;
    int m0 = 0, n0 = t * width;
    if (a.M > 64) {                                  // tiles, in the order of gemm_mx_kernel
        const int grp = t / (GROUP_M * a.tiles_n), w = t % (GROUP_M * a.tiles_n);
        const int g = min((a.M + TM - 1) / TM - grp * GROUP_M, GROUP_M);
        m0 = (grp * GROUP_M + w % g) * TM;
        n0 = w / g * width;
    }
    if (p0 == p1 || r >= rows || m0 + r >= a.M || n0 + col >= a.N)
        return;
    const size_t rec = (size_t)rows * width;
    const float *const w = (const float *)a.C + (size_t)r * width + col;
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
    a.store(m0 + r, n0 + col, sum);
}

constexpr int MX_MAX_PARTS = 4096;

bool mx_few(int M) { return M <= 64; }

int mx_steps(int K) { return (K + 127) / 128; }

// Columns of a strip of few rows: 16 and 32 by gemm_mx_few_kernel, 64 through LDS.  us, 16 |
// 32 | 64 columns (* as 256 parts):
//   1 x 4096 x 4096   5.4 | 7.4 | 13.2     16 x 4096 x 4096   8.4 | 10.6 | 13.4
//   8 x 8192 x 1024   4.6 | 4.1 | 5.9      16 x 8192 x 8192   26.7 | 18.7 | 18.4*
//   1 x 14336 x 4096  14.0 | 12.8 | 13.8   8 x 14336 x 4096   19.5 | 15.5 | 14.1
//   16 x 16384 x 512  5.2 | 4.3 | 4.6      16 x 16384 x 16384  97.6 | 66.8 | 49.6
//   more than 16 rows by the first kernel with 16, 32 and 64 columns, and through LDS:
//   24 x 14336 x 4096 33.9, 24.1, 18.3 | 16.1   64 x 16384 x 4096 74.7, 43.6, 35.5 | 20.3
//   32 x 8192 x 8192  40.6, 27.4, 23.9* | 20.0*
int strip_columns(int M, int N, int K)
{
    if (M > 16)
        return 64;
    return N <= 6144 ? 16 : M <= 4 || K <= 2048 || N <= 10240 ? 32 : 64;
}

// The workgroups that share the strips' steps: one per CU where the steps that the
// longest share is shorter by pay for the second kernel, else a strip each.  us, 0 | 256:
//   16 x 512 x 16384 24.8 | 8.3   16 x 2048 x 8192 13.7 | 11.0   1 x 2048 x 8192 8.7 | 8.6
//   64 x 4096 x 4096 17.9 | 12.3  20 x 6144 x 4096 15.6 | 13.4   20 x 10240 x 4096 15.8 | 17.1
//   64 x 1000 x 2048 10.9 | 7.8   64 x 1000 x 1024 7.2 | 7.3
int strip_parts(int M, int N, int K)
{
    const int columns = strip_columns(M, N, K), waves = columns < 64 ? FW : 1;   // that take a step each
    const int64_t strips = (N + columns - 1) / columns, steps = mx_steps(K);
    const int64_t alone = (steps + waves - 1) / waves, shared = (strips * steps + 256 * waves - 1) / (256 * waves);
    const double step = columns < 64 ? 0.6 + 0.04 * M : 0.3 + 0.045 * ((M + 15) / 16);
    return strips < 256 && (alone - shared) * step > (columns < 64 ? 3.5 : 6) ? 256 : 0;
}

// Estimates in us of a product of more than 64 rows in tiles of 128 x tn on `parts`
// workgroups (0: one each), for the choices below, fitted to the sizes in the table.  A
// workgroup has a CU to itself; a stage takes longer where all CUs draw.  Pieces of
// tiles cost their beginnings and ends, records their way to memory and back, the join 4.
//   us, tn 128 | 256, without and with the best parts:
//   1021 x 16384 x 16384  517       | 448             700 x 8192 x 8192   126, 117 | 111, 113
//   1021 x 4232 x 8224    130, 108  | 110, 94         300 x 12288 x 1024  24, 30   | 21, 33
//   512 x 4096 x 4096     34.3, 29.1 | 54.5, 32.6     128 x 4096 x 4096   31.9, 19.9 | 52, 25
//   200 x 512 x 16384     107, 17.6 | 183, 23.9       300 x 2048 x 512    8.7, 11.8 | 13.4, 14.2
double time_tiles(int64_t tiles, int steps, int tn, int parts)
{
    const double fill = std::min(1.0, (parts ? parts : tiles) / 256.0);
    const double stage = tn == 128 ? 0.83 + 0.17 * fill : 1.42 + 0.33 * fill;
    if (!parts)
        return 5 + (double)((tiles + 255) / 256) * steps * stage;
    const double pieces = parts % tiles ? parts + tiles : parts;
    return 5 + (double)((tiles * steps + parts - 1) / parts) * stage + 10 * (pieces / parts - 1) + 4 +
           2 * pieces * TM * tn * 4 / 6e6;
}

struct TileChoice {
    int tn, parts;
    double time;
};

TileChoice choose_tiles(int M, int N, int K)
{
    TileChoice best = {0, 0, 0.0};
    const int steps = mx_steps(K);
    for (int tn = 128; tn <= 256; tn += 128) {
        const int64_t tiles = (int64_t)((M + TM - 1) / TM) * ((N + tn - 1) / tn);
        const auto look = [&](int64_t parts) {
            if (parts > 256 || parts > tiles * steps)
                return;
            const double t = time_tiles(tiles, steps, tn, (int)parts);
            if (!best.tn || t < best.time)
                best = {tn, (int)parts, t};
        };
        look(0);
        look(256);
        for (int q = 2; q <= steps && q * tiles <= 256; ++q)
            look(q * tiles);
    }
    return best;
}

// Columns of a strip or tile, and how many of those there are
int mx_columns(int M, int N, int K) { return mx_few(M) ? strip_columns(M, N, K) : choose_tiles(M, N, K).tn; }
int mx_units(int M, int N, int K)
{
    const int n = mx_columns(M, N, K);
    return (mx_few(M) ? 1 : (M + TM - 1) / TM) * ((N + n - 1) / n);
}

// The parts that are used: a step each at least, for few rows one for every wave
int64_t mx_parts(int M, int N, int K, int num_parts)
{
    const int64_t steps = (int64_t)mx_units(M, N, K) * mx_steps(K);
    if (steps >= 1ll << 31)      // (counted in 32 bits)
        return 0;
    return std::min<int64_t>(num_parts, mx_few(M) && strip_columns(M, N, K) < 64 ? (steps + FW - 1) / FW : steps);
}

size_t mx_workspace(int M, int N, int K, int num_parts)
{
    return (size_t)mx_parts(M, N, K, num_parts) * 2 * (mx_few(M) ? M : TM) * mx_columns(M, N, K) * 4;
}

template <bool CBF16, int MT>
void launch_mx_few(const MxArgs<CBF16> &a, int columns, hipStream_t s)
{
    auto kernel = a.K % 128 == 0 && (uintptr_t)a.S % 4 == 0 ? gemm_mx_skinny_kernel<CBF16, MT, true>
                                                            : gemm_mx_skinny_kernel<CBF16, MT, false>;
    if constexpr (MT == 1)
        if (columns < 64)
            kernel = columns == 16 ? gemm_mx_few_kernel<CBF16, 1> : gemm_mx_few_kernel<CBF16, 2>;
    hipLaunchKernelGGL(kernel, dim3(a.n_wg), dim3(NT), 0, s, a);
}

template <bool CBF16>
hipError_t launch_mx(MxArgs<CBF16> a, hipStream_t s)
{
    a.n_tiles = mx_units(a.M, a.N, a.K);
    const int tn = mx_columns(a.M, a.N, a.K);
    a.tiles_n = (a.N + tn - 1) / tn;
    a.parts = (int)mx_parts(a.M, a.N, a.K, a.parts);
    a.n_wg = a.parts ? a.parts : a.n_tiles;
    if (mx_few(a.M))
        a.M <= 16   ? launch_mx_few<CBF16, 1>(a, tn, s)
        : a.M <= 32 ? launch_mx_few<CBF16, 2>(a, tn, s)
        : a.M <= 48 ? launch_mx_few<CBF16, 3>(a, tn, s)
                    : launch_mx_few<CBF16, 4>(a, tn, s);
    else
        hipLaunchKernelGGL((tn == 256 ? gemm_mx_kernel<CBF16, 256> : gemm_mx_kernel<CBF16, 128>), dim3(a.n_wg), dim3(NT), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.parts)
        return e;
    const int rows = mx_few(a.M) ? a.M : TM, width = tn;
    hipLaunchKernelGGL(gemm_mx_join_kernel<CBF16>, dim3(a.n_tiles, (rows * width / 4 + 255) / 256), dim3(256), 0, s, a, rows, width);
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
                              void *C, int c_bf16, int activation, int M, int N, int K, int num_parts,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!A || !W || !W_scale || !C)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_parts < 0 || num_parts > MX_MAX_PARTS)
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
    const size_t need = mx_workspace(M, N, K, num_parts);
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
        a.parts = num_parts;
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

ta_status gemm_mxfp4_workspace_bytes(int M, int N, int K, int num_parts, size_t *bytes)
{
    if (!bytes)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    if (num_parts < 0 || num_parts > MX_MAX_PARTS)
        return TA_ERR_INVALID_SHAPE;
    *bytes = mx_workspace(M, N, K, num_parts);
    return TA_OK;
}

ta_status gemm_mxfp4_plan(int M, int N, int K, int *num_parts)
{
    if (!num_parts)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_mx_sizes(M, N, K);
    if (rc != TA_OK)
        return rc;
    *num_parts = mx_few(M) ? strip_parts(M, N, K) : choose_tiles(M, N, K).parts;
    return TA_OK;
}

}  // extern "C"
