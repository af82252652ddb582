// The tiled kernel of the bf16 matrix products (gemm.hip, gemm_epilogue.hip):
// C = A B for A [M, K] and B [K, N], row-major, on the matrix cores.  Its design is
// described at the top of gemm.hip, what products of odd sizes and an epilogue add to
// it at EDGE below.  Internal to libtileattn.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tileattn_gemm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr int BK = 64;       // K per stage
constexpr int NT = 512;      // threads per workgroup (8 waves)
constexpr int NXCD = 8;
constexpr int GROUP_M = 4;   // tile rows per group of the grid order
constexpr int BUF_RSRC_WORD3 = 0x00020000;

struct GArgs {
    const uint16_t *A, *B;
    void *C;
    int M, N, K;
    int tiles_n;     // tiles in a row of C (of a launch's columns)
    int n_tiles;     // tiles of C
    int n_split;     // K ranges per tile; with more than one, C is fp32
                     // [n_split][M][N], one partial product per range
    int n_wg;        // n_tiles * n_split
    // Whole tiles, C stored as it is.  Arguments with EDGE take any M, and N and K
    // in multiples of 8, columns from n_begin on, and store by themselves, four
    // columns from n of rows m, m + step .. at a time, of those that there are:
    // Added<U>::load(args, m, step, n), later store(m, step, n, x, added)
    static constexpr bool EDGE = false;
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// The tile DMA is inline assembly, untracked by the compiler (it would
// otherwise drain the loads in flight before every LDS read, unable to tell
// which buffer they write); the loop waits for it with vmcnt(0).
__device__ __forceinline__ void wait_dma_all() { __builtin_amdgcn_s_waitcnt(0x0F70); }
// wait until at most N of this thread's tile loads are outstanding (N < 16)
template <int N>
__device__ __forceinline__ void wait_dma_upto() { __builtin_amdgcn_s_waitcnt(0x0F70 | N); }

typedef uint32_t u32x4s __attribute__((ext_vector_type(4)));

// raw buffer resource (stride 0, 32-bit format, range-checked) in SGPRs
__device__ __forceinline__ u32x4s buffer_rsrc(const void *base, uint32_t bytes)
{
    const uint64_t a = (uint64_t)(uintptr_t)base;
    return u32x4s{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a),
                  (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xFFFFu),
                  (uint32_t)__builtin_amdgcn_readfirstlane(bytes), (uint32_t)BUF_RSRC_WORD3};
}

// lane l's 16 bytes at byte `voff` of the buffer land at LDS `lds` + 16 l
// (`lds` wave-uniform, passed in M0: the compiler sets M0 for the statement)
__device__ __forceinline__ void dma16(uint32_t lds, uint32_t voff, u32x4s rsrc)
{
    asm volatile("s_nop 0\n\t"   // one wait state between the M0 write and the load
                 "buffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(voff), "s"(rsrc), "{m0}"(__builtin_amdgcn_readfirstlane(lds))
                 : "memory");
}

// What the lanes of a wave wrote to LDS before this, all of its lanes read after it (a
// wave's LDS accesses are carried out in order: this keeps the compiler to the order)
__device__ __forceinline__ void wave_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ uint32_t lds_addr(const void *p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}

__device__ __forceinline__ int a_swz(int r) { return (r >> 1) & 7; }
// B swizzle for the transpose reads of MF x MF blocks: MF = 32 reads four
// rows of 64 bytes per half wave, MF = 16 eight rows (4gq .. +3 of two lane
// groups, 8 apart) of 32 bytes, whose chunk pairs it keeps apart
template <int MF>
__device__ __forceinline__ int b_swz(int r)
{
    return MF == 32 ? 4 * (r & 3) : 2 * (r & 3) + 8 * ((r >> 3) & 1);
}

// KS = 1: the eight waves tile C as 2 x 4.  KS = 2 or 4: KS groups of 8 / KS
// waves, each group tiling C as 1 x (8 / KS) for its share of every K step
// (a wave then reads less of the tiles per flop, most of all of B through
// the transpose read); the groups' sums are added in LDS at the end.
template <int BM, int BN, int KS, int MF>
struct Cfg {
    static constexpr int WPG = 8 / KS;                               // waves per group
    static constexpr int WM = KS == 1 ? BM / 2 : BM, WN = KS == 1 ? BN / 4 : BN / WPG;
    static constexpr int FM = WM / MF, FN = WN / MF;      // MF x MF blocks per wave
    static constexpr int AR = MF * MF / 64;               // accumulator values per lane and block
    static constexpr int KW = 512 / MF;                   // k per MFMA (16 or 32)
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BK * BN * 2;
    static constexpr int A_PER_THREAD = BM * (BK / 8) / NT;   // 16-byte slots
    static constexpr int B_PER_THREAD = BK * (BN / 8) / NT;
    static constexpr int BCH = BN / 8;                    // 16-byte chunks per B row
    static constexpr int PER_STAGE = A_PER_THREAD + B_PER_THREAD;   // loads per thread
};

// ST stages of A and B tiles in LDS: two (double buffering, one tile in
// flight during the MFMAs) or a ring of three or four (ST - 1 tiles in
// flight) for grids of at most one workgroup per CU, where no other
// workgroup's MFMAs cover the wait for a tile.
// SPLIT: C is the fp32 partial products of a.n_split K ranges.  A kernel of its
// own: the range arithmetic in the unsplit one cost 0.5 us (1024 x 8192 x 192,
// fp32 C, 11.6 us with it, 11.1 without).
// EDGE (Args::EDGE): what a tile lacks of its BM rows, BN columns or a last step
// of its 64 rows of B is read from the tile's last row or chunk instead, so that
// nothing outside A and B is addressed; the chunks of a last step that lie past K
// are then cleared in LDS by the threads whose DMA brought them, in A and in B (a
// NaN or infinity times zero would not be).  That step is by itself: tested for in
// the loop it cost 4096 x 8192 x 8192 23 us of 420.  The products are transposed, C^T =
// B^T A^T, which costs nothing (both operands have the same layout) and gives a
// lane four consecutive columns of a row instead of four rows of a column.
template <int BM, int BN, int ST, int KS, int MF, bool CBF16, bool SPLIT, class Args = GArgs>
__global__ __launch_bounds__(NT, 2) void gemm_kernel(Args args)
{
    constexpr bool EDGE = Args::EDGE;
    using C = Cfg<BM, BN, KS, MF>;
    using Acc = typename std::conditional<MF == 32, f32x16, f32x4>::type;
    static_assert(KS == 1 || ((KS == 2 || KS == 4) && C::A_BYTES == 16384 &&
                              C::B_BYTES == 16384 &&
                              C::FM * C::FN * C::AR * 256 * C::WPG == 65536),
                  "a group's sums fill the four 16 KB stage buffers");
    static_assert(ST == 2 || (ST <= 4 && 2 * C::PER_STAGE < 16), "stage count / vmcnt range");
    static_assert((BK / C::KW) % KS == 0, "each group takes whole k-steps of every K step");
    __shared__ __attribute__((aligned(16))) unsigned char abuf[ST][C::A_BYTES];
    __shared__ __attribute__((aligned(16))) unsigned char bbuf[ST][C::B_BYTES];
    unsigned char *const a0 = abuf[0], *const a1 = abuf[1];
    unsigned char *const b0 = bbuf[0], *const b1 = bbuf[1];

    const Args &a = args;
    const int tid = threadIdx.x;
    const int wave = tid >> 6, lane = tid & 63;
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const int col = lane % MF, half = lane / MF;   // lane's column of a block; its k part

    // XCD-contiguous logical tile index, row-major over the tiles of C
    const int per = a.n_wg / NXCD, rem = a.n_wg % NXCD;
    const int xcd = blockIdx.x % NXCD, idx = blockIdx.x / NXCD;
    const int ts = xcd * per + (xcd < rem ? xcd : rem) + idx;
    const uint32_t split = SPLIT ? ts / a.n_tiles : 0;
    const int t = ts - split * a.n_tiles;
    // grouped order: GROUP_M consecutive logical tiles walk down a column of
    // tiles before moving right (fewer in a last group of fewer rows), so the
    // workgroups resident on an XCD cover a GROUP_M x (resident / GROUP_M)
    // block of C and share its A and B panels in that XCD's L2.  Row by row,
    // tile rows that GROUP_M does not divide read B once per row from HBM:
    // 896 x 8192 x 8192 154 -> 130 us, 1280 x 8192 x 8192 252 -> 207.
    const int grp = t / (GROUP_M * a.tiles_n), w = t % (GROUP_M * a.tiles_n);
    const int rows = min((EDGE ? (a.M + BM - 1) / BM : a.M / BM) - grp * GROUP_M, GROUP_M);   // tile rows of this group
    // (w / rows without a division: rows is 1, 2, 3 or 4)
    static_assert(GROUP_M == 4, "the quotient by 1 .. GROUP_M");
    const int tn = rows == 3 ? (int)(((uint64_t)(uint32_t)w * 0xAAAAAAABu) >> 33) : w >> (rows >> 1);
    const int tm = grp * GROUP_M + w - tn * rows;
    const int m0 = tm * BM;
    int n0 = tn * BN;
    if constexpr (EDGE)
        n0 += a.n_begin;
    const int cw = KS == 1 ? wave & 3 : wave % C::WPG;    // column of the wave's block
    const int wm = KS == 1 ? (wave >> 2) * C::WM : 0, wn = cw * C::WN;
    const int kg = KS == 1 ? 0 : wave_u / C::WPG;          // this wave's share of each K step

    // per-lane DMA source offsets within a stage's tiles.  A slot
    // i*NT + 64w + l is row s / 8, stored chunk s % 8 (fetched from chunk
    // (s % 8) ^ a_swz(row)); B slot s is row s / BCH, stored chunk s % BCH
    // (fetched from chunk (s % BCH) ^ b_swz(row)).
    uint32_t a_off[C::A_PER_THREAD], b_off[C::B_PER_THREAD];
#pragma unroll
    for (int i = 0; i < C::A_PER_THREAD; ++i) {
        const int s = i * NT + wave_u * 64 + lane;
        const int r = s / 8, sc = s % 8;
        a_off[i] = (uint32_t)(EDGE ? min(r, a.M - 1 - m0) : r) * a.K * 2 + 16 * (sc ^ a_swz(r));
    }
#pragma unroll
    for (int i = 0; i < C::B_PER_THREAD; ++i) {
        const int s = i * NT + wave_u * 64 + lane;
        const int r = s / C::BCH, sc = s % C::BCH;
        const int ch = sc ^ b_swz<MF>(r);
        b_off[i] = (uint32_t)r * a.N * 2 + 16 * (EDGE ? min(ch, (a.N - n0) / 8 - 1) : ch);
    }

    // this range's K steps (ranges of whole steps, as even as they go; a step is 64 rows
    // and there are at most 64 ranges, so the products are at most K + 63)
    const uint32_t kt_all = EDGE ? (a.K + BK - 1) / BK : a.K / BK;
    int kt_lo = 0, n_kt = kt_all;
    if (SPLIT) {
        kt_lo = kt_all * split / a.n_split;
        n_kt = kt_all * (split + 1) / a.n_split - kt_lo;
    }
    // (the part of a step at K's end comes after the loop, which has no test for it)
    const int k_part = EDGE && (!SPLIT || split + 1 == (uint32_t)a.n_split) ? a.K % BK : 0;
    if (k_part)
        --n_kt;

    const int last_row = EDGE ? min(BM - 1, a.M - 1 - m0) : BM - 1;   // the tile's last row, its columns
    const int cols = EDGE ? min(BN, a.N - n0) : BN;
    auto dma = [&](int kt, unsigned char *as, unsigned char *bs) {
        const int k0 = (kt_lo + kt) * BK;
        const u32x4s ra = buffer_rsrc(a.A + (size_t)m0 * a.K + k0, (uint32_t)(last_row * a.K + BK) * 2);
        const u32x4s rb = buffer_rsrc(a.B + (size_t)k0 * a.N + n0, (uint32_t)((BK - 1) * a.N + cols) * 2);
        const uint32_t la = lds_addr(as), lb = lds_addr(bs);
#pragma unroll
        for (int i = 0; i < C::A_PER_THREAD; ++i)
            dma16(la + (i * NT + wave_u * 64) * 16, a_off[i], ra);
#pragma unroll
        for (int i = 0; i < C::B_PER_THREAD; ++i)
            dma16(lb + (i * NT + wave_u * 64) * 16, b_off[i], rb);
    };

    // a last step of kr < 64 rows of B
    auto dma_part = [&](int kr, unsigned char *as, unsigned char *bs) {
        const int k0 = a.K - kr;
        const u32x4s ra = buffer_rsrc(a.A + (size_t)m0 * a.K + k0, (uint32_t)(last_row * a.K + kr) * 2);
        const u32x4s rb = buffer_rsrc(a.B + (size_t)k0 * a.N + n0, (uint32_t)((kr - 1) * a.N + cols) * 2);
        const uint32_t la = lds_addr(as), lb = lds_addr(bs);
#pragma unroll
        for (int i = 0; i < C::A_PER_THREAD; ++i) {
            const int s = i * NT + wave_u * 64 + lane, ch = (s % 8) ^ a_swz(s / 8);
            dma16(la + (i * NT + wave_u * 64) * 16, a_off[i] - 16 * max(ch - (kr / 8 - 1), 0), ra);
        }
#pragma unroll
        for (int i = 0; i < C::B_PER_THREAD; ++i) {
            const int r = (i * NT + wave_u * 64 + lane) / C::BCH;
            dma16(lb + (i * NT + wave_u * 64) * 16, b_off[i] - (uint32_t)max(r - (kr - 1), 0) * a.N * 2, rb);
        }
        // this thread's chunks past K, before the barrier that lets others read
        wait_dma_all();
#pragma unroll
        for (int i = 0; i < C::A_PER_THREAD; ++i) {
            const int s = i * NT + wave_u * 64 + lane;
            if (8 * ((s % 8) ^ a_swz(s / 8)) >= kr)
                *(u32x4 *)(as + 16 * s) = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < C::B_PER_THREAD; ++i) {
            const int s = i * NT + wave_u * 64 + lane;
            if (s / C::BCH >= kr)
                *(u32x4 *)(bs + 16 * s) = u32x4{0, 0, 0, 0};
        }
        __syncthreads();
    };

    Acc acc[C::FM][C::FN];
#pragma unroll
    for (int i = 0; i < C::FM; ++i)
#pragma unroll
        for (int j = 0; j < C::FN; ++j)
#pragma unroll
            for (int r = 0; r < C::AR; ++r)
                acc[i][j][r] = 0.f;

    // B operand transpose-read addressing (per 16-lane group g = lane / 16,
    // s = lane % 16).  MF = 32: rows 16ks + 8(g >> 1) + (s >> 2) and + 4,
    // columns 16(g & 1) + 4(s & 3) of each 32-column block: the lane then
    // holds 8 consecutive k of one column, k-slot t <-> k = 16ks + 8 half + t.
    // MF = 16: rows 32ks + 8g + (s >> 2) and + 4, columns 4(s & 3) of each
    // 16-column block: k-slot t <-> k = 32ks + 8g + t.
    const int g = lane >> 4, sl = lane & 15;
    const int b_row = MF == 32 ? 8 * (g >> 1) + (sl >> 2) : 8 * g + (sl >> 2);
    const int b_col = MF == 32 ? 16 * (g & 1) + 4 * (sl & 3) : 4 * (sl & 3);

    auto compute = [&](const unsigned char *as, const unsigned char *bs) {
#pragma unroll
        for (int kq = 0; kq < BK / C::KW / KS; ++kq) {
            const int ks = kg * (BK / C::KW / KS) + kq;
            bf16x8 av[C::FM], bv[C::FN];
#pragma unroll
            for (int i = 0; i < C::FM; ++i) {
                // lane: row col of the block, k (KW ks + 8 half ..) = chunk
                // (KW / 8) ks + half of the row
                const int r = wm + MF * i + col;
                av[i] = *(const bf16x8 *)(as + r * (BK * 2) +
                                          16 * (((C::KW / 8) * ks + half) ^ a_swz(r)));
            }
#pragma unroll
            for (int j = 0; j < C::FN; ++j) {
                const int n = wn + MF * j + b_col;
                const int r0 = C::KW * ks + b_row, r1 = r0 + 4;
                const unsigned char *p0 =
                    bs + r0 * (BN * 2) + 16 * ((n >> 3) ^ b_swz<MF>(r0)) + 2 * (n & 7);
                const unsigned char *p1 =
                    bs + r1 * (BN * 2) + 16 * ((n >> 3) ^ b_swz<MF>(r1)) + 2 * (n & 7);
                const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p0);
                const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p1);
                const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
                bv[j] = __builtin_bit_cast(bf16x8, u32x4{l2[0], l2[1], h2[0], h2[1]});
            }
#pragma unroll
            for (int i = 0; i < C::FM; ++i)
#pragma unroll
                for (int j = 0; j < C::FN; ++j)
                    acc[i][j] = EDGE ? mfma(bv[j], av[i], acc[i][j]) : mfma(av[i], bv[j], acc[i][j]);
        }
    };

    if constexpr (ST == 2) {
        if (!EDGE || n_kt > 0)
            dma(0, a0, b0);
        wait_dma_all();
        __syncthreads();
        int kt = 0;
        for (; kt + 1 < n_kt; kt += 2) {
            dma(kt + 1, a1, b1);
            compute(a0, b0);
            wait_dma_all();
            __syncthreads();
            if (kt + 2 < n_kt)
                dma(kt + 2, a0, b0);
            compute(a1, b1);
            wait_dma_all();
            __syncthreads();
        }
        if (kt < n_kt)
            compute(a0, b0);
    } else {
        // ring: K step kt lives in stage kt % ST.  Before step kt, wait for
        // its loads (those of the up to ST - 2 later steps already issued
        // may stay in flight), then one barrier: every thread's part of
        // step kt is in LDS and every wave is done with step kt - 1, whose
        // stage takes step kt + ST - 1.
#pragma unroll
        for (int st = 0; st < ST - 1; ++st)
            if (st < n_kt)
                dma(st, abuf[st], bbuf[st]);
        for (int kt = 0; kt < n_kt; ++kt) {
            const int ahead = min(ST - 2, n_kt - 1 - kt);
            if (ahead >= 2)
                wait_dma_upto<2 * C::PER_STAGE>();
            else if (ahead == 1)
                wait_dma_upto<C::PER_STAGE>();
            else
                wait_dma_all();
            __syncthreads();
            const int nx = kt + ST - 1;
            if (nx < n_kt)
                dma(nx, abuf[nx % ST], bbuf[nx % ST]);
            compute(abuf[kt % ST], bbuf[kt % ST]);
        }
    }

    if (EDGE && k_part) {
        __syncthreads();   // every wave is done with the stage buffers
        dma_part(k_part, a0, b0);
        compute(a0, b0);
    }

    if constexpr (KS > 1) {
        // group 0 adds the other groups' sums, one group per round, in
        // group order.  Accumulator block k = i FN + j of the wave in
        // column cw goes, lane-major, to piece k (AR KB) of the wave's
        // FM FN AR KB of the four 16 KB stage buffers, in buffer order.
        constexpr int PB = C::AR * 256;                         // bytes per block
        constexpr int NB = C::FM * C::FN * PB / 16384;          // 16 KB buffers per wave
        auto piece = [&](int k) {
            const int bi = cw * NB + (k * PB) / 16384;
            unsigned char *base = bi == 0 ? abuf[0] : bi == 1 ? abuf[1] : bi == 2 ? bbuf[0] : bbuf[1];
            return (float *)(base + (k * PB) % 16384);
        };
        __syncthreads();   // every wave is done with the stage buffers
#pragma unroll
        for (int g = 1; g < KS; ++g) {
            if (kg == g) {
#pragma unroll
                for (int i = 0; i < C::FM; ++i)
#pragma unroll
                    for (int j = 0; j < C::FN; ++j) {
                        float *p = piece(i * C::FN + j);
#pragma unroll
                        for (int r = 0; r < C::AR; ++r)
                            p[r * 64 + lane] = acc[i][j][r];
                    }
            }
            __syncthreads();
            if (kg == 0) {
#pragma unroll
                for (int i = 0; i < C::FM; ++i)
#pragma unroll
                    for (int j = 0; j < C::FN; ++j) {
                        const float *p = piece(i * C::FN + j);
#pragma unroll
                        for (int r = 0; r < C::AR; ++r)
                            acc[i][j][r] += p[r * 64 + lane];
                    }
            }
            if (g + 1 < KS)
                __syncthreads();   // read before the next group writes
        }
        if (!EDGE && kg != 0)
            return;
    }

    if constexpr (EDGE) {
        // Lane holds row wm + MF i + col, columns wn + MF j + 8 q + 4 half .. + 3 (four
        // such quads of a 32 x 32 block, one of a 16 x 16 block).  The tile goes
        // through LDS, so that all waves, not one group's two or four, store it (1024 x
        // 4096 x 4096 with an activation and a residual: 74 us without, see below), row
        // by row in whole lines, in a loop: the epilogue's code does not fit the
        // instruction cache if it is unrolled for every accumulator.  A wave's sums
        // have a part of the four stage buffers (16 or 32 KB, what its pieces of the
        // groups' sums had); 16-byte chunk c of row r at c ^ (r % chunks of a row).
        constexpr int ROWB = C::WN * 4, CPR = C::WN / 4;          // bytes and chunks of a part's row
        constexpr int BUF = KS == 1 ? C::A_BYTES : 16384;         // bytes of a stage buffer
        constexpr int PART = KS == 1 ? 16384 : C::WM * ROWB;      // bytes of a wave's part
        constexpr int PH = C::WM * ROWB / PART;                   // row blocks in PH phases
        constexpr int FP = C::FM / PH, RPP = FP * MF;             // blocks, rows per phase
        static_assert(C::A_BYTES == C::B_BYTES && C::FM % PH == 0 && BUF % ROWB == 0 &&
                          PART * (KS == 1 ? 8 : C::WPG) <= 4 * BUF && (KS == 1 || PH == 1), "the waves' parts");
        auto at = [&](int w, int r, int c) {                      // chunk c of wave w's row r
            const int o = w * PART + r * ROWB + 16 * (c ^ (r % CPR));
            unsigned char *const base = o / BUF == 0 ? abuf[0] : o / BUF == 1 ? abuf[1] : o / BUF == 2 ? bbuf[0] : bbuf[1];
            return (f32x4 *)(base + o % BUF);
        };
        // KS = 1: a wave stores its own part; otherwise the eight waves take 16 rows
        // of all parts each
        constexpr int CPS = KS == 1 ? CPR : CPR * C::WPG;         // chunks of a row that is stored
        constexpr int U = KS == 2 ? 4 : 8;                        // steps at a time (128 registers in all)
        constexpr int RPI = 64 / CPS;                             // rows per step
        constexpr int RPW = KS == 1 ? RPP : BM / 8;               // rows of a wave
        static_assert(RPW % (U * RPI) == 0, "whole steps");
        const int lr = lane / CPS, lc = lane % CPS;
        const int n = n0 + (KS == 1 ? wn : 0) + 4 * lc, r_first = KS == 1 ? 0 : wave_u * RPW;
        const int m = m0 + (KS == 1 ? wm : r_first) + lr;          // the row of C of the first step
        // What the epilogue adds from memory is loaded U steps ahead of its use (with four
        // at a time, each waited for, a round of 256 x 256 tiles stood 30 us)
        typename Args::template Added<U> now, next;
        if (!SPLIT)
            now.load(a, m, RPI, n);
        if (KS == 1)
            __syncthreads();   // every wave is done with the stage buffers
#pragma unroll
        for (int ph = 0; ph < PH; ++ph) {
            if (KS > 1)
                wave_exchange();   // (the other groups' sums read before their place is written)
            if (kg == 0) {
#pragma unroll
                for (int i = 0; i < FP; ++i)
#pragma unroll
                    for (int j = 0; j < C::FN; ++j)
#pragma unroll
                        for (int q = 0; q < C::AR / 4; ++q) {
                            const auto &x = acc[ph * FP + i][j];
                            *at(KS == 1 ? wave_u : cw, MF * i + col, (MF * j + 8 * q + 4 * half) / 4) =
                                f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                        }
            }
            if (KS > 1)
                __syncthreads();
            else
                wave_exchange();   // (other lanes of this wave wrote what a lane reads)
#pragma unroll 1
            for (int s = 0; s < RPW; s += U * RPI) {
                const int r = r_first + lr + s;
                f32x4 x[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    x[u] = *at(KS == 1 ? wave_u : lc / CPR, r + u * RPI, lc % CPR);
                const int ms = m + ph * RPP + s;
                if (SPLIT) {
                    const int width = a.N - a.n_begin;
                    float *to = (float *)a.C + ((size_t)split * a.M + ms) * width + n - a.n_begin;
#pragma unroll
                    for (int u = 0; u < U; ++u, to += RPI * width)
                        if (ms + u * RPI < a.M && n < a.N)
                            *(f32x4 *)to = x[u];
                } else {
                    if (ph * RPP + s + U * RPI < PH * RPW)
                        next.load(a, ms + U * RPI, RPI, n);
                    a.store(ms, RPI, n, x, now);
                    now = next;
                }
            }
            if (KS == 1 && ph + 1 < PH)
                wave_exchange();   // read before the next phase's writes
        }
        return;
    }

    // epilogue: lane holds column wn + MF j + col, rows wm + MF i +
    // 8(r/4) + 4half + r%4 (MF = 32) or 4half + r (MF = 16) of the tile
    const size_t c0 = SPLIT ? (size_t)split * a.M * a.N : 0;
#pragma unroll
    for (int i = 0; i < C::FM; ++i)
#pragma unroll
        for (int j = 0; j < C::FN; ++j) {
            const int n = n0 + wn + MF * j + col;
#pragma unroll
            for (int r = 0; r < C::AR; ++r) {
                const int m = m0 + wm + MF * i + (MF == 32 ? 8 * (r >> 2) : 0) + 4 * half + (r & 3);
                if (CBF16)
                    ((uint16_t *)a.C)[(size_t)m * a.N + n] =
                        (uint16_t)pack_bf16(acc[i][j][r], 0.f);
                else
                    ((float *)a.C)[c0 + (size_t)m * a.N + n] = acc[i][j][r];
            }
        }
}

}  // namespace tileattn_gemm
