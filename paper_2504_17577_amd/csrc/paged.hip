// Paged key/value cache for gfx950 (MI355X): new tokens' K and V into the
// pages (kv_cache_append), and attention of one new token per sequence over
// them (attn_decode_paged).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "paged_plan.h"
#include "tileattn.h"

namespace {

using namespace tileattn_detail;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
// a token takes chunk i of its 2 Hkv D / 8, K first.  HBM bounds a prefill (16384
// tokens of 8 heads of 128 dims, 134 MB read and written: 30.6 us, 4.4 TB/s of the
// 4.8 that a copy of 4 GiB reaches; with the ordinary cache policy 34), the loads one
// behind the other (seq and pos, the table, then K or V and the scale) less: 32 tokens
// 3 us, 2047 into 8 bits 6.5 us (2.6 at the copy's rate).
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
    const u32x4 x = __builtin_nontemporal_load(
        (const u32x4 *)(is_v ? a.V + t * a.v_stride + 8 * c : a.K + t * a.k_stride + 8 * c));
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
        __builtin_nontemporal_store(x, (u32x4 *)((uint16_t *)to + row * D + 8 * ch));
    }
}

struct PagedArgs {
    const uint16_t *Q;
    int64_t q_stride;
    const void *K, *V;
    const float *ks, *vs;
    const int *table, *lens;
    void *O;
    float *LSE, *W;
    int o_bf16;
    int B, Hq, Hkv, num_pages, page_shift, max_pages;
    int group, rows, blocks;   // Hq / Hkv; of them per workgroup; row blocks of a group
    int parts;                 // 0: a workgroup per (sequence, K/V head, row block)
    float c;                   // scale * log2(e)
};

// Wave-uniform words that the launch only reads, through the scalar cache: their
// loads are counted apart from the vector loads, which return in order (a page
// looked up behind the loads of V would wait for all of them)
typedef const __attribute__((address_space(4))) int scalar_int;

constexpr int NW = PAGED_NW;
constexpr float LN2 = 0.69314718055994530942f;
constexpr float RESCALE_SLACK = 8.f;
constexpr int DPP_ROR8 = 0x128;   // lanes rotated by eight within rows of sixteen

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x over the four lanes l, l ^ 16, l ^ 32, l ^ 48 that hold one row
__device__ __forceinline__ float max_row(float x)
{
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_row(float x)
{
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// two e4m3 numbers (bytes 0, 1, or 2, 3 with HI) as bf16, exactly
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t w)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HI));
}

// the high halves of (lo, hi) as a pair, and the low ones
__device__ __forceinline__ uint32_t high16(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302); }
__device__ __forceinline__ uint32_t low16(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x05040100); }

// Inclusive sums over the wave's lanes, in the vector ALU (rows of sixteen by
// shifts, then the rows' last lanes broadcast)
__device__ __forceinline__ uint32_t wave_scan(uint32_t n)
{
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xF, 0xF, true);    // row_shr:1, 2, 4, 8
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xF, 0xF, true);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xA, 0xF, false);   // row_bcast:15 to rows 1 and 3
    n += __builtin_amdgcn_update_dpp(0, n, 0x143, 0xC, 0xF, false);   // row_bcast:31 to rows 2 and 3
    return n;
}

__device__ __forceinline__ int len_at(const PagedArgs &a, int i) { return i < a.B ? a.lens[i] : 0; }

// The length and tiles of 64 sequences, one a lane, and where their tiles end
// among the batch's: the kernels find their places from the lengths, 64
// sequences at a time.
struct Lengths {
    int len;
    uint32_t tiles, ends;
};

__device__ __forceinline__ Lengths lengths_at(const PagedArgs &a, int cap, int i)
{
    const int len = len_at(a, i);
    const uint32_t n = i < a.B ? paged_tiles(len, cap) : 0;
    return {len, n, wave_scan(n)};
}

// The batch's tiles of one K/V head and row block, from the first 64 sequences'
__device__ __forceinline__ uint32_t all_tiles(const PagedArgs &a, int cap, int lane, const Lengths &first)
{
    uint32_t n = __builtin_amdgcn_readlane(first.ends, 63);
    for (int i0 = 64; i0 < a.B; i0 += 64)
        n += __builtin_amdgcn_readlane(lengths_at(a, cap, i0 + lane).ends, 63);
    return n;
}

// The sequence that tile t lies in, its length, first tile and tiles of a head
// (HR: K/V heads times row blocks)
struct Place {
    uint32_t b;
    int len;
    uint32_t first, per;
};

__device__ __forceinline__ Place place_of(const PagedArgs &a, uint32_t HR, int cap, int lane, Lengths at, uint32_t t)
{
    uint32_t base = 0;
    for (int i0 = 0;; i0 += 64) {
        const uint64_t after = __builtin_amdgcn_ballot_w64((base + at.ends) * HR > t);   // sequences that end past t
        if (after || i0 + 64 >= a.B) {   // (t is one of the tiles: never the second)
            const int l = after ? __builtin_ctzll(after) : 0;
            const uint32_t own = __builtin_amdgcn_readlane(at.tiles, l);
            return {(uint32_t)(i0 + l), (int)__builtin_amdgcn_readlane(at.len, l),
                    (base + __builtin_amdgcn_readlane(at.ends, l) - own) * HR, own};
        }
        base += __builtin_amdgcn_readlane(at.ends, 63);
        at = lengths_at(a, cap, i0 + 64 + lane);
    }
}

// Attention of one new token per sequence.  HBM bounds it: every key and value is
// read once and feeds the few query heads of its group, the columns of
// v_mfma_f32_16x16x32_bf16: S^T = K Q^T, O^T += V^T P^T.
//
//  * K and V go from memory to the registers they are used in, nothing through
//    LDS.  A lane's 16 bytes of a K row (8 dims of one key) are its operand of the
//    scores, after an exchange between two lanes that lets every load take whole
//    lines.  Of V a lane loads the same 8 dims of eight keys, the keys whose
//    weights the scores left in it, and transposes the 8 x 8 block with byte
//    permutes: operand j of O^T is then dims 8 c16 + j of all lanes.
//  * A wave takes 32 keys a step, on its own, with its own running maximum and
//    sums; the next K is loaded under the softmax and the product with V, the
//    next V under the scores: 16 KB in flight a wave (D = 128, bf16), 128 KB a CU
//    with two workgroups on it.  The waves of a workgroup take a quarter of its
//    blocks each and meet in LDS at the end of a head's keys.
//  * The positions of the whole batch, head by head, are one list of tiles of 16
//    keys per wave; each workgroup takes an even share of it (parts), so a batch
//    of mixed lengths occupies the GPU as one of equal ones does, without the host
//    knowing the lengths.  A head counts two tiles more than it has (without, the
//    shares of many short sequences were the longest: 64 sequences of up to 16384
//    mixed, 124 us instead of 88).  Heads that a share's ends cut leave partial
//    results for attn_paged_merge_kernel.
//  * A 16-key block lies in one page (page_size >= 16), so pages are looked up in
//    scalar registers, a step ahead (through the vector loads, behind those of V,
//    the pages of the next K waited for all of V: 106 us became 139 for B=8 Sk=8191
//    with one workgroup a head).
// Measured, kernel without the merge (32 query and 8 K/V heads of 128 dims): B=8
// Sk=8191 43-45 us (6.0-6.3 TB/s), 64 sequences of up to 16384 mixed, in pages of 16,
// 75-78 us (6.0-6.3 TB/s), B=1 Sk=100001 of 8 bits 36 us (5.7 TB/s); of 8 bits and 64
// dims (16 x 32 heads, 2001 positions) 31 us (4.3 TB/s: a wave's 32 keys are a quarter
// of the bytes in flight, and the softmax's work per key is the same).
template <int D, bool E4M3, int RT>
__global__ __launch_bounds__(64 * NW, 2) void attn_paged_kernel(PagedArgs a)
{
    constexpr int KB = 2;                        // 16-key blocks per wave and step
    constexpr int KS = 16 * KB;
    constexpr int KK = D / 32;                   // k-steps of the scores
    constexpr int ROW = D * (E4M3 ? 1 : 2);      // bytes of a key
    constexpr int KL = ROW / 64;                 // 16-byte loads per lane and key block
    constexpr int DJ = D / 16;                   // dims of a value per lane
    constexpr int VW = DJ * (E4M3 ? 1 : 2) / 4;  // dwords of them
    __shared__ __attribute__((aligned(16))) float po[NW][16 * RT][D];
    __shared__ float ml[NW][2][16 * RT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, g = lane >> 4;
    const int cap = a.max_pages << a.page_shift;
    const uint32_t HR = a.Hkv * a.blocks;

    // the tiles of this workgroup: from tile t of head `hr` (K/V head and row
    // block) of sequence b, `left` of them
    uint32_t b, hr, t, left;
    int len;
    if (a.parts) {
        const Lengths some = lengths_at(a, cap, lane);
        const uint32_t n = all_tiles(a, cap, lane, some) * HR;
        const uint32_t used = paged_parts_used(n, a.parts);
        if (blockIdx.x >= used)
            return;
        const uint32_t begin = even_begin(n, used, blockIdx.x);
        left = even_begin(n, used, blockIdx.x + 1) - begin;
        const Place at = place_of(a, HR, cap, lane, some, begin);
        b = at.b;
        len = at.len;
        hr = (begin - at.first) / at.per;
        t = (begin - at.first) % at.per;
    } else {
        b = blockIdx.x / HR;
        hr = blockIdx.x % HR;
        len = ((scalar_int *)(uintptr_t)a.lens)[b];
        t = 0;
        left = ~0u;
    }

    for (;;) {
        const bool bad_len = len < 0 || len > cap;
        const uint32_t per = paged_tiles(len, cap);
        const uint32_t take = min(left, per - t);
        const int h = hr / a.blocks, r0 = (hr % a.blocks) * a.rows;
        const int rows = min(a.rows, a.group - r0);      // query rows of this block
        const size_t row0 = (size_t)b * a.Hq + (size_t)h * a.group + r0;
        const int k_lo = paged_key(t), end = bad_len ? 0 : min(len, paged_key(t + take));
        // this wave's keys: its share of the blocks, as even as they go
        const int nb = max(end - k_lo + 15, 0) >> 4;
        const int first = k_lo + 16 * (nb * wave / NW), k_hi = min(end, k_lo + 16 * (nb * (wave + 1) / NW));
        const int steps = first < k_hi ? (k_hi - first + KS - 1) / KS : 0;
        scalar_int *const table = (scalar_int *)(uintptr_t)(a.table + (size_t)b * a.max_pages);

        // Q as the B operand: row c16, the dims of the lane's K loads (rows past
        // the last read the last; they are never stored)
        bf16x8 q[RT][KK];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const uint16_t *qp = a.Q + b * a.q_stride + (size_t)(h * a.group + r0 + min(16 * i + c16, rows - 1)) * D;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
                q[i][kk] = __builtin_bit_cast(
                    bf16x8, *(const u32x4 *)(qp + (E4M3 ? 64 * (kk >> 1) + 16 * g + 8 * (kk & 1) : 32 * kk + 8 * g)));
        }
        const float c = a.c * (a.ks ? a.ks[h] : 1.f);

        f32x4 acc[RT][DJ];
        float m_run[RT], l_run[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            m_run[i] = -INFINITY;
            l_run[i] = 0.f;
#pragma unroll
            for (int j = 0; j < DJ; ++j)
                acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // the pages of a step's blocks, and where the head's rows of the blocks are,
        // in bytes from the cache's start; a block past the last key is the last one
        const int last_block = (k_hi - 1) >> 4;
        int page[KB];
        auto lookup = [&](int s) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                page[kb] = table[min(((first + s * KS) >> 4) + kb, last_block) >> (a.page_shift - 4)];
        };
        size_t at[KB];
        bool bad[KB], next_bad[KB];
        auto place = [&](int s) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const int pg = paged_checked(page[kb], a.num_pages);
                const int blk = min(((first + s * KS) >> 4) + kb, last_block);
                const int in = (blk << 4) & ((1 << a.page_shift) - 1);
                at[kb] = ((((size_t)max(pg, 0) * a.Hkv + h) << a.page_shift) + in) * ROW;
                next_bad[kb] = pg < 0;
            }
        };
        u32x4 kr[KB][KL];
        uint32_t vr[KB][4][VW];
        auto load_k = [&]() {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const unsigned char *p = (const unsigned char *)a.K + at[kb];
                if constexpr (KL == 1) {
                    kr[kb][0] = __builtin_nontemporal_load((const u32x4 *)(p + (uint32_t)(c16 * ROW + 16 * g)));
                } else {
#pragma unroll
                    for (int i = 0; i < KL; ++i)   // row 8 (i & 1) + c16 % 8, 16-byte chunk g + 4 (c16 / 8) of line i / 2
                        kr[kb][i] = __builtin_nontemporal_load((const u32x4 *)(
                            p + (uint32_t)((8 * (i & 1) + (c16 & 7)) * ROW + 128 * (i >> 1) + 64 * (c16 >> 3) + 16 * g)));
                }
            }
        };
        auto load_v = [&]() {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const unsigned char *p = (const unsigned char *)a.V + at[kb];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned char *e = p + (uint32_t)((4 * g + i) * ROW + c16 * (4 * VW));
                    if constexpr (VW == 4) {
                        const u32x4 x = __builtin_nontemporal_load((const u32x4 *)e);
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            vr[kb][i][w] = x[w];
                    } else if constexpr (VW == 2) {
                        const u32x2 x = __builtin_nontemporal_load((const u32x2 *)e);
                        vr[kb][i][0] = x[0];
                        vr[kb][i][1] = x[1];
                    } else {
                        vr[kb][i][0] = __builtin_nontemporal_load((const uint32_t *)e);
                    }
                }
            }
        };

        if (steps > 0) {
            lookup(0);
            place(0);
            load_k();
            load_v();
            if (steps > 1)
                lookup(1);
        }
        for (int s = 0; s < steps; ++s) {
            const int key0 = first + s * KS;
            const bool tail = key0 + KS > k_hi;      // uniform
            // The K loads took whole lines of eight rows each (halves of sixteen rows'
            // lines would come from HBM twice); lanes c16 and c16 ^ 8 exchange what the
            // other's row needs: then lane c16 holds chunks 8 l + g and 8 l + 4 + g of row c16
            if constexpr (KL > 1) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < KL; i += 2)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const int x = kr[kb][i][w], y = kr[kb][i + 1][w];
                            kr[kb][i][w] = __builtin_amdgcn_update_dpp(x, y, DPP_ROR8, 0xF, 0xC, false);
                            kr[kb][i + 1][w] = __builtin_amdgcn_update_dpp(y, x, DPP_ROR8, 0xF, 0x3, false);
                        }
            }
            // scores: lane holds keys 16 kb + 4 g + r of row c16
            f32x4 sc[RT][KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    sc[i][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < KK; ++kk) {
                        bf16x8 k;
                        if constexpr (E4M3) {
                            const uint32_t w0 = kr[kb][kk >> 1][2 * (kk & 1)], w1 = kr[kb][kk >> 1][2 * (kk & 1) + 1];
                            k = __builtin_bit_cast(bf16x8, u32x4{e4m3_bf16<false>(w0), e4m3_bf16<true>(w0),
                                                                 e4m3_bf16<false>(w1), e4m3_bf16<true>(w1)});
                        } else {
                            k = __builtin_bit_cast(bf16x8, kr[kb][kk]);
                        }
                        sc[i][kb] = mfma(k, q[i][kk], sc[i][kb]);
                    }
                }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                bad[kb] = next_bad[kb];
            if (s + 1 < steps) {
                place(s + 1);
                load_k();
                if (s + 2 < steps)
                    lookup(s + 2);
            }
            // a page outside the pool makes its keys' scores NaN, and so the row
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                if (bad[kb])
#pragma unroll
                    for (int i = 0; i < RT; ++i)
                        sc[i][kb] = f32x4{NAN, NAN, NAN, NAN};

            // V as the A operand of O^T: k-slot of lane group g <-> keys 32 kp + 4 g
            // + (0..3) and 32 kp + 16 + 4 g + (0..3), as the scores left the weights
            if (tail) {   // what lies behind the last key may be anything
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int w = 0; w < VW; ++w)
                            vr[kb][i][w] = key0 + 16 * kb + 4 * g + i < k_hi ? vr[kb][i][w] : 0u;
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float mx = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (tail)
                            sc[i][kb][r] = key0 + 16 * kb + 4 * g + r < k_hi ? sc[i][kb][r] : -INFINITY;
                        mx = fmaxf(mx, sc[i][kb][r]);
                    }
                mx = max_row(mx);
                const float m_step = mx == -INFINITY ? -INFINITY : mx * c;
                if (__builtin_amdgcn_ballot_w64(m_step > m_run[i] + RESCALE_SLACK)) {
                    const float m_new = fmaxf(m_run[i], m_step);
                    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[i] - m_new);
                    m_run[i] = m_new;
                    l_run[i] *= alpha;
#pragma unroll
                    for (int j = 0; j < DJ; ++j)
                        acc[i][j] *= alpha;
                }
                const float m_use = m_run[i] == -INFINITY ? 0.f : m_run[i];
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][kb][r], c, -m_use));
                        if (tail)   // (scale 0 makes a masked score NaN, not -inf)
                            p = key0 + 16 * kb + 4 * g + r < k_hi ? p : 0.f;
                        sc[i][kb][r] = p;
                        l_run[i] += p;
                    }
            }
#pragma unroll
            for (int kp = 0; kp < KB / 2; ++kp) {
                // The weights as three bf16 numbers that add up to all their 24 bits: with
                // two, cut off, a bf16 O was not the nearest number to the exact one in 215
                // of 32768 places (B=8 Sk=8191), with three it is not in 8.  The loads leave
                // the matrix cores the time: 49 us with two and with three, 8 sequences of
                // 8000 with 32 query heads to a K/V head 26.8 and 27.4
                bf16x8 p[RT][3];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    uint32_t w[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        w[r] = __float_as_uint(sc[i][2 * kp + (r >> 2)][r & 3]);
#pragma unroll
                    for (int n = 0; n < 3; ++n) {
                        p[i][n] = __builtin_bit_cast(bf16x8, u32x4{high16(w[0], w[1]), high16(w[2], w[3]),
                                                                   high16(w[4], w[5]), high16(w[6], w[7])});
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            w[r] = __float_as_uint(__uint_as_float(w[r]) - __uint_as_float(w[r] & 0xFFFF0000u));
                    }
                }
#pragma unroll
                for (int j = 0; j < DJ; j += 2) {
                    uint32_t x0[4], x1[4];   // dims j and j + 1, keys in pairs
#pragma unroll
                    for (int pr = 0; pr < 4; ++pr) {
                        const auto &e = vr[2 * kp + (pr >> 1)][2 * (pr & 1)], &o = vr[2 * kp + (pr >> 1)][2 * (pr & 1) + 1];
                        if constexpr (E4M3) {
                            // bytes j, j + 1 of both keys, paired by dim, then as bf16
                            const uint32_t w = __builtin_amdgcn_perm(o[j >> 2], e[j >> 2], j & 2 ? 0x07030602 : 0x05010400);
                            x0[pr] = e4m3_bf16<false>(w);
                            x1[pr] = e4m3_bf16<true>(w);
                        } else {
                            x0[pr] = low16(e[j >> 1], o[j >> 1]);
                            x1[pr] = high16(e[j >> 1], o[j >> 1]);
                        }
                    }
                    const bf16x8 v0 = __builtin_bit_cast(bf16x8, u32x4{x0[0], x0[1], x0[2], x0[3]});
                    const bf16x8 v1 = __builtin_bit_cast(bf16x8, u32x4{x1[0], x1[1], x1[2], x1[3]});
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int n = 0; n < 3; ++n) {
                            acc[i][j] = mfma(v0, p[i][n], acc[i][j]);
                            acc[i][j + 1] = mfma(v1, p[i][n], acc[i][j + 1]);
                        }
                }
            }
            if (s + 1 < steps)
                load_v();
        }

        // The waves' sums meet in LDS, in wave order.  Lane: row c16, dims
        // DJ (4 g + r) + j; 16-byte chunk ch of row x at ch ^ x.
        __syncthreads();   // (the head before this one has been read)
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const float l = sum_row(l_run[i]);
            const int x = 16 * i + c16;
            if (x < rows) {
                if (g == 0) {
                    ml[wave][0][x] = m_run[i];
                    ml[wave][1][x] = l;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < DJ; j += 4)
                        *(f32x4 *)&po[wave][x][4 * (((DJ * (4 * g + r) + j) / 4) ^ c16)] =
                            f32x4{acc[i][j][r], acc[i][j + 1][r], acc[i][j + 2][r], acc[i][j + 3][r]};
            }
        }
        __syncthreads();
        const bool begins = t == 0, ends = t + take == per;
        float *const rec = begins && ends ? nullptr : a.W + (2 * (size_t)blockIdx.x + begins) * paged_record(a.rows, D);
        const float vs = a.vs ? a.vs[h] : 1.f;
        for (int e = tid; e < rows * (D / 4); e += 64 * NW) {
            const int x = e / (D / 4), ch = e % (D / 4);
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                m = fmaxf(m, ml[w][0][x]);
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = ml[w][0][x];
                const float f = mw == m ? 1.f : __builtin_amdgcn_exp2f(mw - m);
                l += f * ml[w][1][x];
                o += f * *(const f32x4 *)&po[w][x][4 * (ch ^ (x & 15))];
            }
            if (rec) {
                *(f32x4 *)(rec + (size_t)x * D + 4 * ch) = o;
                if (ch == 0) {
                    rec[((size_t)(a.rows + 3) & ~3) * D + x] = m;
                    rec[((size_t)(a.rows + 3) & ~3) * (D + 1) + x] = l;
                }
            } else {
                o *= bad_len ? NAN : len == 0 ? 0.f : vs / l;   // (every score -inf: 0 / 0)
                const size_t at = (row0 + x) * D + 4 * ch;
                if (a.o_bf16)
                    *(u32x2 *)((uint16_t *)a.O + at) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
                else
                    *(f32x4 *)((float *)a.O + at) = o;
                if (ch == 0)
                    a.LSE[row0 + x] = bad_len ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
            }
        }

        left -= take;
        if (!a.parts || left == 0)
            return;
        t = 0;
        if (++hr == HR) {
            hr = 0;
            len = ((scalar_int *)(uintptr_t)a.lens)[++b];
        }
    }
}

// Joins the partial results of the heads that were cut: a workgroup per m_rows
// query rows of a (sequence, K/V head, row block), several threads per 16 bytes
// of them that take every n-th record each, U at a time, and meet in LDS.  It is
// a chain of latencies (4.5 to 6 us), so rows get workgroups of their own while
// there are few.
constexpr int MERGE_T = 512;
template <int D>
__global__ __launch_bounds__(MERGE_T) void attn_paged_merge_kernel(PagedArgs a, int m_rows)
{
    __shared__ __attribute__((aligned(16))) float so[MERGE_T][4];
    __shared__ float sm[MERGE_T], sl[MERGE_T];
    const int tid = threadIdx.x, lane = tid & 63;
    const int cap = a.max_pages << a.page_shift;
    const uint32_t HR = a.Hkv * a.blocks, subs = (a.rows + m_rows - 1) / m_rows;
    const uint32_t b = blockIdx.x / subs / HR, hr = blockIdx.x / subs % HR;
    uint32_t n = 0, before = 0;   // tiles of the batch, and of the sequences before b
    int len = 0;
    for (int i0 = 0; i0 < a.B; i0 += 64) {
        const Lengths some = lengths_at(a, cap, i0 + lane);
        if (b / 64 == (uint32_t)i0 / 64) {
            len = __builtin_amdgcn_readlane(some.len, b % 64);
            before = n + __builtin_amdgcn_readlane(some.ends - some.tiles, b % 64);
        }
        n += __builtin_amdgcn_readlane(some.ends, 63);
    }
    n *= HR;
    const bool bad_len = len < 0 || len > cap;
    const uint32_t per = paged_tiles(len, cap);
    const uint32_t t0 = before * HR + hr * per;
    const uint32_t used = paged_parts_used(n, a.parts);
    const uint32_t p0 = even_part_of(n, used, t0), p1 = even_part_of(n, used, t0 + per - 1);
    if (p0 == p1)
        return;   // a head that one workgroup took whole
    const int h = hr / a.blocks, r0 = (hr % a.blocks) * a.rows;
    const int x0 = blockIdx.x % subs * m_rows;   // the first of these rows in the block
    const int rows = min(m_rows, min(a.rows, a.group - r0) - x0);
    if (rows <= 0)
        return;
    const size_t row0 = (size_t)b * a.Hq + (size_t)h * a.group + r0;
    const size_t pad = (size_t)(a.rows + 3) & ~3, rec = paged_record(a.rows, D);
    const float vs = a.vs ? a.vs[h] : 1.f;

    const int items = rows * (D / 4);            // 16-byte chunks of the head's rows
    // threads per group of records: a power of two of them work on one chunk
    int per_item = 1;
    while (per_item < 16 && items * per_item * 2 <= (int)blockDim.x)
        per_item *= 2;
    const int width = blockDim.x / per_item;        // chunks at a time
    const int k = tid / width;
    for (int e0 = 0; e0 < items; e0 += width) {
        const int e = e0 + tid % width;
        const int x = x0 + min(e, items - 1) / (D / 4), ch = min(e, items - 1) % (D / 4);
        float m = -INFINITY, l = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        constexpr int U = 8;                     // records in flight
        for (uint32_t p = p0 + k; p <= p1; p += U * per_item) {
            float mp[U], lp[U];
            f32x4 op[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t pu = min(p + u * per_item, p1);
                const float *r = a.W + (2 * (size_t)pu + (pu == p0)) * rec;
                op[u] = *(const f32x4 *)(r + (size_t)x * D + 4 * ch);
                mp[u] = r[pad * D + x];
                lp[u] = r[pad * (D + 1) + x];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p + u * per_item > p1)
                    break;
                const float mn = fmaxf(m, mp[u]);
                const float f0 = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                const float f1 = mp[u] == mn ? 1.f : __builtin_amdgcn_exp2f(mp[u] - mn);
                m = mn;
                l = l * f0 + lp[u] * f1;
                o = o * f0 + op[u] * f1;
            }
        }
        __syncthreads();
        *(f32x4 *)so[tid] = o;
        sm[tid] = m;
        sl[tid] = l;
        __syncthreads();
        if (k == 0 && e < items) {
            for (int i = 1; i < per_item; ++i) {
                const int s = tid + i * width;
                const float mn = fmaxf(m, sm[s]);
                const float f0 = m == mn ? 1.f : __builtin_amdgcn_exp2f(m - mn);
                const float f1 = sm[s] == mn ? 1.f : __builtin_amdgcn_exp2f(sm[s] - mn);
                m = mn;
                l = l * f0 + sl[s] * f1;
                o = o * f0 + *(const f32x4 *)so[s] * f1;
            }
            o *= bad_len ? NAN : len == 0 ? 0.f : vs / l;
            const size_t at = (row0 + x) * D + 4 * ch;
            if (a.o_bf16)
                *(u32x2 *)((uint16_t *)a.O + at) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
            else
                *(f32x4 *)((float *)a.O + at) = o;
            if (ch == 0)
                a.LSE[row0 + x] = bad_len ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        }
    }
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

bool heads_ok(int B, int Hq, int Hkv)
{
    return B >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && Hq <= 1 << 16 && (int64_t)B * Hq < 1ll << 24;
}

size_t workspace_need(int group, int D, int num_parts)
{
    return (size_t)num_parts * 2 * paged_record(paged_block_rows(group), D) * 4;
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
                            int num_parts, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!Q || !K_cache || !V_cache || !page_table || !seq_lens || !O || !LSE)
        return TA_ERR_NULL_POINTER;
    const ta_status rc = check_cache(B, Hkv, D, num_pages, page_size, max_pages, cache_e4m3, k_scale, v_scale);
    if (rc != TA_OK)
        return rc;
    const int64_t row = (int64_t)Hq * D;
    if (!heads_ok(B, Hq, Hkv) || q_stride < row || q_stride % 8 || q_stride > 1ll << 30 || num_parts < 0 ||
        num_parts > PAGED_MAX_PARTS)
        return TA_ERR_INVALID_SHAPE;
    const int group = Hq / Hkv, blocks = paged_row_blocks(group);
    if (((int64_t)max_pages * page_size / PAGED_TILE + 1 + PAGED_HEAD) * B * Hkv * blocks >= 1ll << 31)   // tiles in 32 bits
        return TA_ERR_INVALID_SHAPE;
    if (misaligned(Q) || misaligned(K_cache) || misaligned(V_cache) || misaligned(O) || misaligned(LSE) ||
        misaligned(page_table, 4) || misaligned(seq_lens, 4) || misaligned(k_scale, 4) || misaligned(v_scale, 4))
        return TA_ERR_MISALIGNED;
    if (!(scale >= 0.f) || !(scale <= 3.402823466e+38f))
        return TA_ERR_INVALID_SCALE;
    const size_t cb = cache_bytes(Hkv, D, num_pages, page_size, cache_e4m3);
    const size_t need = workspace_need(group, D, num_parts);
    const Span o = {O, (size_t)B * row * (o_bf16 ? 2 : 4)}, l = {LSE, (size_t)B * Hq * 4};
    const Span w = {need ? workspace : nullptr, need};
    const Span in[] = {{Q, (size_t)((B - 1) * q_stride + row) * 2}, {K_cache, cb}, {V_cache, cb},
                       {page_table, (size_t)B * max_pages * 4}, {seq_lens, (size_t)B * 4},
                       {k_scale, (size_t)Hkv * 4}, {v_scale, (size_t)Hkv * 4}};
    if (overlaps(o, l))
        return TA_ERR_ALIASING;
    for (const Span &s : in)
        if (overlaps(o, s) || overlaps(l, s))
            return TA_ERR_ALIASING;
    if (need) {
        if (!workspace || workspace_bytes < need)
            return TA_ERR_WORKSPACE;
        if (misaligned(workspace))
            return TA_ERR_MISALIGNED;
        if (overlaps(w, o) || overlaps(w, l))
            return TA_ERR_ALIASING;
        for (const Span &s : in)
            if (overlaps(w, s))
                return TA_ERR_ALIASING;
    }
    const PagedArgs a = {(const uint16_t *)Q, q_stride, K_cache, V_cache, k_scale, v_scale, page_table, seq_lens, O,
                         LSE, (float *)workspace, o_bf16 != 0, B, Hq, Hkv, num_pages, __builtin_ctz(page_size),
                         max_pages, group, paged_block_rows(group), blocks, num_parts, scale * 1.44269504088896340736f};
    const dim3 grid((unsigned)(num_parts ? num_parts : B * Hkv * blocks)), block(64 * NW);
    hipStream_t s = (hipStream_t)stream;
    const bool two = a.rows > 16;
    const auto kernel =
        D == 64 ? (cache_e4m3 ? (two ? attn_paged_kernel<64, true, 2> : attn_paged_kernel<64, true, 1>)
                              : (two ? attn_paged_kernel<64, false, 2> : attn_paged_kernel<64, false, 1>))
                : (cache_e4m3 ? (two ? attn_paged_kernel<128, true, 2> : attn_paged_kernel<128, true, 1>)
                              : (two ? attn_paged_kernel<128, false, 2> : attn_paged_kernel<128, false, 1>));
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && num_parts) {
        const auto merge = D == 64 ? attn_paged_merge_kernel<64> : attn_paged_merge_kernel<128>;
        const int m_rows = min(a.rows, max(1, B * Hq / 512)), subs = (a.rows + m_rows - 1) / m_rows;
        hipLaunchKernelGGL(merge, dim3((unsigned)(B * Hkv * blocks * subs)),
                           dim3(B * Hq <= 128 ? MERGE_T : MERGE_T / 2), 0, s, a, m_rows);
        e = hipGetLastError();
    }
    return e == hipSuccess ? TA_OK : TA_ERR_LAUNCH;
}

ta_status attn_paged_workspace_bytes(int Hq, int Hkv, int D, int num_parts, size_t *bytes)
{
    if (!bytes)
        return TA_ERR_NULL_POINTER;
    if (!heads_ok(1, Hq, Hkv) || D < 1 || num_parts < 0 || num_parts > PAGED_MAX_PARTS)
        return TA_ERR_INVALID_SHAPE;
    if (D != 64 && D != 128)
        return TA_ERR_UNSUPPORTED;
    *bytes = workspace_need(Hq / Hkv, D, num_parts);
    return TA_OK;
}

ta_status attn_paged_plan(int B, int Hq, int Hkv, int D, int page_size, int max_pages, int *num_parts)
{
    if (!num_parts)
        return TA_ERR_NULL_POINTER;
    if (!heads_ok(B, Hq, Hkv) || D < 1 || page_size < 1 || max_pages < 1)
        return TA_ERR_INVALID_SHAPE;
    if (D != 64 && D != 128)
        return TA_ERR_UNSUPPORTED;
    // Two workgroups per CU share the batch, unless the longest sequence the table
    // has room for is short enough for one workgroup a head, which needs no second
    // kernel.  us on the GPU, one a head | 512 parts (bf16, 128 dims, 32 query and 8
    // K/V heads; the second launch costs the host 4 us besides):
    //   keys   300       500       640       768       900       1024
    //   B=1    7.2|10.5  9.5|10.0  11.4|10.2 12.9|10.3 15.7|10.6 16.0|10.6
    //   B=4    8.6|11.3  10.4|10.7 11.9|10.8 13.5|10.9 16.3|12.8 16.7|12.8
    //   B=32   10.7|16.1 14.1|20.4 16.4|21.4 19.1|25.0 22.7|27.5 24.6|30.1
    //   mixed to 500, 768 and 1000: B=64 12.3|16.3, 18.3|16.9, 19.8|18.7; B=128
    //   19.8|23.9, 24.0|25.0, 28.5|27.0
    // Where heads are many for the longest sequence's length, its workgroup alone is
    // not what the call waits for, and no share stops at each of many short heads.
    // Sequences and K/V heads, mixed to `cap` (64 dims with 32 heads, 128 with 8):
    //   heads >= 2 cap: 64 x 32 to 1024 22.9|33.1, 128 x 32 to 2048 60.5|79.1, 256 x 32 to
    //   4096 194|199, 256 x 8 to 1024 44.3|46.2, 512 x 8 to 2048 116|123
    //   = cap: 64 x 32 to 2048 41.9|41.2, 128 x 32 to 4096 116|117, 256 x 8 to 2048 70|62
    //   = cap / 2: 64 x 32 to 4096 72.9|58.4, 128 x 8 to 2048 56.4|36.6
    const int64_t cap = (int64_t)max_pages * page_size;
    const int64_t heads = (int64_t)B * Hkv * paged_row_blocks(Hq / Hkv);
    *num_parts = cap <= 768 || (cap <= 1024 && heads >= 1024) || heads >= 2 * cap ? 0 : 512;
    return TA_OK;
}

}  // extern "C"
