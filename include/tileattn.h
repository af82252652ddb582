/*
 * tileattn — fused scaled-dot-product attention forward for AMD MI355X
 * (gfx950), as a C ABI.
 *
 * The operation is the tile-fused attention kernel of the TileLang paper
 * (arXiv 2504.17577): scores S = scale * Q K^T, a softmax over keys computed
 * online over key tiles (running row max, rescale of the partial sums by the
 * exponential of the max difference, running row sum, final division), and
 * O = softmax(S) V, without ever storing S in memory.  The paper prints this
 * recurrence in its appendix listing "Implementation of FlashMLA with
 * TileLang" and benchmarks the multi-head forward in its FlashAttention
 * experiment (Section "Numerical Experiments", table "FlashAttention shapes
 * in our benchmark": batch, heads, sequence length, head dim 128, causal).
 *
 * Conventions for every entry point below:
 *   - Layouts are contiguous row-major BHSD: Q and O are [B, Hq, Sq, D],
 *     K and V are [B, Hkv, Sk, D], LSE is [B, Hq, Sq].  There are no stride
 *     arguments.
 *   - The caller owns every buffer.  The library allocates nothing, frees
 *     nothing and keeps no state between calls; calls are thread-safe.
 *   - Calls are asynchronous: they validate, enqueue on `stream` and return.
 *     `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *   - All validation happens before any HIP call: a status other than TA_OK
 *     means nothing was enqueued and no HIP API was touched (except for
 *     TA_ERR_LAUNCH, reported by the HIP runtime after the launch).
 *   - O and LSE are fully overwritten, never accumulated into.
 */
#ifndef TILEATTN_H
#define TILEATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TA_OK = 0,
    TA_ERR_NULL_POINTER = 1,  /* a required pointer is NULL                                 */
    TA_ERR_INVALID_SHAPE = 2, /* a size < 1, Hq % Hkv != 0, causal with Sq > Sk, or an
                                 element count beyond 2^31 per (batch, head) slice         */
    TA_ERR_UNSUPPORTED = 3,   /* D is not 64 or 128, or another value that is not offered   */
    TA_ERR_MISALIGNED = 4,    /* a pointer is not 16-byte aligned                           */
    TA_ERR_INVALID_SCALE = 5, /* scale is negative, NaN or infinite                         */
    TA_ERR_ALIASING = 6,      /* O or LSE overlaps an input or each other                   */
    TA_ERR_LAUNCH = 7,        /* the HIP runtime reported an error for the launch           */
    TA_ERR_WORKSPACE = 8,     /* attn_fwd_split: workspace NULL or smaller than required    */
    TA_ERR_SCRATCH = 9        /* attn_fwd_split_noalloc: partial results larger than
                                 TA_SPLIT_SCRATCH_BYTES                                    */
} ta_status;

/*
 * attn_fwd — O = softmax(scale * Q K^T [+ causal mask]) V and its row
 * log-sum-exp, for bf16 inputs with fp32 accumulation.
 *
 *   Q    device, bf16 [B, Hq, Sq, D]           read only
 *   K    device, bf16 [B, Hkv, Sk, D]          read only
 *   V    device, bf16 [B, Hkv, Sk, D]          read only
 *   O    device, fp32 [B, Hq, Sq, D]           written
 *   LSE  device, fp32 [B, Hq, Sq]              written: natural log of
 *        sum_j exp(scale * q_i . k_j) over the keys row i may see
 *   Hq % Hkv == 0; query head h reads key/value head h / (Hq / Hkv)
 *   causal != 0: key j is visible to query i iff j <= i + (Sk - Sq)
 *        (bottom-right alignment; requires Sq <= Sk so every row sees a key)
 *   scale >= 0, finite; the kernel works in base 2 internally
 *   D in {64, 128}; every pointer 16-byte aligned
 *   stream: hipStream_t as void*
 *
 * The scores are formed in fp32 from bf16 products; the softmax weights are
 * rounded to bf16 (round to nearest even) before the P V product.
 */
ta_status attn_fwd(const void *Q, const void *K, const void *V, float *O, float *LSE,
                   int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal, float scale,
                   void *stream);

/*
 * attn_fwd_bf16out — attn_fwd with O written in bf16 instead of fp32.
 *
 *   O    device, bf16 [B, Hq, Sq, D]           written: each element is the
 *        fp32 value attn_fwd would store, rounded to nearest even
 *   every other argument, the validation and the status codes as attn_fwd;
 *   the aliasing check uses the bf16 size of O
 *
 * For callers that keep activations in bf16 (the usual next consumer of an
 * attention output is a bf16 projection); halves the output traffic.
 */
ta_status attn_fwd_bf16out(const void *Q, const void *K, const void *V, void *O, float *LSE,
                           int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal,
                           float scale, void *stream);

/*
 * attn_fwd_split — attn_fwd with the key range of every query tile split
 * over `num_splits` workgroups, for grids too small to fill the GPU (few
 * heads, short query blocks against long key sequences).
 *
 * Each split computes the softmax result of its rows over its own keys,
 * (O_s, LSE_s), into the workspace; a second kernel merges them exactly:
 * LSE = log sum_s exp(LSE_s) and O = sum_s exp(LSE_s - LSE) O_s.  This is the
 * same rescaling the online softmax applies between key tiles, applied
 * between splits.  Results agree with attn_fwd to within fp32 rounding.
 *
 *   O          device, [B, Hq, Sq, D]: fp32, or bf16 if o_bf16 != 0
 *   num_splits 1..128 requested; splits are whole key tiles, so at most
 *              ceil(Sk / BN) are launched; 1 runs attn_fwd / attn_fwd_bf16out
 *              and ignores the workspace
 *   workspace  device, 16-byte aligned, at least the size
 *              ta_split_workspace_bytes reports (owned by the caller, which
 *              may reuse it once the call's work on `stream` has finished;
 *              its contents on entry do not matter); must not overlap any
 *              other argument (TA_ERR_ALIASING)
 *   other arguments, validation and status codes as attn_fwd;
 *   TA_ERR_WORKSPACE if num_splits > 1 and workspace is NULL or too small
 */
ta_status attn_fwd_split(const void *Q, const void *K, const void *V, void *O, int o_bf16,
                         float *LSE, int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal,
                         float scale, int num_splits, void *workspace, size_t workspace_bytes,
                         void *stream);

/*
 * attn_fwd_split_noalloc — attn_fwd_split for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, and
 * harnesses that forbid hipMalloc.  The per-split partial results go to a
 * static device array inside the library (TA_SPLIT_SCRATCH_BYTES per GPU,
 * allocated when the library's code is loaded on that GPU and held until the
 * process ends) instead of a caller workspace; the call itself allocates and
 * frees nothing.
 *
 *   arguments, results and status codes as attn_fwd_split without the
 *   workspace; TA_ERR_SCRATCH (before any HIP call) if the partial results,
 *   num_splits' * B*Hq*Sq * (D + 1) * 4 bytes for the num_splits' splits
 *   actually launched, exceed TA_SPLIT_SCRATCH_BYTES; num_splits == 1 runs
 *   attn_fwd / attn_fwd_bf16out and touches no scratch.
 *   TA_ERR_LAUNCH also if the runtime cannot report the current device or
 *   the scratch's address on it (looked up once per device, on the first
 *   call there, with that device current).
 *
 * Every call on one GPU uses that GPU's one scratch array: calls whose work
 * overlaps on one GPU (different streams, or different host threads without
 * ordering) race on it and give wrong results.  Calls ordered on one stream
 * are safe.  The scratch keeps the last call's contents; nothing in it needs
 * clearing, since every launched split writes all of its partial rows before
 * the merge reads them.
 */
#define TA_SPLIT_SCRATCH_BYTES (64ull << 20)
ta_status attn_fwd_split_noalloc(const void *Q, const void *K, const void *V, void *O,
                                 int o_bf16, float *LSE, int B, int Hq, int Hkv, int Sq, int Sk,
                                 int D, int causal, float scale, int num_splits, void *stream);

/* Workspace bytes attn_fwd_split needs: num_splits * B*Hq*Sq * (D + 1) * 4
 * for num_splits > 1 (fp32 partial O and LSE per split), 0 for 1.
 * TA_ERR_INVALID_SHAPE / TA_ERR_UNSUPPORTED / TA_ERR_NULL_POINTER as above.
 * No HIP call. */
ta_status ta_split_workspace_bytes(int B, int Hq, int Sq, int D, int num_splits,
                                   size_t *bytes);

/* A split count for attn_fwd_split: 1 when B*Hq*ceil(Sq/BM) workgroups
 * already give two per CU (512), else enough splits to reach that, keeping
 * at least 32 key tiles (2048 keys) per split: shorter splits lose more to
 * the merge kernel's launch and traffic than the extra workgroups win.
 * No HIP call. */
ta_status ta_split_heuristic(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal,
                             int *num_splits);

/* A split count for attn_fwd_split callers that size the workspace after it:
 * as ta_split_heuristic, but with at most 16 query rows per key/value head
 * (Hq / Hkv * Sq <= 16: a decode step) enough splits for one workgroup per
 * (batch, key/value head, split) on each of 256 CUs, and where those are more
 * than 256 already up to four if they even out the rounds, keeping at least 512
 * keys per split.  No HIP call. */
ta_status ta_split_plan(int B, int Hq, int Hkv, int Sq, int Sk, int D, int causal,
                        int *num_splits);

/* Which kernel the attention entry points run for a call of num_splits splits
 * (1 for attn_fwd and attn_fwd_bf16out), for tests and tools: *decode = 1 for
 * the decode kernel, whose workgroups take all query rows of a key/value head
 * (at most 16), 0 for the tiled one, also for short keys in large grids of one
 * or two query heads per key/value head, where it is the faster one.  No HIP
 * call. */
ta_status ta_decode_route(int B, int Hq, int Hkv, int Sq, int Sk, int D, int num_splits,
                          int *decode);

/*
 * mla_decode — multi-head latent attention, one decode step: the
 * computation of the paper's appendix listing "Implementation of FlashMLA
 * with TileLang".  For batch b and query head h, with latent head
 * hk = h / (H / Hkv), over all Skv cache positions t:
 *   s_t = scale * (Q[b,h,:] . KV[b,t,hk,:] + Q_pe[b,h,:] . K_pe[b,t,hk,:])
 *   O[b,h,:] = sum_t softmax(s)_t KV[b,t,hk,:]      (the latent cache is the value)
 *   LSE[b,h] = ln sum_t exp(s_t)
 *
 *   Q     device, bf16 [B, H, Dl]             read only
 *   Q_pe  device, bf16 [B, H, Dr]             read only
 *   KV    device, bf16 [B, Skv, Hkv, Dl]      read only (the listing's layout)
 *   K_pe  device, bf16 [B, Skv, Hkv, Dr]      read only
 *   O     device, fp32 [B, H, Dl]             written
 *   LSE   device, fp32 [B, H]                 written (natural log, scale included)
 *   Dl == 512 and Dr == 64 (else TA_ERR_UNSUPPORTED); H % Hkv == 0
 *   num_splits: 1..128 requested splits of the cache positions (whole tiles
 *   of 32; trailing empty splits are dropped); for more than one, the
 *   per-split results go to `workspace` (device, 16-byte aligned, at least
 *   mla_workspace_bytes(B, H, num_splits) bytes, owned by the caller, no
 *   overlap with any other argument) and a second kernel merges them;
 *   num_splits == 1 ignores the workspace
 *   scale >= 0, finite; every pointer 16-byte aligned; stream as attn_fwd
 * Status codes as attn_fwd (TA_ERR_WORKSPACE for a missing or small
 * workspace).  Scores and sums are fp32, the softmax weights bf16 for the
 * weighted sum of the latent rows.
 */
ta_status mla_decode(const void *Q, const void *Q_pe, const void *KV, const void *K_pe,
                     float *O, float *LSE, int B, int H, int Hkv, int Skv, int Dl, int Dr,
                     float scale, int num_splits, void *workspace, size_t workspace_bytes,
                     void *stream);

/* Workspace bytes mla_decode needs: num_splits * B*H * (Dl + 1) * 4 with
 * Dl = 512 for num_splits > 1, 0 for 1.  No HIP call. */
ta_status mla_workspace_bytes(int B, int H, int num_splits, size_t *bytes);

/* A split count for mla_decode: enough splits of the cache for one
 * workgroup per CU (a workgroup covers up to 128 query heads of one latent
 * head and fills its CU's registers), keeping at least 8 tiles (256 positions) per
 * split.  No HIP call. */
ta_status mla_split_heuristic(int B, int H, int Hkv, int Skv, int *num_splits);

/* A split count for mla_decode callers that size the workspace after it: the
 * one with the smallest time by an estimate that counts the rounds of one
 * workgroup per CU, their tiles and the merge.  No HIP call. */
ta_status mla_split_plan(int B, int H, int Hkv, int Skv, int *num_splits);

/*
 * gemm_bf16 — C = A B: the kernel beneath the paper's Matmul listing
 * (appendix "Matrix Multiplication (Matmul)"), bf16 inputs, fp32
 * accumulation.
 *
 *   A  device, bf16 [M, K] row-major         read only
 *   B  device, bf16 [K, N] row-major         read only
 *   C  device, [M, N] row-major: fp32, or bf16 (rounded to nearest even) if
 *      c_bf16 != 0                             written
 *   M % 128 == 0, N % 128 == 0, K % 64 == 0, and K * N * 2 < 2^31 (else
 *   TA_ERR_UNSUPPORTED, resp. TA_ERR_INVALID_SHAPE for the size); or M == 1,
 *   the matrix-vector product of the paper's V0-V7 shapes (appendix table
 *   "Matrix shapes in our benchmark"), with N % 64 == 0 and K % 8 == 0, which
 *   runs a separate HBM-bound kernel on the vector ALUs; every pointer
 *   16-byte aligned; C must not overlap A or B; stream as attn_fwd.
 * Status codes as attn_fwd; validation before any HIP call.
 */
ta_status gemm_bf16(const void *A, const void *B, void *C, int c_bf16, int M, int N, int K,
                    void *stream);

/*
 * gemm_bf16_split — gemm_bf16 with the K steps of every tile of C split into
 * num_splits ranges that separate workgroups sum, for products with too few
 * 128 x 128 tiles of C to occupy every CU.
 *
 *   num_splits 1..64 (else TA_ERR_INVALID_SHAPE), at most K / 64 (else
 *   TA_ERR_UNSUPPORTED); 1 runs gemm_bf16 and ignores the workspace; for
 *   more, each range's fp32 product goes to `workspace` (device, 16-byte
 *   aligned, at least num_splits * M * N * 4 bytes, owned by the caller, no
 *   overlap with A, B or C; TA_ERR_WORKSPACE if NULL or smaller) and a second
 *   kernel adds them in range order, rounding once if C is bf16
 *   M % 128 == 0 then as well; other arguments and status codes as gemm_bf16
 */
ta_status gemm_bf16_split(const void *A, const void *B, void *C, int c_bf16, int M, int N, int K,
                          int num_splits, void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes gemm_bf16_split needs: num_splits * M * N * 4 for
 * num_splits > 1, 0 for 1.  No HIP call. */
ta_status gemm_split_workspace_bytes(int M, int N, int num_splits, size_t *bytes);

/* A split count for gemm_bf16_split: 1 unless splitting is estimated to be
 * clearly faster (up to 256 tiles of 128 x 128, long K), with at most 512
 * workgroups (tiles x splits).  No HIP call. */
ta_status gemm_split_heuristic(int M, int N, int K, int *num_splits);

/*
 * gemv_bf16_split — the matrix-vector product C[n] = sum_k A[k] B[k][n] of
 * gemm_bf16 with M == 1 (the paper's V0-V7 shapes, appendix table "Matrix
 * shapes in our benchmark"), with the K rows split into num_splits ranges
 * that separate workgroups sum, so that shapes with few column strips
 * still occupy every CU.
 *
 *   A  device, bf16 [K]                       read only
 *   B  device, bf16 [K, N] row-major          read only
 *   C  device, [N]: fp32, or bf16 (rounded to nearest even once, from the
 *      fp32 sum) if c_bf16 != 0                written
 *   N % 64 == 0 and K % 8 == 0 (else TA_ERR_UNSUPPORTED)
 *   num_splits: 1..64 (else TA_ERR_INVALID_SHAPE); 1 runs gemm_bf16's
 *   matrix-vector kernel and ignores the workspace; for more, each range's
 *   fp32 partial sums go to `workspace` (device, 16-byte aligned, at least
 *   gemv_split_workspace_bytes(N, num_splits) bytes, owned by the caller, no
 *   overlap with A, B or C; TA_ERR_WORKSPACE if NULL or smaller) and a
 *   second kernel adds them in range order
 *   every pointer 16-byte aligned; C must not overlap A or B; stream as
 *   attn_fwd
 * Status codes as attn_fwd; validation before any HIP call.  The result
 * does not depend on timing; it differs from the unsplit kernel's in the
 * grouping of the fp32 additions only.
 */
ta_status gemv_bf16_split(const void *A, const void *B, void *C, int c_bf16, int N, int K,
                          int num_splits, void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes gemv_bf16_split needs: num_splits * N * 4 for
 * num_splits > 1, 0 for 1.  No HIP call. */
ta_status gemv_split_workspace_bytes(int N, int num_splits, size_t *bytes);

/* A split count for gemv_bf16_split.  A workgroup sums one strip of 256
 * columns (N % 256 == 0, else 64) over one K range, and two fit a CU; the
 * count chosen is the one whose workgroups (strips x splits, at most 512)
 * fill their last round of the 256 CUs most evenly, with at least 1024 rows
 * per range (fewer workgroups on a tie).  No HIP call. */
ta_status gemv_split_heuristic(int N, int K, int *num_splits);

/*
 * Mamba-2 state-space-duality (SSD) chunk functions: the paper's linear
 * attention workload ("chunk-scan and chunk-state functions from Mamba-2",
 * Section "Numerical Experiments", paragraph "Linear Attention Performance";
 * shapes in the appendix table "Linear Attention shapes in our benchmark").
 * For batch b, head h (group g = h / (nheads / ngroups)) and chunk c of
 * chunk_size positions, with a_l = sum_{l' <= l} dt_{l'} A_h the cumulative
 * log-decay inside the chunk (each call forms it from dt and A itself):
 *   ssd_chunk_state    S_c[p][n] = sum_l exp(a_last - a_l) dt_l x_l[p] Bm_l[n]
 *   ssd_state_passing  H_c = exp(a_last(c)) H_{c-1} + S_c, H_{-1} = 0; writes
 *                      the state each chunk enters with, H_{c-1}
 *   ssd_bmm_chunk      cb[l][s] = Cm_l . Bm_s (both positions in chunk c)
 *   ssd_chunk_scan     y_l[p] = exp(a_l) sum_n H_{c-1}[p][n] Cm_l[n]
 *                             + sum_{s <= l} cb[l][s] exp(a_l - a_s) dt_s x_s[p]
 *                             + D_h x_l[p]
 * Chained, they give the output of the recurrence h_t = exp(dt_t A) h_{t-1} +
 * dt_t x_t Bm_t^T, y_t = h_t Cm_t + D x_t (Mamba-2, "Transformers are SSMs").
 *
 * Layouts (contiguous, row-major; L = seqlen, nc = ceil(L / chunk_size)):
 *   x       device, bf16 [batch, L, nheads, headdim]
 *   Bm, Cm  device, bf16 [batch, L, ngroups, dstate]
 *   dt      device, fp32 [batch, L, nheads]           step sizes (> 0)
 *   A       device, fp32 [nheads]                     decay rates (<= 0)
 *   D       device, fp32 [nheads], or NULL for no skip term
 *   cb      device, fp32 [batch, nc, ngroups, chunk_size, chunk_size]
 *   states, prev_states
 *           device, fp32 [batch, nc, nheads, headdim, dstate]
 *   final_states device, fp32 [batch, nheads, headdim, dstate], or NULL
 *   out     device, fp32 [batch, L, nheads, headdim]
 * A last chunk shorter than chunk_size is handled as if padded with dt = 0
 * and zero x, Bm, Cm: padded positions add nothing (cb rows and columns of
 * padded positions are written as zero; out rows past L are not written).
 * headdim == 64, dstate == 128, chunk_size == 256 (else TA_ERR_UNSUPPORTED);
 * nheads % ngroups == 0 (else TA_ERR_INVALID_SHAPE).  bf16 and output
 * pointers 16-byte aligned, fp32 vectors 4-byte aligned (TA_ERR_MISALIGNED);
 * outputs must not overlap inputs (TA_ERR_ALIASING).  The decay- and
 * dt-weighted operand of each contraction (and, in the chunk scan, the fp32
 * entering state) is rounded to bf16 before the bf16 x bf16 -> fp32 MFMA.
 * Ownership, asynchrony and error behaviour as attn_fwd.
 */
ta_status ssd_chunk_state(const void *x, const void *Bm, const float *dt, const float *A,
                          float *states, int batch, int seqlen, int nheads, int ngroups,
                          int headdim, int dstate, int chunk_size, void *stream);

ta_status ssd_state_passing(const float *states, const float *dt, const float *A,
                            float *prev_states, float *final_states, int batch, int seqlen,
                            int nheads, int headdim, int dstate, int chunk_size, void *stream);

ta_status ssd_bmm_chunk(const void *Cm, const void *Bm, float *cb, int batch, int seqlen,
                        int ngroups, int dstate, int chunk_size, void *stream);

ta_status ssd_chunk_scan(const void *x, const void *Cm, const float *cb, const float *dt,
                         const float *A, const float *prev_states, const float *D, float *out,
                         int batch, int seqlen, int nheads, int ngroups, int headdim,
                         int dstate, int chunk_size, void *stream);

/*
 * ssd_forward — the whole chunked forward in one call: y and the final states
 * of the recurrence above, without the intermediate states, cb or entering
 * states of the four functions in memory (each workgroup walks a head's
 * sequence with the state in registers).  Same inputs, outputs and precision
 * as the four chained: bf16 operands of the contractions, fp32 sums and state.
 * What depends on an infinite or NaN input is not finite, as there; an infinite
 * state gives the infinities of its products with C, and an infinite x (infinite
 * states of both signs) NaN after the step of 64 positions it is in, where the
 * chunk functions give NaN after its chunk of 256.
 *
 *   out          device, fp32 [batch, L, nheads, headdim]        written
 *   final_states device, fp32 [batch, nheads, headdim, dstate], or NULL
 *   num_segments 1..64: the sequence is cut into this many segments (whole
 *                steps of 64 positions; trailing empty ones are dropped) that
 *                run in parallel, for calls with too few heads to fill the
 *                GPU; for more than one, a first kernel writes the state each
 *                segment adds to `workspace` (device, 16-byte aligned, at
 *                least ssd_forward_workspace_bytes(...) bytes, owned by the
 *                caller, no overlap with any other argument;
 *                TA_ERR_WORKSPACE if NULL or smaller); 1 ignores it
 *   nheads <= 131072 and L <= 2^30 (else TA_ERR_INVALID_SHAPE); other
 *   arguments and status codes as the chunk functions
 */
ta_status ssd_forward(const void *x, const void *Bm, const void *Cm, const float *dt, const float *A,
                      const float *D, float *out, float *final_states, int batch, int seqlen,
                      int nheads, int ngroups, int headdim, int dstate, int num_segments,
                      void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes ssd_forward needs for num_segments (0 for one).  No HIP call. */
ta_status ssd_forward_workspace_bytes(int batch, int seqlen, int nheads, int num_segments,
                                      size_t *bytes);

/* A segment count for ssd_forward.  No HIP call. */
ta_status ssd_segment_heuristic(int batch, int seqlen, int nheads, int *num_segments);

/*
 * Paged key/value cache of a decoder's serving step.  K and V of all sequences
 * live in one pool of pages each; a page holds page_size consecutive positions
 * of one sequence, and row b of page_table names the pages of sequence b in
 * order, so that position t of it is row t % page_size of page
 * page_table[b][t / page_size].
 *
 *   K_cache, V_cache  device, [num_pages, Hkv, page_size, D], bf16, or 8-bit
 *                     (OCP e4m3) if cache_e4m3 != 0
 *   k_scale, v_scale  device, fp32 [Hkv], positive, or NULL for 1: an 8-bit
 *                     number c of head h stands for c * scale[h].  NULL for a
 *                     bf16 cache (else TA_ERR_UNSUPPORTED)
 *   page_table        device, int32 [B, max_pages]
 *   D in {64, 128}; page_size a power of two, at least 16 (else
 *   TA_ERR_UNSUPPORTED); max_pages * page_size and Hkv * page_size <= 2^30,
 *   num_pages <= 2^28, Hkv <= 2^16 (else TA_ERR_INVALID_SHAPE).  Caches 16-byte aligned, fp32 and int32
 *   vectors 4-byte aligned.
 * What the arrays on the device hold cannot be checked before the launch; the
 * kernels check every index they take from them, and address nothing outside
 * the caches whatever they hold.
 */

/*
 * kv_cache_append — writes new tokens' keys and values into the paged cache.
 *
 *   K, V      device, bf16 [T, Hkv, D], read only: token t starts k_stride
 *             (v_stride) elements after token t - 1 (at least Hkv * D, at most
 *             2^30, a multiple of 8), so that they can be slices of a fused
 *             projection; 16-byte aligned.  T >= 1 and T * Hkv * D <= 2^34 -
 *             1024 (else TA_ERR_INVALID_SHAPE)
 *   seq       device, int32 [T]: token t belongs to sequence seq[t]; NULL:
 *             token t belongs to sequence t (T <= B, else TA_ERR_INVALID_SHAPE)
 *   pos       device, int32 [T]: its position in that sequence.  A token whose
 *             position is negative (padding) or past the table, whose seq is
 *             not in 0..B-1 or whose page is not in 0..num_pages-1 is left out
 *   K_cache, V_cache  written at those positions only
 *
 * An 8-bit cache takes x / scale rounded to the nearest e4m3 number (to even),
 * beyond +-448 as +-448, infinities too; NaN stays NaN.  Of two tokens of one
 * call with the same place, which one it holds afterwards is not defined, piece
 * of 8 elements by piece.  Caches must not overlap each other or an input
 * (TA_ERR_ALIASING).  Ownership, asynchrony and status codes as attn_fwd.
 */
ta_status kv_cache_append(const void *K, const void *V, int64_t k_stride, int64_t v_stride,
                          const int *seq, const int *pos, void *K_cache, void *V_cache,
                          int cache_e4m3, const float *k_scale, const float *v_scale,
                          const int *page_table, int T, int B, int Hkv, int D, int num_pages,
                          int page_size, int max_pages, void *stream);

/*
 * attn_decode_paged — attention of one new token per sequence over the paged
 * cache: for sequence b of seq_lens[b] positions, query head h and key/value
 * head hk = h / (Hq / Hkv),
 *   s_t = scale * Q[b,h,:] . K_t,  O[b,h,:] = sum_t softmax(s)_t V_t,
 *   LSE[b,h] = ln sum_t exp(s_t)
 * over its positions t (the new token's own included, once appended).
 *
 *   Q         device, bf16 [B, Hq, D], read only: sequence b starts q_stride
 *             elements after sequence b - 1 (at least Hq * D, at most 2^30, a
 *             multiple of 8); 16-byte aligned
 *   seq_lens  device, int32 [B], from 0 to max_pages * page_size.  Length 0 (an
 *             idle slot of a padded batch) gives O = 0 and LSE = -inf.  Any other
 *             value outside, and a page outside 0..num_pages-1 among those of
 *             the sequence's positions, gives NaN in that sequence's O and LSE
 *   O         device, [B, Hq, D]: fp32, or bf16 if o_bf16 != 0      written
 *   LSE       device, fp32 [B, Hq]                                  written
 *   Hq % Hkv == 0, Hq <= 65536, B * Hq < 2^24, and less than 2^31 for B * Hkv *
 *   ceil(Hq / Hkv / 32) * (max_pages * page_size / 64 + 3), the units of 64
 *   positions that the batch could come to (else TA_ERR_INVALID_SHAPE);
 *   scale >= 0, finite; O and LSE 16-byte aligned and apart from each other and
 *   from every input (TA_ERR_ALIASING)
 *   num_parts 0..4096 (else TA_ERR_INVALID_SHAPE): the cached positions of the
 *             whole batch, whatever its lengths, are divided evenly over this
 *             many workgroups, and a second kernel joins the results of the heads
 *             that the division cuts, in order, through `workspace` (device,
 *             16-byte aligned, at least attn_paged_workspace_bytes(...) bytes,
 *             owned by the caller, its contents on entry of no account, no
 *             overlap with any other argument; TA_ERR_WORKSPACE if NULL or
 *             smaller).  0: one workgroup per sequence and key/value head (and
 *             32 query heads of it), no workspace
 *
 * Entries of page_table past a sequence's last page, and what the caches hold
 * past its last position, are never used.  An infinite or NaN key or value of a
 * sequence makes what it enters infinite or NaN.  Scores, softmax weights and sums
 * are fp32; the weights enter the product with V with all 24 bits, as three bf16
 * numbers each.  A bf16 O is the fp32 one, rounded once, to nearest even.
 * Ownership, asynchrony and status codes as attn_fwd.
 */
ta_status attn_decode_paged(const void *Q, int64_t q_stride, const void *K_cache,
                            const void *V_cache, int cache_e4m3, const float *k_scale,
                            const float *v_scale, const int *page_table, const int *seq_lens,
                            void *O, int o_bf16, float *LSE, int B, int Hq, int Hkv, int D,
                            int num_pages, int page_size, int max_pages, float scale,
                            int num_parts, void *workspace, size_t workspace_bytes,
                            void *stream);

/* What a paged cache holds, for the calls that take cache_type */
typedef enum {
    TA_CACHE_BF16 = 0,
    TA_CACHE_E4M3 = 1,
    TA_CACHE_MXFP4 = 2
} ta_cache_type;

/*
 * 4-bit numbers (MXFP4 of the OCP microscaling formats), in caches and weights: rows of
 * n elements (n % 32 == 0) are n / 2 bytes of codes and n / 32 bytes of scales.  A code
 * is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (e2m1); element 2 i of a row is in the
 * low half of byte i, element 2 i + 1 in the high half.  Scale byte e multiplies 32
 * elements by 2^(e - 127); e = 255 makes them NaN.
 *
 * A 4-bit paged cache is laid out as the others are: codes, uint8
 * [num_pages, Hkv, page_size, D / 2], and scales, uint8 [num_pages, Hkv, page_size,
 * D / 32], for K and for V; all 16-byte aligned.
 */

/*
 * qk_norm_rope_append — from the projection to the cache in one pass: norm of the new
 * tokens' queries and keys, head by head, their position rotation, and the append of
 * keys and values to the paged cache.
 *
 *   n(x) = x / sqrt(mean(x^2) + eps) * w      where a weight w is given, else x
 *   y    = R(pos) n(x): of the first rot_dim dims each pair (a, b) becomes
 *          (a cos - b sin, b cos + a sin), the others stay
 *   Q_out[t,h,:] = y of Q[t,h,:];  K_cache takes y of K[t,h,:], V_cache V[t,h,:] itself
 *
 *   Q, K, V   device, bf16 [T, Hq, D] and [T, Hkv, D], read only, with strides between
 *             tokens as kv_cache_append takes them; 16-byte aligned.  Hq 0..65536 (0: Q,
 *             Q_out and q_weight are not looked at), any Hkv >= 1 beside it; 1 <= T < 2^24
 *   q_weight, k_weight  device, bf16 [D], or NULL for no norm; 16-byte aligned
 *   eps       >= 0, finite (else TA_ERR_INVALID_SCALE)
 *   cos_sin   device, fp32 [num_positions, rot_dim], 16-byte aligned: for position p and
 *             pair i the cosine at [p][i] and the sine at [p][rot_dim / 2 + i].  NULL,
 *             with num_positions = rot_dim = 0: no rotation
 *   rot_dim   16..D in steps of 16 (else TA_ERR_UNSUPPORTED)
 *   interleaved  0: pair i is dims (i, rot_dim / 2 + i); else dims (2 i, 2 i + 1)
 *   seq, pos  as kv_cache_append takes them: pos is the token's row of cos_sin too
 *   Q_out     device, bf16 [T, Hq, D], contiguous, 16-byte aligned        written
 *   cache_type  a ta_cache_type (else TA_ERR_UNSUPPORTED)
 *   k_scale, v_scale  bf16: NULL; e4m3: fp32 [Hkv] or NULL, read; MXFP4: the caches'
 *             scale bytes, written with the codes, not NULL
 *
 * Which tokens the cache takes, and two of one place: as kv_cache_append (for MXFP4 the
 * pieces are of 32 elements' codes and of their scale: such a place may end up with
 * the codes of one and the scale of the other).  A token whose
 * position is negative (padding) has zeros in Q_out; one whose position is
 * num_positions or more has NaN there and is left out of the cache.  A token that the
 * cache has no place for has its queries all the same.
 *
 * Queries, and keys for a bf16 cache, are computed in fp32 and rounded once, to nearest
 * even (the norm over all of bf16's range, whatever fp32 makes of its squares).  Keys for
 * 8 and 4 bits are computed in fp64, rounded to fp32 and then to the
 * cache's type; e4m3 as kv_cache_append does.  MXFP4: the scale is the power of two that
 * puts a group's largest number between 3.5 and 7 (at least 2^-126, at most 2^125), the
 * codes are the nearest (to even), beyond 6 as 6, infinities too; a NaN makes its
 * group's scale 255 and its codes 0.  Q_out, the caches and their written scales must
 * not overlap each other or an input (TA_ERR_ALIASING).  Ownership, asynchrony and
 * status codes as attn_fwd.
 */
ta_status qk_norm_rope_append(const void *Q, const void *K, const void *V, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, const void *q_weight, const void *k_weight, float eps,
                              const float *cos_sin, int num_positions, int rot_dim, int interleaved,
                              const int *seq, const int *pos, void *Q_out, void *K_cache, void *V_cache,
                              int cache_type, void *k_scale, void *v_scale, const int *page_table, int T,
                              int B, int Hq, int Hkv, int D, int num_pages, int page_size, int max_pages,
                              void *stream);

/*
 * attn_decode_paged_mxfp4 — attn_decode_paged over a cache held in 4 bits.
 *
 *   K_cache, V_cache  device, codes, uint8 [num_pages, Hkv, page_size, D / 2]
 *   k_scale, v_scale  device, scales, uint8 [num_pages, Hkv, page_size, D / 32],
 *                     16-byte aligned, not NULL
 * Everything else as attn_decode_paged, with its workspace: keys and values
 * enter the products as the numbers they stand for, exactly (those past the largest bf16
 * number as infinity); a scale of 255 within a sequence's positions makes what it enters
 * NaN.
 */
ta_status attn_decode_paged_mxfp4(const void *Q, int64_t q_stride, const void *K_cache,
                                  const void *V_cache, const void *k_scale, const void *v_scale,
                                  const int *page_table, const int *seq_lens, void *O, int o_bf16,
                                  float *LSE, int B, int Hq, int Hkv, int D, int num_pages,
                                  int page_size, int max_pages, float scale, int num_parts,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes attn_decode_paged needs for num_parts (0 for none).  No HIP call. */
ta_status attn_paged_workspace_bytes(int Hq, int Hkv, int D, int num_parts, size_t *bytes);

/* A part count for attn_decode_paged, from the table's capacity (the lengths are on the
 * device).  A caller that knows all sequences to be short behind a large table takes 0
 * instead: one workgroup a head and no second kernel (a sequence of 37 positions 4 us
 * instead of 9.5, 32 of 200 9 instead of 14).  No HIP call. */
ta_status attn_paged_plan(int B, int Hq, int Hkv, int D, int page_size, int max_pages,
                          int *num_parts);

/* The same for attn_decode_paged_mxfp4.  No HIP call. */
ta_status attn_paged_mxfp4_plan(int B, int Hq, int Hkv, int D, int page_size, int max_pages,
                                int *num_parts);

/* Activations of gemm_bf16_epilogue */
typedef enum {
    TA_ACT_NONE = 0,
    TA_ACT_RELU = 1,      /* max(x, 0)                                                    */
    TA_ACT_GELU = 2,      /* x (1 + erf(x / sqrt 2)) / 2                                  */
    TA_ACT_GELU_TANH = 3, /* x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))) / 2            */
    TA_ACT_SILU = 4       /* x / (1 + exp(-x))                                            */
} ta_activation;

/*
 * gemm_bf16_epilogue — C = act(A B + bias) + residual, for any number of rows.
 *
 *   A  device, bf16 [M, K] row-major             read only
 *   B  device, bf16 [K, N] row-major             read only
 *   bias      device, bf16 [N], or NULL          read only
 *   residual  device, [M, N] row-major, of C's type, or NULL; may be C itself
 *             (the sum in place), otherwise read only
 *   C  device, [M, N] row-major: fp32, or bf16 if c_bf16 != 0      written
 *   activation  a ta_activation (else TA_ERR_UNSUPPORTED)
 *   N % 8 == 0 and K % 8 == 0 (else TA_ERR_UNSUPPORTED); N < 2^24, K < 2^22,
 *   M <= 2^20, M * N < 2^35, M * K < 2^40, N * K < 2^40 (else TA_ERR_INVALID_SHAPE);
 *   pointers 16-byte aligned; C apart from A, B and bias, and from residual
 *   unless it is C
 *   num_splits  1..64 (else TA_ERR_INVALID_SHAPE): ranges of K that separate
 *               workgroups sum (up to 64 rows: about this many per 128 columns;
 *               more rows: at most K / 64 of them, and for the columns only that
 *               do not fill the GPU in 256 x 256 tiles); for more than one, each
 *               range's fp32 product goes to `workspace`
 *               (device, 16-byte aligned, at least
 *               gemm_epilogue_workspace_bytes(...) bytes, owned by the caller, no
 *               overlap with any other argument; TA_ERR_WORKSPACE if NULL or
 *               smaller) and a second kernel adds them in range order
 *
 * Sums, bias, activation and residual are fp32; a bf16 C is rounded once, to
 * nearest even.  Ownership, asynchrony and status codes as gemm_bf16.
 */
ta_status gemm_bf16_epilogue(const void *A, const void *B, const void *bias, const void *residual,
                             void *C, int c_bf16, int activation, int M, int N, int K,
                             int num_splits, void *workspace, size_t workspace_bytes,
                             void *stream);

/* Workspace bytes gemm_bf16_epilogue needs, 0 for one range.  No HIP call. */
ta_status gemm_epilogue_workspace_bytes(int M, int N, int K, int num_splits, size_t *bytes);

/* A split count for gemm_bf16_epilogue: 1 unless the workgroups of one range
 * would leave CUs without work.  No HIP call. */
ta_status gemm_epilogue_plan(int M, int N, int K, int *num_splits);

/* How many of the first columns of C gemm_bf16_epilogue computes in 256 x 256 tiles,
 * whole rounds of one per CU, for tests and tools: 0 (the other kernels take them all)
 * to N.  No HIP call. */
ta_status gemm_epilogue_route(int M, int N, int K, int num_splits, int *large_columns);

/*
 * gemm_mxfp4_epilogue — C = act(A W^T + bias) + residual, for any number of rows, with
 * the weights in 4 bits (MXFP4, described at qk_norm_rope_append).
 *
 *   A        device, bf16 [M, K] row-major                          read only
 *   W        device, codes, uint8 [N, K / 2]: a row holds the weights of one output
 *   W_scale  device, scales, uint8 [N, K / 32]; any alignment       read only
 *   bias, residual, C, c_bf16, activation  as gemm_bf16_epilogue
 *   N % 8 == 0 and K % 32 == 0 (else TA_ERR_UNSUPPORTED); sizes up to those of
 *   gemm_bf16_epilogue; A, W, bias, residual, C and workspace 16-byte aligned; C apart
 *   from A, W, W_scale and bias, and from residual unless it is C
 *   num_parts  0..4096 (else TA_ERR_INVALID_SHAPE): the steps of K, 128 columns each, of
 *               all strips (up to 64 rows) or tiles (more) of C are divided evenly over
 *               this many workgroups, fewer where there are not as many steps (eight for
 *               each, in strips); a second kernel adds what the division cuts, in order
 *               of K, through `workspace` (device, at least
 *               gemm_mxfp4_workspace_bytes(...) bytes, owned by the caller, no overlap with
 *               any other argument; TA_ERR_WORKSPACE if NULL or smaller).  0: one
 *               workgroup per strip or tile, no workspace
 *
 * The weights enter the products as the numbers that they stand for, exactly (those past
 * the largest bf16 number as infinity); a scale of 255 makes its row's column of C NaN.
 * Sums, bias, activation and residual are fp32; a bf16 C is rounded once, to nearest
 * even.  Ownership, asynchrony and status codes as gemm_bf16.
 */
ta_status gemm_mxfp4_epilogue(const void *A, const void *W, const void *W_scale, const void *bias,
                              const void *residual, void *C, int c_bf16, int activation, int M,
                              int N, int K, int num_parts, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Workspace bytes gemm_mxfp4_epilogue needs for num_parts (0 for none).  No HIP call. */
ta_status gemm_mxfp4_workspace_bytes(int M, int N, int K, int num_parts, size_t *bytes);

/* A part count for gemm_mxfp4_epilogue.  No HIP call. */
ta_status gemm_mxfp4_plan(int M, int N, int K, int *num_parts);

/*
 * sample_logits — the next token of each row of logits, by temperature, top-k, top-p and
 * min-p, from a given uniform number.
 *
 * Row b's tokens are in order by falling logit, those of equal logits by index.  With the
 * weights w_i = exp((x_i - max x) / T), of that order are kept: the first top_k; of
 * these each token before which there is less than top_p of their weight; each with
 * w_i >= min_p; and the first in any case.  The token is the first, by index, up to which
 * the kept tokens' weights sum to more than u of their whole sum, and logp the logarithm
 * of its share of all tokens' weight: (x - max x) / T - ln sum_i w_i.
 *
 *   logits  device, fp32, or bf16 if l_bf16 != 0, [B, V]: row b starts stride elements
 *           after row b - 1 (0 to 2^30); aligned to its type               read only
 *   u       device, fp32 [B], 0 <= u < 1 (what is outside: as the nearest inside)
 *   temperature  device, fp32 [B], or NULL for 1.  0, negative or NaN: the largest logit
 *           (of several the first), whatever u and the filters, logp for T = 1; others are
 *           taken as 1e-30 to 1e30
 *   top_k   device, int32 [B], or NULL; 0, negative, or V and more: without
 *   top_p   device, fp32 [B], or NULL; 1 and more: without; 0, negative or NaN: the first
 *           alone
 *   min_p   device, fp32 [B], or NULL; 0 and less: without; more than 1 or NaN: the first
 *           alone
 *   token   device, int32 [B]                                              written
 *   logp    device, fp32 [B]                                               written
 *   1 <= B <= 65536, 1 <= V <= 2^20 (else TA_ERR_INVALID_SHAPE); token and logp apart from
 *   each other and every input (TA_ERR_ALIASING)
 *   workspace  device, 16-byte aligned, at least sample_logits_workspace_bytes(...) bytes,
 *           owned by the caller, its contents on entry of no account, no overlap with any
 *           other argument; TA_ERR_WORKSPACE if NULL or smaller
 *
 * A logit of -inf is never chosen.  A row with NaN or +inf in it, or with -inf only, has
 * token -1 and logp NaN.  Weights are computed in fp64 and added exactly, as whole
 * multiples of 2^-43 (a token of less than half of that is never chosen), so that results
 * do not depend on the order of additions; logp's sum is in fp32 and fp64.  Ownership,
 * asynchrony and status codes as attn_fwd.
 */
ta_status sample_logits(const void *logits, int64_t stride, int l_bf16, const float *u,
                        const float *temperature, const int *top_k, const float *top_p,
                        const float *min_p, int *token, float *logp, int B, int V,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes sample_logits needs for logits of one type (0 where one workgroup takes a
 * row: of up to 32768 logits or, from 128 rows on, up to 69627 in fp32 and 139255 in bf16).
 * No HIP call. */
ta_status sample_logits_workspace_bytes(int B, int V, int l_bf16, size_t *bytes);

/* The same for either type: fp32's, bf16 needs no more.  No HIP call. */
ta_status sample_workspace_bytes(int B, int V, size_t *bytes);

/*
 * ta_schedule — host-side tile schedule of attn_fwd, for tests and tools.
 * For the query tile `q_tile` (rows q_tile*BM .. q_tile*BM+BM-1, BM from
 * ta_tile_shape) it reports how many key tiles of BN keys the kernel visits
 * (n_kv_tiles; tiles past it are skipped because every key in them is
 * masked) and the first visited tile that needs per-element masking
 * (first_masked; == n_kv_tiles if none).  Pure integer logic, no HIP call.
 * Returns TA_ERR_INVALID_SHAPE for sizes < 1, q_tile out of range, or causal
 * with Sq > Sk; TA_ERR_UNSUPPORTED for D not 64/128; TA_ERR_NULL_POINTER.
 */
ta_status ta_schedule(int Sq, int Sk, int D, int causal, int q_tile,
                      int *n_kv_tiles, int *first_masked);

/* Query rows (BM) and keys (BN) per tile for head dim D; TA_ERR_UNSUPPORTED
 * for D not 64/128.  No HIP call. */
ta_status ta_tile_shape(int D, int *BM, int *BN);

/* Static text for a status code (never NULL). */
const char *ta_status_string(ta_status s);

/* Library version, major*10000 + minor*100 + patch. */
int ta_version(void);

#ifdef __cplusplus
}
#endif

#endif /* TILEATTN_H */
