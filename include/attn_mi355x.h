/*
 * attn_mi355x.h -- C ABI of libattn_mi355x.so: exact softmax attention, forward and backward,
 * for AMD MI355X (gfx950).
 *
 * What is computed (arXiv 2410.09397, "On Fine-Grained I/O Complexity of Attention Backward
 * Passes"; the paper's S = A_1 X, A_2, h = A_3 Y are the Q, K, V of this interface):
 *   forward  (Sec. 3.1, forward definition; App. B.4, definitions of A, l, f, O)
 *       s_ij = scale * <Q_i, K_j> over visible (i, j);  l_i = sum_j exp(s_ij);
 *       O_i = sum_j exp(s_ij) / l_i * V_j;              LSE_i = log l_i
 *   backward (App. B.4, definitions of q and p; Sec. 3.1, backward gradient; the tiling follows
 *             the large-cache phase-2 algorithm of App. D for d <= 256 and the four-phase
 *             small-cache algorithm of App. C for d > 256)
 *       f_ij = exp(s_ij - LSE_i);  v_i = <dO_i, O_i>;  q_ij = <dO_i, V_j>;  p_ij = f_ij (q_ij - v_i)
 *       dV_j = sum_i f_ij dO_i;  dK_j = scale sum_i p_ij Q_i;  dQ_i = scale sum_j p_ij K_j
 * The paper has no scale and no mask; scale multiplies Q K^T, and a pair (i, j) is visible iff
 * (!causal || j <= i) and, when a block mask is given, the mask keeps block (i/block, j/block).
 * A query with no visible key gets O = 0, LSE = -inf and contributes no gradient.
 *
 * Conventions
 *   - Every tensor pointer is DEVICE memory owned by the caller.  Q, K, V, O, dO, dQ, dK, dV are
 *     [batch, heads, n, d] with element strides (stride_b, stride_h, stride_n, 1), the same for
 *     all of them; LSE is contiguous [batch, heads, n] float.  Outputs are overwritten.
 *     Gradients do not overlap what their call reads, but for one: with ATTN_BF16, d in {64, 128, 256, 512, 1024} and ATTN_BWD_AUTO one
 *     of dQ, dK and dV may have the memory of O, whose rows are read before they are written.
 *   - All work is enqueued on `stream` (a hipStream_t passed as void*, NULL = default stream);
 *     calls return without synchronising.  The library allocates no device memory and keeps no
 *     state between calls (attn_bwd_noalloc alone keeps the device address of its scratch array,
 *     per GPU, behind a mutex); scratch comes from the caller's workspace (attn_workspace_bytes).
 *     Entry points may be called from several host threads at once.
 *   - Arguments are validated on the host before anything is launched; a failed call launches
 *     nothing and leaves outputs untouched.  batch * heads * n == 0 is a valid empty call.
 *   - Supported: d a multiple of 8 for ATTN_BF16 (pointers and strides 16-byte aligned), any d
 *     for ATTN_F32, 1 <= d <= 512.  ATTN_BF16 runs bf16-MFMA kernels with fp32 accumulation for
 *     d in {64, 128, 256} (block masks: block == 128; fused, nothing n x n leaves the chip) and
 *     for d in {512, 1024} without block mask and n <= 32768 (four-phase path through the
 *     workspace; d = 1024 is supported there only); every other supported case, ATTN_F32 always,
 *     runs in fp32 arithmetic: on the matrix cores for d <= 128 (ATTN_F32) or d <= 256 (ATTN_BF16) and
 *     mask blocks that are a multiple of 16 (ATTN_BF16 with d <= 128: of 32), on fp32 FMA kernels beyond and for
 *     sequences of up to 2 to 6 rows in some hundreds of heads or more.
 *   - The same call gives the same bits (but for dQ of the one-pass tilings, see below).  How a head's sums are shared out
 *     over the waves depends on batch * heads and n: the bits of a head may differ in the last places
 *     between calls with other heads beside it.  Where a call and its masked form run on the same kernels (blocks of 128
 *     for d in {64, 128, 256} in bf16; the matrix-core kernels of fp32 arithmetic), a mask that keeps every block gives
 *     the bits of the call without one, and one that keeps the lower triangle, with causal = 1, those of the causal call.
 */
#ifndef ATTN_MI355X_H
#define ATTN_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ATTN_OK = 0,
    ATTN_ERR_INVALID_ARG = 1, /* null pointer, negative size, misaligned stride, malformed mask */
    ATTN_ERR_UNSUPPORTED = 2, /* valid request outside the supported set (d, dtype) */
    ATTN_ERR_WORKSPACE = 3,   /* workspace missing or smaller than attn_workspace_bytes() */
    ATTN_ERR_DEVICE = 4       /* the HIP runtime reported an error at launch */
} attn_status;

typedef enum { ATTN_F32 = 0, ATTN_BF16 = 1 } attn_dtype;

/*
 * Tilings of the bf16 backward.  All compute the same gradients; they
 * differ in which block stays on chip, i.e. in the cache size M they need and in the traffic they
 * cause (the trade-off of Thm 1.1 / Sec. 4), and exist side by side so that it can be measured.
 *   ATTN_BWD_AUTO          the library's choice (the fastest measured for the shape); where that is the
 *                          next one, small calls run its two owners in one launch, with the same bits
 *   ATTN_BWD_TWO_KERNEL    a query-block owner forms dQ and a key-block owner forms dK, dV; both
 *                          recompute f and p (14 d multiply-adds per pair for 10 d counted); no
 *                          atomics, every output bit-reproducible; d in {64, 128, 256}
 *   ATTN_BWD_ONEPASS_K64   one key-block owner (64 keys) forms all five products once and adds its
 *   ATTN_BWD_ONEPASS_K128  dQ tiles with fp32 atomic adds into a zeroed array in the workspace,
 *                          which a last kernel scales and rounds to bf16 (K128: 128 keys per owner,
 *                          half the atomic volume); dK, dV bit-reproducible, dQ up to the order of
 *                          the additions; d in {64, 128}
 *   ATTN_BWD_PART_DQ       measurement aids: one kernel of ATTN_BWD_TWO_KERNEL alone, so that a caller
 *   ATTN_BWD_PART_DKDV     can time it with events of its own.  PART_DQ writes dQ (and v into the
 *                          workspace) and leaves dK, dV untouched; PART_DKDV writes dK, dV, leaves dQ
 *                          untouched and reads the v (and, under a block mask, nothing else) that an
 *                          earlier TWO_KERNEL or PART_DQ call left in the same workspace
 *   ATTN_BWD_FOUR_PHASE    the four-phase small-cache scheme of App. C (f and p through the workspace) at
 *                          a head dimension where the fused kernels are the default: d in {128, 256}
 *                          (it is what d in {512, 1024} run anyway); no block mask, n <= 32768
 *   ATTN_BWD_SPLIT_D       fused kernels whose owned block is 32 rows with the contraction over d split
 *                          over the waves of a workgroup: the fused alternative where the four-phase
 *                          scheme is the default, d = 512 (also d = 256); no block mask; bit-reproducible
 * A tiling that does not exist for the shape gives ATTN_ERR_UNSUPPORTED; the generic fp32 kernels
 * ignore the field, and so does the forward.
 */
typedef enum {
    ATTN_BWD_AUTO = 0,
    ATTN_BWD_TWO_KERNEL = 1,
    ATTN_BWD_ONEPASS_K64 = 2,
    ATTN_BWD_ONEPASS_K128 = 3,
    ATTN_BWD_PART_DQ = 4,
    ATTN_BWD_PART_DKDV = 5,
    ATTN_BWD_FOUR_PHASE = 6,
    ATTN_BWD_SPLIT_D = 7
} attn_bwd_tiling;

typedef struct {
    int32_t batch, heads, n, d;
    float scale;        /* multiplies Q K^T; callers usually pass 1/sqrt(d) */
    int32_t causal;     /* 0 or 1: key j visible to query i iff j <= i */
    int32_t dtype;      /* attn_dtype of Q, K, V, O, dO, dQ, dK, dV */
    int32_t bwd_tiling; /* attn_bwd_tiling; 0 unless a particular tiling is to be measured */
    int64_t stride_b, stride_h, stride_n; /* in elements; the d axis has stride 1; stride_n < 2^22 */
} attn_desc;

/*
 * Block mask: an nblk x nblk pattern of kept blocks, nblk = ceil(n / block), in both compressed
 * orientations (DEVICE int32 arrays, caller owned):
 *   row_ptr[nblk+1], col_idx[nnz]: key blocks kept for each query-block row, ascending;
 *   col_ptr[nblk+1], row_idx[nnz]: query blocks kept for each key-block column, ascending.
 * The two must describe the same set; attn_blockmask_validate checks host copies.
 * nmasks == 0 or 1: one pattern shared by all (batch, head) pairs.  nmasks == batch * heads: one
 * pattern per pair, mask m = b * heads + h; the arrays are the concatenations of the per-mask
 * arrays, row_ptr and col_ptr with nblk + 1 entries per mask that index the concatenated col_idx
 * and row_idx directly (entry 0 of mask m equals entry nblk of mask m - 1; mask 0 starts at 0).
 * (The paper's sparse bound, Thm 4.5, only counts non-zero entries: it covers both.)
 */
typedef struct {
    int32_t block;
    int32_t nblk;
    const int32_t *row_ptr, *col_idx;
    const int32_t *col_ptr, *row_idx;
    int32_t nmasks;
} attn_blockmask;

/* Bytes of device scratch that attn_fwd, attn_bwd and attn_bwd_blocksparse need for `desc`
 * (one figure that covers all three; 0 if desc or mask is invalid).  For d <= 256 it holds the
 * [batch, heads, n] row sums v (under a block mask also two lists of ceil(n / 128) block indices:
 * the order in which the workgroups take the blocks) and, for the one-pass tilings, the fp32
 * [batch, heads, n, d] array in which dQ is summed; for d > 256 (App. C path) the row sums and
 * the n x n matrices f and p of every (batch, head) in bf16, with n rounded up to 256. */
size_t attn_workspace_bytes(const attn_desc *desc, const attn_blockmask *mask /* nullable */);

/* Forward: writes O [batch, heads, n, d] and LSE [batch, heads, n].  `mask` may be NULL.
 * `workspace` is read only when d > 256 and may be NULL otherwise. */
attn_status attn_fwd(const attn_desc *desc, const attn_blockmask *mask, const void *Q,
                     const void *K, const void *V, void *O, float *LSE, void *workspace,
                     size_t workspace_bytes, void *stream);

/* Backward without block mask: dQ, dK, dV from Q, K, V, the forward's O and LSE, and dO. */
attn_status attn_bwd(const attn_desc *desc, const void *Q, const void *K, const void *V,
                     const void *O, const void *dO, const float *LSE, void *dQ, void *dK,
                     void *dV, void *workspace, size_t workspace_bytes, void *stream);

/*
 * attn_bwd for callers that cannot allocate or pass device scratch (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same kernels and the same result as
 * attn_bwd, with the scratch taken from a fixed array of ATTN_NOALLOC_SCRATCH_BYTES that the
 * library holds on every GPU it runs on until the process ends.  It calls no hipMalloc, hipFree or
 * other allocating routine.  A desc whose attn_workspace_bytes(desc, NULL) exceeds the array gives
 * ATTN_ERR_WORKSPACE and launches nothing (d <= 256 needs 4 bytes per (batch, head, query) for the
 * two-kernel tiling: 2 Mi rows fit).  Every call on one GPU uses that GPU's one array, which keeps
 * the previous call's contents (nothing in it has to start at zero: every kernel writes what it
 * later reads): calls that overlap in time on one GPU, on whatever streams, race.
 */
#define ATTN_NOALLOC_SCRATCH_BYTES (8u << 20)
attn_status attn_bwd_noalloc(const attn_desc *desc, const void *Q, const void *K, const void *V,
                             const void *O, const void *dO, const float *LSE, void *dQ, void *dK,
                             void *dV, void *stream);

/* Backward under a block mask (the sparse setting of Sec. 4.3; the paper gives bounds for it,
 * no algorithm).  `mask` must not be NULL.  Gradients of fully masked key rows are zero. */
attn_status attn_bwd_blocksparse(const attn_desc *desc, const attn_blockmask *mask,
                                 const void *Q, const void *K, const void *V, const void *O,
                                 const void *dO, const float *LSE, void *dQ, void *dK, void *dV,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Weight gradient of the paper's loss (Def. 3.2 and the backward gradient of Sec. 3.1; the
 * no-cache algorithm of App. C.1 states the same product step by step): with
 *     S = A_1 X (queries), A_2 (keys), h = A_3 Y (values), f, q, p as above,
 *     g = dL/dX = scale * A_1^T p A_2            one d x d matrix per (batch, head), float32.
 * A_1, A_2, A_3 and dO are [batch, heads, n, d] (here contiguous: stride_n == d, stride_h ==
 * n * d, stride_b == heads * n * d), X and Y are contiguous [batch, heads, d, d], row-major
 * (X[k][c]: input feature k, output feature c), g is contiguous [batch, heads, d, d].  dO is the
 * gradient of the loss with respect to the attention output (the paper's O - E).
 * The two projections, the forward, the dQ part of the backward and the product A_1^T dQ all run
 * on the device; queries, values, O and dQ pass through the workspace in bf16.
 * Supported: ATTN_BF16, d in {64, 128, 256}, no block mask; anything else -> ATTN_ERR_UNSUPPORTED.
 * attn_wgrad_workspace_bytes returns 0 for an invalid or unsupported desc.
 */
size_t attn_wgrad_workspace_bytes(const attn_desc *desc);
attn_status attn_bwd_wgrad(const attn_desc *desc, const void *A1, const void *A2, const void *A3,
                           const void *X, const void *Y, const void *dO, float *g,
                           void *workspace, size_t workspace_bytes, void *stream);

/* Checks HOST copies of a block mask (nmasks patterns, 0 counts as 1): monotone pointers that
 * continue from one pattern to the next, strictly ascending in-range indices,
 * nblk == ceil(n / block), and that the two orientations of every pattern hold the same pairs. */
attn_status attn_blockmask_validate(int32_t block, int32_t nblk, int32_t n, int32_t nmasks,
                                    const int32_t *row_ptr, const int32_t *col_idx,
                                    const int32_t *col_ptr, const int32_t *row_idx);

/*
 * Measurement aid (no part of the attention path; the paper has no counterpart): launches a
 * register-only loop of independent dense bf16 MFMAs (32x32x16) on every CU, two waves per SIMD,
 * `iters` iterations of 8 MFMAs per wave.  `operands`: 0 = random bf16 operands held in registers,
 * 1 = all-zero operands, 2 = random operands with the B operand of every MFMA read from LDS as a fresh
 * 1 KB fragment requested one MFMA ahead (what the attention kernels do), 3 = as 2 plus four fp32
 * multiply-adds and one exponential per MFMA (about the vector arithmetic of the backward kernels),
 * 4 = the instruction stream of one wave of the dK / dV kernel per 64 x 64 tile at d = 128 with every
 * dependency taken out (per 32 MFMAs: 16 ds_read_b128 and 32 ds_read_b64_tr_b16 fragment reads, 16
 * exponentials, 64 multiply-adds, 16 bf16 packs, 8 LDS writes, 8 KB of global_load_lds tile copy out of
 * a 1 MB window, two workgroup barriers); `iters` still counts 8 MFMAs, a tile is four of them.
 * The rate it sustains is the ceiling of any kernel built on that instruction for operands of
 * that kind: under matrix load the shader clock follows the power the data's switching activity
 * draws.  Asynchronous on `stream`; the caller times it.
 *   clock_ghz  DEVICE float[1], caller owned: shader clock seen by one workgroup over the run
 *              (cycle counter against the 100 MHz constant-rate counter), valid after the stream
 *              has been synchronised
 *   flops      HOST double[1]: floating-point operations the launch executes
 * Errors: ATTN_ERR_INVALID_ARG (iters outside 1 .. 4 000 000, i.e. about a second of GPU time;
 * operands outside 0 .. 4; null pointers), ATTN_ERR_DEVICE.
 */
attn_status attn_mfma_ceiling(int32_t iters, int32_t operands, float *clock_ghz, double *flops,
                              void *stream);

/*
 * Attention with a sliding window and shared keys, forward and backward.  As attn_fwd and attn_bwd, causal, with
 *   - heads query heads that share kv_heads key heads: query head h reads key head h / (heads / kv_heads), and dK, dV of a key
 *     head are the sums over its query heads;
 *   - a window: a pair (i, j) is visible iff j <= i and (window == 0 or i - j < window or j < sinks), i.e. a query sees itself, the
 *     window - 1 keys in front of it and the first `sinks` keys of the sequence; window == 0 is plain causal attention;
 *   - sequences of different lengths: with `lens` (DEVICE int32 [batch], may be NULL: n each) rows of sequence b from lens[b] on are
 *     padding: keys there are visible to nobody and never read into a sum, queries there get O = 0, LSE = -inf and gradients 0.
 *     (Values below 0 or above n count as 0 and n.)
 * Q, O, dO, dQ are [batch, heads, n, d] with the q_ strides, K, V, dK, dV [batch, kv_heads, n, d] with the kv_ strides (in
 * elements, d axis 1); LSE is contiguous [batch, heads, n].  Outputs are overwritten and overlap nothing else (a call with batch, heads or n
 * 0 has nothing to do: it writes nothing, not dK and dV of keys that no head reads either); a stride of an axis with more than one entry is at least d.
 * Supported: 1 <= d <= 256; ATTN_F32; ATTN_BF16 with d, strides and pointers as for attn_fwd.  ATTN_BF16 runs bf16-MFMA kernels with fp32
 * accumulation (d = 64, 128 and 256 fill them, other d run at the next of these), ATTN_F32 fp32 arithmetic on the matrix cores.  The same call
 * gives the same bits.
 * Precision, ATTN_BF16: the weights P and dS are rounded to bf16 for the products that use them, at every d.  attn_fwd and attn_bwd round them at d = 64, 128
 * and 256 only: at other d a causal call without a window or shared heads is more exact through those (distance from 64 bits over the norm 1.6 to
 * 1.7e-3, of O and of the gradients, against 2.0 and 2.4e-3 here), in about the same time.  ATTN_F32: a step takes longer than the full causal one of attn_fwd
 * and attn_bwd where the window is more than about a tenth of the sequence (three times as long without a window).
 * A NaN or an infinity in a row inside a sequence may reach every query whose tile of keys it lies in, also those that do not see it.
 * The work goes with the number of visible pairs: tiles that no query of a block sees are neither read nor computed.
 */
typedef struct {
    int32_t batch, heads, kv_heads, n, d;
    float scale;
    int32_t window, sinks; /* 0: no window; sinks count only under a window */
    int32_t dtype;         /* attn_dtype */
    int32_t reserved;      /* 0 */
    int64_t q_stride_b, q_stride_h, q_stride_n;
    int64_t kv_stride_b, kv_stride_h, kv_stride_n;
} attn_win_desc;

/* Device scratch of attn_win_bwd (row sums v, and partial sums of keys whose work is shared out); attn_win_fwd needs none.  0 if desc is invalid. */
size_t attn_win_workspace_bytes(const attn_win_desc *desc);
attn_status attn_win_fwd(const attn_win_desc *desc, const int32_t *lens, const void *Q, const void *K, const void *V,
                         void *O, float *LSE, void *stream);
attn_status attn_win_bwd(const attn_win_desc *desc, const int32_t *lens, const void *Q, const void *K, const void *V,
                         const void *O, const void *dO, const float *LSE, void *dQ, void *dK, void *dV,
                         void *workspace, size_t workspace_bytes, void *stream);

/*
 * Paged cache of keys and values, and the attention of new tokens over it (serving: one token per sequence, a chunk, or a batch of
 * both).  A page holds page_size consecutive tokens of one sequence for all key heads; table[b][x] (DEVICE int32, rows
 * table_stride apart) is the page of tokens x * page_size .. of sequence b.  lens[b] counts the tokens of sequence b in the cache,
 * the new ones included: these are its last, and have rows q_ptr[b] .. q_ptr[b + 1] - 1 of Q, O, K, V (q_ptr: DEVICE int32
 * [batch + 1], ascending; NULL: max_q rows each, row b * max_q first).  The order of a step is attn_cache_write, then
 * attn_paged_fwd with the same desc.
 *   pages   K, V [num_pages] x [kv_heads] x [page_size] x [d] with page_stride_p, _h, _n (elements, d axis 1; any order)
 *   ATTN_CACHE_PLAIN  pages hold values of `dtype`
 *   ATTN_CACHE_FP8    pages hold e4m3 codes, K_exp and V_exp ([num_pages, kv_heads, page_size] bytes, contiguous) an exponent byte e
 *                     per row: a code c stands for c 2^(e - 127), where 2^(e - 127) is the smallest power of two that brings the row's
 *                     largest magnitude to 448 or less (at least 2^-126; 1 for a row of zeros).  Codes are rounded to nearest, ties
 *                     to even; NaN and infinities become NaN and do not count for the largest magnitude.
 * Query t of a sequence is at position i = lens[b] - (its new tokens) + t and sees key j iff j <= i and (window == 0 or
 * i - j < window or j < sinks).  A query in front of position 0 sees nothing: O = 0, LSE = -inf.
 * max_q and max_len bound the new tokens and the lengths (they size the launches; what lies beyond them is not worked on; max_len <=
 * max_pages * page_size).  Pages that no query sees are not read, and their entries of the table are not used for an access; an
 * entry outside 0 .. num_pages - 1 where a query sees tokens makes the result meaningless, but no access leaves the cache:
 * attn_cache_write skips such tokens, attn_cache_read gives zeros for them.  Rows beyond the sequences' own are not written.
 * Supported: page_size a power of two from 8 to 4096, 1 <= d <= 256, d % 8 == 0 for ATTN_BF16 and ATTN_CACHE_FP8, batch <= 65535; with
 * ATTN_BF16 strides are multiples of 8 and pointers 16-byte aligned, strides of quantised pages are multiples of 8 (of 16 for d a multiple
 * of 64).  ATTN_BF16 runs bf16-MFMA kernels (quantised pages: with d in {64, 128, 256}), everything else fp32 arithmetic.
 */
typedef enum { ATTN_CACHE_PLAIN = 0, ATTN_CACHE_FP8 = 1 } attn_cache_kind;

typedef struct {
    int32_t batch, heads, kv_heads, d;
    int32_t total_q;            /* rows of Q, O, K, V */
    int32_t max_q, max_len;     /* most new tokens, most tokens of a sequence */
    int32_t page_size, num_pages, max_pages; /* max_pages: entries of a row of the table */
    float scale;
    int32_t window, sinks;
    int32_t dtype;              /* attn_dtype of Q, O, K, V */
    int32_t kind;               /* attn_cache_kind */
    int32_t reserved;           /* 0 */
    int64_t q_stride_n, q_stride_h;   /* Q, O [total_q, heads, d] */
    int64_t kv_stride_n, kv_stride_h; /* K, V [total_q, kv_heads, d] */
    int64_t page_stride_p, page_stride_h, page_stride_n;
    int64_t table_stride;
} attn_paged_desc;

typedef struct { /* DEVICE memory, caller owned */
    void *K, *V;
    uint8_t *K_exp, *V_exp;         /* ATTN_CACHE_FP8, else NULL */
    const int32_t *table, *lens, *q_ptr;
} attn_cache;

/* The new tokens' K and V into the pages; their places are overwritten, nothing else is. */
attn_status attn_cache_write(const attn_paged_desc *desc, const attn_cache *cache, const void *K, const void *V, void *stream);
/* The last tokens of every sequence (as many as q_ptr says) out of the pages into K and V, in order and dequantised. */
attn_status attn_cache_read(const attn_paged_desc *desc, const attn_cache *cache, void *K, void *V, void *stream);
/* Device scratch of attn_paged_fwd: sums of the parts into which a long cache is split when there are few rows.  0 if desc is invalid. */
size_t attn_paged_workspace_bytes(const attn_paged_desc *desc);
/* O [total_q, heads, d] and LSE, contiguous [total_q, heads] float, of the new tokens. */
attn_status attn_paged_fwd(const attn_paged_desc *desc, const attn_cache *cache, const void *Q, void *O, float *LSE,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * Trees of drafted tokens over the paged cache (speculative decoding).  The new tokens of a sequence are not one continuation but several that
 * share their beginnings: each follows the context or an earlier one of them.  The order of a step is attn_cache_write (lens counts all
 * drafted tokens), attn_tree_mask once, attn_tree_fwd for every layer, and attn_tree_commit for the branch that was accepted.
 *   parents  DEVICE int32 [total_q]: the number, among the new tokens of its sequence, of the token that a row follows; -1 (or any number that is
 *            not an earlier token's): it follows the context
 *   mask     DEVICE words [total_q] x [(max_q + 31) / 32], rows mask_stride words apart: bit u % 32 of word u / 32 of a row says that it sees new token
 *            u of its sequence.  attn_tree_mask sets the bits of a row's own token and of those that lead to it; any other bits may be set instead
 * A query sees the tokens in front of the new ones (the context) and the new ones of its mask.  The r-th of these, in their order, is at
 * position r and the query at the last one's: under a window it sees those less than `window` away from it, and the first `sinks`.  Of the context
 * the last `window` tokens and the first `sinks` are read.  A query that sees nothing: O = 0, LSE = -inf.  max_q <= 1024.
 * attn_tree_mask takes batch, total_q, max_q and q_ptr as in attn_paged_desc and attn_cache; rows of no sequence, and rows from max_q on, are not written.
 * attn_tree_fwd is attn_paged_fwd with the mask in the place of the order of the new tokens: a mask whose row t has bits 0 .. t gives what that gives
 * (not the same bits: its key tiles differ).  Its workspace is attn_tree_workspace_bytes: sums in fp32 of every workgroup that there may be, 128 rows of d (16 or 32 with few
 * rows), known from desc alone: 137 MB for 64 sequences with 64 drafted tokens, h32 k8 d = 128, 35 MB for one.  ATTN_BF16 rounds weights to bf16 as attn_paged_fwd does.
 */
attn_status attn_tree_mask(int32_t batch, int32_t total_q, int32_t max_q, const int32_t *q_ptr, const int32_t *parents, uint32_t *mask,
                           int64_t mask_stride, void *stream);
size_t attn_tree_workspace_bytes(const attn_paged_desc *desc);
attn_status attn_tree_fwd(const attn_paged_desc *desc, const attn_cache *cache, const uint32_t *mask, int64_t mask_stride, const void *Q, void *O,
                          float *LSE, void *workspace, size_t workspace_bytes, void *stream);
/* Of the new tokens those that row leaf[b] of a sequence sees stay, behind the context, in their order: their rows move there, and new_lens[b] (DEVICE
 * int32 [batch], overlaps no input) is the number of tokens that are left.  leaf[b] (DEVICE int32 [batch]) counts within the sequence's new tokens; any other
 * number, -1 say: none stays.  The slots behind the new length hold what they held.  A token whose page, or the page that it moves to, is outside the
 * cache does not move.  A page of new tokens belongs to one sequence (as attn_cache_write needs it); pages of the context may be shared.
 * Of desc the sizes of Q, O, K and V, scale and window do not matter (heads may be kv_heads).  A call with batch, heads, total_q or
 * max_q 0 has nothing to do and writes nothing, not new_lens either. */
attn_status attn_tree_commit(const attn_paged_desc *desc, const attn_cache *cache, const uint32_t *mask, int64_t mask_stride, const int32_t *leaf,
                             int32_t *new_lens, void *stream);

/*
 * Eviction from the paged cache by accumulated attention weight.  weight[b][h][j] is what the queries have paid to the token in slot j of key head h so far:
 *     out[b][h][j] = decay * in[b][h][j] + sum exp(scale <Q, K_j> - LSE)     over the new tokens that see j and the query heads of the group,
 * by attn_cache_weigh, with the visibility and the LSE of attn_paged_fwd (a query with LSE = -inf adds nothing).  Behind a tree step its new tokens are the accepted ones: Q and LSE are
 * the rows of those, which the caller brings together, with the lengths that attn_tree_commit left.  New tokens start at zero: `in` is read
 * for the tokens in front of them only, and may be NULL (zeros).  Slots below lens[b] are written, others not.  `out` may be `in` (with the same strides).
 * Every token of the cache is worked on, those of sequences without new tokens too: they keep decay times their weight.  Q and LSE (contiguous [total_q,
 * heads]) may be NULL if heads, total_q or max_q is 0; a call with batch, kv_heads or max_len 0 writes nothing.  batch * kv_heads * ceil(max_len / 32) < 2^24.
 * Arithmetic as attn_paged_fwd, weights in fp32.
 */
typedef struct { /* DEVICE memory; strides in elements, the slots' is 1 and those of batches and heads at least max_len */
    const float *in;
    float *out;
    int64_t in_stride_b, in_stride_h, out_stride_b, out_stride_h;
    float decay;      /* finite */
    int32_t reserved; /* 0 */
} attn_weights;
/* Device scratch of attn_cache_weigh: sums of the parts that many new tokens are shared out in; 256: none, and `workspace` may be NULL (so it is with
 * attn_tree_workspace_bytes and attn_evict_workspace_bytes).  0 if desc is invalid. */
size_t attn_weigh_workspace_bytes(const attn_paged_desc *desc);
attn_status attn_cache_weigh(const attn_paged_desc *desc, const attn_cache *cache, const void *Q, const float *LSE, const attn_weights *weights,
                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * attn_cache_evict: of every sequence of more than `budget` tokens each key head keeps `budget`, for itself: those at positions in front of `first`, the
 * `recent` latest ones, and of the others those with the largest weights (a tie: the lower slot; NaN is less than anything).  Kept tokens in slots from
 * `budget` on move into slots that have become free below, both in ascending order; all others stay where they are, so that what moves is as little as can
 * be.  Their weights and positions move with them.  Attention without a window does not depend on the order of the keys; under a window, slots are not
 * positions any more.
 * Positions: a token in slot s < kept[b] is at pos[b][h][s], one behind at seen[b] - lens[b] + s: slots from kept[b] on hold the latest tokens, in their order, the
 * last at position seen[b] - 1.  seen counts all tokens that the sequence has had; NULL: lens.  kept: new_lens of the last eviction; NULL: 0, and so it is
 * without pos.  weight_out and pos_out (may be NULL without pos) get the values of the tokens that stay, in slots 0 .. new_lens[b] - 1; they may be weight
 * and pos themselves, with the same strides.  new_lens[b] = min(lens[b], budget), in memory of its own.  A token whose page, or the page that it moves to, is
 * outside the cache does not move.
 * max_len - budget bounds how many tokens move, whatever the lengths are: up to 64 (a sequence that decodes, a page of tokens over its budget) a call is one launch without a workspace, beyond it
 * is two, and beyond max_len = 4096 the first has larger workgroups.  So give a tight max_len where it is known: 64 sequences of 1040 tokens, budget 1024, 14 us with max_len 1040 or 1056, 23
 * with 2048 or 4096, 30 with 8192 or more.
 * A page of a sequence that is cut down belongs to it alone: of a page that two tables name, or one table twice, copies are made first.
 * A call with batch, kv_heads or max_len 0 writes nothing.  first + recent <= budget, budget >= 1.  Of desc batch, kv_heads, d, max_len, the pages' fields, dtype and kind matter.
 */
typedef struct { /* DEVICE memory; strides in elements, that of the slots is 1 */
    int32_t budget, first, recent;
    int32_t reserved; /* 0 */
    const float *weight;
    const int32_t *pos, *kept, *seen;
    float *weight_out;
    int32_t *pos_out, *new_lens;
    int64_t stride_b, stride_h;         /* weight, pos: at least max_len */
    int64_t out_stride_b, out_stride_h; /* weight_out, pos_out: at least min(max_len, budget) */
} attn_eviction;
/* Device scratch of attn_cache_evict: the slots between which tokens move.  0 if desc or budget is invalid. */
size_t attn_evict_workspace_bytes(const attn_paged_desc *desc, int32_t budget);
attn_status attn_cache_evict(const attn_paged_desc *desc, const attn_cache *cache, const attn_eviction *eviction, void *workspace,
                             size_t workspace_bytes, void *stream);

/* Static description of a status code. */
const char *attn_status_str(attn_status s);

#ifdef __cplusplus
}
#endif
#endif /* ATTN_MI355X_H */
