/*
 * ultratex.h -- C ABI of libultratex.so: the foreground hot path of UltraTex
 * (arXiv 2609.23169) on one AMD Instinct MI355X (gfx950).
 *
 * The path: Background Token Dropping packs the foreground tokens of the
 * unified multi-view sequence (Sec. 3.2), block lists are built from a block
 * mask (Sec. 3.3, Eq. 7), block-sparse attention runs forward and backward
 * over the packed sequence (Sec. 3.3, Eq. 8), and the packed tokens are
 * written back to the full token grid (Sec. 3.2, Eq. 4; Sec. 3.4, Eq. 9).
 *
 * Conventions shared by every call:
 *  - Pointers are DEVICE pointers unless the name ends in _host.
 *  - The caller allocates and owns every buffer; the library allocates no
 *    device memory and keeps no pointer after a call returns. Buffers must
 *    stay alive until the work queued on `stream` has completed.
 *  - Every call is asynchronous on `stream` (a hipStream_t; NULL is the null
 *    stream). The only host synchronisations are the optional *_host outputs,
 *    which wait for the stream before returning.
 *  - Arguments are validated before anything is launched. On a bad argument a
 *    call returns a non-zero ut_status, launches nothing and records a message
 *    readable with ut_last_error() (per calling thread). A HIP runtime error
 *    returns UT_ERR_HIP with the HIP error text. No C++ exception crosses the
 *    ABI.
 *  - Token and block indices are int32; byte offsets are computed in 64 bits.
 *  - Block lists passed to the attention calls are trusted. With the
 *    environment variable UT_VALIDATE set (to anything but "0") those calls
 *    first copy the lists to the host, waiting for the stream, and return
 *    UT_ERR_INVALID_ARG unless every row is strictly ascending within
 *    [0, Nk) and the pointer array starts at 0 and never decreases.
 *  - bf16 is IEEE binary32 truncated to its upper 16 bits (stored as uint16),
 *    results rounded to nearest even.
 */
#ifndef ULTRATEX_H
#define ULTRATEX_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define UT_ABI_VERSION 3

typedef enum {
  UT_OK = 0,
  UT_ERR_INVALID_ARG = 1, /* null / misaligned pointer, bad size or count   */
  UT_ERR_UNSUPPORTED = 2, /* a head_dim or block size the kernels lack      */
  UT_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required     */
  UT_ERR_CAPACITY = 4,    /* an output holds fewer entries than produced    */
  UT_ERR_HIP = 5          /* a HIP runtime or launch error                  */
} ut_status;

/* Element types of the foreground step calls. */
typedef enum {
  UT_BF16 = 0,
  UT_F32 = 1
} ut_dtype;

/* Message for the last non-OK status returned on this thread ("" if none). */
const char* ut_last_error(void);

/* UT_ABI_VERSION of the loaded library. */
int ut_abi_version(void);

/* ------------------------------------------------------------------------
 * Kernel timing (a tracing aid). With tracing on, every kernel the library
 * launches is bracketed by two HIP events recorded on the stream it runs on;
 * ut_trace_read waits for those events and returns per-kernel totals in
 * first-launch order, then forgets them. Off by default. It costs two event
 * records per launch and is meant for eager launches, not graph capture.
 *
 * ut_trace_enable  on != 0 starts recording, 0 stops (records already made
 *                  stay until read). Always UT_OK.
 * ut_trace_read    consumes the records made since the last read: fills
 *                  out[0 .. min(n, max_entries)) and returns n, the number of
 *                  distinct kernels among them (entries past max_entries are
 *                  dropped; out may be NULL with max_entries = 0); -1 with
 *                  ut_last_error() set if an event could not be read (a HIP
 *                  error).
 * Names are the kernel's with its head_dim and block where it has them, e.g.
 * "bsattn_fwd<128,128>", "bwd_dkdv<128,128>", "gather_rows".
 * ---------------------------------------------------------------------- */
typedef struct {
  char name[48];
  int64_t count;      /* launches recorded */
  double total_ms;    /* summed durations */
  double min_ms;
  double max_ms;
} ut_kernel_time;
ut_status ut_trace_enable(int on);
int ut_trace_read(ut_kernel_time* out, int max_entries);

/* ------------------------------------------------------------------------
 * Background Token Dropping (Sec. 3.2, "Mask Construction and Sequence
 * Compression"): the retained set M_fg of a per-view token-grid foreground
 * mask and the Gather_{M_fg} of a full-sequence hidden state.
 *
 * fg_mask     [L] uint8, the unified sequence's token-grid masks laid out
 *             view-major then row-major; nonzero = foreground (kept).
 * x_full      [L, row_bytes] rows to gather, or NULL for the index map only.
 * row_bytes   bytes per row; a positive multiple of 16 (e.g. 3072 bf16 =
 *             6144). x_full and x_packed must be 16-byte aligned.
 * x_packed    [capacity, row_bytes] output; NULL iff x_full is NULL.
 * capacity    rows available in kept_idx and x_packed.
 * kept_idx    [capacity] int32 output: kept positions in ascending order
 *             (packed row k is full row kept_idx[k]).
 * inv_idx     [L] int32 output (NULL to skip): packed index of each position,
 *             -1 where dropped.
 * n_kept      [1] int32 device output: the number of kept positions (written
 *             even when it exceeds capacity; then only `capacity` entries are
 *             written and the host cannot tell without reading it).
 * n_kept_host optional host output: if non-NULL the call waits for the stream,
 *             stores the count, and returns UT_ERR_CAPACITY if it exceeds
 *             capacity.
 * workspace   device scratch of ut_drop_background_workspace_size(L) bytes,
 *             4-byte aligned; contents need not be initialised.
 * Errors: L < 1 or L >= 2^31, null required pointers, row_bytes not a
 *         positive multiple of 16, misalignment, capacity < 0 ->
 *         UT_ERR_INVALID_ARG; workspace too small -> UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_drop_background_workspace_size(int64_t L);
ut_status ut_drop_background(const uint8_t* fg_mask, int64_t L,
                             const void* x_full, int64_t row_bytes,
                             void* x_packed, int64_t capacity,
                             int32_t* kept_idx, int32_t* inv_idx,
                             int32_t* n_kept, int64_t* n_kept_host,
                             void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* ------------------------------------------------------------------------
 * Write-back of the packed foreground rows (Sec. 3.2, Eq. 4: only positions
 * in M_fg are updated; Sec. 3.4, Eq. 9: every other position keeps the
 * background the caller pre-filled, Gaussian noise or the tiled z_bg).
 *
 * x_packed  [n_kept, row_bytes] rows to write.
 * kept_idx  [n_kept] int32 full-sequence positions, each in [0, L); the
 *           positions must be distinct (as ut_drop_background produces).
 * row_bytes positive multiple of 16; both row buffers 16-byte aligned.
 * x_full    [L, row_bytes] in/out: row kept_idx[k] <- packed row k; rows not
 *           listed are untouched.
 * n_kept = 0 is a no-op. kept_idx contents are trusted (not range-checked).
 * ---------------------------------------------------------------------- */
ut_status ut_scatter_foreground(const void* x_packed, const int32_t* kept_idx,
                                int64_t n_kept, int64_t row_bytes, void* x_full,
                                hipStream_t stream);

/* ------------------------------------------------------------------------
 * Block index (Sec. 3.3, Eq. 7; the sets S_i of Eq. 8): from a binary block
 * mask M_c per (batch, head), the list of selected key blocks of every query
 * block (ascending j) and the transpose, the list of query blocks that select
 * each key block (ascending i), both in compressed-row form.
 *
 * block_mask [B, H, Nq, Nk] uint8, nonzero = the pair (i, j) is computed.
 * q_rowptr   [B*H*Nq + 1] int32 out: row r = (b*H + h)*Nq + i spans
 *            q_cols[q_rowptr[r] .. q_rowptr[r+1]).
 * q_cols     [cap] int32 out: key-block indices j.
 * kv_colptr  [B*H*Nk + 1] int32 out: column c = (b*H + h)*Nk + j spans
 *            kv_rows[kv_colptr[c] .. kv_colptr[c+1]).
 * kv_rows    [cap] int32 out: query-block indices i.
 * cap        entries available in q_cols and kv_rows; entries past cap are
 *            not written.
 * nnz_host   optional: if non-NULL the call waits, stores the number of
 *            nonzero mask entries, and returns UT_ERR_CAPACITY if > cap.
 * workspace  device scratch of ut_build_block_index_workspace_size(B, H, Nq,
 *            Nk) bytes. That size is 0 for every shape: the per-row and
 *            per-column counts are written straight into q_rowptr and
 *            kv_colptr and replaced by offsets in place, so the build needs
 *            no memory beyond its outputs. NULL with workspace_bytes = 0 is
 *            valid; the arguments keep the signature uniform with the other
 *            calls that take scratch.
 * Errors: any of B, H, Nq, Nk < 1, B*H > 65535, B*H*Nq*Nk >= 2^31 (the
 *         offsets are int32), null or misaligned pointers, cap < 0 ->
 *         UT_ERR_INVALID_ARG; workspace_bytes below the required size ->
 *         UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_build_block_index_workspace_size(int32_t B, int32_t H, int32_t Nq,
                                           int32_t Nk);
ut_status ut_build_block_index(const uint8_t* block_mask, int32_t B, int32_t H,
                               int32_t Nq, int32_t Nk, int32_t* q_rowptr,
                               int32_t* q_cols, int32_t* kv_colptr,
                               int32_t* kv_rows, int64_t cap, int64_t* nnz_host,
                               void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/* ------------------------------------------------------------------------
 * Block-sparse attention forward (Sec. 3.3, Eq. 5 and Eq. 8): for each
 * (batch b, head h, query block i), O_i = softmax(Q_i K_{S_i}^T * scale)
 * V_{S_i}; key blocks outside S_i are never read.
 *
 * q, k, v   bf16 [B, N, H, D] contiguous (token-major, heads interleaved:
 *           the layout of a [N, H*D] projection output), 16-byte aligned.
 * o         bf16 [B, N, H, D] output.
 * lse       fp32 [B, H, N] output: natural-log log-sum-exp of each query
 *           row's scaled scores over its retained keys; -inf for a row whose
 *           S_i is empty (its O row is 0).
 * D         head_dim, 64 or 128. block: b_q = b_kv, 64 or 128.
 * Nq = Nk = ceil(N / block); the last block may be short (keys beyond N are
 *           excluded, rows beyond N are neither computed nor stored).
 * q_rowptr, q_cols  the row lists of ut_build_block_index for [B, H, Nq, Nq].
 *           Contents are trusted: each j must lie in [0, Nq).
 * softmax_scale  the score scale, 1/sqrt(D) in the paper; must be finite
 *           and > 0 (the kernels track the running maximum of the scaled
 *           scores, which a zero or negative scale would turn into a
 *           minimum, and mask keys with -inf scores).
 * Errors: unsupported D / block, or one sample's [N, H, D] bf16 tensor of
 *         2 GiB or more -> UT_ERR_UNSUPPORTED; N < 1, B or H < 1,
 *         null or misaligned pointers, a scale that is not finite and
 *         positive -> UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
ut_status ut_bsattn_fwd(const void* q, const void* k, const void* v, void* o,
                        float* lse, int32_t B, int32_t N, int32_t H, int32_t D,
                        int32_t block, const int32_t* q_rowptr,
                        const int32_t* q_cols, float softmax_scale,
                        hipStream_t stream);

/* ------------------------------------------------------------------------
 * Block-sparse attention backward: gradients of Eq. 8 with the block mask
 * held constant (the paper's third training stage runs this attention; it
 * prints no gradient formula). With P = softmax of the retained scores:
 * dV = P^T dO, dP = dO V^T, delta = rowsum(dO o O), dS = P o (dP - delta),
 * dQ = scale dS K, dK = scale dS^T Q. No atomics: results are deterministic.
 *
 * q, k, v, o, dout  bf16 [B, N, H, D] (o and lse from ut_bsattn_fwd).
 * lse               fp32 [B, H, N].
 * dq, dk, dv        bf16 [B, N, H, D] outputs (fully overwritten).
 * q_rowptr, q_cols, kv_colptr, kv_rows  both lists of ut_build_block_index.
 * workspace         device scratch, 16-byte aligned, of at least
 *                   ut_bsattn_bwd_workspace_size(B, N, H) bytes (8 per query
 *                   row): the row log-sum-exp in log2 units and
 *                   -delta = -rowsum(dO o O) as two planes of 4 bytes per row.
 *                   Bytes past that, from the next 256-byte boundary, hold
 *                   a flag per query block (4 bytes each), a map of 4 bytes
 *                   per pair and bf16 dS tiles of 2 block^2 bytes each (32
 *                   KiB at block 128), one per retained pair in column-list
 *                   order: the dK/dV pass writes the tiles that fit, and every
 *                   query block whose tiles all fit takes dQ from them (one
 *                   product per pair); the other query blocks recompute S and
 *                   dP (three products per pair). The row and column lists
 *                   must describe the same mask, as ut_build_block_index
 *                   makes them. ut_bsattn_bwd_workspace_size_stored(B, N, H,
 *                   block, nnz) is the size at which all nnz pairs fit.
 *                   Either way the results agree to rounding (dS is bf16 in
 *                   both).
 * Errors: as ut_bsattn_fwd, plus UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_bsattn_bwd_workspace_size(int32_t B, int32_t N, int32_t H);
/* Workspace with room for the dS tiles of nnz retained pairs (the nnz of
 * ut_build_block_index); 0 for block not 64 or 128, nnz < 0 or invalid sizes. */
size_t ut_bsattn_bwd_workspace_size_stored(int32_t B, int32_t N, int32_t H,
                                           int32_t block, int64_t nnz);
ut_status ut_bsattn_bwd(const void* q, const void* k, const void* v,
                        const void* o, const void* dout, const float* lse,
                        void* dq, void* dk, void* dv, int32_t B, int32_t N,
                        int32_t H, int32_t D, int32_t block,
                        const int32_t* q_rowptr, const int32_t* q_cols,
                        const int32_t* kv_colptr, const int32_t* kv_rows,
                        float softmax_scale, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * ut_bsattn_bwd without a workspace argument, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving or
 * training loops, harnesses that forbid hipMalloc. Arguments, outputs and
 * errors are those of ut_bsattn_bwd; the call allocates nothing (no hipMalloc,
 * hipFree or allocating library routine) and runs the same kernels.
 *
 * Scratch: a built-in device array of 32 MiB per GPU, part of the library's
 * code object (loaded with it on each GPU the library runs on and held until
 * the process ends). It holds the 8 bytes per query row of the statistics
 * planes, so B*H*N may be at most 4,194,304 (e.g. 24 heads x 174,762
 * tokens); larger problems return UT_ERR_WORKSPACE and launch nothing. Every
 * call on one GPU shares that GPU's array: calls that overlap in time on one
 * GPU (concurrent streams, threads) race on it and must be serialised by the
 * caller. Each call writes every row it reads, so nothing needs clearing
 * between calls. The UT_VALIDATE list check is not applied here (it copies
 * the lists to the host and waits for the stream).
 * ---------------------------------------------------------------------- */
ut_status ut_bsattn_bwd_noalloc(const void* q, const void* k, const void* v,
                                const void* o, const void* dout,
                                const float* lse, void* dq, void* dk, void* dv,
                                int32_t B, int32_t N, int32_t H, int32_t D,
                                int32_t block, const int32_t* q_rowptr,
                                const int32_t* q_cols, const int32_t* kv_colptr,
                                const int32_t* kv_rows, float softmax_scale,
                                hipStream_t stream);

/* ------------------------------------------------------------------------
 * Variable-length batches of the two attention calls: B samples of differing
 * kept-token counts packed back to back in one launch. The paper buckets
 * training samples by their foreground token count (Sec. 4.1, Implementation
 * Details) because the count differs from asset to asset; packing lets one
 * launch serve a bucket whose counts still differ. Each sample attends only
 * within itself, with the same math as ut_bsattn_fwd / ut_bsattn_bwd.
 *
 * q, k, v, o, dout, dq, dk, dv  bf16 [T, H, D]: sample b holds tokens
 *           [cu_seqlens[b], cu_seqlens[b+1]).
 * cu_seqlens  device int32 [B + 1], 0 = cu[0] <= cu[1] <= ... <= cu[B] = T.
 * T         packed tokens (int64, below 2^31; T = 0 launches nothing).
 * max_seqlen  >= every sample's length; sizes the block grid:
 *           Nb = ceil(max_seqlen / block) blocks per sample.
 * lse       fp32 [H, T] (head-major over the packed tokens).
 * q_rowptr, q_cols (and kv_colptr, kv_rows)  lists of ut_build_block_index
 *           over a [B, H, Nb, Nb] block mask. Sample b uses its leading
 *           ceil(len_b / block) block rows and columns; list entries past
 *           them are ignored, and its last block may be short.
 * workspace (backward) at least ut_bsattn_bwd_varlen_workspace_size(T, H)
 *           bytes; past the next 256-byte boundary, dS tiles as in
 *           ut_bsattn_bwd (ut_bsattn_bwd_varlen_workspace_size_stored(B, T,
 *           max_seqlen, H, block, nnz) holds all of them).
 * Offsets are clamped to [0, T] and lengths to max_seqlen inside the
 * kernels, so bad offsets cannot reach outside the tensors; tokens covered by
 * no sample are left unwritten. With UT_VALIDATE set, cu_seqlens is checked
 * as described above (UT_ERR_INVALID_ARG otherwise).
 * Errors: as the uniform calls, with max_seqlen in the role of N.
 * ---------------------------------------------------------------------- */
ut_status ut_bsattn_fwd_varlen(const void* q, const void* k, const void* v,
                               void* o, float* lse, const int32_t* cu_seqlens,
                               int32_t B, int64_t T, int32_t max_seqlen,
                               int32_t H, int32_t D, int32_t block,
                               const int32_t* q_rowptr, const int32_t* q_cols,
                               float softmax_scale, hipStream_t stream);
size_t ut_bsattn_bwd_varlen_workspace_size(int64_t T, int32_t H);
size_t ut_bsattn_bwd_varlen_workspace_size_stored(int32_t B, int64_t T,
                                                  int32_t max_seqlen, int32_t H,
                                                  int32_t block, int64_t nnz);
ut_status ut_bsattn_bwd_varlen(const void* q, const void* k, const void* v,
                               const void* o, const void* dout,
                               const float* lse, void* dq, void* dk, void* dv,
                               const int32_t* cu_seqlens, int32_t B, int64_t T,
                               int32_t max_seqlen, int32_t H, int32_t D,
                               int32_t block, const int32_t* q_rowptr,
                               const int32_t* q_cols, const int32_t* kv_colptr,
                               const int32_t* kv_rows, float softmax_scale,
                               void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/* ------------------------------------------------------------------------
 * Top-K block selection (Sec. 3.3, Eq. 6 and Eq. 7): the block mask M_c of
 * block-sparse attention from mean-pooled query and key blocks. Per (b, h),
 * pool(X)_i is the mean of block i's token rows (a short last block averages
 * its real tokens), S_c = pool(Q) pool(K)^T, and row i of the mask keeps the
 * k_keep largest entries of S_c[i, :]. Equal scores are taken lower j first.
 * No block is forced (the diagonal included). The output feeds
 * ut_build_block_index.
 *
 * q, k        bf16 [B, N, H, D] contiguous, 16-byte aligned.
 * D           a multiple of 8, at most 512. block: >= 1.
 * k_keep      blocks kept per row, >= 1 (floor(rho N_k) in the paper; the
 *             caller computes it); k_keep >= Nk keeps every block.
 * prefix_blocks  P in [0, Nk]: leading blocks of always-kept tokens (the
 *             text tokens of the joint sequence, 512 in the paper's token
 *             counts): rows i < P keep every block, every row keeps blocks
 *             j < P, and the k_keep best blocks are chosen among j >= P.
 * block_mask  uint8 [B, H, Nk, Nk] output, Nk = ceil(N / block); 1 = kept.
 * workspace   device scratch of ut_topk_block_mask_workspace_size bytes
 *             (the pooled rows, fp32), 16-byte aligned.
 * Scores are fp32 (sums in order over tokens and over d); a row whose
 * k-th and (k+1)-th scores differ by less than the fp32 rounding of that
 * arithmetic may differ from an exact-arithmetic selection, and is then still
 * a valid Top-K of the fp32 scores. Inputs must be finite.
 * Errors: sizes < 1, D not a multiple of 8 or > 512, B > 65535, null or
 *         misaligned pointers, k_keep < 1, prefix_blocks outside [0, Nk] ->
 *         UT_ERR_INVALID_ARG; a row of
 *         scores too long for one workgroup's LDS (Nk + D > 16384) ->
 *         UT_ERR_UNSUPPORTED; workspace too small -> UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_topk_block_mask_workspace_size(int32_t B, int32_t N, int32_t H, int32_t D,
                                         int32_t block);
ut_status ut_topk_block_mask(const void* q, const void* k, int32_t B, int32_t N,
                             int32_t H, int32_t D, int32_t block, int32_t k_keep,
                             int32_t prefix_blocks, uint8_t* block_mask, void* workspace,
                             size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Foreground-only Euler update (Sec. 3.2, Eq. 4): at every retained position
 * i = kept_idx[k], z[i, :] += dt * v[k, :] with dt = t_prev - t_curr; all
 * other positions keep their values (the initial noise).
 *
 * z         fp32 [L, C] in/out, 16-byte aligned.
 * v         [n_kept, C] packed velocities, UT_BF16 or UT_F32, aligned to
 *           8 (bf16) or 16 (fp32) bytes.
 * C         channels per token, a positive multiple of 4.
 * kept_idx  [n_kept] int32, distinct positions (as ut_drop_background
 *           produces); entries outside [0, L) are skipped.
 * Each element is one fp32 fused multiply-add (one rounding). n_kept = 0 is
 * a no-op.
 * Errors: L < 1, C not a positive multiple of 4, n_kept < 0 or > L, bad
 *         dtype, non-finite dt, null or misaligned pointers ->
 *         UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
ut_status ut_euler_update_foreground(float* z, int64_t L, int64_t C, const void* v,
                                     ut_dtype v_dtype, const int32_t* kept_idx,
                                     int64_t n_kept, float dt, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Foreground flow-matching loss (Sec. 3.2, Eq. 3, with the target velocity
 * eps - z_tgt of Eq. 1-2): with i = kept_idx[k],
 *   loss = sum_{k, c} (v[k, c] - (eps[i, c] - z0[i, c]))^2 / (n_kept C)
 * (the mean over retained tokens and channels), and optionally its gradient
 *   grad[k, c] = 2 (v[k, c] - (eps[i, c] - z0[i, c])) / (n_kept C).
 *
 * v         [n_kept, C] model prediction, v_dtype.
 * eps, z0   [L, C] noise and clean target latent on the full grid, x_dtype.
 *           Rows not listed in kept_idx are never read.
 * loss      [1] fp32 device output (0 when n_kept = 0).
 * grad      [n_kept, C] fp32 device output, or NULL.
 * workspace device scratch of ut_fg_flow_loss_workspace_size() bytes,
 *           8-byte aligned (per-workgroup partial sums).
 * Differences and squares are taken in fp64 and summed in a fixed order: the
 * loss is deterministic and within a few fp64 roundings of exact before its
 * final rounding to fp32. Alignment as for ut_euler_update_foreground.
 * Errors: as ut_euler_update_foreground, plus UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_fg_flow_loss_workspace_size(void);
ut_status ut_fg_flow_loss(const void* v, ut_dtype v_dtype, const void* eps, const void* z0,
                          ut_dtype x_dtype, int64_t L, int64_t C,
                          const int32_t* kept_idx, int64_t n_kept, float* loss,
                          float* grad, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* ------------------------------------------------------------------------
 * Composite latent for foreground-aware decoding (Sec. 3.4, Eq. 9): row i of
 * z_mix is the denoised packed row inv_idx[i] where position i was retained,
 * and otherwise row i mod bg_rows of the canonical background latent z_bg
 * (one view's token grid, tile-repeated over the views).
 *
 * x_packed  [n_kept, row_bytes] packed rows (NULL allowed when n_kept = 0).
 * inv_idx   [L] int32, the inverse map of ut_drop_background: the packed
 *           index of each position, -1 where dropped. Entries outside
 *           [0, n_kept) take the background row.
 * z_bg      [bg_rows, row_bytes]. z_mix: [L, row_bytes] output (every row
 *           written). row_bytes: a positive multiple of 16; the row buffers
 *           16-byte aligned. A byte copy: any element type.
 * Errors: L < 1 or >= 2^31, bg_rows < 1, n_kept < 0 or > L, row_bytes not
 *         a positive multiple of 16, null or misaligned pointers ->
 *         UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
ut_status ut_composite_latent(const void* x_packed, int64_t n_kept,
                              const int32_t* inv_idx, int64_t L, const void* z_bg,
                              int64_t bg_rows, int64_t row_bytes, void* z_mix,
                              hipStream_t stream);

/* ------------------------------------------------------------------------
 * Token-grid foreground masks from alpha masks (Sec. 3.2, "Mask Construction
 * and Sequence Compression"): a token is foreground when any pixel of its
 * patch x patch block has alpha > threshold; the result is then dilated by a
 * (2 radius + 1)^2 square, clipped at each view's border. (The paper gives
 * neither rule; these are the readings taken.)
 *
 * alpha       uint8 [V, Hp, Wp], 16-byte aligned; Hp and Wp multiples of
 *             patch; patch a positive multiple of 16 (16 in the paper: the
 *             latent token grid is 1/16 of the image).
 * threshold   0..255. radius: 0..16 (0 = no dilation).
 * token_mask  uint8 [V, Hp / patch, Wp / patch] output, 1 = foreground.
 * workspace   ut_token_mask_workspace_size bytes (the undilated mask),
 *             unused (may be NULL) when radius = 0.
 * Errors: bad sizes, patch, threshold or radius, null or misaligned pointers
 *         -> UT_ERR_INVALID_ARG; workspace too small -> UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
size_t ut_token_mask_workspace_size(int32_t V, int32_t Hp, int32_t Wp, int32_t patch);
ut_status ut_token_mask_from_alpha(const uint8_t* alpha, int32_t V, int32_t Hp,
                                   int32_t Wp, int32_t patch, int32_t threshold,
                                   int32_t radius, uint8_t* token_mask, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Rotary positions with several axes (view, row, column; time, height, width)
 * on query and key rows, with the per-head RMS norm of queries and keys in
 * front where the model has one. Kept tokens rotate by their positions in the
 * full multi-view grid (Sec. 3.2), which they read through kept_idx.
 *
 *   pairs p = 0 .. R/2 - 1 of a head's first R = sum of the axes' sizes d_a
 *   elements; pair p is the i-th of its axis a, in the order of the axes:
 *   angle = pos[row, a] * theta^(-2 i / d_a),
 *   (u, v) -> (u cos - v sin, v cos + u sin); elements R .. D - 1 pass through.
 *   With weights, before that: x -> x / sqrt(mean(x^2) + eps) * weight per head.
 *
 * q, k       [n, Hq, D] and [n, Hk, D] rows, UT_BF16 or UT_F32 (`dtype`),
 *            16-byte aligned; Hk = 0: no keys (k, k_out ignored). A batch of
 *            B samples is n = B N rows.
 * q_out, k_out  outputs; q_out may be q and k_out k (with equal strides), and
 *            otherwise must not overlap the inputs.
 * strides_host  HOST array of the elements from token to token of {q, k, q_out,
 *            k_out}, or NULL for rows back to back; each at least H D and a
 *            multiple of 8 (bf16) or 4 (fp32). A token's heads are contiguous.
 * D          head_dim, a multiple of 8 up to 256.
 * pos        fp32 [pos_rows, n_axes] coordinates (fractions are fine).
 * token_idx  int32 [n]: token i reads row token_idx[i] (the kept_idx of
 *            ut_drop_background); an index outside [0, pos_rows) is not rotated,
 *            the norm still applies. NULL: token i reads row i mod pos_rows.
 * axis_dims_host  HOST array of the n_axes (1 to 4) sizes d_a, positive and even.
 * theta      base of the frequencies, finite and > 0.
 * pairs      UT_ROPE_NEAR: pair p is elements 2p and 2p + 1; UT_ROPE_FAR: p and
 *            p + R/2 (R a multiple of 8).
 * q_weight, k_weight  [D] norm weights (`w_dtype`), or both NULL: no norm.
 * eps        finite and > 0 where there are weights, else ignored.
 * Angles are formed in fp64 and reduced to one turn, everything else is fp32
 * with one rounding to `dtype`. n = 0 is a no-op.
 * Errors: sizes, strides, axes, theta or eps out of range, null or misaligned
 *         pointers, one weight without the other -> UT_ERR_INVALID_ARG; a
 *         head_dim outside the above, far pairs with R % 8 != 0, a stride of
 *         2^31 or more -> UT_ERR_UNSUPPORTED.
 *
 * Backward: from the gradients of q_out and k_out those of q and k, and with
 * weights those of the weights, summed over tokens and heads.
 *
 * dq_out, dk_out  gradients of the outputs, as q_out and k_out.
 * q, k       the forward's inputs; read only with weights, else may be NULL.
 * dq, dk     outputs; dq may be dq_out and dk dk_out (with equal strides).
 * strides_host  {dq_out, dk_out, q, k, dq, dk}, or NULL.
 * dq_weight, dk_weight  fp32 [D] outputs, written (not added to); required
 *            with weights (dk_weight only with Hk > 0), else ignored.
 * workspace  with weights, device scratch of ut_qk_rope_bwd_workspace_size(D)
 *            bytes, 16-byte aligned; else unused.
 * No atomics: results are deterministic. With n = 0 the weights' gradients
 * are set to 0.
 * Errors: as the forward, plus UT_ERR_WORKSPACE.
 * ---------------------------------------------------------------------- */
typedef enum {
  UT_ROPE_NEAR = 0,
  UT_ROPE_FAR = 1
} ut_rope_pairs;
ut_status ut_qk_rope_fwd(const void* q, const void* k, void* q_out, void* k_out,
                         const int64_t* strides_host, ut_dtype dtype, int64_t n, int32_t Hq,
                         int32_t Hk, int32_t D, const float* pos, int64_t pos_rows,
                         const int32_t* token_idx, const int32_t* axis_dims_host, int32_t n_axes,
                         double theta, ut_rope_pairs pairs, const void* q_weight,
                         const void* k_weight, ut_dtype w_dtype, float eps, hipStream_t stream);
size_t ut_qk_rope_bwd_workspace_size(int32_t D);
ut_status ut_qk_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k,
                         void* dq, void* dk, const int64_t* strides_host, ut_dtype dtype, int64_t n,
                         int32_t Hq, int32_t Hk, int32_t D, const float* pos, int64_t pos_rows,
                         const int32_t* token_idx, const int32_t* axis_dims_host, int32_t n_axes,
                         double theta, ut_rope_pairs pairs, const void* q_weight,
                         const void* k_weight, ut_dtype w_dtype, float eps, float* dq_weight,
                         float* dk_weight, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* ------------------------------------------------------------------------
 * Cross attention: the image tokens' queries attend to an encoder's states
 * (text, a reference image) of another length, O = softmax(Q K^T * scale) V
 * over the keys in use, every query of a sample to every key of it.
 *
 * q, o, dout, dq  bf16 [B, Nq, Hq, D]; k, v, dk, dv  bf16 [B, Nk, Hk, D]; Hq a
 *           multiple of Hk: query head h reads key head h / (Hq / Hk), whose
 *           gradients are summed over its query heads. 16-byte aligned. Outputs
 *           must not overlap inputs. Nq, Nk >= 0.
 * D         head_dim, a multiple of 8 up to 128.
 * lse       fp32 [B, Hq, Nq]: natural-log log-sum-exp of each row's scaled
 *           scores; -inf for a row without keys in use (its O row is 0, its dQ
 *           row 0).
 * strides_host  HOST array of the elements from token to token, in the order
 *           {q, k, v, o} forward and {q, k, v, o, dout, dq, dk, dv} backward, or
 *           NULL for rows back to back; each at least H D, a multiple of 8 and
 *           below 2^22. Samples follow each other: sample b starts N strides
 *           after sample b - 1. A token's heads are contiguous.
 * key_mask  uint8 [B, Nk], nonzero = in use, or NULL: all in use. Rows of k and
 *           v that are not in use may hold anything (NaN included) and get zero
 *           gradients. Any alignment.
 * softmax_scale  finite and > 0.
 * workspace device scratch of the size query's bytes (0 for most shapes of the
 *           forward: it is used where few queries meet many keys), 16-byte
 *           aligned; need not be initialised. Two calls that may run at the same
 *           time need one each.
 * No atomics: results are deterministic.
 * Errors: sizes or strides out of range, Hq % Hk != 0, 2^27 rows of a head or
 *         more (B Nq Hq, B Nk Hk), backward launches of 2^24 workgroups (B Hk
 *         ceil(Nk / 128); T H D / 1024 where work is split), null or misaligned
 *         pointers -> UT_ERR_INVALID_ARG; a head_dim outside the above, a stride of 2^22 or
 *         more -> UT_ERR_UNSUPPORTED; UT_ERR_WORKSPACE. The size queries return 0
 *         for sizes that the calls refuse.
 *
 * Backward: dS = P o (dO V^T - rowsum(dO o O)), dQ = scale dS K,
 * dK = scale dS^T Q, dV = P^T dO; o and lse from the forward.
 *
 * Variable lengths: B samples packed back to back on both sides.
 *
 * q, o, dout, dq  bf16 [Tq, Hq, D]; k, v, dk, dv  bf16 [Tk, Hk, D]; lse fp32
 *           [Hq, Tq]; key_mask uint8 [Tk] or NULL.
 * cu_seqlens_q, cu_seqlens_k  device int32 [B + 1]: sample b holds query tokens
 *           [cu_q[b], cu_q[b+1]) and key tokens [cu_k[b], cu_k[b+1]); they start
 *           at 0, never decrease and end at or before Tq and Tk. A sample may
 *           have no queries or no keys.
 * max_seqlen_q, max_seqlen_k  at least every sample's lengths.
 * zero_rest 0: rows at and past cu_seqlens[B] of the outputs are left as they
 *           were; else they are set to 0 and lse there to -inf.
 * Offsets are clamped to [0, T] and lengths to max_seqlen inside the kernels, so
 * bad offsets cannot reach outside the tensors. With UT_VALIDATE set both offset
 * arrays are checked first (UT_ERR_INVALID_ARG otherwise).
 * ---------------------------------------------------------------------- */
size_t ut_xattn_fwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk,
                                   int32_t D);
ut_status ut_xattn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                       const int64_t* strides_host, const uint8_t* key_mask, int32_t B, int32_t Nq,
                       int32_t Nk, int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                       void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t ut_xattn_fwd_varlen_workspace_size(int32_t B, int64_t Tq, int32_t max_seqlen_q,
                                          int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D);
ut_status ut_xattn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                              const int64_t* strides_host, const uint8_t* key_mask,
                              const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                              int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                              int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                              int32_t zero_rest, void* workspace, size_t workspace_bytes,
                              hipStream_t stream);
size_t ut_xattn_bwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk,
                                   int32_t D);
ut_status ut_xattn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                       const float* lse, void* dq, void* dk, void* dv, const int64_t* strides_host,
                       const uint8_t* key_mask, int32_t B, int32_t Nq, int32_t Nk, int32_t Hq,
                       int32_t Hk, int32_t D, float softmax_scale, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);
size_t ut_xattn_bwd_varlen_workspace_size(int32_t B, int64_t Tq, int64_t Tk, int32_t max_seqlen_q,
                                          int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D);
ut_status ut_xattn_bwd_varlen(const void* q, const void* k, const void* v, const void* o,
                              const void* dout, const float* lse, void* dq, void* dk, void* dv,
                              const int64_t* strides_host, const uint8_t* key_mask,
                              const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                              int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                              int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                              int32_t zero_rest, void* workspace, size_t workspace_bytes,
                              hipStream_t stream);

/* ------------------------------------------------------------------------
 * Window attention: a query sees the keys around it and a few first ones,
 * O = softmax(Q K^T * scale) V over the visible keys in use. Self attention of the
 * packed image tokens (a text prefix as the first keys), or Nq queries at the end
 * of Nk keys.
 *
 * Query i of a sample's nq sits at position p = i + nk - nq of its nk keys. Key j is
 * visible to it where
 *   p - window_left <= j <= p + window_right, or
 *   j < n_sink and (window_right > 0 or j <= p):
 * with window_right = 0 no query sees a later key, otherwise every query sees the
 * sinks. A query in front of the keys (p < 0) may see none.
 *
 * window_left, window_right  >= 0, or -1: no bound on that side.
 * n_sink    >= 0; more than the keys is as many as there are.
 * Everything else - tensors, strides_host, key_mask (keys in use, sinks
 * included), lse, workspace, packed samples, zero_rest, errors - is as in
 * ut_xattn_*. The size queries take the window too. A row without visible keys in
 * use: o = 0, lse = -inf, zero gradients. Keys that no query sees may hold
 * anything and get zero gradients; inf or NaN in a key that some query sees may reach
 * the other queries of its 128-row tile, as 0 times it (mark padding in key_mask).
 * delta = rowsum(dO o O) is formed from the stored o, except for rows that see 16
 * keys or fewer (key_mask aside), and rows of a 128-row tile whose visible keys in use
 * all lie in one 64-key tile: theirs is rowsum(P o dP) in fp32.
 * No atomics: results are deterministic. How they are rounded goes by the sizes of the
 * call (small ones carry dS with more bits), so that a sample's gradients may differ
 * in their last bits with the number of samples beside it.
 * Errors: also window_left or window_right < -1, n_sink < 0 -> UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
size_t ut_swattn_fwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk,
                                    int32_t D, int32_t window_left, int32_t window_right,
                                    int32_t n_sink);
ut_status ut_swattn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                        const int64_t* strides_host, const uint8_t* key_mask, int32_t B,
                        int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk, int32_t D,
                        int32_t window_left, int32_t window_right, int32_t n_sink,
                        float softmax_scale, void* workspace, size_t workspace_bytes,
                        hipStream_t stream);
size_t ut_swattn_fwd_varlen_workspace_size(int32_t B, int64_t Tq, int32_t max_seqlen_q,
                                           int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D,
                                           int32_t window_left, int32_t window_right,
                                           int32_t n_sink);
ut_status ut_swattn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                               const int64_t* strides_host, const uint8_t* key_mask,
                               const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                               int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                               int32_t Hq, int32_t Hk, int32_t D, int32_t window_left,
                               int32_t window_right, int32_t n_sink, float softmax_scale,
                               int32_t zero_rest, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);
size_t ut_swattn_bwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk,
                                    int32_t D, int32_t window_left, int32_t window_right,
                                    int32_t n_sink);
ut_status ut_swattn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                        const float* lse, void* dq, void* dk, void* dv, const int64_t* strides_host,
                        const uint8_t* key_mask, int32_t B, int32_t Nq, int32_t Nk, int32_t Hq,
                        int32_t Hk, int32_t D, int32_t window_left, int32_t window_right,
                        int32_t n_sink, float softmax_scale, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);
size_t ut_swattn_bwd_varlen_workspace_size(int32_t B, int64_t Tq, int64_t Tk, int32_t max_seqlen_q,
                                           int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D,
                                           int32_t window_left, int32_t window_right,
                                           int32_t n_sink);
ut_status ut_swattn_bwd_varlen(const void* q, const void* k, const void* v, const void* o,
                               const void* dout, const float* lse, void* dq, void* dk, void* dv,
                               const int64_t* strides_host, const uint8_t* key_mask,
                               const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                               int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                               int32_t Hq, int32_t Hk, int32_t D, int32_t window_left,
                               int32_t window_right, int32_t n_sink, float softmax_scale,
                               int32_t zero_rest, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/* ------------------------------------------------------------------------
 * Attention over a cache of keys and values: T tokens of each sample, the next
 * one (T = 1), a chunk of a prompt, or a tree of drafted tokens to be verified, whose
 * own keys and values are in the cache already.
 *
 * q, o      bf16 [B, T, Hq, D], T >= 1.
 * k_cache, v_cache  bf16 [B, capacity, Hk, D]. Sample b's tokens attend to slots
 *           0 .. cache_len[b] - 1 and to their own T slots behind them; what later
 *           slots hold is not used, nor those in front of every token's window. Of a
 *           slot that some token's window or sinks hold, or one of the T, inf or NaN in V
 *           may reach the sample's other tokens, hidden from them or not, as 0 times it
 *           (in K it reaches those alone that see the slot): pad drafted tokens with
 *           finite values.
 * cache_len device int32 [B]: slots in use before the T tokens, 0 .. capacity - T
 *           (clamped to that; checked first under UT_VALIDATE).
 * tree      device uint64 [B, T], T <= 64: bit u of word (b, t) set = token t sees
 *           token u's slot (its ancestors and itself); bits past T are ignored. NULL: a
 *           chain, token t sees the tokens 0 .. t.
 * window_left, n_sink  as in ut_swattn_*, with window_right = 0: token t sits at
 *           position cache_len[b] + t, in a tree behind the tokens that it sees,
 *           cache_len[b] + their number less itself. With a tree the window has to hold
 *           every drafted token, window_left >= T - 1 (or -1), and sinks count in front
 *           of cache_len[b] only.
 * lse       fp32 [B, Hq, T].
 * strides_host  HOST {q, k_cache, v_cache, o} or NULL, as in ut_xattn_fwd: sample b's
 *           slots start capacity strides after those of sample b - 1.
 * weights_in, weights_out  fp32 [B, Hk, capacity], or weights_out NULL: not wanted.
 *           weights_out[b, hk, j] = weights_in[b, hk, j] + the sum, over the T tokens and
 *           the heads of the group, of the softmax weight of slot j, for every slot (of
 *           weights_in alone where nothing sees it). weights_in NULL: zeros;
 *           weights_out may be weights_in, but not overlap it otherwise.
 * workspace as in ut_xattn_fwd, of the size query's bytes (with_weights: nonzero for
 *           a call with weights_out).
 * A token that sees no slot (a tree word of 0 in front of an empty cache): o = 0,
 * lse = -inf. No atomics: results are deterministic.
 * Errors: those of ut_xattn_fwd; T < 1 or > capacity, a tree with T > 64 or
 *         0 <= window_left < T - 1, weights_in without weights_out or overlapping it,
 *         launches of 2^32 threads (never below 2^21 sample-heads, B Hk)
 *         -> UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
size_t ut_cache_attn_workspace_size(int32_t B, int32_t T, int32_t capacity, int32_t Hq, int32_t Hk,
                                    int32_t D, int32_t window_left, int32_t n_sink,
                                    int32_t with_weights);
ut_status ut_cache_attn(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                        const int64_t* strides_host, const int32_t* cache_len, const uint64_t* tree,
                        const float* weights_in, float* weights_out, int32_t B, int32_t T,
                        int32_t capacity, int32_t Hq, int32_t Hk, int32_t D, int32_t window_left,
                        int32_t n_sink, float softmax_scale, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * The weights alone, of some of the tokens: after a tree has been verified, those
 * that were accepted.
 *
 * q, k_cache, lse, cache_len, tree, window_left, n_sink, softmax_scale  of the
 *           ut_cache_attn call, lse its output.
 * strides_host  HOST {q, k_cache} or NULL.
 * tokens    device uint64 [B], T <= 64: bit t of word b set = token t counts. NULL: all.
 * Errors: as above; tokens with T > 64 -> UT_ERR_INVALID_ARG.
 * ---------------------------------------------------------------------- */
ut_status ut_cache_weights(const void* q, const void* k_cache, const float* lse,
                           const int64_t* strides_host, const int32_t* cache_len,
                           const uint64_t* tree, const uint64_t* tokens, const float* weights_in,
                           float* weights_out, int32_t B, int32_t T, int32_t capacity, int32_t Hq,
                           int32_t Hk, int32_t D, int32_t window_left, int32_t n_sink,
                           float softmax_scale, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Eviction: of each sample and key head the slots that stay, by the weight that
 * they have received, moved together into another cache.
 *
 * With n = cache_len[b] slots in use: all of them where n <= n_keep. Otherwise the first
 * n_sink, the last n_recent, and of those between them the n_keep - n_sink -
 * n_recent with the largest weights; of equal weights the lower slots stay, -0 counts
 * as 0, and NaN is below every number. The kept slots keep their order.
 *
 * k_cache, v_cache  bf16 [B, capacity, Hk, D]; k_out, v_out [B, capacity_out, Hk, D].
 * weights   fp32 [B, Hk, capacity]; weights_out [B, Hk, capacity_out]: the kept
 *           slots' weights, then zeros.
 * cache_len device int32 [B] (clamped to [0, capacity]; checked first under
 *           UT_VALIDATE); len_out int32 [B]: min(cache_len, n_keep).
 * kept_idx  int32 [B, Hk, n_keep]: the slots that stay, ascending, then -1.
 * strides_host  HOST {k_cache, v_cache, k_out, v_out} or NULL, as in ut_xattn_fwd.
 * zero_rest 0: rows of k_out and v_out at and past n_keep are left as they were;
 *           else they are set to 0. Rows from len_out to n_keep are set to 0 always.
 * n_keep >= 1, n_sink >= 0, n_recent >= 0, n_sink + n_recent <= n_keep <=
 * capacity_out; B < 65536. Outputs must not overlap inputs or each other (checked; k_out
 * and v_out may be interleaved views of one buffer, of one stride).
 * Errors: sizes (2^27 rows of K or V of a head, 2^24 rows of weights, or more),
 *         strides, null or misaligned pointers, overlap
 *         -> UT_ERR_INVALID_ARG; a head_dim that is no multiple of 8 up to 128, a
 *         stride of 2^22 or more -> UT_ERR_UNSUPPORTED.
 * ---------------------------------------------------------------------- */
ut_status ut_cache_evict(const void* k_cache, const void* v_cache, const float* weights,
                         const int32_t* cache_len, void* k_out, void* v_out, float* weights_out,
                         int32_t* len_out, int32_t* kept_idx, const int64_t* strides_host, int32_t B,
                         int32_t capacity, int32_t capacity_out, int32_t Hk, int32_t D,
                         int32_t n_keep, int32_t n_sink, int32_t n_recent, int32_t zero_rest,
                         hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ULTRATEX_H */
