/*
 * b2sp -- SPMM, SDDMM and FusedMM over a CSR sparsity pattern S on NVIDIA B200 (sm_100a).
 *
 * C ABI.  Plain pointers and sizes only; `stream` is a cudaStream_t passed as void*
 * (NULL = the legacy default stream).
 *
 * Storage (paper, section "Matrix Storage Layout", Fig. 1):
 *   S  is M x K in compressed sparse row form: row_ptr[M+1], col_idx[nnz], values[nnz];
 *      int32, 0-based; row i owns positions row_ptr[i] <= p < row_ptr[i+1].  Any valid CSR is
 *      accepted: rows may be empty, and the column indices of a row need be neither sorted
 *      nor unique (each stored entry is its own term and its own SDDMM output slot).
 *   Dense operands are fp32, row-major, with a leading dimension counted in elements
 *      (ld >= number of columns).
 *   Names: the paper's (A, I_A; C; B; D; E) are here (S; A; B; D; O); its single letter N is
 *      split into Kd (length of the sampled dot product) and N (width of D and O).
 *
 * Conventions for the device entry points (b2sp_spmm, b2sp_sddmm, b2sp_fusedmm):
 *   - every data pointer is a DEVICE pointer on the current device; the caller owns all of
 *     them, including the workspace; the library allocates nothing;
 *   - inputs are read-only; outputs are fully overwritten (never accumulated into; an empty
 *     row gives a zero output row, Alg. 2 line 1);
 *   - the call enqueues kernels on `stream` and returns without synchronising; it may be captured
 *     into a CUDA graph (make one ordinary call first: it does the library's one-time driver queries);
 *   - `workspace` is scratch of at least b2sp_workspace_bytes(...) bytes, 256-byte aligned;
 *     its contents are overwritten by every call, so two calls that may overlap in time on
 *     the GPU (different streams) need different workspaces, and so do calls that two host threads
 *     make at once on one stream (their kernels may take turns);
 *   - argument errors are reported synchronously with no kernel launched; a launch failure
 *     is reported as B2SP_ERR_CUDA; nothing traps, asserts or exits.
 *   - M = 0, nnz = 0 and zero widths are valid (outputs of the stated size are zero-filled).
 *
 * `algo` selects the kernel family:
 *   B2SP_ALGO_AUTO     the library chooses (fastest family whose preconditions hold);
 *   B2SP_ALGO_ROW      CUDA-core row kernels, rows taken longest-first (binned by length);
 *   B2SP_ALGO_ROW_NAT  the same kernels, rows in natural order (no binning pass);
 *   B2SP_ALGO_TILE     dense-tile tensor-core kernels (tcgen05 + tensor memory, every operand
 *                      split into two tf32 numbers so that fp32 accuracy is kept).  A pre-pass
 *                      over col_idx builds a table of 32-column windows; it also detects rows
 *                      whose columns are not strictly increasing, in which case the row kernels
 *                      produce the result instead (decided on the device, inside the same call).
 *                      B2SP_ERR_UNSUPPORTED if the sizes are outside the family (SDDMM/FusedMM:
 *                      Kd > 128), B2SP_ERR_WORKSPACE if the workspace is too small for it.
 *   B2SP_ALGO_TILE_PREPARED  as TILE, but the window table is taken from the workspace, where an
 *                      earlier b2sp_prepare_pattern call for the same S left it (see there).
 * Floating-point results of the families differ in summation order only; all stay within
 * |x - exact| <= 1e-5 * sum|terms| + 1e-6.
 *
 * Non-finite inputs.  The row kernels touch exactly the entries Eq. 1-3 name and follow IEEE
 * propagation.  The dense-tile kernels multiply whole windows of S, positions without a stored entry
 * included (by zero), so they only run when every element of A, B and D -- referenced by a stored
 * entry or not -- is finite and small enough for its tf32 hi part to be finite (|x| below about
 * 3.4e38 * (1 - 2^-11)): the operand pre-pass of every call checks this on the device, and otherwise
 * the row kernels produce that call's result (the check is per call and costs no extra launch).
 * Not checked, and undefined (NaN or Inf) on the dense-tile kernels: stored values s_p that are not
 * finite, and inputs so large that a dot product A_i . B_j overflows fp32 at ANY position (i, j) of
 * S, stored or not (the dense-tile kernels form all of them).
 */
#ifndef B2SP_H
#define B2SP_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    B2SP_OK = 0,
    B2SP_ERR_INVALID_ARG = 1, /* negative size, NULL required pointer, ld < width, nnz > 2^31-1 */
    B2SP_ERR_UNSUPPORTED = 2, /* explicit algo whose preconditions do not hold */
    B2SP_ERR_BAD_CSR = 3,     /* b2sp_validate_csr: row_ptr not monotone / col_idx out of range */
    B2SP_ERR_CUDA = 4,        /* a CUDA runtime call or a kernel launch failed */
    B2SP_ERR_WORKSPACE = 5,   /* workspace NULL, misaligned or too small */
    B2SP_ERR_TIMEOUT = 6,     /* a bounded device-side wait expired (reported by b2sp_device_status) */
    B2SP_ERR_TOO_LARGE = 7    /* the problem does not fit the library's built-in scratch array */
} b2sp_status;

enum { B2SP_ALGO_AUTO = 0, B2SP_ALGO_ROW = 1, B2SP_ALGO_ROW_NAT = 2, B2SP_ALGO_TILE = 3,
       B2SP_ALGO_TILE_PREPARED = 4 };
enum { B2SP_OP_SPMM = 0, B2SP_OP_SDDMM = 1, B2SP_OP_FUSEDMM = 2 };

/* Library version (major*10000 + minor*100 + patch). */
int b2sp_version(void);

/* Static, human-readable name of a status code. */
const char *b2sp_status_string(b2sp_status s);

/*
 * Bytes of device workspace an op needs for the given sizes: an upper bound over all algo values
 * the sizes allow (always a multiple of 256, never 0).  `op` is one of B2SP_OP_*.  Unused sizes
 * (Kd for SPMM, N for SDDMM) may be 0.  Returns 0 on invalid arguments.
 */
size_t b2sp_workspace_bytes(int op, int M, int K, int Kd, int N, long long nnz);

/*
 * The same for one algo value: B2SP_ALGO_AUTO gives what the automatic choice will use (the row
 * family's few bytes per row when it would not pick the dense-tile family), B2SP_ALGO_ROW /
 * B2SP_ALGO_ROW_NAT the row family's size, B2SP_ALGO_TILE / B2SP_ALGO_TILE_PREPARED the dense-tile
 * family's (0 if these sizes are outside that family).  Returns 0 on invalid arguments.
 */
size_t b2sp_workspace_bytes_algo(int op, int algo, int M, int K, int Kd, int N, long long nnz);

/*
 * Pattern analysis shared by the dense-tile kernels of all three ops (work assignment and index
 * staging: where the paper's kernels cut each row's ja array into blocks of VLC = 32 entries on the
 * fly, this library cuts each row into windows of 32 columns once).  Builds, in `workspace`, the
 * table of (first position, occupancy mask) per row and window from row_ptr / col_idx and records
 * which arrays it was built from.  Any later b2sp_spmm / b2sp_sddmm / b2sp_fusedmm call with
 * algo = B2SP_ALGO_TILE_PREPARED, the same workspace and the same M, K, nnz, row_ptr, col_idx
 * skips its own pre-pass.  The caller promises that the contents of row_ptr and col_idx did not
 * change in between; a workspace that does not hold a matching table (never prepared, prepared for
 * another S, or used by a B2SP_ALGO_ROW call since) is detected on the device and the row kernels
 * produce the result instead.  `workspace` must be at least as large as b2sp_workspace_bytes says
 * for the ops that will use it.  Asynchronous on `stream`.
 */
b2sp_status b2sp_prepare_pattern(int M, int K, long long nnz, const int *row_ptr, const int *col_idx,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * SPMM, Eq. 2 / Alg. 2 (SPMM-ROW):  O[i, :] = sum over stored entries (s, k) of row i of
 * s * D[k, :].
 *   M, K, N     S is M x K, D is K x N, O is M x N
 *   nnz         number of stored entries (= row_ptr[M])
 *   row_ptr, col_idx, values   CSR of S (device, read-only)
 *   D, ldd      dense K x N (device, read-only), leading dimension >= N
 *   O, ldo      dense M x N (device, written), leading dimension >= N; must not alias an input
 */
b2sp_status b2sp_spmm(int M, int K, int N, long long nnz,
                      const int *row_ptr, const int *col_idx, const float *values,
                      const float *D, long long ldd, float *O, long long ldo,
                      void *workspace, size_t workspace_bytes, int algo, void *stream);

/*
 * SDDMM, Eq. 1 / Alg. 1 (SDDMM-ROW), with the sampled value scaled by the stored one:
 *   out_values[p] = s_p * sum_{l < Kd} A[i, l] * B[j, l]   for the p-th stored entry (i, j).
 * The paper samples with an all-ones pattern; pass s_values = NULL for that (s_p = 1).
 * The result's sparsity pattern is S's: row_ptr and col_idx are not modified and out_values
 * follows the order of col_idx.
 *   A, lda      dense M x Kd (device, read-only);  B, ldb  dense K x Kd (device, read-only)
 *   out_values  nnz floats (device, written); may be the same pointer as s_values
 *               (in-place, as the paper overwrites its avalues array)
 */
b2sp_status b2sp_sddmm(int M, int K, int Kd, long long nnz,
                       const int *row_ptr, const int *col_idx, const float *s_values,
                       const float *A, long long lda, const float *B, long long ldb,
                       float *out_values,
                       void *workspace, size_t workspace_bytes, int algo, void *stream);

/*
 * FusedMM, Eq. 3 / Alg. 3 (FusedMM-ROW):  O = (S .* (A * B^T)) * D, i.e. the SDDMM values of a
 * row are consumed by the SPMM sweep of the same row without being written to global memory.
 * (One exception, a measured trade: the dense-tile family recomputes the sampled values once per
 * 128-column tile of O, so with N > 256 -- and with 128 < N <= 256 when Kd > 64 and S has at least
 * 3e7 cells -- it writes them once into the workspace and runs its SPMM stage on them, inside the same
 * call.)  s_values may be NULL (all ones).  Arguments as in the two ops above.
 */
b2sp_status b2sp_fusedmm(int M, int K, int Kd, int N, long long nnz,
                         const int *row_ptr, const int *col_idx, const float *s_values,
                         const float *A, long long lda, const float *B, long long ldb,
                         const float *D, long long ldd, float *O, long long ldo,
                         void *workspace, size_t workspace_bytes, int algo, void *stream);

/*
 * The three ops with bfloat16 dense operands and fp32 accumulation -- the variant the paper's conclusion
 * names as its next step.  A, B and D are bfloat16 (the upper 16 bits of an fp32 value; pointers passed as
 * const void*, leading dimensions in elements); the stored values of S, all sums and the outputs stay fp32.
 * Everything else (CSR conventions, workspace from b2sp_workspace_bytes, algo, prepared pattern tables,
 * stream, error behaviour) is as for the fp32 entry points above.  Results satisfy the same bound against
 * Eq. 1-3 evaluated exactly on the bfloat16 values: every product of two bfloat16 numbers is exact in
 * fp32, only the order of the fp32 sums differs.  The row kernels gather half the bytes per dense row;
 * the dense-tile kernels need no lo halves for operands that are exact in tf32, i.e. one tensor-core
 * product per GEMM1 term instead of three and two per GEMM2 term.  The row kernels load
 * four elements at a time where every operand's address, width and leading dimension is a multiple of
 * four elements, two where all are even, single ones otherwise (A on the dense-tile kernels: eight-element
 * loads where it is 16-byte aligned with a leading dimension that is a multiple of 8).
 */
b2sp_status b2sp_spmm_bf16(int M, int K, int N, long long nnz,
                           const int *row_ptr, const int *col_idx, const float *values,
                           const void *D, long long ldd, float *O, long long ldo,
                           void *workspace, size_t workspace_bytes, int algo, void *stream);
b2sp_status b2sp_sddmm_bf16(int M, int K, int Kd, long long nnz,
                            const int *row_ptr, const int *col_idx, const float *s_values,
                            const void *A, long long lda, const void *B, long long ldb,
                            float *out_values,
                            void *workspace, size_t workspace_bytes, int algo, void *stream);
b2sp_status b2sp_fusedmm_bf16(int M, int K, int Kd, int N, long long nnz,
                              const int *row_ptr, const int *col_idx, const float *s_values,
                              const void *A, long long lda, const void *B, long long ldb,
                              const void *D, long long ldd, float *O, long long ldo,
                              void *workspace, size_t workspace_bytes, int algo, void *stream);

/*
 * FusedMM (Eq. 3 / Alg. 3) on a batch of independent problems of the same sizes in one call -- the rows
 * of Alg. 3 are independent work units, and so are whole problems: e.g. the (batch x heads) problems of
 * sparse attention, O_b = (S_b .* (Q_b * K_b^T)) * V_b.  One pattern pre-pass, one operand pre-pass and one
 * kernel launch cover all problems (CTAs of all problems are in flight together).
 *   batch            number of problems (>= 1)
 *   M, K, Kd, N      sizes of every problem, as for b2sp_fusedmm
 *   row_ptr, row_ptr_stride   problem b's row pointers are row_ptr + b * row_ptr_stride (M + 1 of them,
 *                    starting at 0: positions count inside the problem's own col_idx array);
 *                    row_ptr_stride >= M + 1, or 0 when all problems share one pattern
 *   col_idx, s_values, nnz_stride   problem b's column indices (and stored values, if s_values is not
 *                    NULL) are col_idx + b * nnz_stride (s_values + b * nnz_stride); nnz_stride is at least
 *                    every problem's entry count (row_ptr_b[M]); with a shared pattern pass nnz_stride = that
 *                    count for the size queries and the family choice -- then s_values is shared too
 *                    (stride 0 is taken when row_ptr_stride is 0)
 *   A, lda, stride_a (and B, D, O likewise)   problem b's operand is A + b * stride_a, row-major with
 *                    leading dimension lda; an input's stride may be 0 (operand shared by all problems);
 *                    outputs must not overlap: stride_o >= (M - 1) * ldo + N
 * Workspace: b2sp_workspace_bytes_batched(...) bytes.  algo as for b2sp_fusedmm; B2SP_ALGO_ROW and
 * B2SP_ALGO_ROW_NAT both take the rows in natural order; B2SP_ALGO_TILE_PREPARED needs a table built by
 * b2sp_prepare_pattern_batched with the same batch, M, K, nnz_stride, row_ptr, row_ptr_stride and col_idx.
 * B2SP_ALGO_AUTO chooses the family from the density nnz_stride / (M * K).  Outputs wider than 256
 * columns (where a single problem takes two phases, see b2sp_fusedmm) run on the row kernels.
 * Every other convention (device pointers, asynchronous on `stream`, outputs overwritten, patterns that
 * are not strictly sorted handled by the row kernels inside the same call) is b2sp_fusedmm's.
 */
size_t b2sp_workspace_bytes_batched(int batch, int M, int K, int Kd, int N, long long nnz_stride);
b2sp_status b2sp_prepare_pattern_batched(int batch, int M, int K, long long nnz_stride, const int *row_ptr,
                                         long long row_ptr_stride, const int *col_idx, void *workspace,
                                         size_t workspace_bytes, void *stream);
b2sp_status b2sp_fusedmm_batched(int batch, int M, int K, int Kd, int N, long long nnz_stride,
                                 const int *row_ptr, long long row_ptr_stride, const int *col_idx,
                                 const float *s_values, const float *A, long long lda, long long stride_a,
                                 const float *B, long long ldb, long long stride_b, const float *D, long long ldd,
                                 long long stride_d, float *O, long long ldo, long long stride_o, void *workspace,
                                 size_t workspace_bytes, int algo, void *stream);
/* The same with bfloat16 A, B, D (see b2sp_fusedmm_bf16): e.g. sparse attention on bfloat16 Q, K, V. */
b2sp_status b2sp_fusedmm_batched_bf16(int batch, int M, int K, int Kd, int N, long long nnz_stride,
                                      const int *row_ptr, long long row_ptr_stride, const int *col_idx,
                                      const float *s_values, const void *A, long long lda, long long stride_a,
                                      const void *B, long long ldb, long long stride_b, const void *D, long long ldd,
                                      long long stride_d, float *O, long long ldo, long long stride_o, void *workspace,
                                      size_t workspace_bytes, int algo, void *stream);

/*
 * Attention over a CSR pattern, forward and backward: FusedMM with a softmax over each row of sampled products,
 *
 *   O_i = sum_j p_ij V_j,   p_ij = exp(scale Q_i . K_j - lse_i),   lse_i = log sum_j exp(scale Q_i . K_j),
 *
 * the sums over the columns j that row i of the pattern stores.  A row that stores nothing (or whose products are all
 * -inf) gives a zero row of O and lse_i = -inf.  Only stored positions count: what Q, K, V or dO hold in rows that no
 * entry names, NaN and infinities too, does not enter the results.  (By tiles, see below, bfloat16 results can move by their own rounding with it, fp32
 * ones keep their bits while it is finite.  Rows that meet a NaN or an infinity in a tile, stored or not, are taken entry by entry there, a warp
 * each: right, but slow.  Padding is best zeros.)
 *
 * batch x heads problems of the same sizes; heads / kv_heads neighbouring query heads share one head of K and V.  The pattern (M x K, no
 * stored values) belongs to all problems (patterns = 1), to a sequence (patterns = batch) or to a problem (patterns =
 * batch * heads, sequence by sequence); pattern p has its row pointers, counted from 0, at row_ptr + p * row_ptr_stride and its
 * column indices at col_idx + p * nnz_stride; nnz_stride >= every row_ptr_p[M].
 * Operands are b2sp_heads: element (b, h, i, e) of a [batch][heads][rows][d] operand is data[b * stride_batch + h * stride_head +
 * i * ld + e], strides in elements; an input's strides may be 0, the elements of an output must not overlap, nor lie in an input.  Q, O, dO, dQ have `heads`
 * heads of M rows; K, V, dK, dV have kv_heads heads of K rows.  lse is fp32 [batch][heads][M].  d <= 256.
 * The fp32 entry points take and give fp32; the _bf16 ones bfloat16 (lse, sums and softmax statistics stay fp32).
 *
 * Patterns that more than one call uses are analysed once: b2sp_attention_count_tiles says how many 128 x 128 tiles hold an entry
 * (it synchronises `stream`), b2sp_attention_plan_bytes how much device memory a plan of that many takes, and
 * b2sp_attention_prepare builds it there.  The problem names the plan and the pattern it was built from, whose contents must not have
 * changed.  The backward pass needs a plan; the forward pass without one takes the row kernels (each stored entry is its own term
 * then), which suits a pattern that is used once.  A plan needs distinct columns in each row, in any order, and at most
 * 4194304 columns; b2sp_attention_plan_status (which synchronises) reports B2SP_ERR_BAD_CSR for a plan whose pattern has a column twice in
 * a row, a column out of range or row pointers that are not monotone within [0, nnz_stride]: such a plan must not be used.
 *
 * algo: B2SP_ALGO_ROW = CUDA-core row kernels (any sizes and alignment); B2SP_ALGO_TILE = tcgen05 kernels over the tiles of the plan, for
 * scale > 0 and
 *   bfloat16: d <= 128; where d is a multiple of 8 every operand's address and strides have to be multiples of 16 bytes (other widths are
 *             copied into the workspace).  The weights p (and, backward, p (dp - delta)) are rounded to bfloat16 before the second
 *             products, as the operands are; the row kernels do not round them.
 *   fp32:     d <= 128, any alignment; above 64 the products of the tiles lie in the workspace, 64 KB a tile and problem (backward 128), up to
 *             2 GB of them.  Every number is taken apart into three bfloat16 numbers that add up to it (below about 2^-110 the last one
 *             loses bits); products keep what is above 2^-23 of each term.
 * B2SP_ERR_UNSUPPORTED otherwise.  B2SP_ALGO_AUTO chooses by the number of entries and tiles.
 * Results do not depend on the order in which anything runs: the same call gives the same bits.
 * workspace: b2sp_attention_workspace_bytes bytes, as for the ops above (b2sp_device_status reads it too).
 */
typedef struct { void *data; long long ld, stride_head, stride_batch; } b2sp_heads;
typedef struct {
    int batch, heads, kv_heads, M, K, d, patterns;
    float scale;
    const int *row_ptr; long long row_ptr_stride;
    const int *col_idx; long long nnz_stride;
    const void *plan;        /* NULL: none */
    long long plan_tiles;    /* what b2sp_attention_count_tiles said */
} b2sp_attention_problem;
/* workspace: 256 bytes; tiles_host: HOST pointer.  Synchronises `stream`. */
b2sp_status b2sp_attention_count_tiles(int patterns, int M, int K, long long nnz_stride, const int *row_ptr, long long row_ptr_stride,
                                       const int *col_idx, void *workspace, size_t workspace_bytes, long long *tiles_host,
                                       void *stream);
/* 0 on invalid arguments. */
size_t b2sp_attention_plan_bytes(int patterns, int M, int K, long long nnz_stride, long long tiles);
b2sp_status b2sp_attention_prepare(int patterns, int M, int K, long long nnz_stride, const int *row_ptr, long long row_ptr_stride,
                                   const int *col_idx, long long tiles, void *plan, size_t plan_bytes, void *stream);
b2sp_status b2sp_attention_plan_status(const void *plan, void *stream);
/* Bytes for the forward (backward = 0) or the backward call of a type, whatever algo; 0 on invalid arguments. */
size_t b2sp_attention_workspace_bytes(const b2sp_attention_problem *problem, int backward);
size_t b2sp_attention_workspace_bytes_bf16(const b2sp_attention_problem *problem, int backward);
b2sp_status b2sp_attention(const b2sp_attention_problem *problem, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                           const b2sp_heads *O, float *lse, void *workspace, size_t workspace_bytes, int algo, void *stream);
b2sp_status b2sp_attention_bf16(const b2sp_attention_problem *problem, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                                const b2sp_heads *O, float *lse, void *workspace, size_t workspace_bytes, int algo, void *stream);
/*
 * dQ, dK, dV of sum(O * dO) from O and lse as the forward call left them; the probabilities are computed again, never stored.
 *   delta_i = dO_i . O_i;  ds_ij = p_ij (dO_i . V_j - delta_i);  dQ_i = scale sum_j ds_ij K_j;  dK_j = scale sum_i ds_ij Q_i;
 *   dV_j = sum_i p_ij dO_i
 * dK and dV of a shared head are summed over its query heads (and only over the sequences of its own b: with inputs shared by
 * stride 0 the caller adds the gradients up).
 */
b2sp_status b2sp_attention_backward(const b2sp_attention_problem *problem, const b2sp_heads *Q, const b2sp_heads *K, const b2sp_heads *V,
                                    const b2sp_heads *O, const float *lse, const b2sp_heads *dO, const b2sp_heads *dQ,
                                    const b2sp_heads *dK, const b2sp_heads *dV, void *workspace, size_t workspace_bytes, int algo,
                                    void *stream);
b2sp_status b2sp_attention_backward_bf16(const b2sp_attention_problem *problem, const b2sp_heads *Q, const b2sp_heads *K,
                                         const b2sp_heads *V, const b2sp_heads *O, const float *lse, const b2sp_heads *dO,
                                         const b2sp_heads *dQ, const b2sp_heads *dK, const b2sp_heads *dV, void *workspace,
                                         size_t workspace_bytes, int algo, void *stream);

/*
 * A cache of keys or values in 4 bits, and attention over it: the serving form of the above.
 *
 * A cache has heads x slots rows of d elements in G = ceil(d / 32) groups of 32 neighbours.  Row (h, slot): 16 G bytes of codes at
 * codes + h * code_stride_head + slot * code_ld, G bfloat16 scales at scales + h * scale_stride_head + slot * scale_ld (elements).
 *   scale s = bf16(max |x| / 7) of the group; code = clamp(rint(x / s), -7, 7) + 8 (8 if s = 0), half to even throughout;
 *   halfword g G + c of the codes (g = 0..7, c = 0..G-1) holds elements 32 c + 4 g + {0, 1, 2, 3}, the first in the lowest four bits.
 * A group with a NaN or an infinity gets the scale NaN, and reads as NaN.  codes: 16-byte aligned address and strides.  scales: address a multiple
 * of 4 bytes (8 for G = 4); strides multiples of G elements where G is 2 or 4.  Strides of 2^32 and more (bytes of codes, elements of all else;
 * b2sp_attention_kv4: a row's of 2^31) are B2SP_ERR_UNSUPPORTED.
 *
 * b2sp_kv4_write quantises X[tokens][heads][d] (ld, stride_head) into the rows `slots` (device, one per token); a slot outside [0, cache
 * slots) is skipped (padding), and of several tokens with one slot the last one's row stays.  Up to 1024 tokens need no workspace.
 * b2sp_kv4_read gives the rows back, rounded once to the output type; slots outside the cache read as zeros.
 * b2sp_attention_kv4: M query tokens, each with its own list of slots: row_ptr[M+1] (from 0), col_idx = slots (each stored one is its own term; those
 * outside the cache are left out, as are entries from nnz on), O and lse as for b2sp_attention with lse[M][heads]; Q, O: token i, head h at data + i * ld +
 * h * stride_head, bfloat16; d <= 128; heads / kv_heads neighbouring query heads share a head of the caches.  A weight times the scale of its
 * value's group is rounded to eleven bits before the second product (weights below 2^-14 of the row's largest: to within 2^-25 of that largest
 * one), whatever the scales; everything else is fp32.
 * Any M, but made for few tokens with long rows: a row is cut into parts when there are few.
 */
typedef struct {
    void *codes; long long code_ld, code_stride_head;
    void *scales; long long scale_ld, scale_stride_head;
    int slots;
} b2sp_kv4;
size_t b2sp_kv4_write_workspace_bytes(int tokens, int slots);   /* 0 on invalid arguments */
b2sp_status b2sp_kv4_write(int tokens, int heads, int d, const float *X, long long ld, long long stride_head, const int *slots,
                           const b2sp_kv4 *cache, void *workspace, size_t workspace_bytes, void *stream);
b2sp_status b2sp_kv4_write_bf16(int tokens, int heads, int d, const void *X, long long ld, long long stride_head, const int *slots,
                                const b2sp_kv4 *cache, void *workspace, size_t workspace_bytes, void *stream);
b2sp_status b2sp_kv4_read(int tokens, int heads, int d, const int *slots, const b2sp_kv4 *cache, float *X, long long ld,
                          long long stride_head, void *stream);
b2sp_status b2sp_kv4_read_bf16(int tokens, int heads, int d, const int *slots, const b2sp_kv4 *cache, void *X, long long ld,
                               long long stride_head, void *stream);
size_t b2sp_attention_kv4_workspace_bytes(int M, int heads, int kv_heads, int d, long long nnz);
b2sp_status b2sp_attention_kv4(int M, int heads, int kv_heads, int d, long long nnz, const int *row_ptr, const int *col_idx,
                               const void *Q, long long ldq, long long stride_head_q, const b2sp_kv4 *keys, const b2sp_kv4 *values,
                               float scale, void *O, long long ldo, long long stride_head_o, float *lse, void *workspace,
                               size_t workspace_bytes, void *stream);

/*
 * A cache of keys or values in pages, in the operands' own type (fp32, or bfloat16 in the _bf16 forms), for serving.
 *
 * A cache has `pages` pages of `page` rows for each of kv_heads heads: row r of page c, head h begins at element
 * c * stride_page + h * stride_head + r * ld of data; data and all strides are multiples of 16 bytes (so rows of any width d are padded to that; what lies
 * behind d is neither used nor changed).  Request r's position p lies in row p % page of page entries[r * ld + p / page] of its tables (b2sp_page_tables:
 * requests x width entries); an entry outside [0, pages) stands for no page: nothing is written there, and its positions are left out.
 * A token i of a call belongs to request rows[i] (rows = NULL: to request i) and sees its first seen[i] positions, as many as the table reaches; a
 * token whose request is not in [0, requests) sees nothing.  Lengths below 0 count as 0.  All of these numbers are on the device; the host gives sizes only.
 * Results do not depend on the order in which anything runs.
 *
 * b2sp_paged_tables makes a step's tables.  Request r has lengths[r] positions and gets max(added[r], 0) more; added[r] < 0: it ends.
 *   free_pages, free_room, free_count: a stack of the pages that no request has, free_count (device) of them in free_pages[0 .. free_room).  The pages
 *     of the requests that end are pushed in order of requests (those beyond free_room are lost), then the pages that are missing are popped and entered
 *     in the tables, again in order of requests.  Popped pages stay in the array, and entries of requests that end stay in the tables.
 *   lengths_out[requests]: positions after the step.  row_ptr[requests + 1]: prefix sums of the new tokens (2^31 - 1 at most, as all sums here).
 *   rows, seen, slots (tokens of each: the step's room): of each new token its request, its position + 1, and its slot, page * (rows of a page) + row, as
 *     b2sp_kv4_write and b2sp_attention_kv4 count slots.  No page for it: seen = 0, slot = -1.  Behind the last token: -1, 0, -1.
 *   counts[4]: free pages after the step (the next step's free_count; negative: so many were missing), new tokens, those of them that found no free
 *     page, no place in their table or none in `tokens`, pages taken.
 *   Nothing that the call reads is changed but by the pushes: with the old lengths and count a step that did not fit can be made again, and repeating a
 *   step gives the same.  A step that found too few pages (counts[0] < 0) has to be made again, with fewer tokens or more requests that end, before there is
 *   another: its lengths_out counts positions that no page holds.  A call with free_count < 0 does nothing and says so: lengths_out are the lengths, no token
 *   is new, counts are free_count, 0, the new tokens that it did not take, 0.  So steps may be queued before the host has seen the first one's counts.
 *   Entries within the lengths and numbers on the stack that are no page for another reason are the caller's: a token there gets slot -1 and does not count
 *   as one without a page, and a request that ends gives them back as they are.
 *   lengths_out and counts must not lie in lengths or free_count.  At most 8192 requests; pages * page < 2^31.
 * b2sp_paged_lists gives the slots that tokens see as lists for b2sp_attention_kv4 over caches whose rows are given out by pages: row_ptr[M + 1],
 *   col_idx[entries]; lists are cut where `entries` end, -1 stands for a missing page and behind the last list.
 * b2sp_paged_write copies the new rows into the pages: request r's tokens row_ptr[r] .. row_ptr[r + 1] - 1 of K and V (token t, head h at t * ld + h *
 *   stride_head) become its positions from lengths[r] (BEFORE the step) on.  means (NULL: none): [pages][kv_heads][d], its ld unused; the mean of K's
 *   rows of every page that gets rows, over those that are filled, is entered there.  Sums in fp32, rounded once.  A page that gets rows must belong to one
 *   request alone.  At most 8192 requests, d <= 1024.
 * b2sp_paged_select chooses pages by a score, (sum of the queries of the head's group) . (mean of the page), formed in 64 bits: of the pages that a token
 *   sees the first `first`, the last `last` and the best others, `keep` in all; of equal scores the lower page; NaN scores last.  lists[M][kv_heads][keep]: ascending
 *   indices into the request's table, -1 behind the last.  means->page: rows of the cache's pages.  first + last <= keep, d <= 256;
 *   strides of the means below 2^32 bytes.
 * b2sp_attention_paged: O and lse[M][heads] as for b2sp_attention_kv4, of M tokens over the positions that they see, or (lists not NULL) those of them
 *   that lie in the pages listed for the token and key head: of a list's entries the first ones count, as many as the token sees pages; each is its own
 *   term, in any order, and one that is no page seen is left out.  Q, O: token i, head h at i * ld + h * stride_head.
 *   Any M, but made for few tokens with long rows: a row is cut into parts and joined; neighbouring tokens of one request read its rows together.  d <= 256;
 *   strides below 2^32 bytes.  O may be Q itself, with its strides.
 * Other than that no call may write to what it reads (K and V of a write may be rows of the caches that it leaves as they are), nor may its outputs share
 *   memory: calls whose arguments show that they do are refused.  Rows of one tensor between those of another are fine.  At most 2^30 tokens.
 */
typedef struct {
    void *data; long long ld, stride_head, stride_page;
    int pages, page;
} b2sp_pages;
typedef struct {
    int *entries; long long ld;
    int requests, width;
} b2sp_page_tables;
b2sp_status b2sp_paged_tables(const b2sp_page_tables *tables, int pages, int page, const int *lengths, const int *added, int *free_pages,
                              int free_room, const int *free_count, int tokens, int *lengths_out, int *row_ptr, int *rows, int *seen, int *slots,
                              int *counts, void *stream);
b2sp_status b2sp_paged_lists(int M, const b2sp_page_tables *tables, int pages, int page, const int *rows, const int *seen, long long entries,
                             int *row_ptr, int *col_idx, void *stream);
b2sp_status b2sp_paged_write(int tokens, int kv_heads, int d, const float *K, long long ldk, long long stride_head_k, const float *V, long long ldv,
                             long long stride_head_v, const int *row_ptr, const int *lengths, const b2sp_page_tables *tables,
                             const b2sp_pages *k_pages, const b2sp_pages *v_pages, const b2sp_pages *means, void *stream);
b2sp_status b2sp_paged_write_bf16(int tokens, int kv_heads, int d, const void *K, long long ldk, long long stride_head_k, const void *V, long long ldv,
                                  long long stride_head_v, const int *row_ptr, const int *lengths, const b2sp_page_tables *tables,
                                  const b2sp_pages *k_pages, const b2sp_pages *v_pages, const b2sp_pages *means, void *stream);
size_t b2sp_paged_select_workspace_bytes(int M, int kv_heads, int width);   /* 0 on invalid arguments */
b2sp_status b2sp_paged_select(int M, int heads, int kv_heads, int d, const float *Q, long long ldq, long long stride_head_q, const b2sp_pages *means,
                              const b2sp_page_tables *tables, const int *rows, const int *seen, int keep, int first, int last, int *lists,
                              void *workspace, size_t workspace_bytes, void *stream);
b2sp_status b2sp_paged_select_bf16(int M, int heads, int kv_heads, int d, const void *Q, long long ldq, long long stride_head_q,
                                   const b2sp_pages *means, const b2sp_page_tables *tables, const int *rows, const int *seen, int keep, int first, int last,
                                   int *lists, void *workspace, size_t workspace_bytes, void *stream);
size_t b2sp_attention_paged_workspace_bytes(int M, int heads, int kv_heads, int d);   /* 0 on invalid arguments; either type */
b2sp_status b2sp_attention_paged(int M, int heads, int kv_heads, int d, const float *Q, long long ldq, long long stride_head_q,
                                 const b2sp_pages *k_pages, const b2sp_pages *v_pages, const b2sp_page_tables *tables, const int *rows, const int *seen,
                                 const int *lists, int keep, float scale, float *O, long long ldo, long long stride_head_o, float *lse, void *workspace,
                                 size_t workspace_bytes, void *stream);
b2sp_status b2sp_attention_paged_bf16(int M, int heads, int kv_heads, int d, const void *Q, long long ldq, long long stride_head_q,
                                      const b2sp_pages *k_pages, const b2sp_pages *v_pages, const b2sp_page_tables *tables, const int *rows,
                                      const int *seen, const int *lists, int keep, float scale, void *O, long long ldo, long long stride_head_o,
                                      float *lse, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Host-buffer forms of the three ops: every data pointer is a HOST pointer (pinned memory
 * makes the copies asynchronous and faster, pageable memory also works).  Each call copies
 * its inputs to the device, runs the device entry point above with algo = B2SP_ALGO_AUTO,
 * copies the result back and synchronises `stream` before returning.  Device memory comes
 * from a stream-ordered memory pool that the library creates for itself on each device at first
 * use (the process's default pool and its settings are not touched) and is returned to that pool
 * before the call ends; the pool keeps freed blocks for the next call.  Dense operands are
 * contiguous (ld = number of columns).  The workspace's device status word is read back with the
 * result: B2SP_ERR_TIMEOUT if a bounded wait inside a kernel gave up (outputs undefined).
 */
b2sp_status b2sp_spmm_host(int M, int K, int N, long long nnz,
                           const int *row_ptr, const int *col_idx, const float *values,
                           const float *D, float *O, void *stream);
b2sp_status b2sp_sddmm_host(int M, int K, int Kd, long long nnz,
                            const int *row_ptr, const int *col_idx, const float *s_values,
                            const float *A, const float *B, float *out_values, void *stream);
b2sp_status b2sp_fusedmm_host(int M, int K, int Kd, int N, long long nnz,
                              const int *row_ptr, const int *col_idx, const float *s_values,
                              const float *A, const float *B, const float *D, float *O,
                              void *stream);

/*
 * SPMM without any allocation, for callers that cannot obtain device memory of their own.
 * (The paper has no counterpart; this is a deployment convenience, not part of its method.)
 *
 * Who needs it: code that runs where cudaMalloc is not an option -- a plug-in inside a serving
 * process that gave all device memory to its own arena at start-up, or a latency-critical loop
 * that must not trigger the device-wide synchronisation an allocation can cause.  Such a caller
 * owns inputs and outputs but has no workspace to offer, so this entry point keeps the row-binning
 * workspace in a fixed array inside the library's device image instead.
 *
 * Same result and same argument meaning as b2sp_spmm with B2SP_ALGO_ROW (all data pointers are
 * device pointers; O is fully overwritten), minus the workspace and algo arguments.
 *
 * Limits and rules:
 *   - M <= B2SP_STATIC_SCRATCH_MAX_ROWS, otherwise B2SP_ERR_TOO_LARGE and nothing is enqueued.
 *     K, N and nnz are unrestricted.
 *   - The array (512 bytes + 4 bytes per row of the limit, about 257 KiB) is part of the library's
 *     device image: every GPU on which the image gets loaded holds it until the process exits.
 *   - The first call on each device looks up the array's device address.  With CUDA's lazy module
 *     loading that look-up is also what loads the library's device image on that GPU, and the
 *     driver reserves room for the array (and the code) at that moment; it may synchronise the
 *     device.  So make the first call at start-up: with the device current, BEFORE the host
 *     process's arena takes the remaining device memory, outside any latency-critical loop and
 *     before starting any stream capture.  Later calls on that device do no such work.
 *   - All calls on a device share the one array, and it keeps whatever the previous call left.  The
 *     part that must start from zero is cleared at the start of each call, so back-to-back calls on
 *     one stream are fine; two calls that can overlap on the GPU (different streams, or different
 *     host threads with different streams) race on it and give wrong results.  Use b2sp_spmm with
 *     separate workspaces for concurrent work.
 *   - The entry point itself calls no cudaMalloc / cudaFree / pool allocator and launches only a
 *     small memset and kernels on `stream`; it does not synchronise.
 */
#define B2SP_STATIC_SCRATCH_MAX_ROWS 65536
b2sp_status b2sp_spmm_static_scratch(int M, int K, int N, long long nnz,
                                     const int *row_ptr, const int *col_idx, const float *values,
                                     const float *D, long long ldd, float *O, long long ldo,
                                     void *stream);

/*
 * Debug helper: checks on the device that row_ptr[0] = 0, row_ptr is non-decreasing,
 * row_ptr[M] = nnz and 0 <= col_idx[p] < K.  Synchronises `stream`.  `workspace` needs 256
 * bytes.  Returns B2SP_OK or B2SP_ERR_BAD_CSR.
 */
b2sp_status b2sp_validate_csr(int M, int K, long long nnz, const int *row_ptr, const int *col_idx,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * Reads back (synchronising `stream`) the status word device code left in `workspace` during
 * the most recent op that used it: B2SP_OK, or B2SP_ERR_TIMEOUT if a bounded wait inside a
 * kernel gave up (the outputs of that call are then undefined).
 */
b2sp_status b2sp_device_status(const void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* B2SP_H */
