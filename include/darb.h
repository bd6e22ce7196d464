/*
 * darb.h -- C ABI of the MI355X (gfx950) DARB library.
 *
 * DARB (density-adaptive regular-block pruning, Ren et al., AAAI-20) stores a
 * pruned weight matrix W [M x N] as follows (section 3.2):
 *   - every row r has a power-of-two block size b_r chosen from its irregular-
 *     pruning row density;
 *   - the row is split into ceil(N / b_r) blocks of b_r columns (the last one
 *     may be shorter);
 *   - each block keeps exactly one weight, its largest-magnitude element
 *     (block-max weight masking, section 3.1), together with that element's
 *     position inside the block (a log2(b_r)-bit index, held either in one
 *     byte or bit-packed, see darb_pack_offsets).
 *
 * Storage order ("grouped layout"): rows are grouped by block size, smallest
 * block size first, rows of one group in ascending original index, and the
 * blocks of a row in ascending order.  Row r's retained weights are
 * values[row_start[r] + k], k < ceil(N / b_r); its block k covers columns
 * [k*b_r, k*b_r + b_r) and keeps column k*b_r + offsets[row_start[r] + k].
 * Grouping by block size follows the paper's remark that power-of-two density
 * groups make the storage regular: every group is one dense 2-D array.
 *
 * Conventions for every call:
 *   - Return value 0 on success, a negative DARB_E_* code otherwise; on error
 *     no output is written and darb_last_error() returns a detail string
 *     (thread-local).  No C++ exception crosses this boundary.
 *   - "device" pointers are HIP device memory of the current device (for
 *     example a torch CUDA tensor's data_ptr()); "host" pointers are ordinary
 *     host memory.  All buffers are owned by the caller; the library never
 *     allocates device memory.
 *   - stream is a hipStream_t (NULL = the null stream).  Device calls only
 *     enqueue work on it and return; the caller synchronises before reading
 *     outputs.  Calls on different streams that write the same buffers race.
 *   - A plan is host memory created by darb_plan_create and released by
 *     darb_plan_destroy.  One plan may be used from several threads for device
 *     calls once uploaded; create/upload/destroy are not thread-safe.
 *   - Sizes: 1 <= M < 2^31, 1 <= N <= 2^31 - 256 (a plan's products form column
 *     indices in 32 bits); block sizes are powers of two in [1, 128].
 */
#ifndef DARB_H
#define DARB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DARB_OK 0
#define DARB_E_INVALID (-1)      /* null pointer, bad size, bad bound, bad density, bad stride */
#define DARB_E_DTYPE (-2)        /* dtype or dtype combination not supported */
#define DARB_E_NOT_UPLOADED (-3) /* device call on a plan without device metadata */
#define DARB_E_HIP (-4)          /* a HIP runtime call or kernel launch failed */
#define DARB_E_NOMEM (-5)        /* host allocation failed */
#define DARB_E_WORKSPACE (-6)    /* workspace too small */

/* DARB_BF16 is taken by the evaluation and retraining calls only (logits, layer norm, the gated
 * recurrence, parameters and their gradients); the format and its products are fp32 or fp16. */
typedef enum { DARB_F32 = 0, DARB_F16 = 1, DARB_BF16 = 2 } darb_dtype;

/* Rounding of a row density to a power-of-two fraction (section 3.2). */
typedef enum {
    /* always round the density up: b_r = largest power of two with b_r * d_r <= 1 */
    DARB_ROUND_FLOOR = 0,
    /* the paper's rule: round up when d_r >= D (the matrix density), down when d_r < D */
    DARB_ROUND_PAPER = 1
} darb_round;

typedef struct darb_plan darb_plan;

/* One block-size group of the grouped layout. */
typedef struct {
    int32_t log2b;      /* block size is 1 << log2b                       */
    int32_t reserved;
    int64_t first_row;  /* index in storage order of the group's first row */
    int64_t rows;       /* rows in the group                               */
    int64_t first_elem; /* slot of the group's first retained weight       */
    int64_t nblk;       /* retained weights per row = ceil(N / b)          */
    int64_t first_word; /* packed offsets: the group's first 32-bit word   */
} darb_bin;

typedef struct {
    int64_t M, N;
    int64_t nnz;             /* retained weights = sum_r ceil(N / b_r)    */
    int64_t workspace_bytes; /* device workspace darb_plan_upload needs   */
    int64_t packed_words;    /* uint32 words of the bit-packed offsets    */
    int32_t nbins;           /* non-empty block-size groups, <= 8         */
    int32_t reserved;
    darb_bin bins[8];        /* ascending block size                      */
} darb_plan_info_t;

/*
 * Block sizes and layout from row densities (section 3.2).
 *   row_density  host fp64 [M], each in [0, 1]: the fraction of row r that
 *                irregular magnitude pruning keeps (section 3.1 obtains it from
 *                the irregular mask without pruning for real).
 *   matrix_density  D in [0, 1], the whole matrix's kept fraction; used by
 *                DARB_ROUND_PAPER only (a row with d_r == D rounds up).
 *   round_mode   a darb_round value.
 *   b_min, b_max powers of two, 1 <= b_min <= b_max <= 128; the block size is
 *                clamped to [b_min, b_max].  A row of density 0 gets b_max.
 *   out          receives the new plan (host memory), or NULL on error.
 * 1 <= M < 2^31, 1 <= N <= 2^31 - 256, and the plan may hold at most 2^55
 * retained weights.
 * Errors: DARB_E_INVALID, DARB_E_NOMEM.
 */
int darb_plan_create(int64_t M, int64_t N, const double *row_density, double matrix_density,
                     int round_mode, int b_min, int b_max, darb_plan **out);

/*
 * darb_plan_create from kept counts: row_density[r] = row_count[r] / N and
 * matrix_density = kept / (M * N), as produced by darb_prune_counts.
 *   row_count  host int64 [M], each in [0, N];  kept in [0, M * N]
 * Errors: DARB_E_INVALID, DARB_E_NOMEM.
 */
int darb_plan_create_counts(int64_t M, int64_t N, const int64_t *row_count, int64_t kept,
                            int round_mode, int b_min, int b_max, darb_plan **out);

/*
 * The plan built on the device, from kept counts in device memory (the flow of
 * section 3.2 from the irregular mask to block sizes, with darb_prune_counts' output
 * left where it is).  The same block-size rule as darb_plan_create_counts, in both
 * rounding modes and with the same results; the storage order and the per-row table
 * are written straight into `workspace`, which becomes the plan's device workspace
 * (the plan comes back uploaded on the current device; darb_plan_upload is refused
 * for it).  Only the group sizes (32 int64) travel to the host, so the call waits for
 * `stream`.  darb_plan_export copies the tables back from the device.
 *   row_count  device int64 [M], 8-byte aligned, each in [0, N] (as darb_prune_counts
 *              writes them; larger values count as N, negative ones as 0)
 *   kept       the matrix's kept count k, in [0, M * N] (D = k / (M N))
 *   workspace  device, 256-byte aligned, >= darb_plan_device_workspace(M) bytes; it must
 *              stay allocated and unmodified while the plan is used
 * Other arguments as for darb_plan_create.
 * Errors: DARB_E_INVALID, DARB_E_WORKSPACE, DARB_E_NOMEM, DARB_E_HIP.
 */
int darb_plan_device_workspace(int64_t M, int64_t *bytes);
int darb_plan_create_device(int64_t M, int64_t N, const int64_t *row_count, int64_t kept,
                            int round_mode, int b_min, int b_max, void *workspace,
                            int64_t workspace_bytes, void *stream, darb_plan **out);

/* Sizes and groups of a plan.  Errors: DARB_E_INVALID (null pointer). */
int darb_plan_info(const darb_plan *plan, darb_plan_info_t *info);

/*
 * Copy the plan's host metadata out.  Any output may be NULL to skip it.
 *   log2b      host uint8 [M]: log2 of each original row's block size
 *   row_start  host int64 [M]: first slot of each original row
 *   perm       host int32 [M]: original index of the row stored i-th
 */
int darb_plan_export(const darb_plan *plan, uint8_t *log2b, int64_t *row_start, int32_t *perm);

/*
 * Copy the plan's device metadata (the storage order and a per-row table of
 * first slot and block size) into a caller-owned device workspace of at least
 * info.workspace_bytes bytes (256-byte aligned) on `stream`, wait for the copy
 * to finish, and remember the workspace for later device calls on the current
 * device.  The workspace must stay allocated and unmodified while the plan is
 * used on the device.  Re-uploading to another workspace is allowed.
 * Errors: DARB_E_INVALID, DARB_E_WORKSPACE, DARB_E_NOMEM, DARB_E_HIP.
 */
int darb_plan_upload(darb_plan *plan, void *workspace, int64_t workspace_bytes, void *stream);

/* Release a plan (NULL is ignored).  Does not touch the device workspace. */
void darb_plan_destroy(darb_plan *plan);

/*
 * BMWM encode (section 3.1, with section 3.2's per-row block size): for every
 * row and block keep the element whose magnitude is largest -- magnitude is the
 * stored bit pattern with the sign bit cleared, compared as an unsigned
 * integer, so equal magnitudes (including +0 / -0) go to the lowest column --
 * and write its bits and its in-block index.
 *   wdtype   DARB_F32 or DARB_F16
 *   W        device [M x ldw] row-major, ldw >= N (elements)
 *   values   device [nnz] of wdtype, grouped layout
 *   offsets  device uint8 [nnz], grouped layout
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_encode(const darb_plan *plan, int wdtype, const void *W, int64_t ldw, void *values,
                uint8_t *offsets, void *stream);

/*
 * Decode to the masked dense matrix: W_out[r, c] = the retained value if c is
 * row r's kept column of its block, +0.0 otherwise.  Every element of the
 * [M x N] region is written.  Used to check the format against dense products.
 *   W_out    device [M x ldw] of wdtype, ldw >= N
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_decode(const darb_plan *plan, int wdtype, const void *values, const uint8_t *offsets,
                void *W_out, int64_t ldw, void *stream);

/*
 * y = W_darb x (sections 2 and 3.2: only retained weights are read, each
 * block's offset selects the one activation it multiplies).  Products and
 * sums in fp32; y is overwritten.
 *   (wdtype, xdtype) in {(F32, F32), (F16, F16), (F16, F32)}
 *   x  device [N] of xdtype;  y  device fp32 [M], original row order
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_spmv(const darb_plan *plan, int wdtype, const void *values, const uint8_t *offsets,
              int xdtype, const void *x, float *y, void *stream);

/*
 * Y = W_darb X for a batch of B activation vectors (same definition as
 * darb_spmv, column by column).  X is [N x B] row-major with leading dimension
 * ldx >= B (the B values of one input feature are contiguous); Y is fp32
 * [M x B] row-major with ldy >= B, overwritten.  B >= 1.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_spmm(const darb_plan *plan, int wdtype, const void *values, const uint8_t *offsets,
              int xdtype, int64_t B, const void *X, int64_t ldx, float *Y, int64_t ldy,
              void *stream);

/*
 * Bit-packed offsets (section 4.2: the kept weight's position inside a block of
 * size b needs log2 b bits, not a byte).  Layout: inside each block-size group
 * (log2 b = l) the retained weights are numbered j = 0, 1, ... in storage order
 * and cut into runs of 32; run j / 32 occupies l consecutive uint32 words, and
 * weight j's index is bits (j % 32) * l ... (j % 32) * l + l - 1 of its run read
 * as one little-endian bit string (bit i of the run is bit i % 32 of word i / 32).
 * Groups follow each other in ascending block size starting at word
 * bins[g].first_word; a group with b = 1 has no words (every index is 0).  The
 * whole form is info.packed_words words, which may be 0 (then `packed` may be
 * NULL).  `packed` is device memory, 4-byte aligned.
 *
 * darb_pack_offsets converts the byte offsets darb_encode writes (every one must
 * be < b; only its low log2 b bits are stored) to the packed form, overwriting
 * every packed word; darb_unpack_offsets converts back, writing all nnz bytes.
 * Errors: DARB_E_INVALID, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_pack_offsets(const darb_plan *plan, const uint8_t *offsets, uint32_t *packed,
                      void *stream);
int darb_unpack_offsets(const darb_plan *plan, const uint32_t *packed, uint8_t *offsets,
                        void *stream);

/*
 * darb_spmv and darb_spmm reading the offsets in the packed form above.  Every
 * other argument, and the result bit for bit, is as for the byte-offset calls.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_spmv_packed(const darb_plan *plan, int wdtype, const void *values,
                     const uint32_t *packed, int xdtype, const void *x, float *y, void *stream);
int darb_spmm_packed(const darb_plan *plan, int wdtype, const void *values,
                     const uint32_t *packed, int xdtype, int64_t B, const void *X, int64_t ldx,
                     float *Y, int64_t ldy, void *stream);

/*
 * INT8 retained weights.  Section 4.2's storage accounting assumes weights
 * quantised to INT8 without fixing a scheme; this one is symmetric with one fp32
 * scale per row.  For row r with a = max |v| over its retained values (fp32, fp16
 * widened exactly): inv = 127 / a, code q = rint(v * inv) (ties to even) clamped to
 * [-127, 127], scale s_r = a / 127 -- each a single correctly rounded fp32
 * operation, so the codes are exact.  Rows with a < 2^-120 (127 / a would
 * overflow) get s_r = 0 and all-zero codes.  Values must be finite.
 *   darb_quantize_i8
 *     values   device, the format's values (wdtype DARB_F32 or DARB_F16), nnz
 *     codes    device int8 [nnz], slot order like values, overwritten
 *     scales   device fp32 [M], indexed by original row, overwritten
 *   darb_spmv_i8 / darb_spmm_i8: y[r] = s_r * sum_k q[r,k] * x[k * b_r + off[r,k]],
 *     summed in fp32 and scaled once; as darb_spmv / darb_spmm (same layouts, x/X
 *     fp32 or fp16, Y fp32) with the offsets from exactly one of `offsets` (one byte
 *     each) and `packed` (darb_pack_offsets' words; with offsets NULL, packed may be
 *     NULL only when the plan has no packed words).  Passing both is an error.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_quantize_i8(const darb_plan *plan, int wdtype, const void *values, int8_t *codes,
                     float *scales, void *stream);
int darb_spmv_i8(const darb_plan *plan, const int8_t *codes, const float *scales,
                 const uint8_t *offsets, const uint32_t *packed, int xdtype, const void *x,
                 float *y, void *stream);
int darb_spmm_i8(const darb_plan *plan, const int8_t *codes, const float *scales,
                 const uint8_t *offsets, const uint32_t *packed, int xdtype, int64_t B,
                 const void *X, int64_t ldx, float *Y, int64_t ldy, void *stream);

/*
 * Irregular magnitude pruning, the step DARB starts from (section 3.2: the
 * irregular mask is computed only to measure each row's density; irregular
 * pruning keeps the K largest-magnitude weights, section 2).  Keeps the k
 * elements of W with the largest magnitude -- the stored bits with the sign
 * cleared, compared as unsigned integers, as in darb_encode; among equal
 * magnitudes the lower flat index r * N + c first -- and writes how many each
 * row keeps.  No mask is materialised.
 *   wdtype     DARB_F32 or DARB_F16
 *   W          device [M x ldw] row-major, ldw >= N (elements)
 *   k          0 <= k <= M * N
 *   counts     device int64 [M], 8-byte aligned, overwritten
 *   workspace  device, 256-byte aligned, >= the size darb_prune_workspace
 *              returns (about M*N/4 bytes: room for the keys whose leading digit
 *              lies in a small bracket around the threshold's, which the later
 *              passes read instead of W from about 20 MiB of W on); its
 *              contents on entry do not change the counts (from 64 MiB of W a
 *              workspace last used by this call runs fastest: it leaves the part the
 *              next call's sample adds into at zero; other contents may cost that
 *              call passes over W)
 * Work is enqueued on `stream` only (several kernels, no host synchronisation);
 * calls sharing a workspace must not overlap.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_HIP.
 */
int darb_prune_workspace(int64_t M, int64_t N, int wdtype, int64_t *bytes);
int darb_prune_counts(int64_t M, int64_t N, int wdtype, const void *W, int64_t ldw, int64_t k,
                      int64_t *counts, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * darb_prune_counts for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation): the same
 * arguments and the same counts, bit for bit, without the workspace.  Its scratch
 * is a fixed 8 MiB array in the library's device code, one per device, held until
 * the process ends; the first call on a device looks up that device's copy (no
 * allocation).  The array holds the per-row counters (16 bytes per row), so M is
 * limited to 483 296 rows (larger M: DARB_E_INVALID, naming the limit);
 * the rest is candidate room, and a matrix whose candidates do not fit takes more
 * passes over W with the same result.  Every call on a device shares its array and
 * leaves its contents there (each call clears what must start at zero), so calls
 * that overlap on one device -- on different streams or threads -- race.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_HIP.
 */
int darb_prune_counts_noalloc(int64_t M, int64_t N, int wdtype, const void *W, int64_t ldw,
                              int64_t k, int64_t *counts, void *stream);

/*
 * One LSTM layer over a sequence with DARB-stored weights (the recurrent
 * models of section 4.1): no bias, gate order (i, f, g, o),
 *   gates_t = W_ih x_t + W_hh h_{t-1},
 *   c_t = sigmoid(f) * c_{t-1} + sigmoid(i) * tanh(g),  h_t = sigmoid(o) * tanh(c_t).
 * W_ih is [4H x I] and W_hh is [4H x H], both of wdtype, each with its own
 * uploaded plan.  The input products of all steps are computed first as one
 * darb_spmm with B = T * batch.  The time steps then run as one launch whose
 * workgroups keep W_hh and exchange h through the workspace.  That takes T >= 16, W_hh
 * rows of at most 512 retained weights, no stream capture, H of 16 to 4095 at batch <= 16,
 * 2048 at batch <= 32, 1024 at batch <= 64, and W_hh's weights in the workgroups'
 * registers: the ceil(H / 32) units of each (of 32) hold at most 1536 chunks of 16 weights
 * (1024 at batch > 32), each gate row in whole chunks.  Such launches take turns on a
 * device, each once all that its own stream ordered before it has ended; a workgroup's
 * waits are bounded, and a sequence whose workgroups could not all run at once (another
 * process holding the device) is computed again without waiting, with the same result bit
 * for bit but some tens of milliseconds later.  Otherwise each time step is one launch: a
 * workgroup per hidden unit computes the unit's four gate rows of W_hh h_{t-1} and the
 * cell (batch <= 64 and a multiple of 4, or batch <= 16; W_hh rows of at most 512 retained
 * weights); other shapes run the recurrent product and the cell as two launches.  The
 * three add in different orders: they give the same result within the product tolerance,
 * so a captured call, which takes no sequence launch, and an eager one may differ in the
 * last bits.  For the same arguments the call is deterministic.  The workspace also holds
 * the second buffer of h that the steps alternate with `h`, or the exchange's.
 *   x_seq      device fp32 [I x T*batch], column t*batch + n
 *   h_seq      device fp32 [H x T*batch], receives h_t in columns t*batch + n
 *   h, c       device fp32 [H x batch], initial state in, final state out
 *   workspace  device fp32, 16-byte aligned, at least 4H*T*batch + 4H*batch floats
 *              (darb_lstm_workspace)
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_HIP.
 */
int darb_lstm_layer(const darb_plan *wih_plan, const void *wih_values,
                    const uint8_t *wih_offsets, const darb_plan *whh_plan,
                    const void *whh_values, const uint8_t *whh_offsets, int wdtype,
                    int64_t H, int64_t T, int64_t batch, const float *x_seq, float *h_seq,
                    float *h, float *c, float *workspace, int64_t workspace_floats,
                    void *stream);

/* Workspace floats darb_lstm_layer needs for (H, T, batch).  Errors: DARB_E_INVALID. */
int darb_lstm_workspace(int64_t H, int64_t T, int64_t batch, int64_t *floats);

/* ------------------------------------------------------------------------------------
 * Evaluating and retraining a DARB layer (section 4.1 retrains the retained weights after
 * pruning): log probabilities with their gradient, layer norm, the product's gradients and
 * the optimizer's step.
 *
 * Activations are [features x batch] as everywhere here.  The first two take either memory
 * order: element (f, b) lies at f * feature_stride + b * batch_stride (elements), and one of
 * the two strides is 1 (batch_stride: the order of the products' X and Y; feature_stride: a
 * batch of rows).  Along an axis of size 1 the stride is not used and may be anything.  The
 * other stride is at least the unit axis' length (one token or one feature that is only read
 * may have 0: the same element everywhere).  Sums and statistics are fp32; results of a 16-bit
 * type are rounded once, to nearest even.  All calls are deterministic.
 */

/*
 * Log probabilities of given tokens under logits z [V x B]: per column (token),
 *   lse = log sum_v e^z[v],  logprob = z[target] - lse,
 *   entropy = - sum_v p_v log p_v,  p_v = e^(z[v] - lse),
 * and the `top` greatest logits' log probabilities and classes, greatest first, equal ones
 * by the lower class.  A logit of -inf has probability 0 and adds nothing to the entropy.
 * A column of nothing but -inf has lse and log probabilities -inf and entropy 0; one that
 * holds a NaN or +inf has NaN for all three (its alternatives are still ordered, NaN first).
 * A negative target means that the column has none: logprob 0.  A target of V or more: NaN.
 *   zdtype       DARB_F32, DARB_F16 or DARB_BF16
 *   z            device [V x B], 1 <= V < 2^31, 1 <= B < 2^31
 *   targets      device int64 [B], or NULL (no column has a target)
 *   top          0 ... 64, at most V
 *   logprob, entropy, lse      device fp32 [B]
 *   top_logprob  device fp32 [B x top]; top_index device int64 [B x top] (NULL if top is 0)
 *   workspace    device, 256-byte aligned, >= darb_token_logprobs_workspace's bytes; NULL
 *                where those are 0 (rows that one workgroup reads)
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_HIP.
 */
int darb_token_logprobs_workspace(int zdtype, int64_t V, int64_t B, int64_t z_feature_stride,
                                  int64_t z_batch_stride, int64_t top, int64_t *bytes);
int darb_token_logprobs(int zdtype, int64_t V, int64_t B, const void *z, int64_t z_feature_stride,
                        int64_t z_batch_stride, const int64_t *targets, int64_t top,
                        float *logprob, float *entropy, float *lse, float *top_logprob,
                        int64_t *top_index, void *workspace, int64_t workspace_bytes,
                        void *stream);

/*
 * The gradient of sum_b (grad_logprob[b] logprob[b] + grad_entropy[b] entropy[b]):
 *   dz[v] = grad_logprob (1[v = target] - p_v) - grad_entropy p_v (log p_v + entropy),
 * from the lse (and entropy) of darb_token_logprobs; p_v log p_v is zero where p_v is.  A
 * column without a target gets none of the first part, one of nothing but -inf (lse = -inf) is zero
 * altogether, and one whose target is V or more is NaN.
 *   grad_logprob  device fp32 [B] or NULL (zeros)
 *   entropy, grad_entropy  device fp32 [B], both or neither NULL; not all three NULL
 *   dz            device [V x B] of zdtype, the unit stride along z's axis; may be z itself
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_HIP.
 */
int darb_token_logprobs_grad(int zdtype, int64_t V, int64_t B, const void *z,
                             int64_t z_feature_stride, int64_t z_batch_stride,
                             const int64_t *targets, const float *lse, const float *grad_logprob,
                             const float *entropy, const float *grad_entropy, void *dz,
                             int64_t dz_feature_stride, int64_t dz_batch_stride, void *stream);

/*
 * Layer norm of the columns of x [H x B]:
 *   mean = sum_h x / H,  rstd = 1 / sqrt(sum_h (x - mean)^2 / H + eps),
 *   y = (x - mean) rstd weight + bias.
 *   xdtype        type of x and y: DARB_F32, DARB_F16 or DARB_BF16
 *   wdtype        type of weight and bias: DARB_F32 or xdtype
 *   weight, bias  device [H], each may be NULL (ones, zeros)
 *   eps           >= 0 (0: a constant column divides by zero)
 *   y             device [H x B], the unit stride along x's axis; may be x itself
 *   mean, rstd    device fp32 [B], each may be NULL
 * 1 <= H < 2^31, 1 <= B < 2^31.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_HIP.
 */
int darb_layer_norm(int xdtype, int wdtype, int64_t H, int64_t B, const void *x,
                    int64_t x_feature_stride, int64_t x_batch_stride, const void *weight,
                    const void *bias, double eps, void *y, int64_t y_feature_stride,
                    int64_t y_batch_stride, float *mean, float *rstd, void *stream);

/*
 * Its gradients from dy [H x B] (type and axis of x), x, and the mean and rstd it returned:
 * with xh = (x - mean) rstd and a = dy weight,
 *   dx = rstd (a - sum_h a / H - xh sum_h a xh / H),
 *   dweight = sum_b dy xh,  dbias = sum_b dy   (fp32 [H], in an order that H and B fix).
 *   dx            device [H x B] of xdtype, the unit stride along x's axis; may be dy itself
 *                 or x itself
 *   weight        as given to darb_layer_norm (NULL: ones)
 *   dx, dweight, dbias   each may be NULL (not computed), not all three
 *   workspace     device, 256-byte aligned, >= darb_layer_norm_workspace's bytes
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_HIP.
 */
int darb_layer_norm_workspace(int64_t H, int64_t B, int64_t *bytes);
int darb_layer_norm_grad(int xdtype, int wdtype, int64_t H, int64_t B, const void *dy,
                         int64_t dy_feature_stride, int64_t dy_batch_stride, const void *x,
                         int64_t x_feature_stride, int64_t x_batch_stride, const float *mean,
                         const float *rstd, const void *weight, void *dx,
                         int64_t dx_feature_stride, int64_t dx_batch_stride, float *dweight,
                         float *dbias, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * The gradients of Y = W_darb X (darb_spmm; darb_spmv with B = 1) with the mask fixed:
 *   dvalues[s] = sum_b dY[r, b] X[c, b]   for the slot s that keeps column c of row r,
 *   dX[c, b]   = sum over the slots s of column c of values[s] dY[r, b].
 * They run over an index of the retained weights by column, which darb_transpose makes from
 * the byte offsets (the same index for the same offsets, bit for bit).  It stays valid as long
 * as the offsets do: a program that retrains the values makes it once.
 *   index     device, 256-byte aligned, >= darb_transpose_bytes bytes; the plan must keep
 *             fewer than 2^31 weights
 * darb_spmm_grad:
 *   wdtype, values, xdtype, B, X, ldx   as for darb_spmm
 *   dY        device fp32 [M x B], leading dimension ldy >= B
 *   dvalues   device fp32 [nnz], overwritten, or NULL
 *   dX        device fp32 [N x B], leading dimension lddx >= B, overwritten (a column that no
 *             row keeps: zeros), or NULL; not both NULL
 *   workspace device, 256-byte aligned, >= darb_spmm_grad_workspace's bytes: none for a small
 *             dY (then it may be NULL), at most 72 bytes a weight and 4 KiB a row
 * values may be NULL if dX is, X if dvalues is.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_NOT_UPLOADED, DARB_E_WORKSPACE, DARB_E_HIP.
 */
int darb_transpose_bytes(const darb_plan *plan, int64_t *bytes);
int darb_transpose(const darb_plan *plan, const uint8_t *offsets, void *index,
                   int64_t index_bytes, void *stream);
int darb_spmm_grad_workspace(const darb_plan *plan, int64_t B, int64_t *bytes);
int darb_spmm_grad(const darb_plan *plan, const void *index, int wdtype, const void *values,
                   int xdtype, int64_t B, const void *X, int64_t ldx, const float *dY,
                   int64_t ldy, float *dvalues, float *dX, int64_t lddx, void *workspace,
                   int64_t workspace_bytes, void *stream);

/*
 * AdamW with decoupled weight decay over many tensors at once.  Step t >= 1:
 *   m = m b1 + g (1 - b1),  v = v b2 + g g (1 - b2),
 *   p = p (1 - lr decay) - (m / (sqrt(v) rs + eps)) (lr / (1 - b1^t)),
 *   rs = 1 / sqrt(1 - b2^t),
 * each operation one correctly rounded fp32 operation in this order, the scalars computed in
 * fp64 and rounded to fp32; g is the gradient times *grad_scale.  Where a tensor has a
 * master, p is the master and the parameter receives its rounding.
 *
 * States in 8 bits: blocks of 256 consecutive elements share an fp32 scale, the greatest
 * magnitude of the block.  A code c > 0 of m (7 bits, and the sign in bit 7) stands for the
 * fp32 number with the bits (c + 889) << 20 times the scale, one of v (8 bits) for the bits
 * (c + 1777) << 19; code 0 stands for 0.  A step rounds the new state x with random bits:
 * with q = |x| (1 / scale) the code is (bits of q + r) >> 20 (19), less 889 (1777), from 0
 * (v > 0: 1) to 127 (255), where r has its upper 16 bits below the shift from a hash of the
 * element's number, the tensor's and the seed: h is x0 = element + tensor * 0xBB67AE85 + seed
 * after x ^= x >> 16, x *= 0x9E3779B9, x ^= x >> 15, x *= 0xB504F333, x ^= x >> 16 (modulo
 * 2^32); m takes its low half, v its high half.  A block whose greatest magnitude is below
 * 2^-120 becomes 0; one that holds an infinity or NaN gets scale NaN.
 *
 * darb_adamw_create copies the table of tensors into the caller's workspace (on `stream`,
 * waiting for it); the tensors and the workspace stay allocated while the handle is used, and
 * no tensor's memory may overlap another's.  The handle is host memory; release it with
 * darb_adamw_destroy.
 *   bits        32 (m, v: fp32 [n]) or 8 (m, v: uint8 [n]; m_scale, v_scale: fp32
 *               [ceil(n / 256)]); all zeros is the initial state
 *   n           0 <= n < 2^39
 *   decay       the tensor's weight decay, >= 0
 * darb_adamw_step:
 *   grads       host array of `count` device pointers, [n] of the type in gdtypes; NULL: the
 *               tensor is left as it is (and its entry of gdtypes is not read)
 *   grad_scale  device fp32 [1] or NULL (1)
 *   lr >= 0, 0 <= beta1, beta2 < 1, eps >= 0, step >= 1
 * darb_adamw_moments writes the values that the states stand for: host arrays of `count`
 * device pointers to fp32 [n]; either array, or any pointer in it, may be NULL.
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_NOMEM, DARB_E_HIP.
 */
typedef struct darb_adamw darb_adamw;
typedef struct {
    void *param;       /* device [n] of dtype */
    float *master;     /* device [n], or NULL */
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    double decay;
    int32_t dtype;     /* DARB_F32, DARB_F16 or DARB_BF16 */
    int32_t reserved;  /* 0 */
} darb_adamw_tensor;

int darb_adamw_workspace(const darb_adamw_tensor *tensors, int64_t count, int64_t *bytes);
int darb_adamw_create(const darb_adamw_tensor *tensors, int64_t count, int bits, void *workspace,
                      int64_t workspace_bytes, void *stream, darb_adamw **out);
int darb_adamw_step(const darb_adamw *adamw, const void *const *grads, const int *gdtypes,
                    int64_t count, double lr, double beta1, double beta2, double eps,
                    int64_t step, const float *grad_scale, uint32_t seed, void *stream);
int darb_adamw_moments(const darb_adamw *adamw, float *const *m, float *const *v, int64_t count,
                       void *stream);
void darb_adamw_destroy(darb_adamw *adamw);

/*
 * A gated linear recurrence over sequences, the recurrent layer that is retrained here: column
 * t * batch + n of an operand [H x T*batch] is step t of sequence n, as in darb_lstm_layer.
 *   DARB_RECURRENCE_GATE    f = sigmoid(gate),  h_t = f_t h_{t-1} + (1 - f_t) x_t
 *   DARB_RECURRENCE_LINEAR  f = gate,           h_t = f_t h_{t-1} + x_t
 * elementwise, from h_{-1} = h0.  T = 1 is the single step of a program that generates: h0 and
 * h_last may be the same buffer.
 *   dtype     type of gate, x and h: DARB_F32, DARB_F16 or DARB_BF16; the state between steps
 *             and h0, h_last are fp32
 *   gate, x   device [H x T*batch], any order, one for all such operands (strides as above)
 *   resets    device uint8 [T*batch] or NULL: where it is not 0 a sequence starts, and the state
 *             before it counts as 0, whatever it was (packed texts)
 *   h0        device fp32 [H x batch], either order, or NULL (zeros)
 *   h         device [H x T*batch] of dtype, receives every state; may be gate or x itself
 *   h_last    device fp32 [H x batch], either order, or NULL: the state after the last step
 * Steps are joined as maps h -> a h + b, a being a product of gates: gates above 1 in magnitude
 * (linear form) are right as long as no product of consecutive ones leaves the range of fp32.  A
 * state that is not finite makes those after it not finite, up to the next start.
 *   workspace device, 256-byte aligned, >= darb_gated_recurrence_workspace's bytes (back: 0, or
 *             1 for the gradients); NULL where those are 0
 * H, T, batch >= 1, H < 2^31, T * batch < 2^31.
 *
 * Gradients, from dh [H x T*batch] (by every state) and dh_last (by the last one; NULL: zeros),
 * with g_t = dh_t + f_{t+1} g_{t+1} (nothing from a start), g_{T-1} = dh_{T-1} + dh_last:
 *   gate form    dgate_t = (h_{t-1} - x_t) g_t f_t (1 - f_t),  dx_t = (1 - f_t) g_t
 *   linear form  dgate_t = h_{t-1} g_t,                        dx_t = g_t   (x is not read: NULL)
 *   dh0 = f_0 g_0 (zeros where step 0 is a start)
 *   h          as darb_gated_recurrence returned it; h0 as it was given
 *   dgate, dx  device [H x T*batch] of dtype; each may be dh, gate or x itself, neither may be h
 *   dh0        device fp32 [H x batch], either order, or NULL; may be dh_last or h0 itself
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_HIP.
 */
typedef enum { DARB_RECURRENCE_GATE = 0, DARB_RECURRENCE_LINEAR = 1 } darb_recurrence;

/* A device matrix: element (f, b) at p + f * feature_stride + b * batch_stride (elements). */
typedef struct {
    void *p;
    int64_t feature_stride, batch_stride;
} darb_matrix;

int darb_gated_recurrence_workspace(int dtype, int back, int64_t H, int64_t T, int64_t batch,
                                    int64_t *bytes);
int darb_gated_recurrence(int dtype, int form, int64_t H, int64_t T, int64_t batch,
                          const darb_matrix *gate, const darb_matrix *x, const uint8_t *resets,
                          const darb_matrix *h0, const darb_matrix *h, const darb_matrix *h_last,
                          void *workspace, int64_t workspace_bytes, void *stream);
int darb_gated_recurrence_grad(int dtype, int form, int64_t H, int64_t T, int64_t batch,
                               const darb_matrix *dh, const darb_matrix *gate,
                               const darb_matrix *x, const darb_matrix *h, const uint8_t *resets,
                               const darb_matrix *h0, const darb_matrix *dh_last,
                               const darb_matrix *dgate, const darb_matrix *dx,
                               const darb_matrix *dh0, void *workspace, int64_t workspace_bytes,
                               void *stream);

/*
 * The clipped policy loss over token log probabilities (darb_token_logprobs), and its gradients,
 * which darb_token_logprobs_grad takes: with r = e^(logprob - old), q = ref - logprob,
 *   L_b = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (e^q - 1 - q)
 *         - entropy_coef entropy,
 *   loss = sum_b weight_b L_b,  kl = sum_b weight_b (e^q - 1 - q),
 *   clipped = sum of the weights of the tokens whose ratio's part is the clipped one (and so has
 *   no gradient),
 *   grad_logprob = weight (-r A where not clipped, - kl_coef (e^q - 1)),
 *   grad_entropy = -weight entropy_coef.
 * A token of weight 0 adds nothing and has gradient 0, whatever its other values are.
 *   logprob, old, advantage   device fp32 [B], 1 <= B < 2^31
 *   weight        device fp32 [B], or NULL (1 / B each)
 *   ref           device fp32 [B], or NULL (kl is 0; kl_coef must be 0 then); with kl_coef 0 it
 *                 changes kl alone, whatever it holds
 *   entropy       device fp32 [B], with grad_entropy, or NULL both (entropy_coef 0)
 *   clip_low, clip_high   >= 0 (clip_low of 1 or more: no lower bound); kl_coef >= 0
 * r and e^q are formed in fp32: past its range (an exponent above 88.7) they count as infinite, but
 * an A of 0 times a finite r is 0.
 *   stats         device fp32 [3]: loss, kl, clipped
 *   grad_logprob, grad_entropy   device fp32 [B]; may be any of the inputs of that size
 *   workspace     device, 256-byte aligned, >= darb_policy_loss_workspace's bytes; NULL where
 *                 those are 0
 * Errors: DARB_E_INVALID, DARB_E_WORKSPACE, DARB_E_HIP.
 */
int darb_policy_loss_workspace(int64_t B, int64_t *bytes);
int darb_policy_loss(int64_t B, const float *logprob, const float *old, const float *advantage,
                     const float *weight, const float *ref, const float *entropy,
                     double clip_low, double clip_high, double kl_coef, double entropy_coef,
                     float *stats, float *grad_logprob, float *grad_entropy, void *workspace,
                     int64_t workspace_bytes, void *stream);

/*
 * The preference loss of `pairs` pairs of sequences over token log probabilities, and its gradient.
 * Sequences 0 ... P-1 are the preferred ones, P ... 2P-1 the others of the same pairs.  With
 * s = a sequence's sum of logprob - ref, m_p = beta (s_p - s_{P+p}),
 *   loss = sum_p weight_p (-(1 - smoothing) log sigma(m_p) - smoothing log sigma(-m_p)),
 *   grad_logprob = weight_p beta (smoothing - sigma(-m_p)) for the tokens of sequence p, the
 *   negative for those of P + p.
 *   starts        NULL: B = T * 2P, token t of sequence s at t * 2P + s (the columns of an operand
 *                 [V x T*batch] with batch 2P; a padded place has logprob and ref 0).  Or device
 *                 int64 [2P + 1], never decreasing: sequence s holds the tokens starts[s] ...
 *                 starts[s + 1] - 1; tokens before the first and behind the last sequence have
 *                 gradient 0.  What lies outside [0, B] is taken as 0 or B.
 *   logprob       device fp32 [B], 1 <= B < 2^31; ref device fp32 [B], or NULL (zeros)
 *   weight        device fp32 [P], or NULL (1 / P each); a pair of weight 0 adds nothing and has
 *                 gradient 0, whatever its margin is
 *   beta          finite, >= 0; smoothing in [0, 1)
 *   loss          device fp32 [1]; margin device fp32 [P] (m_p)
 *   grad_logprob  device fp32 [B]; may be logprob or ref itself
 * 1 <= P < 2^30.
 * Errors: DARB_E_INVALID, DARB_E_HIP.
 */
int darb_preference_loss(int64_t pairs, int64_t B, const float *logprob, const float *ref,
                         const int64_t *starts, const float *weight, double beta,
                         double smoothing, float *loss, float *margin, float *grad_logprob,
                         void *stream);

/*
 * The orthogonalised update of weight matrices: a matrix u is divided by its norm and its singular
 * values taken towards 1 by steps of a quintic, X = u / (|u| + eps) (Frobenius norm),
 *   X = a X + (b A + c A A) X,  A = X X^T (X with at most as many rows as columns),
 *   (a, b, c) = (3.4445, -4.7750, 2.0315),
 * after five of which those from 0.01 of |u| up lie between 0.68 and 1.21.
 * darb_orthogonalize writes that X of each matrix; darb_muon_step makes one optimizer step with
 *   m = momentum m + (1 - momentum) g,  u = momentum m + (1 - momentum) g  (nesterov; else m)
 *   p = p (1 - lr decay) - lr scale X.
 * Sums and m are fp32 or more.  A result is as accurate as fp32 products make it, whatever its type,
 * and rounded to that type once; X is held to 2^-22 of each element, and not below 2^-40, so that of a
 * matrix whose norm is far below eps (its X far below 1) less is left.  The same call gives the same bits; a matrix together with others
 * may differ from it alone in how its sums are rounded.
 * A matrix that holds an infinity or NaN becomes NaN; zeros stay zeros.
 *   dtype, gdtype   DARB_F32, DARB_F16 or DARB_BF16, of param and of grad
 *   param       device [rows x cols], unit column stride, leading dimension ld_param >= cols
 *               (darb_orthogonalize: receives X; may be grad itself)
 *   master      device fp32 [rows x cols] at the same leading dimension, or NULL: a copy that the
 *               step updates and rounds into param
 *   grad        device [rows x cols], unit column stride, leading dimension ld_grad >= cols;
 *               NULL (darb_muon_step): the tensor is left as it is
 *   momentum    device fp32 [rows x cols], contiguous (darb_orthogonalize: NULL)
 *   scale, decay  finite, decay >= 0
 *   fp16_products   0; or 1: a result of 16 bits (without a master) may take its products from
 *               operands of fp16, in less time: it is off by 1 to 3 10^-3 of its norm before it is
 *               rounded.  Without effect on other results, and where a side is below 64.
 *   reserved    0
 *   rows, cols  1 <= rows, cols < 2^20
 *   tensors     host array of `count` >= 1, read during the call; no memory overlaps
 *   steps       1 ... 16;  momentum in [0, 1), lr >= 0, eps > 0 (finite)
 *   grad_scale  device fp32 [1] that multiplies every gradient, or NULL (1)
 *   workspace   device, 256-byte aligned, >= darb_muon_workspace's bytes for these tensors: 16 to 24
 *               an element (16 + 8 shorter side / longer side, sides padded to multiples of 32) of
 *               the largest group that is taken at once, of up to 28 tensors and 4 GiB or a single one
 * Errors: DARB_E_INVALID, DARB_E_DTYPE, DARB_E_WORKSPACE, DARB_E_HIP.
 */
typedef struct {
    void *param;
    float *master;
    const void *grad;
    float *momentum;
    int64_t rows, cols, ld_param, ld_grad;
    double scale, decay;
    int32_t dtype, gdtype;
    int32_t fp16_products, reserved;
} darb_muon_tensor;

int darb_muon_workspace(const darb_muon_tensor *tensors, int64_t count, int64_t *bytes);
int darb_muon_step(const darb_muon_tensor *tensors, int64_t count, double lr, double momentum,
                   int nesterov, int steps, double eps, const float *grad_scale, void *workspace,
                   int64_t workspace_bytes, void *stream);
int darb_orthogonalize(const darb_muon_tensor *tensors, int64_t count, int steps, double eps,
                       void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Measurement helpers (not part of DARB).  darb_stream_read reads `bytes`
 * bytes (a multiple of 16, 16-byte aligned) of device memory and writes one
 * float per workgroup derived from them into `sink` (device, >= 8192 floats)
 * so the reads cannot be elided; darb_stream_copy copies `bytes` bytes
 * (multiple of 16, both 16-byte aligned).  They give the HBM read and copy
 * rates the DARB kernels are compared with.
 */
int darb_stream_read(const void *buf, int64_t bytes, float *sink, void *stream);
/*
 * The same read in other launch shapes, to find the fastest plain read of a given
 * size: `threads` per workgroup (64, 128, 256, 512 or 1024) each issuing `vectors`
 * 16-byte loads (1, 2, 4 or 8; the pairs 64/1, 64/2, 128/1, 128/2, 128/8, 512/8
 * and 1024/8 are not built) before using any of them.  The loaded data decides
 * whether anything is written to `sink` (device, >= 8192 floats); real data never
 * produces the value that would, so the launch is the read alone.
 * Errors: DARB_E_INVALID (also for a shape that is not built), DARB_E_HIP.
 */
int darb_stream_read_shape(const void *buf, int64_t bytes, int threads, int vectors, float *sink,
                           void *stream);
int darb_stream_copy(void *dst, const void *src, int64_t bytes, void *stream);

/* Text for a DARB_E_* code (static storage). */
const char *darb_strerror(int code);

/* Detail of the last error on the calling thread ("" if none). */
const char *darb_last_error(void);

/* Library version as major*10000 + minor*100 + patch. */
int darb_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DARB_H */
