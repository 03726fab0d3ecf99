/*
 * fasq.h - product-quantized (PQ) weight matmul for AMD Instinct MI355X (gfx950).
 *
 * The operation (FASQ, Sec. 3.1.2, Eq. lut-accumulate; Sec. 2.2):
 *
 *   A weight matrix W_hat with N output features and K input features is never
 *   stored densely.  Each output row n is cut along K into S = K / d
 *   sub-vectors of length d, and sub-vector s is replaced by the id u(n, s) of
 *   one of C fp16 codewords:
 *
 *       W_hat[n, s*d + i] = codebook[u(n, s) * d + i]        (0 <= i < d)
 *       y[m, n]           = sum_s dot(x[m, s*d : s*d + d], codebook[u(n, s)])
 *                         = (x . W_hat^T)[m, n]
 *
 *   One codebook is shared by every sub-vector of the matrix (the paper's
 *   per-subspace tables with all tables equal).
 *
 * Layouts (all buffers are DEVICE memory, owned and allocated by the caller):
 *   x        fp16 [M x K], row-major, contiguous.
 *   y        fp16 [M x N], row-major, contiguous; every element is written
 *            (no zeroing needed).  Accumulation is fp32; each output is rounded
 *            to fp16 (round to nearest even) exactly once.
 *   codebook fp16 [C x d], row-major.
 *   idx      N rows of R = fasq_idx_row_bytes(K, d, idx_bits) bytes, back to
 *            back (row n starts at byte n*R).  Within a row the ids form one
 *            least-significant-bit-first bit stream: id s occupies stream bits
 *            [idx_bits*s, idx_bits*s + idx_bits), and stream bit t is bit
 *            (t mod 8) of byte (t div 8).  So idx_bits = 8 is one byte per id,
 *            16 a little-endian byte pair, and 12 packs two ids in three bytes
 *            (b0 = u0 & 0xFF, b1 = (u0 >> 8) | (u1 & 0xF) << 4, b2 = u1 >> 4).
 *            The pad bits of an odd 12-bit row are ignored.
 *
 * Conventions:
 *   - Every call is asynchronous on `stream` (0 = the null stream).  The
 *     library allocates no device memory and, outside launch lists (below),
 *     keeps no pointer after returning, so the calls may be captured in a
 *     hipGraph.  The plain entry
 *     points use no scratch memory; the _ex calls and the encoder take a
 *     caller-owned workspace argument for theirs.
 *   - Argument checks run before any HIP call.  A bad argument returns
 *     FASQ_ERR_INVALID_ARG and launches nothing.  A failed launch returns
 *     FASQ_ERR_HIP.  fasq_last_error() then describes the failure (per calling
 *     thread).  A fault inside a kernel surfaces at the caller's next
 *     synchronisation.
 *   - Preconditions that are NOT checked: every id is < C (an id >= C reads
 *     outside the codebook); x, y, idx and codebook do not overlap.
 *   - Calls that share no output buffer may run concurrently from any thread.
 *   - Results are deterministic: the same inputs give the same bits.
 */
#ifndef FASQ_H
#define FASQ_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FASQ_ABI_VERSION 8

typedef enum {
  FASQ_OK = 0,
  FASQ_ERR_INVALID_ARG = 1, /* a size, pointer or format argument is invalid */
  FASQ_ERR_UNSUPPORTED = 2, /* valid, but no kernel handles this combination */
  FASQ_ERR_HIP = 3,         /* the HIP runtime reported an error */
  FASQ_ERR_HOST_MEMORY = 4  /* host memory for a launch list could not be allocated */
} fasq_status;

/*
 * Decode regime (FASQ Sec. 4.1, the batch-1 GEMV of the decode phase):
 * y[M x N] = x[M x K] . W_hat^T.  Tuned for M <= 16 (M = 1 is token-by-token
 * decode); any M >= 1 is accepted and computed correctly.  This is also the
 * batch-adaptive entry point the paper leaves to future work (Sec. 4.4,
 * batch size): rows of x beyond 16, or operands the decode kernels cannot
 * hold on chip, go to the prefill kernel of fasq_pq_gemm.
 *
 *   x, M, K     activations, fp16 [M x K]
 *   N           output features (rows of the index table)
 *   idx         packed ids, N rows of fasq_idx_row_bytes(K, d, idx_bits) bytes
 *   idx_bits    8, 12 or 16
 *   d           sub-vector length, d >= 1, K % d == 0
 *   codebook, C fp16 [C x d], 1 <= C <= 2^idx_bits
 *   y           output, fp16 [M x N]
 *   stream      HIP stream the kernels are queued on
 *
 * Returns FASQ_OK, FASQ_ERR_INVALID_ARG (M, K, N < 1; d < 1; K % d != 0;
 * idx_bits not in {8, 12, 16}; C outside [1, 2^idx_bits]; a NULL pointer) or
 * FASQ_ERR_HIP.
 */
fasq_status fasq_pq_gemv(const void* x, int64_t M, int64_t K, int64_t N,
                         const void* idx, int idx_bits, int d,
                         const void* codebook, int64_t C,
                         void* y, hipStream_t stream);

/*
 * Decode regime over several weight matrices that read the same activations
 * (FASQ Sec. 4.1; in a decoder layer the q, k and v projections share their
 * input, and so do the gate and up projections): for i < count,
 *
 *   y[i][M x N[i]] = x[M x K] . W_hat_i^T
 *
 * with W_hat_i given by idx[i] (N[i] rows of fasq_idx_row_bytes(K, d,
 * idx_bits) bytes) and codebook[i] (fp16 [C[i] x d]).  x, M, K, idx_bits and d
 * are shared; every array holds `count` entries and lives in HOST memory,
 * while the buffers it points to are device memory.  For M <= 16 up to eight
 * matrices run in one launch; when no grouped kernel applies (d = 3, for
 * instance) the matrices are computed one call after another.  Every y[i] is
 * bit-for-bit what fasq_pq_gemv would write for matrix i alone.
 *
 * Returns FASQ_ERR_INVALID_ARG when count < 1, an array is NULL, or any
 * matrix fails the checks of fasq_pq_gemv (fasq_last_error() names the
 * matrix); FASQ_ERR_HIP on a launch error.  The y buffers must not overlap
 * one another or any input.
 */
fasq_status fasq_pq_gemv_batched(const void* x, int64_t M, int64_t K, int count,
                                 const void* const* idx, const int64_t* N,
                                 const void* const* codebook, const int64_t* C,
                                 void* const* y, int idx_bits, int d, hipStream_t stream);

/*
 * Prefill regime (FASQ Sec. 4.2: many tokens share one weight matrix).  Same
 * operation, arguments, layouts and errors as fasq_pq_gemv; built for M in the
 * tens to thousands.  Weight tiles are decoded from the ids into on-chip
 * memory and contracted with matrix-core (MFMA) instructions, fp16 inputs,
 * fp32 accumulation.
 */
fasq_status fasq_pq_gemm(const void* x, int64_t M, int64_t K, int64_t N,
                         const void* idx, int idx_bits, int d,
                         const void* codebook, int64_t C,
                         void* y, hipStream_t stream);

/*
 * fasq_pq_gemm with a workspace (FASQ Sec. 4.2 splits the subspaces, i.e. K,
 * over blocks; Sec. 4.4 tunes the split for the prefill length).  When the
 * output tiles alone leave compute units idle (small M or N), the tuned
 * kernel also splits K over up to 8 workgroups per tile, which write fp32
 * partial sums to the workspace; a second kernel adds them in a fixed order
 * and rounds once to fp16 (deterministic for a given shape and device).
 *
 *   workspace  device scratch of at least fasq_pq_gemm_ex_workspace_bytes()
 *              bytes (4-byte aligned; may be NULL when that is 0); contents
 *              are overwritten.  A NULL or smaller workspace runs exactly
 *              fasq_pq_gemm (no split).
 *
 * Other arguments, layouts and errors as fasq_pq_gemm, plus
 * FASQ_ERR_INVALID_ARG for workspace_bytes < 0.
 */
fasq_status fasq_pq_gemm_ex(const void* x, int64_t M, int64_t K, int64_t N,
                            const void* idx, int idx_bits, int d,
                            const void* codebook, int64_t C,
                            void* y, void* workspace, int64_t workspace_bytes,
                            hipStream_t stream);

/* Workspace bytes fasq_pq_gemm_ex splits K with on the current device (0
 * when it would not split), -1 for invalid sizes. */
int64_t fasq_pq_gemm_ex_workspace_bytes(int64_t M, int64_t K, int64_t N, int idx_bits, int d, int64_t C);

/*
 * The paper's own prefill kernel design (FASQ Sec. 4.2, Alg. 3), kept for
 * comparison with fasq_pq_gemm: per token and subspace a lookup table of the
 * C dot products x_s . codebook[k] is built in LDS (fp32), and every output
 * feature adds up its table entries.  No matrix cores.  Same arguments,
 * layouts and errors as fasq_pq_gemm, plus FASQ_ERR_UNSUPPORTED when d is not
 * in {1, 2, 4, 8} or C > 2048 (the tables would not fit in LDS).
 */
fasq_status fasq_pq_gemm_lut(const void* x, int64_t M, int64_t K, int64_t N,
                             const void* idx, int idx_bits, int d,
                             const void* codebook, int64_t C,
                             void* y, hipStream_t stream);

/*
 * Decode regime with the paper's general codebook layout (FASQ Sec. 3.1.1:
 * T_cluster is [N_ss x K_s x SZ_ss], one codebook per subspace; Eq.
 * lut-accumulate):
 *
 *   y[m, n] = sum_s dot(x[m, s*d : (s+1)*d], codebook[s * cb_stride + u(n, s) * d .. + d])
 *
 *   cb_stride  0: one codebook [C x d] shared by every subspace (exactly
 *              fasq_pq_gemv); C * d: one codebook per subspace, the S = K / d
 *              books back to back, fp16 [S x C x d].  Other values are invalid.
 *   workspace  device scratch of at least fasq_pq_gemv_ex_workspace_bytes()
 *              bytes (4-byte aligned; NULL when that is 0), for the fp32
 *              partial sums of the K split; contents are overwritten
 *
 * Other arguments, layouts and errors as fasq_pq_gemv.  With per-subspace
 * books and M <= 16 the tuned kernel splits K over workgroups whose books fit
 * in LDS and adds the partials in a fixed order (deterministic; each token's
 * output has the bits a call with that token alone gives); for M > 1 it needs
 * d <= 4 and x 16-byte aligned with K * 2 a multiple of 16.  Other shapes, or
 * a workspace that is too small, take the general kernel.  With one shared
 * codebook the call is fasq_pq_gemv, except that the workspace lets the
 * prefill GEMM split K as fasq_pq_gemm_ex does where the GEMM takes the call:
 * beyond 16 tokens, where no decode kernel applies, and, from 12 tokens on,
 * where the decode kernel would stage x in slabs, the GEMM keeps its codebook
 * in LDS and the decode kernel's own K split (below) would leave compute units
 * idle (the measured crossover of Sec. 4.4's batch-size trade-off);
 * and it lets the decode kernel for 3 to 16 tokens split K over workgroups
 * where the rows of x outweigh a workgroup's share of the ids (tall K, few
 * rows: 2 to 8 segments, at most 4 MiB of fp32 partials, added in segment
 * order by a second kernel; deterministic, though not the bits of the
 * unsplit call).
 */
fasq_status fasq_pq_gemv_ex(const void* x, int64_t M, int64_t K, int64_t N,
                            const void* idx, int idx_bits, int d,
                            const void* codebook, int64_t C, int64_t cb_stride,
                            void* y, void* workspace, int64_t workspace_bytes,
                            hipStream_t stream);

/* Workspace bytes fasq_pq_gemv_ex uses on the current device for these sizes
 * (per-subspace books: the tuned kernel's partials; one shared codebook: the
 * K split of the GEMM fallback), 0 when none is used, -1 for invalid sizes. */
int64_t fasq_pq_gemv_ex_workspace_bytes(int64_t M, int64_t K, int64_t N, int idx_bits, int d,
                                        int64_t C, int64_t cb_stride);

/*
 * fasq_pq_gemv_ex for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation).
 * Same operation, arguments (minus the workspace), layouts and results as
 * fasq_pq_gemv_ex: the scratch that call would take from a caller workspace
 * (the per-subspace K split, the decode kernel's K split, or the K split of
 * the GEMM fallback) comes from
 * a static device array the library holds on every GPU it runs on, of
 * fasq_noalloc_scratch_bytes() = FASQ_NOALLOC_SCRATCH_BYTES bytes, kept until
 * the process ends.  The call allocates nothing: no hipMalloc, no allocating
 * library routine.  Its device address is looked up once per device, on the
 * first call made with that device current.
 *
 * Every call on one GPU shares that GPU's array, and the array keeps the last
 * call's contents: calls that overlap on one GPU (concurrent streams or
 * threads) race on it and must be serialised by the caller.  Calls on
 * different GPUs do not interact.
 *
 * Returns FASQ_ERR_INVALID_ARG for the checks of fasq_pq_gemv_ex and when
 * fasq_pq_gemv_ex_workspace_bytes() of these sizes exceeds the array
 * (fasq_last_error() gives both figures; such calls need fasq_pq_gemv_ex
 * with a workspace), FASQ_ERR_HIP when the array cannot be located or a
 * launch fails.
 */
#define FASQ_NOALLOC_SCRATCH_BYTES (16 * 1024 * 1024)
fasq_status fasq_pq_gemv_ex_noalloc(const void* x, int64_t M, int64_t K, int64_t N,
                                    const void* idx, int idx_bits, int d,
                                    const void* codebook, int64_t C, int64_t cb_stride,
                                    void* y, hipStream_t stream);

/* Bytes of the per-device scratch array of fasq_pq_gemv_ex_noalloc. */
int64_t fasq_noalloc_scratch_bytes(void);

/*
 * Calibration-free PQ encoding of one weight matrix (FASQ Sec. 3.1.1, Alg. 1):
 * Lloyd's k-means over the N * K / d sub-vectors of w, with one codebook of C
 * codewords shared by every subspace (the format the matmul entry points
 * consume).  No calibration data: only the weights.
 *
 *   w              fp16 [N x K], row-major; sub-vector p = n * (K / d) + s is
 *                  w[n, s*d : (s+1)*d]; finite, |w| < 128 (unchecked)
 *   d, C, idx_bits sub-vector length (1 <= d <= 16), codewords, id width
 *   init_codebook  fp16 [C x d], the starting codewords (for example C
 *                  distinct sub-vectors of w chosen at random); may be the
 *                  same buffer as `codebook`
 *   iters          Lloyd iterations (assignment, then update), >= 0
 *   codebook       out: fp16 [C x d], the codewords after `iters` updates
 *   idx            out: N rows of fasq_idx_row_bytes(K, d, idx_bits) bytes,
 *                  the nearest codeword of every sub-vector under the final
 *                  codebook, in the packed format of fasq_pq_gemv
 *   workspace      device scratch of at least
 *                  fasq_pq_encode_workspace_bytes(N, K, d, C) bytes, 8-byte
 *                  aligned; its contents are overwritten
 *
 * Arithmetic (the paper leaves it open): squared distances in fp32, summed
 * over the d components in order without fused multiply-add, the lowest index
 * winning a tie; cluster sums formed exactly (every fp16 value is a multiple
 * of 2^-24), the mean divided out in fp64 and rounded to fp16 (nearest, ties
 * to even); an empty cluster keeps its codeword.  The result does not depend
 * on scheduling: repeated calls give identical bits.
 *
 * Asynchronous on `stream`; the caller owns every buffer.  Returns
 * FASQ_ERR_INVALID_ARG (sizes; d does not divide K; idx_bits not in
 * {8, 12, 16}; C outside [1, 2^idx_bits]; iters < 0; a NULL or misaligned
 * pointer; a workspace that is too small), FASQ_ERR_UNSUPPORTED (d > 16) or
 * FASQ_ERR_HIP.
 */
fasq_status fasq_pq_encode(const void* w, int64_t N, int64_t K, int d, int64_t C, int idx_bits,
                           const void* init_codebook, int iters, void* codebook, void* idx,
                           void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Workspace bytes fasq_pq_encode needs for these sizes; -1 if they are invalid
 * (N, K < 1; d does not divide K; C outside [1, 65536]). */
int64_t fasq_pq_encode_workspace_bytes(int64_t N, int64_t K, int d, int64_t C);

/*
 * Launch lists: the kernel launches of a sequence of library calls, recorded
 * once and queued again as often as needed, for callers that issue the same
 * calls with the same buffers at every step (a serving loop's decode step, a
 * benchmark) and want to pay only for the launches: no argument checks, no
 * kernel selection, no HIP graph.  Between fasq_launch_list_begin and
 * fasq_launch_list_end, every fasq_* compute call made on the calling thread
 * (fasq_pq_gemv, _batched, _ex, _ex_noalloc, fasq_pq_gemm, _ex, _lut,
 * fasq_pq_reconstruct, fasq_pq_encode, and the entry points between the
 * projections below) validates its arguments and chooses its kernels as usual,
 * then appends its launches (kernel, grid, block, LDS bytes and a copy of the
 * argument values) to the list instead of queueing them; its `stream` argument
 * is ignored.  fasq_launch_list_run queues every recorded
 * launch, in recording order, on `stream`.  A run computes what the recorded
 * calls would have computed at that point of the stream, bit for bit.
 *
 * The list holds the device addresses the calls were given (inputs, outputs,
 * workspaces, the static array of fasq_pq_gemv_ex_noalloc): they must stay
 * valid while the list may run, and a run reads and writes their contents as
 * they are when it executes.  A list records for the device current at
 * fasq_launch_list_begin and runs only with that device current (its
 * recorded launches from later begin/end pairs are appended and must be on
 * the same device).  A call that fails while recording returns its error and
 * may leave part of its launches in the list: destroy such a list.
 *
 *   fasq_launch_list_create   *list = a new, empty list.  FASQ_ERR_INVALID_ARG
 *                             (list is NULL), FASQ_ERR_HOST_MEMORY.
 *   fasq_launch_list_begin    the calling thread records into `list`.
 *                             FASQ_ERR_INVALID_ARG when list is NULL, the
 *                             thread already records a list, the list records
 *                             on another thread, or it holds launches for
 *                             another device; FASQ_ERR_HIP when no device is
 *                             current.
 *   fasq_launch_list_end      stop recording.  FASQ_ERR_INVALID_ARG when
 *                             `list` does not record on the calling thread.
 *   fasq_launch_list_run      queue the launches on `stream` (asynchronous).
 *                             FASQ_ERR_INVALID_ARG when list is NULL, it
 *                             records, the calling thread records a list, or
 *                             another device is current; FASQ_ERR_HIP when a
 *                             launch fails (fasq_last_error() names which;
 *                             the launches before it are queued).  An empty
 *                             list queues nothing.  Runs from several threads
 *                             may share a list.
 *   fasq_launch_list_size     launches recorded, -1 for a NULL list.
 *   fasq_launch_list_destroy  free the list (and stop recording into it on the
 *                             calling thread); NULL is ignored.  Launches
 *                             already queued are not affected.  No other
 *                             thread may record into the list, or run it,
 *                             while it is destroyed, and no thread may
 *                             record into a list that another thread runs.
 */
typedef struct fasq_launch_list fasq_launch_list;
fasq_status fasq_launch_list_create(fasq_launch_list** list);
fasq_status fasq_launch_list_begin(fasq_launch_list* list);
fasq_status fasq_launch_list_end(fasq_launch_list* list);
fasq_status fasq_launch_list_run(const fasq_launch_list* list, hipStream_t stream);
int64_t fasq_launch_list_size(const fasq_launch_list* list);
void fasq_launch_list_destroy(fasq_launch_list* list);

/*
 * Decode W_hat explicitly (the reconstruction the paper's reconstruction-free
 * kernels avoid, Sec. 3.1.2).  Writes fp16 [N x K] to `w`; every element is a
 * bit-for-bit copy of a codebook entry (signed zeros, subnormals, NaN
 * payloads preserved).  Diagnostic only: it is how the decoder is tested.
 * Errors as for fasq_pq_gemv.
 */
fasq_status fasq_pq_reconstruct(const void* idx, int64_t N, int64_t K, int idx_bits, int d,
                                const void* codebook, int64_t C, void* w,
                                hipStream_t stream);

/*
 * ---------------------------------------------------------------------------
 * Between the projections of a decoder layer: rotary positions and the write
 * of a paged cache, attention over that cache, the residual stream's norms,
 * and low-rank adapters beside the projections.  As everywhere in the
 * library the values are fp16, sums and softmax statistics are fp32, every
 * call is asynchronous on `stream`, allocates nothing and can be captured in
 * a hipGraph or recorded into a launch list.  What changes from step to step
 * (positions, slots, lengths, page tables, adapter ids) is read from device
 * memory when the kernels run, so one recorded step serves every step of the
 * same shape.  Zero tokens (T or M = 0) is a valid call that launches
 * nothing.  Strides are in elements; the last dimension of every tensor is
 * contiguous.  Inputs may be broadcast (strides of 0), what is written may not:
 * its strides of more than one row are at least D.
 * ---------------------------------------------------------------------------
 */

/*
 * A paged cache of keys and values: element i of head h in slot t of page p
 * is k[p * page_stride + t * slot_stride + h * head_stride + i], and the same
 * for v.  So [pages x page_size x heads x D] and [pages x heads x page_size x
 * D] are both caches.  Offsets are formed in 64 bits.
 */
typedef struct {
  void* k;
  void* v;
  int64_t num_pages;
  int64_t page_size;
  int64_t page_stride, slot_stride, head_stride;
} fasq_kv_cache;

/*
 * Rotary table: table[p][i] = (cos(p w_i), sin(p w_i)) * scale for positions
 * 0 <= p < positions and the `half` frequencies w_i of inv_freq, a HOST array
 * (copied during the call).  Angles are formed in 64 bits and each value is
 * rounded to fp32 once, so that the table is as good at position 131072 as
 * at 0.  Scaled variants for long contexts differ in w and scale only.
 *
 *   table  out: fp32 [positions x half x 2], 8-byte aligned
 *
 * Returns FASQ_ERR_INVALID_ARG (half outside [1, 128]; positions < 1 or above
 * 2^31; a NULL or misaligned pointer) or FASQ_ERR_HIP.
 */
fasq_status fasq_rope_table(const double* inv_freq, int half, int64_t positions, double scale,
                            float* table, hipStream_t stream);

/*
 * Rotary positions of T new tokens, and the write of their keys and values
 * to the cache.  For each token t and head of q and k:
 *
 *   x = head, or, with a norm weight w,  x = head / sqrt(mean(head^2) + eps) * w
 *   (x_a, x_b) -> (x_a c - x_b s, x_b c + x_a s),  (c, s) = table[positions[t]][i]
 *
 * for the rot / 2 pairs i: (a, b) = (i, i + rot / 2), or (2i, 2i + 1) with
 * `interleaved`.  Dimensions from rot on are not turned.  q goes to q_out; k
 * and the unchanged v go to cache slot slots[t] = page * page_size + offset.
 * Arithmetic is fp32, rounded to fp16 once.
 *
 *   q, q_out    fp16 [T x Hq x D] with token and head strides; q_out may be q
 *               (with the same strides).  Both NULL: keys and values only
 *   k, v        fp16 [T x Hkv x D] with strides; both NULL (cache and slots
 *               are then not used): queries only
 *   D           1 <= D <= 256
 *   table, table_positions, rot
 *               the table of fasq_rope_table with rot / 2 frequencies; rot
 *               even, 0 <= rot <= D.  rot = 0: no rotation (table and
 *               positions are not used)
 *   positions   int32 [T]; a position outside [0, table_positions) turns its
 *               token into NaN (in q_out and in the cache's k)
 *   slots       int32 [T], distinct; a slot outside [0, num_pages *
 *               page_size) is not written (padding tokens: -1)
 *   q_norm, k_norm  fp16 [D] or NULL
 *
 * Returns FASQ_ERR_INVALID_ARG or FASQ_ERR_HIP.
 */
fasq_status fasq_rope_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, int Hq,
                             void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                             const void* k, int64_t k_token_stride, int64_t k_head_stride,
                             const void* v, int64_t v_token_stride, int64_t v_head_stride, int Hkv,
                             int64_t T, int D, const float* table, int64_t table_positions, int rot,
                             int interleaved, const int32_t* positions, const int32_t* slots,
                             const void* q_norm, const void* k_norm, float eps,
                             const fasq_kv_cache* cache, hipStream_t stream);

/*
 * Attention of the new tokens of B requests over a paged cache that already
 * holds their keys and values.  Request b has the tokens q_start[b] <= t <
 * q_start[b + 1] of q (n of them, in the order of their positions) and the
 * first kv_len[b] slots of its pages: key j is slot j % page_size of page
 * pages[b][j / page_size].  Token i of the request stands at position
 * p = kv_len[b] - n + i and sees the keys
 *
 *   j <= p (causal) or j < kv_len[b];  with window > 0 also j > p - window
 *
 *   s_j = scale * q . k_j;   out = sum_j exp(s_j - lse) v_j,  lse = log sum_j exp(s_j)
 *
 * with query head h on cache head h / (Hq / Hkv).  A token that sees no key
 * gets out = 0 and lse = -inf.  Keys and values that a token does not see do
 * not reach its output, whatever they hold (NaN and infinities included), and
 * what is stored past kv_len is never used.
 * The weights exp(s_j - lse) are rounded to fp16 (relative 2^-12 down to 2^-21
 * of a token's largest one, in steps of at most 2^-31 of it below).
 *
 *   q, out      fp16 [T x Hq x D] with token and head strides, which do not
 *               overlap; tokens outside every request are neither read nor written;
 *               T * (Hq / Hkv) <= 2^30
 *   cache       16-byte aligned, strides multiples of 8
 *   D           a multiple of 8, 8 <= D <= 256
 *   pages       int32 [B x max_pages], row stride page_row_stride; entries
 *               past a request's last page are not used, others lie in
 *               [0, num_pages) (an entry outside is read as the nearest page)
 *   B           requests, at most 2^16; 0 only with T = 0 (as max_pages)
 *   q_start     int32 [B + 1], not decreasing, within [0, T]
 *   kv_len      int32 [B], at most max_pages * page_size (more is cut there),
 *               which is at most 2^31 - 1024
 *   lse         fp32 [T x Hq], contiguous, or NULL
 *   workspace   device scratch of fasq_paged_attention_workspace_bytes()
 *               bytes (16-byte aligned) for the fp32 partial results, where
 *               the keys of a tile are split over workgroups; joined in a
 *               fixed order by a second kernel.  NULL or a smaller one: no
 *               split (slower where there are few tokens and long caches)
 *
 * The keys are split by what q_start and kv_len hold when the kernels run, so
 * the bits of a request's result may depend on the others in the batch; the
 * same batch gives the same bits.
 *
 * Returns FASQ_ERR_INVALID_ARG, FASQ_ERR_UNSUPPORTED (D not a multiple of 8
 * or above 256) or FASQ_ERR_HIP.
 */
fasq_status fasq_paged_attention(const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t T, int Hq,
                                 const fasq_kv_cache* cache, int Hkv, int D,
                                 const int32_t* pages, int64_t page_row_stride, int64_t max_pages,
                                 const int32_t* q_start, const int32_t* kv_len, int64_t B,
                                 float scale, int causal, int64_t window,
                                 void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                                 void* workspace, int64_t workspace_bytes, hipStream_t stream);

/*
 * What attention may have besides (fasq_paged_attention_ex).  A field that is 0
 * or NULL is not there; with all of them so the call is fasq_paged_attention.
 *
 *   softcap  c > 0: a score s becomes c * tanh(s / c).  2^-10 <= c <= 1024, |scale|
 *            <= 2^64; a capped score is off by at most 2^-21 c
 *   slopes   fp32 [Hq]: query head h at position p adds -slopes[h] * |p - j| to its
 *            score with key j (before a cap).  2^-24 <= |scale| <= 2^64; slopes[h] / scale
 *            within fp32, and negative ones times the longest distance too
 *   spans    int32 [T x 2]: token t sees the keys spans[t][0] <= j < spans[t][1]
 *            (cut to what there is) in place of causal and window (window must
 *            be 0): documents packed into one request, prefixes that are read in
 *            both directions, windows over other positions
 *   tree     int32 [T rows of tree_words words, tree_stride words apart]: of the
 *            request's n new tokens, which are its last n keys, token t sees the
 *            i-th exactly if bit i % 32 of its word i / 32 is set (itself among
 *            them); words past tree_words are zero, bits from n on are not used.
 *            The keys before the new tokens it sees all, or those of its span;
 *            causal is not used and window must be 0.  Not with slopes
 */
typedef struct {
  float softcap;
  const float* slopes;
  const int32_t* spans;
  const int32_t* tree;
  int64_t tree_stride, tree_words;
} fasq_attention_scores;

/*
 * fasq_paged_attention with scores and masks of the call's own; `scores` NULL:
 * none.  Everything else, the workspace too, is as there: a token that sees no
 * key gets out = 0 and lse = -inf, and what a token does not see does not reach
 * its output, whatever it holds.
 *
 * Returns FASQ_ERR_INVALID_ARG, FASQ_ERR_UNSUPPORTED (as there; softcap above
 * 1024; slopes with tree) or FASQ_ERR_HIP.
 */
fasq_status fasq_paged_attention_ex(const void* q, int64_t q_token_stride, int64_t q_head_stride, int64_t T, int Hq,
                                    const fasq_kv_cache* cache, int Hkv, int D,
                                    const int32_t* pages, int64_t page_row_stride, int64_t max_pages,
                                    const int32_t* q_start, const int32_t* kv_len, int64_t B,
                                    float scale, int causal, int64_t window, const fasq_attention_scores* scores,
                                    void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                                    void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Workspace bytes fasq_paged_attention splits keys with on the current device
 * for T tokens of B requests (0 when it would not split), -1 for invalid
 * sizes. */
int64_t fasq_paged_attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D);

/*
 * What stands between a model's logits and a token (fasq_process_logits).  Row r
 * belongs to request s = requests[r].  A field that is NULL is not there.
 *
 *   requests      int32 [R]; NULL: row r is request r (S = R).  A row whose request
 *                 lies outside [0, S) is not written
 *   S             requests, at most 2^24
 *   tokens        int32 [S rows of max_tokens, token_stride apart]: a request's
 *                 prompt and then its answer so far, token_count[s] of them (int32
 *                 [S]; cut to max_tokens, at most 2^30), the first prompt_len[s]
 *                 (int32 [S]; NULL: none) the prompt.  Ids outside [0, V) do not count
 *   repetition    fp32 [S], positive: a logit x of a token that occurs becomes
 *                 x * (1 / repetition) if x > 0, else x * repetition
 *   frequency     fp32 [S]: less frequency * n + presence for a token that occurs n
 *   presence      > 0 times in the answer
 *   bias_ids      int32 [S x max_bias] (at most 2^24) and bias_values fp32: added to these tokens'
 *   bias_values   logits; a token's last entry counts, ids outside [0, V) do not
 *   temperature   fp32 [S]: times 1 / temperature where that is positive (one below 2^-128
 *                 counts as that; infinity makes every finite logit 0)
 *   allowed       int32 [R rows of ceil(V / 32) words, allowed_stride apart]: a token
 *                 whose bit v % 32 of word v / 32 is clear becomes -inf, whatever it was
 *   draft_tokens  int32 [R], q_start int32 [S + 1], tree as in fasq_attention_scores:
 *   q_start, tree the rows of request s are q_start[s] <= r < q_start[s + 1], row r has
 *                 drafted draft_tokens[r], and the tokens of the rows that its bits
 *                 name (itself among them) are counted with its answer
 */
typedef struct {
  const int32_t* requests;
  int64_t S;
  const int32_t* tokens;
  int64_t token_stride, max_tokens;
  const int32_t* token_count;
  const int32_t* prompt_len;
  const float* repetition;
  const float* presence;
  const float* frequency;
  const int32_t* bias_ids;
  const float* bias_values;
  int64_t max_bias;
  const float* temperature;
  const int32_t* allowed;
  int64_t allowed_stride;
  const int32_t* draft_tokens;
  const int32_t* q_start;
  const int32_t* tree;
  int64_t tree_stride, tree_words;
} fasq_token_rules;

/*
 * R rows of V logits under the rules of `rules`, applied in the order above:
 * penalties, bias, temperature, mask.  Arithmetic is fp32, an operation at a
 * time (reciprocals rounded before they are used).
 *
 *   logits  fp16, or fp32 with logits_fp32; rows `stride` elements apart.  V <= 2^30
 *   out     fp16 or fp32 (out_fp32), rows out_stride apart, or NULL; may be logits
 *           (of the same type and stride), and overlaps nothing else
 *   choice  int32 [R] or NULL: the token of the largest value (before it is
 *           rounded to out), the lowest of equal ones; NaN is larger than
 *           all; -1 where every value is -inf
 *   lse     fp32 [R] or NULL: the logarithm of the sum of the values' exponentials
 *   workspace  device scratch of fasq_process_logits_workspace_bytes() bytes, 16-byte
 *           aligned, overwritten; not used without choice and lse
 *
 * Returns FASQ_ERR_INVALID_ARG or FASQ_ERR_HIP.
 */
fasq_status fasq_process_logits(const void* logits, int logits_fp32, int64_t stride, int64_t R, int64_t V,
                                const fasq_token_rules* rules, void* out, int out_fp32, int64_t out_stride,
                                int32_t* choice, float* lse, void* workspace, int64_t workspace_bytes,
                                hipStream_t stream);

/* Workspace bytes fasq_process_logits needs for choice or lse on the current
 * device; -1 for invalid sizes. */
int64_t fasq_process_logits_workspace_bytes(int64_t R, int64_t V);

/*
 * The residual stream between two blocks: the block's output y is normed (if
 * post_weight), gated (if gate), scaled and added to the stream, and the norm
 * that the next block reads is taken of the sum (if weight):
 *
 *   u     = y / sqrt(mean(y^2) + eps) * post_weight   or   y
 *   x_new = x + scale * gate * u
 *   h     = x_new / sqrt(mean(x_new^2) + eps) * weight
 *
 * over each of M rows of N values.  Arithmetic is fp32 throughout (h is taken
 * of the unrounded x_new); x_out and h are rounded to fp16 once.
 *
 *   x, y         fp16 [M x N], contiguous; y NULL: x_new = x (post_weight and
 *                gate must be NULL, x_out may be)
 *   post_weight, weight  fp16 [N] or NULL
 *   gate         fp16: [N] with gate_stride 0, or [M x N] with gate_stride N;
 *                NULL: 1
 *   x_out        fp16 [M x N] or NULL; may be x or y
 *   h            fp16 [M x N]; NULL exactly when weight is; may be x or y,
 *                not x_out
 *
 * Returns FASQ_ERR_INVALID_ARG (sizes; eps not positive and finite; nothing to
 * write) or FASQ_ERR_HIP.
 */
fasq_status fasq_residual_norm(const void* x, const void* y, int64_t M, int64_t N, const void* post_weight,
                               const void* gate, int64_t gate_stride, float scale, const void* weight, float eps,
                               void* x_out, void* h, hipStream_t stream);

/*
 * Low-rank adapters of many requests beside `count` projections that read the
 * same activations (q + k + v, gate + up, or one): for i < count and each of
 * M tokens with adapter a = adapters[m],
 *
 *   y[i][m] = base[i][m] + scales[a] * B[i][a] . (A[i][a] . x[m])
 *
 * and y[i][m] = base[i][m] where a lies outside [0, L) (a request without an
 * adapter).  base is what the shared projection gave (fasq_pq_gemv, _gemm and
 * their kin).  The low-rank values A x are fp32 and enter the second product
 * with 22 bits (those below 2^-17 of a token's largest in steps of 2^-38 of it),
 * sums are fp32, and y is rounded to fp16 once.
 * Adapters of a smaller rank than r are padded with zero rows in A.
 *
 *   x         fp16 [M x K]
 *   adapters  int32 [M], device memory: any order, any mix
 *   L, r      adapters in the pool, their rank (1 <= r <= 256)
 *   scales    fp32 [L]
 *   N, A, B, base, y   HOST arrays of `count` entries: sizes, and device
 *             buffers fp16 [L x r x K], [L x N[i] x r], [M x N[i]], [M x N[i]];
 *             N[i] <= 2^31 - 2^17; y[i] may be base[i]; base[i] NULL: zero
 *   workspace device scratch of fasq_lora_workspace_bytes() bytes, 16-byte
 *             aligned; contents are overwritten
 *
 * count is 1 to 8.  The K sum of a token does not depend on the other tokens'
 * values.  Returns FASQ_ERR_INVALID_ARG (sizes, count, a NULL or misaligned
 * pointer, a workspace that is too small), FASQ_ERR_UNSUPPORTED (r > 256) or
 * FASQ_ERR_HIP.
 */
fasq_status fasq_lora_batched(const void* x, int64_t M, int64_t K, const int32_t* adapters, int64_t L, int r,
                              const float* scales, int count, const int64_t* N, const void* const* A,
                              const void* const* B, const void* const* base, void* const* y,
                              void* workspace, int64_t workspace_bytes, hipStream_t stream);

/* Workspace bytes fasq_lora_batched needs for these sizes on the current
 * device; -1 if they are invalid. */
int64_t fasq_lora_workspace_bytes(int64_t M, int64_t K, int r, int count);

/*
 * Bytes of one packed index row: ceil((K / d) * idx_bits / 8).  Each of the
 * K / d sub-vectors of a row stores one codeword id of ceil(log2 K_s) bits
 * (FASQ Sec. 3.2, the index term of the storage footprint); ids are packed
 * as the bit stream described at the top of this file.  Returns -1 when
 * K < 1, d < 1, K % d != 0 or idx_bits is not 8, 12 or 16.  Host only.
 */
int64_t fasq_idx_row_bytes(int64_t K, int d, int idx_bits);

/* Static, human-readable name of a status code. */
const char* fasq_status_string(fasq_status s);

/*
 * Detail of the calling thread's most recent failed call ("" if none).  The
 * string stays valid until the thread's next fasq_* call.
 */
const char* fasq_last_error(void);

/* FASQ_ABI_VERSION of the built library. */
int fasq_abi_version(void);

/*
 * Diagnostic: the name of the kernel instantiation that fasq_pq_gemv
 * (regime 0), fasq_pq_gemm (regime 1) or fasq_pq_gemv_batched over two or
 * more matrices of these sizes (regime 2) would launch with 16-byte-aligned
 * buffers, e.g. "k_gemv_m1<8, 2, 2, 0, 0>" (template arguments in
 * declaration order).  Launches nothing; needs a current HIP
 * device.  Returns "" for invalid arguments or when no device is available.
 * The string is thread-local and valid until the thread's next fasq_* call.
 */
const char* fasq_pq_plan(int regime, int64_t M, int64_t K, int64_t N, int idx_bits, int d, int64_t C);

#ifdef __cplusplus
}
#endif

#endif /* FASQ_H */
