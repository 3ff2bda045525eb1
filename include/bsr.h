/*
 * bsr.h -- C ABI of the GB300 (sm_103a) block-sparse-row x dense product.
 *
 * Section 2.2 of "Algorithm to Compilation Co-design: An Integrated View of
 * Neural Network Sparsity" (Guo and Huang, 2021) stores a pruned weight
 * W[M, K] in Block Sparse Row form -- block values, block column indices and
 * block-row pointers, following SciPy -- and multiplies only the kept blocks
 * with the input tensor. Eq. 3 partitions W into blocks; here a block is
 * R x C: R consecutive rows of W (output features) by C consecutive columns
 * (input features). MB = M/R block rows, KB = K/C block columns.
 *
 *   indptr[MB+1]     int32, indptr[0] = 0, non-decreasing, indptr[MB] = nnzb
 *   indices[nnzb]    int32 block-column index, strictly ascending inside a row
 *   data[nnzb][R][C] block values, row-major inside each block
 *
 * The product (the paper's linear/attention projection, Y = X W^T + b):
 *   Y[n, i*R + r] = bias[i*R + r]
 *                 + sum_{p = indptr[i]}^{indptr[i+1]-1} sum_{c<C} X[n, indices[p]*C + c] * data[p][r][c]
 * with X[N, K] and Y[N, M] row-major. Element types: BSR_F32 (fp32 data, X
 * and Y, fp32 accumulation) or BSR_BF16 (bf16 data, X and Y, fp32
 * accumulation, Y rounded to nearest even). bias is always fp32 or NULL.
 * Plain TF32 is never used for BSR_F32. fp32 blocks of 32 or more rows with
 * 16 or 32 columns, and 16-row blocks of such width in weights of at least
 * 2^20 elements (M K), run on the tensor cores as 3xTF32: each operand is split
 * into a tf32 high part and a tf32 low part (the remainder) and the product is
 * hi*hi + hi*lo + lo*hi, accumulated in fp32. The dropped lo*lo term and the
 * rounding of the low parts leave a relative error near 2^-20 per product,
 * inside the fp32 tolerance |dY| <= 1e-5 * (sum |x||w| + |b|). Calls of 512
 * or more tokens on fp32 blocks that only the generic kernel would take
 * otherwise (64 or 128 rows with 1 to 8 columns) run on the gathered-K
 * tensor-core kernel, 3xTF32 in the same way. Every other fp32 shape
 * multiplies in plain fp32 FMA.
 *
 * Conventions.
 *  - Every call returns a status; the library never aborts, prints or traps.
 *  - Pointers marked "device" are global-memory pointers of the device that
 *    was current when the handle was created (for bsr_from_dense: the
 *    current device).
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *    stream). Work is enqueued on it; calls say when they synchronise.
 *  - Supported shapes: 1 <= R, C and R*C <= 4096, M % R == 0, K % C == 0,
 *    MB + 1, KB and nnzb below 2^31.
 *  - One handle must not run bsr_spmm on two streams at once (the split-row
 *    workspace and staging buffers belong to the handle).
 *  - bsr_residual_norm, bsr_gated and their backward calls, bsr_expert_* and bsr_fp8_*
 *    have no handle: they work on the current device and keep nothing between calls but the choice of
 *    tiles for the last 16 sizes (per thread; a size that is not among them costs a
 *    forward call of the gated block 0.5 us more, a backward call 5 to 14, one of
 *    65536 tokens 22). Scratch memory is the caller's, a buffer to each call in
 *    flight.
 */
#ifndef BSR_H
#define BSR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BSR_OK = 0,
    BSR_ERR_INVALID_ARG = 1, /* NULL where a pointer is needed, negative size, aliasing, bad threshold */
    BSR_ERR_SHAPE = 2,       /* M % R or K % C non-zero, sizes beyond int32 indexing */
    BSR_ERR_UNSUPPORTED = 3, /* block shape or dtype not supported */
    BSR_ERR_CAPACITY = 4,    /* output arrays of bsr_from_dense too small */
    BSR_ERR_STRUCTURE = 5,   /* indptr/indices are not a canonical BSR structure */
    BSR_ERR_ALIGNMENT = 6,   /* X or Y not 16-byte aligned, bias not 4-byte aligned */
    BSR_ERR_CUDA = 7,        /* a CUDA runtime call or kernel launch failed */
    BSR_ERR_TIMEOUT = 8,     /* a bounded device-side wait gave up (reported by bsr_check_device_status) */
    BSR_ERR_ALLOC = 9        /* device or host allocation failed */
} bsr_status_t;

typedef enum { BSR_F32 = 0, BSR_BF16 = 1 } bsr_dtype_t;

typedef struct bsr_handle_s *bsr_handle_t;
typedef struct bsr_plan_s *bsr_plan_t;

/*
 * bsr_from_dense -- build the BSR arrays of a dense weight on the GPU
 * (Section 2.2: "data values, indices, and indptr").
 *
 * W        device, [M, K] row-major, element type dt.
 * R, C     block shape. threshold: a block is kept iff at least one element
 *          w has !(|w| <= threshold) in fp32 (so NaN keeps its block, -0.0
 *          never does). threshold must be >= 0 and not NaN.
 * indptr   device, MB+1 int32, always written on success and on CAPACITY.
 * indices  device, capacity_blocks int32; data: device, capacity_blocks*R*C
 *          elements. Kept blocks appear in ascending column order per row,
 *          their values copied bit for bit (sub-threshold values included).
 * Query:   indices == NULL, data == NULL, capacity_blocks == 0 -> BSR_OK,
 *          *nnzb_out = number of kept blocks, only indptr written.
 * If capacity_blocks < nnzb: BSR_ERR_CAPACITY, *nnzb_out set, indices/data
 *          untouched. nnzb_out (host) may be NULL.
 * Synchronises `stream` once (to read nnzb). Temporary device memory is
 * allocated and freed inside the call.
 */
bsr_status_t bsr_from_dense(const void *W, int64_t M, int64_t K, int R, int C, float threshold,
                            bsr_dtype_t dt, int32_t *indptr, int32_t *indices, void *data,
                            int64_t capacity_blocks, int64_t *nnzb_out, void *stream);

/*
 * bsr_create -- analyse a BSR structure and build its execution schedule
 * (the counterpart of the paper's task buffer and auto-scheduler, Section
 * 2.2: tasks with identical structure are reused).
 *
 * indptr, indices, data: device arrays as described above. They are
 * BORROWED: the caller keeps them alive and unmodified until bsr_destroy.
 * Validates the structure on the host (one device-to-host copy of indptr and
 * indices, synchronous): indptr[0] == 0, non-decreasing, indices strictly
 * ascending per row and < K/C; otherwise BSR_ERR_STRUCTURE.
 * Owns: the schedule (shared with other handles of identical structure),
 * the work list, copies of data in the layouts of the kernels that calls may
 * run (bf16 weights among them as zero-filled rows of K: up to 2 M K bytes,
 * where that is at most 1 GB or 64 times the blocks), a device status word and
 * workspaces. *out receives the handle.
 */
bsr_status_t bsr_create(const int32_t *indptr, const int32_t *indices, const void *data, int R,
                        int C, int64_t M, int64_t K, bsr_dtype_t dt, bsr_handle_t *out);

/*
 * bsr_reserve -- size the handle's workspaces for up to N_max tokens so that
 * later bsr_spmm calls with N <= N_max allocate nothing (needed before
 * capturing bsr_spmm in a CUDA graph). Synchronous.
 */
bsr_status_t bsr_reserve(bsr_handle_t h, int64_t N_max);

/*
 * bsr_spmm -- Y[N, M] = X[N, K] W^T + bias[M] over the kept blocks.
 *
 * X, Y     row-major, element type of the handle, 16-byte aligned, not
 *          overlapping (else BSR_ERR_ALIGNMENT / BSR_ERR_INVALID_ARG).
 *          Both device pointers, or both host pointers: with host pointers
 *          the call copies X in and Y out on `stream` through device staging
 *          buffers owned by the handle; Y is valid once `stream` has
 *          synchronised.
 * bias     device, fp32 [M], or NULL for zero.
 * N        tokens; N == 0 is a no-op returning BSR_OK.
 * Asynchronous on `stream`; never synchronises unless a workspace must grow
 * beyond what bsr_reserve sized (then it allocates). Kernel launch failures
 * return BSR_ERR_CUDA.
 */
bsr_status_t bsr_spmm(bsr_handle_t h, const void *X, const float *bias, void *Y, int64_t N,
                      void *stream);

/*
 * bsr_check_device_status -- synchronise the device and return the first
 * error a kernel of this handle recorded (BSR_ERR_TIMEOUT when a bounded
 * wait gave up), then clear it. BSR_OK if none. Structure errors are not
 * reported here: bsr_create validates indptr/indices on the host and the
 * kernels take the structure from the handle's own copy of what it validated.
 */
bsr_status_t bsr_check_device_status(bsr_handle_t h);

/*
 * bsr_get_call_info -- which kernel a bsr_spmm call of N tokens runs, and how
 * many launches it makes, as "key=value" lines:
 *   kernel    "xstage" (SIMT, per task), "xcol" (SIMT, column lists), "tcgen05"
 *             (tensor cores, block by block), "dense" (tensor cores, bf16 weight
 *             as zero-filled tiles), "gk" (tensor cores, gathered columns),
 *             "tcp" (opt-in), "generic", or "none" (N = 0)
 *   launches  kernel launches of the call (with the reduce pass, if any)
 * Arguments as for bsr_get_schedule; BSR_ERR_INVALID_ARG for N < 0 too.
 */
bsr_status_t bsr_get_call_info(bsr_handle_t h, int64_t N, char *buf, size_t len);

/*
 * bsr_get_schedule -- a text description of the handle's schedule: kernel
 * variant, the kernels that it holds operands for (a call's is chosen from its
 * token count: bsr_get_call_info), execution block height and width (exec_R x exec_C: max(R, 16) x 64
 * where small or narrow bf16 blocks run on the tensor cores as zero-filled
 * tiles), tile sizes, work items, split
 * rows, launches per call, the schedule-cache statistics and the task sizes
 * each kernel can run (items per CTA; the size a call uses is chosen per
 * call from its token count), as "key=value" lines. Writes at most len bytes
 * including the terminating NUL into buf (truncating). Returns
 * BSR_ERR_INVALID_ARG for a NULL handle or buffer.
 */
bsr_status_t bsr_get_schedule(bsr_handle_t h, char *buf, size_t len);

/*
 * bsr_spmm_noalloc -- bsr_spmm for callers that cannot allocate device memory.
 *
 * The paper has no counterpart: this is a deployment aid. Some callers may
 * not call cudaMalloc at the point where they run the product: code inside
 * a CUDA graph capture (allocation there is not allowed), code bound to a
 * fixed memory budget or to its own allocator, and latency-critical loops
 * where an allocation's implicit device synchronisation is unacceptable.
 * bsr_spmm allocates when a call needs more split-row workspace than the
 * handle holds; this entry point never does.
 *
 * Same product and arguments as bsr_spmm, except that X and Y must be device
 * pointers (host buffers would need staging memory: BSR_ERR_INVALID_ARG).
 * The fp32 partial tiles of block rows that the schedule splits across CTAs
 * go to one scratch array compiled into the library, of
 * BSR_NOALLOC_SCRATCH_BYTES bytes, which every GPU that loads the library
 * holds until the process exits. A call needs slots * N * exec_R * 4 bytes
 * of it ("slots" and "exec_R" as reported by bsr_get_schedule; exec_R is the
 * block height the kernels run, 16 for small or narrow bf16 blocks re-blocked
 * for the tensor cores, else R); a larger call returns BSR_ERR_CAPACITY and
 * launches nothing.
 * The first call on a device looks up the array's device address
 * (cudaGetSymbolAddress, with that device current) and keeps it: make that
 * first call before any stream capture. All calls share the one array, so
 * calls whose kernels may run at the same time on the GPU (on streams with
 * no ordering between them) race and produce wrong results. The array keeps
 * the last call's contents; every element a call reads is written earlier
 * in the same call, so nothing is cleared.
 * Calls no cudaMalloc, cudaFree or allocating library routine.
 */
#define BSR_NOALLOC_SCRATCH_BYTES (32u << 20)
bsr_status_t bsr_spmm_noalloc(bsr_handle_t h, const void *X, const float *bias, void *Y, int64_t N,
                              void *stream);

/*
 * bsr_spmm_batch -- n products that share one input: Y_i = X · W_iᵀ + b_i.
 *
 * The paper prunes BERT (Section 2.3), whose self-attention applies several
 * weights (query, key, value) to the same activations; this entry point takes
 * such products together. Products whose weights run on the same kernel
 * configuration -- the per-task SIMT kernel with the same dtype, block shape and
 * task layout for the call's N, the column-list SIMT kernel with the same block
 * height, the block-by-block tensor-core kernel with the same dtype and block
 * height, or the dense-tile kernel with any block shapes -- are fused into one grid, up to 64 per launch, so one
 * product's last, partly filled wave overlaps the others' work; products on
 * the generic kernel run one after another on the same stream. Each output
 * is bit-identical to what bsr_spmm gives for the same arguments.
 *
 *   handles[n]  distinct handles, all on one device, one dtype and one K;
 *               BSR_ERR_INVALID_ARG for a NULL or repeated handle or a device
 *               or dtype mismatch, BSR_ERR_SHAPE for a K mismatch.
 *   X           device, [N, K] row-major, 16-byte aligned; read by all.
 *   biases      NULL (no bias anywhere) or n entries, each NULL or a device
 *               fp32 [M_i] array (4-byte aligned).
 *   Ys[n]       device, [N, M_i] row-major, 16-byte aligned; no output may
 *               overlap X, a bias or another output (BSR_ERR_INVALID_ARG).
 *   N           tokens; n == 0 or N == 0 is a no-op returning BSR_OK.
 *   stream      as in bsr_spmm. Host buffers are not accepted (BSR_ERR_INVALID_ARG).
 *
 * Asynchronous; like bsr_spmm it may grow a handle's split-row workspace (with
 * one stream synchronisation) unless bsr_reserve sized it for N beforehand.
 */
bsr_status_t bsr_spmm_batch(const bsr_handle_t *handles, int n, const void *X, const float *const *biases,
                            void *const *Ys, int64_t N, void *stream);

/*
 * bsr_plan_create -- a fixed sequence of n products, Y_i = X_i · W_iᵀ + b_i,
 * captured once into a CUDA graph that bsr_plan_launch replays.
 *
 * Section 2.2: the task scheduler keeps BSR tasks in a buffer, reuses
 * identical tasks and schedules similar ones next to each other. Identical
 * structures already share one schedule (bsr_create's cache); a plan adds the
 * adjacency for a whole sequence, such as every projection of a BERT model
 * (Section 2.3), and removes the per-call host work: validation, workspace
 * sizing and launch set-up happen here, once.
 *
 *   handles[n]   the weights (a handle may appear more than once); all on the
 *                current device, which must be the one they were created on.
 *                Each must outlive the plan (the plan uses its block values
 *                and status word); the plan owns its split-row workspaces, so
 *                later bsr_spmm calls on the same handles do not disturb it.
 *   X[n]         device, [N_i, K_i] row-major, 16-byte aligned.
 *   biases       NULL (no bias) or n entries, each NULL or device fp32 [M_i].
 *   Y[n]         device, [N_i, M_i] row-major, 16-byte aligned; Y_i must not
 *                overlap X_i or b_i.
 *   N[n]         tokens per product (>= 0; 0 is a no-op product).
 *   independent  0: the products run in the given order, one call each, so a
 *                later X may be an earlier Y (a chain of layers).
 *                1: the caller states that no product reads what another
 *                writes -- checked: no Y_i may overlap any X_j, b_j or other
 *                Y_j (BSR_ERR_INVALID_ARG otherwise) -- and the plan may
 *                reorder: products that share X and N are grouped in first-
 *                appearance order of their X, inside a group products whose
 *                kernels share a template come next to each other (handles
 *                that share a schedule adjacent) and run as fused grids as in
 *                bsr_spmm_batch (a handle repeated inside a group starts a new
 *                fused call). Outputs are bit-identical to bsr_spmm calls.
 *   out          receives the plan.
 *
 * The buffers are bound at capture: a replay reads the current contents of
 * X_i and b_i and writes Y_i. Synchronous (allocates the workspaces, captures
 * on a private stream); enqueues no device work. Errors: BSR_ERR_INVALID_ARG
 * (NULL, negative N, aliasing, host or foreign-device pointers),
 * BSR_ERR_ALIGNMENT, BSR_ERR_ALLOC, BSR_ERR_CUDA (capture or instantiation).
 */
bsr_status_t bsr_plan_create(const bsr_handle_t *handles, const void *const *X, const float *const *biases,
                             void *const *Y, const int64_t *N, int n, int independent, bsr_plan_t *out);

/* bsr_plan_launch -- replay the plan's graph on `stream` (asynchronous; the
 * products' device-side errors are reported per handle by
 * bsr_check_device_status). Two replays of one plan must not overlap in time
 * (they share the plan's workspaces). */
bsr_status_t bsr_plan_launch(bsr_plan_t plan, void *stream);

/* bsr_plan_get_order -- what the plan runs: order[k] = the product executed
 * k-th and call[k] = the index of the library call (one bsr_spmm, or one
 * fused bsr_spmm_batch group) that runs it, for k < n; products with N = 0
 * run nothing and are not listed, entries past the executed products are -1
 * (either array may be NULL); *n_kernels (if not NULL) = the kernel launches
 * in the graph. */
bsr_status_t bsr_plan_get_order(bsr_plan_t plan, int *order, int *call, int n, int *n_kernels);

/* bsr_plan_destroy -- release the graph and the workspaces. NULL is a no-op. */
void bsr_plan_destroy(bsr_plan_t plan);

/*
 * ---- The residual step between two blocks
 *
 * A transformer layer adds the output of a block (of bsr_spmm, of a
 * feed-forward block) to its residual stream; a norm may stand before and
 * after the block, a gate and a scale at its end:
 *
 *   t[n]  = post(y[n])
 *   h'[n] = alpha * h[n] + scale * gate[n / gate_tokens] * t[n]
 *   z[n]  = pre(h'[n])                       (the next block's input)
 *
 * post and pre: BSR_NORM_NONE (the row itself), BSR_NORM_LAYER
 * (x - mean) / sqrt(var + eps) * w + b with the biased variance, or BSR_NORM_RMS
 * x / sqrt(mean(x^2) + eps) * w + b. All arithmetic is in fp32; h' and z are
 * rounded once each, z is made from the unrounded h'.
 */
typedef enum { BSR_NORM_NONE = 0, BSR_NORM_LAYER = 1, BSR_NORM_RMS = 2 } bsr_norm_t;

typedef struct {
    int64_t D;             /* features, 1 .. 16384 (else BSR_ERR_SHAPE) */
    int64_t gate_tokens;   /* consecutive tokens that share a row of the gate: >= 1 with a gate, else unused */
    bsr_dtype_t block_dt;  /* element type of y, z, gate and their gradients */
    bsr_dtype_t stream_dt; /* element type of h, h' and their gradients: block_dt, or BSR_F32 beside bf16 blocks */
    bsr_norm_t post, pre;
    float post_eps, pre_eps;
    float alpha;
    const float *scale;            /* device fp32 [D], or NULL for 1 */
    const float *post_w, *post_b;  /* device fp32 [D], or NULL for 1 and 0; NULL without the norm */
    const float *pre_w, *pre_b;
} bsr_residual_norm_t;

/*
 * bsr_residual_norm -- h' and z from y and h.
 *
 * y, h     device, [N, D] row-major, 16-byte aligned. h NULL: no stream yet (0).
 * gate     device, [ceil(N / gate_tokens), D], 16-byte aligned, or NULL for 1.
 * h_out    receives h', or NULL where only z is wanted.
 * z        receives z; NULL if and only if pre is BSR_NORM_NONE (then h_out is needed).
 * A plain norm of y: h, gate and h_out NULL, post BSR_NORM_NONE.
 * h_out may be h and z may be y (the same addresses); outputs overlap nothing
 * else (BSR_ERR_INVALID_ARG). Device buffers only. N == 0 is a no-op.
 * Asynchronous on `stream`; allocates nothing. The current device's buffers.
 */
bsr_status_t bsr_residual_norm(const bsr_residual_norm_t *p, const void *y, const void *h, const void *gate, void *h_out,
                               void *z, int64_t N, void *stream);

/* The gradients of the parameters; each device, or NULL where not wanted (and
 * NULL where the parameter is absent). dgate has the gate's shape and type. */
typedef struct {
    void *dgate;
    float *dscale, *dpost_w, *dpost_b, *dpre_w, *dpre_b;
} bsr_residual_norm_grads_t;

/* Bytes of workspace of a backward call of N tokens (0 for N == 0), with or
 * without a gate of p->gate_tokens tokens a row. */
bsr_status_t bsr_residual_norm_workspace(const bsr_residual_norm_t *p, int64_t N, size_t *bytes);

/*
 * bsr_residual_norm_backward -- the gradients of y, h and the parameters, from
 * y, the h' that the forward call returned and the gradients of h' and z.
 *
 * h_out    the forward call's h'; needed if pre is a norm, else unused.
 * dh_out   the gradient of h' from what else reads it, or NULL for 0.
 * dz       the gradient of z; NULL if and only if pre is BSR_NORM_NONE.
 * dy, dh   receive the gradients of y and h; each may be NULL. dh may be dh_out,
 *          dy may be y or dz (the same addresses); else nothing overlaps.
 * grads    written, not added to (zeros for N == 0); NULL: none wanted.
 * ws       device, 16-byte aligned, of at least the bytes that
 *          bsr_residual_norm_workspace gives (else BSR_ERR_CAPACITY); used until
 *          the call's kernels have run.
 * Sums over tokens are added in a fixed order: the same call gives the same bits.
 */
bsr_status_t bsr_residual_norm_backward(const bsr_residual_norm_t *p, const void *y, const void *h_out, const void *gate,
                                        const void *dh_out, const void *dz, void *dy, void *dh,
                                        const bsr_residual_norm_grads_t *grads, int64_t N, void *ws, size_t ws_bytes,
                                        void *stream);

/*
 * ---- The gated feed-forward block
 *
 *   G = X Wg' + bg,  U = X Wu' + bu,  H = act(G) * U      (elementwise)
 *
 * with dense weights: the paper prunes a transformer's attention projections,
 * its feed-forward weights stay dense. H is what a down projection (bsr_spmm)
 * takes. X [N, K], Wg and Wu [F, K], H [N, F], row-major, element type dt; bg and
 * bu fp32 [F] or NULL. Sums are held in fp32 and G and U are not rounded before
 * H is. Sizes: F, K in 1 .. 2^20, N in 0 .. 2^30, N F and N K below 2^38.
 *
 * fp32 operands run on the tensor cores as three bf16 parts each, whose sum they
 * are, and a product as the six part products that are not below 2^-24 of it,
 * added in fp32 (one or two tokens: in plain fp32): |dG| <= 1e-5 (sum |x||w| + |b|),
 * as for bsr_spmm. With bf16 operands the tensor cores' own sums run over up to 16384
 * products before they are added up in fp32, and lose up to 7e-9 of a sum of one sign
 * with each product (about 1e-9 of one of mixed signs): at most 2^-13, where a result
 * in bf16 is rounded by up to 2^-8. Only dbg and dbu, which are fp32, show it (1.2e-6
 * at K = 1024).
 */
typedef enum {
    BSR_ACT_SILU = 0,      /* g / (1 + e^-g) */
    BSR_ACT_GELU = 1,      /* g Phi(g), Phi the normal distribution (erf) */
    BSR_ACT_GELU_TANH = 2, /* g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2 */
    BSR_ACT_RELU = 3,      /* max(g, 0) */
    BSR_ACT_SIGMOID = 4    /* 1 / (1 + e^-g) */
} bsr_act_t;

/* Bytes of workspace of a call of N tokens; `backward` 0 or 1. May be 0. */
bsr_status_t bsr_gated_workspace(int64_t N, int64_t F, int64_t K, bsr_dtype_t dt, int backward, size_t *bytes);

/*
 * bsr_gated -- H from X.
 *
 * X, Wg, Wu, H: device, 16-byte aligned; H overlaps no other buffer.
 * ws       device, 16-byte aligned, of at least the bytes that bsr_gated_workspace
 *          gives (else BSR_ERR_CAPACITY); used until the call's kernels have run.
 * Asynchronous on `stream`; allocates nothing; reads the weights as they are when
 * its kernels run. N == 0 is a no-op. Device buffers of the current device only.
 */
bsr_status_t bsr_gated(const void *X, const void *Wg, const void *Wu, const float *bg, const float *bu, void *H, int64_t N,
                       int64_t F, int64_t K, bsr_dtype_t dt, bsr_act_t act, void *ws, size_t ws_bytes, void *stream);

/*
 * bsr_gated_backward -- the gradients from dH [N, F], with G and U computed again
 * from the forward call's arguments:
 *
 *   dG = dH U act'(G), dU = dH act(G)       (relu'(0) = 0)
 *   dX = dG Wg + dU Wu, dWg = dG' X, dWu = dU' X, dbg = sum_n dG, dbu = sum_n dU
 *
 * dX [N, K], dWg and dWu [F, K] (element type dt, 16-byte aligned), dbg and dbu
 * fp32 [F]: written, not added to; each NULL where not wanted, but dWg and dWu
 * both or neither, and dbg or dbu only beside bg or bu. For N == 0 the weights'
 * gradients are zeros. No output overlaps another buffer. For BSR_BF16, dG and dU
 * are rounded as operands of dX, dWg and dWu (not for dbg and dbu): to bf16, and up
 * to 128 tokens to 16 bits.
 */
bsr_status_t bsr_gated_backward(const void *X, const void *Wg, const void *Wu, const float *bg, const float *bu,
                                const void *dH, void *dX, void *dWg, void *dWu, float *dbg, float *dbu, int64_t N, int64_t F,
                                int64_t K, bsr_dtype_t dt, bsr_act_t act, void *ws, size_t ws_bytes, void *stream);

/*
 * ---- Rows sorted by expert
 *
 * A layer of E experts sends every token to k of them. Sorted by expert, an
 * expert's tokens are one run of rows, which one product takes (bsr_fp8_product
 * with groups, or bsr_gated on the run); the results are added up again with the
 * router's weights:
 *
 *   c_e = number of choices of expert e,  offsets[0] = 0,
 *   offsets[e + 1] = offsets[e] + align * ceil(c_e / align)
 *   place[n, j]  = offsets[e] + the number of earlier choices of e, in the order
 *                  of n k + j; -1 if the choice is no expert (outside 0 .. E - 1)
 *   source[r]    = the n k + j of row r, -1 where there is none
 *   Xs[r] = X[source[r] / k], zeros in the rows of an expert's run behind its last
 *   Y[n]  = sum_j weights[n, j] Ys[place[n, j]]     (j with a place only)
 */
typedef struct {
    int64_t N;         /* tokens, below 2^30 */
    int64_t R;         /* rows of source, Xs and Ys: at least bsr_expert_capacity's, below 2^31 */
    int k, E, align;   /* 1 .. 64 choices of a token, 1 .. 1024 experts, 1 .. 1024 */
    int32_t *offsets;  /* device [E + 1] */
    int32_t *place;    /* device [N, k] */
    int32_t *source;   /* device [R] */
} bsr_experts_t;

/* The rows that N tokens take at most: the least R of bsr_experts_t. */
bsr_status_t bsr_expert_capacity(int64_t N, int k, int E, int align, int64_t *rows);

/*
 * bsr_expert_order -- offsets, place and source from each token's choices.
 *
 * experts  device int32 [N, k]; a value outside 0 .. E - 1 is a dropped choice, an
 *          expert may be chosen twice. R below the capacity: BSR_ERR_CAPACITY.
 * Nothing is read back: the arrays are used on the device by the calls below and
 * by bsr_fp8_product. Asynchronous on `stream`; allocates nothing. Same input, same bits.
 */
bsr_status_t bsr_expert_order(const bsr_experts_t *p, const int32_t *experts, void *stream);

/*
 * bsr_expert_rows -- Xs [R, D] from X [N, D] (device, 16-byte aligned, type dt,
 * D in 1 .. 2^20, D R below 2^38).
 * Rows from offsets[E] on are left as they were. Its gradient is bsr_expert_sum of
 * dXs without weights. Entries of place outside 0 .. R - 1 are not sent, here and
 * in the calls below. N == 0 is a no-op. Nothing overlaps.
 */
bsr_status_t bsr_expert_rows(const bsr_experts_t *p, const void *X, void *Xs, int64_t D, bsr_dtype_t dt, void *stream);

/*
 * bsr_expert_sum -- Y [N, D] from Ys [R, D]; weights: device fp32 [N, k], or NULL for
 * 1. Sums in fp32, in the order of j, rounded once; a token without a place gets
 * zeros. Rows that no choice has are not read.
 */
bsr_status_t bsr_expert_sum(const bsr_experts_t *p, const void *Ys, const float *weights, void *Y, int64_t D, bsr_dtype_t dt,
                            void *stream);

/*
 * bsr_expert_sum_backward -- dYs[place[n, j]] = weights[n, j] dY[n], zeros in an
 * expert's rows behind its last, and dweights[n, j] = the product of dY[n] and
 * Ys[place[n, j]] summed over features (0 without a place). dYs or dweights may be
 * NULL; dweights needs weights and Ys (else unused). Rows from offsets[E] on are left as they were.
 */
bsr_status_t bsr_expert_sum_backward(const bsr_experts_t *p, const void *Ys, const float *weights, const void *dY, void *dYs,
                                     float *dweights, int64_t D, bsr_dtype_t dt, void *stream);

/*
 * ---- Products in 8-bit floating point
 *
 * An operand is a matrix of 8-bit values with a scale, a power of two, for each block
 * of 128 columns (the axis that the product sums over) of a row, or of 128 rows:
 *
 *   x[r, c] is q[r, c] * scale[c / 128, r / tile]
 *
 * The product reads the scales as exponents, a byte 127 + log2(scale) for each row and
 * block in the order that the tensor cores take them: with w = ceil(rows / 128), that of
 * row r and block b at byte
 *
 *   ((b / 4) * w + r / 128) * 512 + (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4
 *
 * Y = a b' + bias:  Y[n, m] = bias[m] + sum_k a[n, k] b[m, k], in the tensor cores'
 * fp32 accumulators, which lose at most 4e-9 of a sum of one sign with each column (on
 * average 2e-10 of 1024 columns, 6e-10 of 16384); they are added up in fp32 every 1024 columns, for bf16 results every 16384 at least.
 * A layer X W': a = X by rows, b = W by rows with tiles of 128. Its gradients:
 * dX = dY W: b = W by columns; dW = dY' X: a = dY and b = X, both by columns.
 */
typedef enum { BSR_E4M3 = 0, BSR_E5M2 = 1 } bsr_fp8_t;
typedef struct {
    int64_t batch;         /* matrices, one behind the other, at most 65535; 1 but for the weights of experts */
    int64_t rows, cols;    /* below 2^31; batch * rows * (cols rounded up to 128) up to 2^38 */
    int tile;              /* rows that share a scale: 1 or 128 */
    bsr_fp8_t type;
    void *q;               /* device, 16-byte aligned: [batch, rows, cols rounded up to 128], zeros past cols */
    uint8_t *exponent;     /* device, 16-byte aligned: [batch, ceil(cols / 512), ceil(rows / 128), 512] */
    float *scale;          /* device [batch, ceil(cols / 128), ceil(rows / tile)], or NULL: written by
                              bsr_fp8_quantize for who reads q, not read by the product */
} bsr_fp8_matrix_t;

/*
 * bsr_fp8_quantize -- x [batch, R, C] (device, 16-byte aligned, type dt) in 8 bits.
 *
 * rows     [batch, R, C]: blocks along C. columns: [batch, C, R], x transposed, blocks
 *          along R. Either may be NULL; with both, their batch, tile and type agree.
 * A block's scale is the least power of two that brings its largest |x| to at most
 * 448 (e4m3) or 57344 (e5m2), at least 2^-126; 1 for a block of zeros. So each value is rounded
 * once, to nearest even. Values that are not finite become NaN, and do not count
 * for the scale.
 * used     device int32 [1], or NULL for R (batch 1): rows of x from *used on are not read
 *          and count as zeros of a block; in rows, they and their scales are left as they
 *          were (with tile 128, a block in use in part has one scale: that of its rows in
 *          use), in columns the blocks of 128 that begin at or after *used.
 * Asynchronous on `stream`; allocates nothing. Nothing overlaps.
 */
bsr_status_t bsr_fp8_quantize(const void *x, bsr_dtype_t dt, const bsr_fp8_matrix_t *rows, const bsr_fp8_matrix_t *columns,
                              const int32_t *used, void *stream);

typedef enum {
    BSR_GROUP_NONE = 0,
    BSR_GROUP_ROWS = 1,     /* rows offsets[e] .. offsets[e + 1] - 1 of a meet b's matrix e */
    BSR_GROUP_COLUMNS = 2   /* Y[e] sums over the columns offsets[e] .. offsets[e + 1] - 1, multiples of 128 or the end */
} bsr_group_t;

/* Bytes of workspace of a product; may be 0. a and b: their sizes, no arrays. */
bsr_status_t bsr_fp8_product_workspace(const bsr_fp8_matrix_t *a, const bsr_fp8_matrix_t *b, bsr_dtype_t dt, bsr_group_t group,
                                       int64_t groups, size_t *bytes);

/*
 * bsr_fp8_product -- Y = a b' + bias.
 *
 * a, b     of as many columns; types may differ; a.batch is 1.
 * Y        device, 16-byte aligned, type dt: [a.rows, b.rows], by BSR_GROUP_COLUMNS
 *          [groups, a.rows, b.rows]. Overlaps nothing.
 * bias     device fp32 [b.batch, b.rows], or NULL; not by BSR_GROUP_COLUMNS.
 * groups   1 .. 1024 experts, offsets: device int32 [groups + 1], ascending, within a's rows
 *          or columns; read on the device. Of columns, multiples of 128 (orders of align 128, 256, ...), or a.cols
 *          and more, the end: at any other, the matrices Y[e] of the runs that it ends are NaN, and
 *          bsr_check_status returns BSR_ERR_INVALID_ARG.
 *          BSR_GROUP_ROWS: b.batch is groups; rows in no expert's run are left as they were.
 *          BSR_GROUP_NONE: offsets NULL, groups unused, b.batch 1.
 * ws       device, 16-byte aligned, of at least the bytes that bsr_fp8_product_workspace
 *          gives (else BSR_ERR_CAPACITY); used until the call's kernels have run.
 * Asynchronous on `stream`; allocates nothing. Same input, same bits.
 */
bsr_status_t bsr_fp8_product(const bsr_fp8_matrix_t *a, const bsr_fp8_matrix_t *b, const float *bias, void *Y, bsr_dtype_t dt,
                             bsr_group_t group, const int32_t *offsets, int64_t groups, void *ws, size_t ws_bytes, void *stream);

/*
 * bsr_check_status -- synchronise the current device and return the first error
 * that a kernel of bsr_gated, bsr_gated_backward or bsr_fp8_product recorded there
 * (BSR_ERR_TIMEOUT when a bounded wait gave up, BSR_ERR_INVALID_ARG for offsets inside a
 * block of columns), then clear it. BSR_OK if none.
 */
bsr_status_t bsr_check_status(void);

/* bsr_destroy -- release what the handle owns (not the borrowed arrays). NULL is a no-op. */
void bsr_destroy(bsr_handle_t h);

/* bsr_status_str -- a static, human-readable name for a status code. */
const char *bsr_status_str(bsr_status_t s);

#ifdef __cplusplus
}
#endif
#endif /* BSR_H */
