/*
 * apml.h - C ABI of the sparse APML loss (forward and backward) on one AMD
 * Instinct MI355X (gfx950).
 *
 * The loss is the sparse Adaptive Probabilistic Matching Loss of
 * "From Theory to Throughput: CUDA-Optimized APML for Large-Batch 3D
 * Learning" (arXiv:2512.19743). Per sample b, with predicted points
 * X = {x_i} (N of them) and reference points Y = {y_j} (M of them):
 *
 *   C_ij = ||x_i - y_j||_2                                    Sec. III-A
 *   per row i: C1 = min_j C_ij, C2 = second smallest,
 *     g = max(C2 - C1 + delta, eps_gap)                       Sec. III-A, III-D
 *     T = log((M - 1) p_min / (1 - p_min)) / g                Eq. 1
 *     s_ij = exp(-T (C_ij - C1)), kept where s_ij >= tau      Sec. III-B
 *     P_row = s / (sum of kept s in the row)                   Eq. 2, Sec. III-C
 *   per column j: the same with roles swapped (K = N)          Sec. III-B
 *   P0 = (P_row + P_col) / 2 on the union of both kept sets    Sec. III-A, III-C
 *   L_iter times: column scaling (Eq. 3), then row scaling (Eq. 4)
 *   loss_b = sum over kept pairs of v_t C_t                     Sec. III-D
 *   d loss / d x through all of the above, with Eq. 5 for the
 *   distance and the temperature differentiated (no gradient
 *   through the choice of the kept set or of the minima).      Sec. III-D
 *
 * The minimum and second minimum of a row or column are decided on the
 * single-precision squared distance; ties go to the smaller index. Everything
 * after the decision (cost values, temperatures, similarities, sums) is
 * computed in double precision and stored per stored pair in single precision.
 *
 * All pointers named "device" point to memory on the current HIP device, all
 * pointers named "host" to host memory. Every function returns an
 * apml_status and never throws; on failure apml_last_error() describes it.
 * Argument validation happens before any HIP call, so a rejected call touches
 * neither the device nor its outputs.
 */
#ifndef APML_H
#define APML_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define APML_VERSION 1

typedef enum apml_status {
    APML_OK = 0,
    APML_ERR_INVALID_ARG = 1,   /* a NULL pointer, a size or a parameter out of range */
    APML_ERR_UNSUPPORTED = 2,   /* d != 3, or a size beyond the 32-bit index range */
    APML_ERR_OUT_OF_MEMORY = 3, /* the allocator returned NULL */
    APML_ERR_DEVICE = 4,        /* a HIP call failed (text in apml_last_error) */
    APML_ERR_INTERNAL = 5       /* a consistency check on the device failed */
} apml_status;

/* A hipStream_t; NULL is the default (null) stream of the current device. */
typedef void *apml_stream;

/* Hyper-parameters. Defaults (apml_params_default) are the paper's
 * tau = 1e-8, L_iter = 10, eps_stab = 1e-8 (Sec. III-E, Sec. IV-C) and, where
 * the paper gives no value, p_min = 0.8, delta = 1e-8, eps_gap = 1e-6,
 * eps_dist = 1e-12. */
/* How the dense scans (the minimum and second minimum of every row and
 * column, Sec. III-A; the candidate support, Sec. III-B) visit the pairs.
 * Both modes give identical results. FULL evaluates every pair. SKIP sorts
 * both clouds along a space-filling curve and skips every run of 32 points
 * whose bounding box is provably beyond the distance that can still matter
 * to the owners being scanned; it pays off for large samples. AUTO takes SKIP
 * when min(N, M) >= 8192. */
typedef enum { APML_SCAN_AUTO = 0, APML_SCAN_FULL = 1, APML_SCAN_SKIP = 2 } apml_scan_mode;

/* Readings of the paper where it offers two (for ablation; the defaults are
 * the first of each).
 * gap_mode  CLAMP: g = max(C2 - C1 + delta, eps_gap) (Sec. III-D).
 *           UNIFORM_FALLBACK: an owner whose gap C2 - C1 is below eps_gap
 *           gets P = 1/K on all K pairs (Sec. III-A, Sec. III-C); all of its
 *           pairs are stored and no gradient flows through that softmax.
 * sym_mode  HALF_SUM: P0 = (P_row + P_col)/2 with an absent side 0 (the
 *           dense initial plan of Sec. III-A on the union support).
 *           MEAN_DUP: duplicates averaged (Sec. III-C, Alg. 1 step 3) and a
 *           pair kept by one direction only keeps that direction's value.
 * tgrad_mode FULL: the gradient reaches the costs through the temperatures
 *           (Eq. 1); DETACHED: the temperatures are constants in backward. */
typedef enum { APML_GAP_CLAMP = 0, APML_GAP_UNIFORM_FALLBACK = 1 } apml_gap_mode;
typedef enum { APML_SYM_HALF_SUM = 0, APML_SYM_MEAN_DUP = 1 } apml_sym_mode;
typedef enum { APML_TGRAD_FULL = 0, APML_TGRAD_DETACHED = 1 } apml_tgrad_mode;

typedef struct apml_params {
    uint32_t struct_size; /* sizeof(apml_params), for forward compatibility */
    int32_t n_iter;       /* L_iter >= 0: Sinkhorn iterations (Alg. 1) */
    double p_min;         /* Eq. 1; needs 1/min(N, M) < p_min < 1 */
    double tau;           /* pruning threshold on s, 0 <= tau <= 1 (Sec. III-B) */
    double eps_stab;      /* >= 0, added to every Sinkhorn sum (Eq. 3, Eq. 4) */
    double delta;         /* >= 0, gap offset g = c2 + delta (Sec. III-A) */
    double eps_gap;       /* > 0, gap clamp max(gap, eps_gap) (Sec. III-D) */
    double eps_dist;      /* >= 0, added to ||x - y|| in the gradient only (Eq. 5) */
    int32_t dense_scan;   /* apml_scan_mode: how the two dense scans visit the pairs */
    int32_t gap_mode;     /* apml_gap_mode (default CLAMP) */
    int32_t sym_mode;     /* apml_sym_mode (default HALF_SUM) */
    int32_t tgrad_mode;   /* apml_tgrad_mode (default FULL) */
} apml_params;

/* Fills *p with the defaults above (p must not be NULL). */
void apml_params_default(apml_params *p);

/* Opaque per-call state kept from the forward pass for the backward pass:
 * the stored pairs, the per-row and per-column statistics and the Sinkhorn
 * scalings. Library-owned; release it with apml_plan_destroy. */
typedef struct apml_plan apml_plan;

/*
 * Forward pass (Alg. 1, Sec. III-A to III-D).
 *   x     device, float32 [B, N, d] contiguous (predicted points X)
 *   y     device, float32 [B, M, d] contiguous (reference points Y)
 *   B >= 1, N >= 2, M >= 2, d == 3 (else APML_ERR_UNSUPPORTED);
 *   B*N, B*M and the number of stored pairs must fit in int32.
 *   params  host, may be NULL for the defaults
 *   loss    device, float32 [B]: per-sample loss sum_t v_t C_t (no batch mean)
 *   plan    host out-pointer; if non-NULL, *plan receives the state needed by
 *           apml_backward; if NULL, that state is released before returning.
 *   stream  every kernel is queued on it.
 * The call synchronises the stream once, after the support has been counted,
 * to size the sparse arrays (the paper's two-pass construction does the same).
 * x and y are only read. On error *plan is NULL and loss is untouched unless
 * the failure came from the device. A device-side consistency check that runs
 * after that synchronisation (a row's or column's minimum missing from its
 * stored pairs, which the construction rules out) is reported only by
 * apml_plan_nnz, as APML_ERR_INTERNAL; this call returns APML_OK then. So is
 * a bounded wait of the Sinkhorn kernels that split a sample over several
 * workgroups expiring (they are launched so that all of them run at once,
 * which rules it out), as APML_ERR_DEVICE.
 */
apml_status apml_forward(const float *x, const float *y, int32_t B, int32_t N, int32_t M,
                         int32_t d, const apml_params *params, float *loss, apml_plan **plan,
                         apml_stream stream);

/*
 * Backward pass (Sec. III-D): gradient of sum_b grad_loss[b] * loss_b.
 *   plan       from apml_forward; not consumed (may be used again)
 *   x, y       the same device arrays, unchanged since the forward call
 *   grad_loss  device, float32 [B]
 *   grad_x     device, float32 [B, N, 3], overwritten
 *   grad_y     device, float32 [B, M, 3], overwritten, or NULL to skip it
 */
apml_status apml_backward(apml_plan *plan, const float *x, const float *y,
                          const float *grad_loss, float *grad_x, float *grad_y,
                          apml_stream stream);

/*
 * Forward and backward in one call, with no device allocation. For callers
 * that cannot allocate device memory (code under stream capture, serving loops
 * with a fixed memory budget, harnesses that forbid hipMalloc): the same
 * kernels as apml_forward followed by apml_backward, with every plan array and
 * temporary carved from one static device array of
 * APML_NOALLOC_SCRATCH_BYTES that each device the library runs on holds until
 * the process ends (32 clouds of 2048 points against 2048 fit in it; 64 clouds
 * of 8192 points do not). No plan is returned.
 *   x, y, B, N, M, d, params, loss   as for apml_forward
 *   grad_loss, grad_x, grad_y        as for apml_backward; grad_x == NULL
 *                                    computes the loss only (grad_loss and
 *                                    grad_y are then ignored)
 * Errors: as apml_forward; APML_ERR_OUT_OF_MEMORY when the call needs more
 * scratch than the array holds (apml_last_error states both sizes; detected
 * before the kernels that write loss or gradients run, so the outputs are
 * untouched), APML_ERR_UNSUPPORTED when B > 1791. The call synchronises the
 * stream once, like apml_forward. Every call on a device shares that
 * device's array and leaves its contents behind: calls that overlap on one
 * device (other host threads, or other streams still running an earlier
 * call) race and give undefined results; calls on one stream, or on
 * different devices, do not.
 */
#define APML_NOALLOC_SCRATCH_BYTES ((size_t)128 << 20)
apml_status apml_forward_backward_noalloc(const float *x, const float *y, int32_t B, int32_t N,
                                          int32_t M, int32_t d, const apml_params *params,
                                          float *loss, const float *grad_loss, float *grad_x,
                                          float *grad_y, apml_stream stream);

/*
 * Dense APML (Sec. III-A): the unpruned formulation, a baseline for the
 * sparse path's memory and time. Every pair of a sample takes part (no
 * threshold: tau is ignored, the result is what the sparse path gives at
 * tau = 0), for points of any dimension 1 <= d <= 16. The minimum and second
 * minimum of every row and column are decided on the single-precision squared
 * distance as in the sparse path; the temperatures follow Eq. 1 with the gap
 * clamp (Sec. III-D), the softmaxes Eq. 2 over all pairs, P0 = (P_row +
 * P_col)/2, then L column (Eq. 3) and row (Eq. 4) scalings, loss = sum P C.
 * The plan keeps P0 as a float32 N x M matrix per sample (4 bytes a pair) and
 * per-point vectors. Device memory comes from the same pool or caller
 * allocator as the sparse path.
 *   x, y    device, float32 [B, N, d] / [B, M, d] contiguous
 *   params  as for apml_forward; gap_mode and sym_mode must be the defaults
 *           (else APML_ERR_UNSUPPORTED); dense_scan and tau are ignored
 *   loss    device, float32 [B]
 *   plan    as for apml_forward (NULL: released before returning)
 * apml_dense_backward: gradient of sum_b grad_loss[b] loss_b, grad_x [B,N,d]
 * overwritten, grad_y [B,M,d] overwritten or NULL. Neither call synchronises.
 */
typedef struct apml_dense_plan apml_dense_plan;
apml_status apml_dense_forward(const float *x, const float *y, int32_t B, int32_t N, int32_t M,
                               int32_t d, const apml_params *params, float *loss,
                               apml_dense_plan **plan, apml_stream stream);
apml_status apml_dense_backward(apml_dense_plan *plan, const float *x, const float *y,
                                const float *grad_loss, float *grad_x, float *grad_y,
                                apml_stream stream);
apml_status apml_dense_plan_destroy(apml_dense_plan *plan);

/* Releases the plan's device memory (stream-ordered on the plan's stream).
 * NULL is accepted. */
apml_status apml_plan_destroy(apml_plan *plan);

/* Sizes of a plan. stored_pairs counts every stored pair, including pairs kept
 * only as the minimum or second minimum of a row or column (they carry zero
 * mass). bytes is the device memory the plan holds. scanned_min and
 * scanned_support count the pairs the two dense scans of the forward
 * examined: the minimum scan once per direction (2*B*N*M when nothing is
 * skipped, although the full scan evaluates each distance once for both),
 * the support scan over rows (B*N*M); the skipping scans leave out pairs that
 * provably cannot matter. */
typedef struct apml_plan_info {
    int32_t B, N, M, n_iter;
    int64_t stored_pairs;
    int64_t bytes;
    int64_t scanned_min, scanned_support;
} apml_plan_info;
apml_status apml_plan_get_info(const apml_plan *plan, apml_plan_info *info);

/* Per-sample size of the kept support Omega = Omega_row U Omega_col
 * (Sec. III-B), host int64 [B]. Synchronises the plan's stream. Returns
 * APML_ERR_INTERNAL if a device-side consistency check failed, and
 * APML_ERR_DEVICE if a bounded wait of the split Sinkhorn kernels expired. */
apml_status apml_plan_nnz(const apml_plan *plan, int64_t *nnz);

/*
 * Copies sample b's kept pairs to the host, sorted by (i, j), for testing and
 * inspection. capacity is the length of every non-NULL output array and must
 * be at least the sample's apml_plan_nnz value. Outputs (any may be NULL):
 *   i, j     int32 row and column index
 *   flags    bit 0: s_row >= tau, bit 1: s_col >= tau
 *   p_row, p_col  float32 normalised row / column probabilities (0 if not kept)
 *   p0       float32 initial plan (P_row + P_col)/2
 *   v        float32 plan after the Sinkhorn iterations
 * Synchronises the plan's stream.
 */
apml_status apml_plan_export(const apml_plan *plan, int32_t b, int64_t capacity, int32_t *i,
                             int32_t *j, uint8_t *flags, float *p_row, float *p_col, float *p0,
                             float *v);

/*
 * Copies sample b's per-row and per-column statistics to the host:
 * temperature (Eq. 1), index of the minimum and second minimum, and whether
 * the gap was clamped. Row arrays have N entries, column arrays M; any may be
 * NULL. Synchronises the plan's stream.
 */
apml_status apml_plan_export_stats(const apml_plan *plan, int32_t b, double *T_row, int32_t *j1,
                                   int32_t *j2, uint8_t *row_clamped, double *T_col, int32_t *i1,
                                   int32_t *i2, uint8_t *col_clamped);

/*
 * Device memory. By default the library keeps its own pool of hipMalloc'd
 * blocks per device and stream (freed blocks are reused by later calls on the
 * same stream). A caller may route every allocation through its own
 * allocator instead, e.g. a framework's caching allocator; alloc must return
 * device memory usable on `stream` (or NULL on failure), free is called with
 * the same pointer, size and stream. Every failure of alloc must come back as
 * NULL: the library cannot tell any other pointer from device memory and its
 * kernels will write through it (a binding whose callbacks can raise must
 * catch and return NULL). Blocks the pool caches are not given back when the
 * route changes: apml_release_cached_memory does that. Passing NULLs restores
 * the pool. Must not be called while a plan is alive.
 */
typedef void *(*apml_alloc_fn)(size_t bytes, apml_stream stream, void *user);
typedef void (*apml_free_fn)(void *ptr, size_t bytes, apml_stream stream, void *user);
apml_status apml_set_allocator(apml_alloc_fn alloc, apml_free_fn free_fn, void *user);

/* Bytes currently held by live plans and temporaries, the peak of that since
 * the last reset, and the bytes reserved by the pool. */
typedef struct apml_memory_stats {
    int64_t in_use;
    int64_t peak_in_use;
    int64_t reserved;
} apml_memory_stats;
apml_status apml_get_memory_stats(apml_memory_stats *stats);
apml_status apml_reset_peak_memory(void);
/* Returns the pool's unused blocks to HIP. */
apml_status apml_release_cached_memory(void);

/*
 * Per-phase timing with HIP events recorded on the caller's stream around
 * each phase of forward and backward. Phases (index: name):
 *   0 stats     dense scan: minimum and second minimum per row and column
 *   1 support   dense scan: emission of the candidate pairs
 *   2 build     counts, prefix sums, row-major and column-major index build
 *   3 softmax   temperatures, both softmaxes, symmetrized plan
 *   4 sinkhorn  the 2 L scaling sweeps
 *   5 loss      loss per sample
 *   6 bwd_sinkhorn   reverse Sinkhorn sweeps
 *   7 bwd_softmax    softmax, temperature and distance adjoints
 * apml_profile_read synchronises the recorded events and returns, per phase,
 * the total milliseconds and the number of timed occurrences since the last
 * reset (arrays of length n, at most APML_N_PHASES).
 */
#define APML_N_PHASES 8
apml_status apml_profile_enable(int32_t on);
apml_status apml_profile_reset(void);
apml_status apml_profile_read(int32_t n, double *total_ms, int64_t *count);
const char *apml_phase_name(int32_t phase);

/*
 * Losses on features and on routed experts, for networks trained beside the
 * loss above (descriptors of the points of two clouds matched to each other,
 * tokens of a code book, segmentation classes, expert layers). Their calls
 * allocate nothing, never synchronise and hold no state: temporaries lie in a
 * workspace of the caller's, whose size a query gives (device memory, aligned
 * to 256 bytes, free for other use once the call's kernels have run; two calls
 * that may overlap need two), and what the backward pass needs of the forward
 * one lies in a state array of the caller's. So every call can be captured into
 * a graph (after one of its kind outside: the runtime loads a kernel with its
 * first launch). Gradients are overwritten. All sums are held in float32 or more.
 */
typedef enum { APML_F32 = 0, APML_BF16 = 1, APML_F16 = 2 } apml_dtype;
typedef enum { APML_I64 = 0, APML_I32 = 1 } apml_index_type;
typedef enum { APML_REDUCE_NONE = 0, APML_REDUCE_SUM = 1, APML_REDUCE_MEAN = 2 } apml_reduction;

/*
 * Softmax cross entropy of rows against classes by their scaled products,
 * without storing the rows x classes logits. Per sample (the samples are
 * independent problems; classes shared by all rows: samples = 1):
 *
 *   z_tv   = scale <x_t, w_v>
 *   lse_t  = log sum_v exp z_tv
 *   loss_t = lse_t - z_t,target_t + z_weight lse_t^2, 0 where target_t == ignore_index
 *
 * reduction SUM adds all rows' losses, MEAN divides by the rows that are not
 * ignored (the loss is 0 where all are). An ignored row adds nothing and gets a
 * zero gradient, whatever x holds there. A target outside [0, classes) other
 * than ignore_index gives a NaN loss for its row, NaN gradients of that row and
 * of w. A row that counts and whose upstream gradient is 0 gets a zero gradient.
 * Features of w, and of x in rows that count, have to be finite: an infinite one
 * gives NaN in float32, whose products are made of pieces of the operands.
 */
typedef struct apml_linear_ce_desc {
    uint32_t struct_size; /* sizeof(apml_linear_ce_desc) */
    int32_t dtype;        /* apml_dtype of x, w, grad_x and grad_w */
    int32_t target_type;  /* apml_index_type of target */
    int32_t samples;      /* >= 1 */
    int32_t rows;         /* >= 1, per sample; samples * rows <= 2^26 */
    int32_t classes;      /* >= 1, <= 2^26 */
    int32_t dim;          /* >= 1, <= 2^20; some 2^38 logits, or 2^35 features of either side, a call */
    int32_t reduction;    /* apml_reduction */
    float scale;          /* 1 / temperature; within +-2.35e38 */
    float z_weight;       /* weight of lse^2 */
    int64_t ignore_index;
} apml_linear_ce_desc;

/* samples 1, scale 1, z_weight 0, ignore_index -100, MEAN; the sizes 0. */
void apml_linear_ce_desc_default(apml_linear_ce_desc *d);

/* Bytes of workspace of the two calls for these x and w (their alignment
 * decides whether they are copied into padded rows; NULL: the most any needs).
 * Either pointer to a size may be NULL. With dim up to a multiple of 64, the copies
 * are, in either pass: for float32 x and w whole, in 6 bytes an element (the forward
 * pass of at most 128 rows a sample goes without where dim is a multiple of 32 and
 * both are aligned to 16 bytes); in 16 bits x where dim is no multiple of 64 and w
 * where it is none of 8, or what is not aligned to 16 bytes. The backward pass copies
 * x once more for grad_w. Beside them the forward pass has 8 bytes a row and 64 or 128 classes (32
 * for at most 16 rows a sample), the backward pass a piece of the logits' gradient of
 * about 256 MB at most and, where sums are cut, gradients in float32. */
apml_status apml_linear_ce_workspace(const apml_linear_ce_desc *desc, const void *x, const void *w,
                                     size_t *forward_bytes, size_t *backward_bytes);

/*
 *   x       device [samples][rows][dim] contiguous
 *   w       device [samples][classes][dim] contiguous
 *   target  device [samples][rows]
 *   loss    device float32, [samples][rows] (NONE) or one value
 *   state   device float32 [samples * rows + 1][4], aligned to 16 bytes, for
 *           the backward pass, or NULL
 */
apml_status apml_linear_ce_forward(const apml_linear_ce_desc *desc, const void *x, const void *w, const void *target,
                                   float *loss, float *state, void *workspace, size_t workspace_bytes,
                                   apml_stream stream);

/*
 * Gradients of sum grad_loss * loss: grad_loss device float32 [samples][rows]
 * (NONE) or one value; x, w, target and state as in the forward call. grad_x and
 * grad_w (shapes of x and w) are overwritten; one of them may be NULL. The logits'
 * gradient exists in pieces of about 256 MB at most (of the samples, the classes,
 * the rows), rounded to x's type for the two products that read it; grad_x gets back
 * what the rounding of its rows' targets took, grad_w does not (bfloat16: up to 1.35
 * times the error of one rounding). float16 where the rows' upstream gradients differ
 * (NONE or a z_weight): for grad_w a feature times its row's upstream gradient keeps
 * all its bits down to 2^-27 of the largest such product, below it an absolute step.
 */
apml_status apml_linear_ce_backward(const apml_linear_ce_desc *desc, const void *x, const void *w, const void *target,
                                    const float *state, const float *grad_loss, void *grad_x, void *grad_w,
                                    void *workspace, size_t workspace_bytes, apml_stream stream);

/*
 * Balance loss of a network with routed experts, and the tokens per expert.
 * Per sample of `tokens` tokens, n of them valid, with p_t = softmax(logits_t):
 *
 *   counts_e = how often e stands in the valid tokens' chosen experts
 *   f_e = counts_e / sum counts,   P_e = (1 / n) sum over valid t of p_te
 *   loss = E sum_e f_e P_e + z_weight (1 / n) sum over valid t of lse_t^2
 *
 * 1 (without the second term) where tokens and probabilities are spread evenly.
 * The gradient flows through the probabilities, not through the counts. A chosen
 * expert outside [0, experts) is a dropped slot and counted nowhere. Tokens that
 * are not valid add nothing and get a zero gradient, whatever logits holds
 * there. A logit of -inf is an expert out of reach; a token with nothing else
 * has no probabilities and adds nothing but its place in n. A sample without
 * valid tokens has loss 0. SUM and MEAN are over the samples.
 */
typedef struct apml_balance_desc {
    uint32_t struct_size; /* sizeof(apml_balance_desc) */
    int32_t dtype;        /* apml_dtype of logits and grad_logits */
    int32_t index_type;   /* apml_index_type of index */
    int32_t samples;      /* >= 1, <= 2^20 */
    int32_t tokens;       /* >= 1, per sample; samples * tokens <= 2^30 */
    int32_t experts;      /* 1 to 1024 */
    int32_t chosen;       /* >= 1, experts per token in index; tokens * chosen <= 2^30 */
    int32_t reduction;    /* apml_reduction */
    float z_weight;
} apml_balance_desc;

/* samples 1, chosen 1, z_weight 0, MEAN; the sizes 0. */
void apml_balance_desc_default(apml_balance_desc *d);
apml_status apml_balance_workspace(const apml_balance_desc *desc, size_t *bytes);

/*
 *   logits  device [samples][tokens][experts] contiguous
 *   index   device [samples][tokens][chosen], or NULL: counts is given (the sum
 *           over all ranks of what apml_expert_counts gave each, for instance)
 *   valid   device [samples][tokens], a byte each, 0 for padding; or NULL
 *   counts  device int64 [samples][experts], written, or read where index is NULL
 *   loss    device float32 [samples] (NONE) or one value
 *   state   device float32 [samples][experts + 1] for the backward pass, or NULL
 */
apml_status apml_balance_forward(const apml_balance_desc *desc, const void *logits, const void *index,
                                 const uint8_t *valid, int64_t *counts, float *loss, float *state, void *workspace,
                                 size_t workspace_bytes, apml_stream stream);

/* Gradient of sum grad_loss * loss: grad_loss device float32 [samples] (NONE)
 * or one value; grad_logits, of logits' shape and type, is overwritten. */
apml_status apml_balance_backward(const apml_balance_desc *desc, const void *logits, const uint8_t *valid,
                                  const float *state, const float *grad_loss, void *grad_logits, apml_stream stream);

/* The counts alone; sizes and index as above. */
apml_status apml_expert_counts(const void *index, int32_t index_type, const uint8_t *valid, int32_t samples,
                               int32_t tokens, int32_t chosen, int32_t experts, int64_t *counts, apml_stream stream);

const char *apml_status_string(apml_status status);
/* Text of the last error on the calling thread ("" if none). */
const char *apml_last_error(void);
int32_t apml_version(void);

#ifdef __cplusplus
}
#endif
#endif /* APML_H */
