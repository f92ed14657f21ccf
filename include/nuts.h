/*
 * nuts.h - C ABI of the MI355X lock-step NUTS sampler.
 *
 * The library runs many independent No-U-Turn-Sampler chains on one GPU.  The
 * recursive tree doubling of each chain is turned into an explicit per-chain
 * program counter and stack, and only chains that stand at the same program
 * point are stepped together - the program-counter batching of Radul et al.,
 * "Automatically batching control-intensive programs for modern accelerators"
 * (Section 3, Algorithm 2), specialised by hand to the sampler the paper
 * evaluates (Section 4).  The unit of work the paper counts is one evaluation
 * of the target's log-density gradient (Section 4.1); here that is one
 * leapfrog step, i.e. one leaf of a NUTS tree.
 *
 * All functions return 0 on success and a negative NUTS_E_* code otherwise; a
 * human-readable reason is then available from nuts_last_error().  No C++
 * exception crosses this boundary.  On an argument error nothing is written to
 * any output buffer.  The library never falls back to the CPU: without a GPU
 * every call that needs one fails with NUTS_E_DEVICE.
 */
#ifndef NUTS_H_
#define NUTS_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { NUTS_OK = 0, NUTS_E_INVALID_ARG = -1, NUTS_E_ALLOC = -2, NUTS_E_DEVICE = -3, NUTS_E_UNSUPPORTED = -4 };

/* Arithmetic type of the target data, the chain states and out_states.  Energies,
 * log-weights and U-turn dot products are binary64 in both cases. */
enum { NUTS_F32 = 0, NUTS_F64 = 1 };

/* The categorical operators (last sections) take NUTS_F32 and these two: bfloat16, binary16. */
enum { NUTS_BF16 = 2, NUTS_F16 = 3 };

/* Type of an array of classes. */
enum { NUTS_I32 = 0, NUTS_I64 = 1 };

/* Target families (the paper's two test problems, Section 4, plus the two
 * element-wise Gaussians of the benchmark configurations). */
enum {
    NUTS_TARGET_STD_NORMAL = 0,            /* log p = -1/2 |x|^2                                   */
    NUTS_TARGET_GAUSS_DENSE_PRECISION = 1, /* log p = -1/2 x' P x                                  */
    NUTS_TARGET_GAUSS_DIAG = 2,            /* log p = -1/2 sum_i x_i^2 / sigma_i^2                 */
    NUTS_TARGET_LOGISTIC_REGRESSION = 3    /* sum_n [y_n z_n - log(1+e^{z_n})] - |x|^2/(2 s^2), z = X x */
};

/* Which kernel family nuts_sample_ex uses. */
enum {
    NUTS_VARIANT_AUTO = 0,
    NUTS_VARIANT_WAVE = 1,  /* one wavefront per chain, vectors striped over the 64 lanes; any target/shape.
                               AUTO steps dense Gaussians of 128 < dim <= 512 whose matrix is not banded in
                               lock step, 4 or 8 wavefronts per workgroup with their products on the matrix
                               cores, and keeps those of banded ones (dim <= 2048) in registers; it reports
                               both under this number.  Asked for by it the general kernel runs: the same
                               bits as for banded matrices, another order of the sums for the others        */
    NUTS_VARIANT_TILE = 2,  /* 16 chains per workgroup in lock step, gradient as MFMA GEMMs (logistic
                               regression, binary64, dim <= 32, max_tree_depth <= 12); when dim = 1 mod 4
                               and a column of X is the same non-zero value in every row (an intercept),
                               that column's share of the logits is added ahead of the others' instead of
                               in its place among them: another order of the same sum.  Up to 4 chains per
                               compute unit, and up to 8 in short runs on many rows, it steps 4 chains per
                               workgroup instead of 16 (the same bits).
                               AUTO extends the family to dim <= 128 and to binary32 data sets that are too
                               small for the grid kernels, and reports it under this number                 */
    NUTS_VARIANT_ELEM = 3,  /* one wavefront per chain with the moving trajectory end held in registers
                               (standard normal / diagonal Gaussian, dim <= 1024 binary32, <= 512 binary64;
                               AUTO runs the same kernel up to dim = 2048 and reports it as WAVE there)     */
    NUTS_VARIANT_GRID = 4,  /* every gradient round is a chip-wide binary32 MFMA GEMM over the data rows
                               (logistic regression, binary32, dim <= 128; up to 1024 chains are resident
                               at a time, further chains wait in a queue); this variant returns only when
                               sampling has finished.  Targets of up to 1.5e6 elements (of 17 to 32 features:
                               12 000 rows) run in one launch that holds every compute unit, one such run at
                               a time on a device: calls of a process take turns, and a call waits while
                               other work holds compute units (where that goes on, or the stream has
                               only some of them, it runs on as many as it gets: the same bits);
                               larger ones in two launches a round, beyond 128 chains
                               divided between two or four streams, the caller's and others that the target
                               owns, forked from and joined to the caller's stream by events; chains that want
                               a gradient are packed together, so idle ones cost next to nothing           */
    NUTS_VARIANT_DENSE = 5, /* one wavefront per chain, moving trajectory end in registers, precision matrix in LDS
                               (dense Gaussian, dim <= 128)                                                 */
    NUTS_VARIANT_QUAD = 6   /* four chains per wavefront, their precision-matrix products together as MFMA blocks
                               with the matrix in LDS in operand order (dense Gaussian, binary64, dim <= 128,
                               max_tree_depth <= 12); chosen automatically for matrices that are not banded
                               from 2560 chains on                                                          */
};

typedef struct nuts_target nuts_target; /* opaque; owns device copies of its data */

/* All pointers in the descriptor are HOST pointers to arrays of `dtype`; they are
 * copied (and re-laid-out) during nuts_create_target and may be freed afterwards. */
typedef struct {
    int32_t kind;          /* NUTS_TARGET_*                                                    */
    int32_t dtype;         /* NUTS_F32 / NUTS_F64                                              */
    int64_t dim;           /* d >= 1                                                           */
    const void* precision; /* GAUSS_DENSE_PRECISION: d*d row-major, symmetric                  */
    const void* scales;    /* GAUSS_DIAG: sigma_i > 0, d values                                */
    const void* X;         /* LOGISTIC_REGRESSION: n_data*d row-major design matrix            */
    const void* y;         /* LOGISTIC_REGRESSION: n_data labels in {0,1}                      */
    int64_t n_data;        /* LOGISTIC_REGRESSION: n_data >= 1                                 */
    double prior_scale;    /* LOGISTIC_REGRESSION: prior N(0, prior_scale^2 I), > 0            */
} nuts_target_desc;

/* Counters of the last nuts_sample* call on a target (see nuts_get_stats). */
typedef struct {
    uint64_t leaf_slots_issued; /* chain slots handed to the batched gradient step over all lock-step
                                   rounds, idle and padded slots included.  Kernels whose chains do not
                                   step together (wave, element-wise) hold every slot for the whole
                                   launch: they charge, per launch, slots x the gradient count of the
                                   busiest slot                                                        */
    uint64_t leaf_slots_useful; /* of those, slots that carried a leapfrog step (= sum of out_n_leapfrog) */
    uint64_t extra_grad_evals;  /* gradient evaluations that are not leapfrog steps (initial points)   */
    uint64_t rounds;            /* lock-step rounds, summed over workgroups                            */
    double kernel_ms;           /* duration of the sampler kernel, from HIP events on its stream       */
    uint64_t phase_ticks[3];    /* kernels with a phase clock: shader-clock ticks spent in {control, batched
                                   gradient, step completion}, summed as `rounds` is (divide by it)    */
    int32_t variant;            /* NUTS_VARIANT_* that ran                                             */
    int32_t grid_blocks;        /* workgroups launched                                                 */
} nuts_stats;

/* When chains may start their next iteration (Section 4.2 of the paper compares the two).
 * FREE: a chain goes on as soon as its own trajectory is finished, so gradient steps of different
 *   iterations are batched together (what program-counter batching allows).
 * TRAJECTORY: no chain starts iteration i+1 before every chain of the call has finished iteration i
 *   (all a batching scheme that follows the control structure of the chain program can do).  One
 *   launch per iteration; the gradient at each iteration's starting point is evaluated again
 *   (counted in extra_grad_evals, never in out_n_leapfrog).
 * Both give bit-identical outputs. */
enum { NUTS_SCHEDULE_FREE = 0, NUTS_SCHEDULE_TRAJECTORY = 1 };

/* How the points of a trajectory are weighted when one of them is selected.
 * MULTINOMIAL (default): weight exp(H0 - H) per leaf, subtrees summarised by the log of their summed weights.
 * SLICE: the form of the No-U-Turn Sampler as first published (Hoffman & Gelman, JMLR 2014, Algorithm 3),
 *   which is what Section 4.1 of the paper batches: a height u is drawn uniformly below exp(-H0) once per
 *   iteration (draw purpose 5), a leaf is a candidate iff exp(-H) >= u and stays valid while
 *   exp(-H) > u exp(-1000); subtrees are summarised by their candidate counts; the right half's
 *   proposal is taken with probability count_R / (count_L + count_R), a new half with min(1, count_new / count_tree).
 * Everything else (doubling, U-turn tests, depth limit, leaf_steps, outputs) is shared. */
enum { NUTS_SAMPLER_MULTINOMIAL = 0, NUTS_SAMPLER_SLICE = 1 };

/* Options of nuts_sample_ex; zero-initialise for the defaults. */
typedef struct {
    const void* init_states; /* DEVICE, dtype, [n_chains][dim]; NULL: x0 ~ N(0, I) drawn from `seed`     */
    int64_t first_chain;     /* global id of chain 0 (enters the random-number keys); default 0.  A run
                                of chains [a, a+n) equals columns [a, a+n) of a larger run.              */
    int32_t variant;         /* NUTS_VARIANT_*                                                           */
    int32_t leaf_steps;      /* leapfrog steps per tree leaf, 1..NUTS_MAX_LEAF_STEPS; 0 means 1.  Section 4.1
                                of the paper takes 4 so that the control around a leaf is paid once per 4
                                gradients.  Only a leaf's end state is a candidate and enters the U-turn
                                and energy tests; out_n_leapfrog counts leapfrog steps (leaf_steps per
                                leaf); the subtree-selection draw is keyed by that count at the merge.   */
    int32_t schedule;        /* NUTS_SCHEDULE_*                                                          */
    int32_t sampler;         /* NUTS_SAMPLER_*                                                           */
} nuts_sample_options;
#define NUTS_MAX_LEAF_STEPS 64

/* Create a target, i.e. the fixed synthetic posterior the chains sample from (the
 * paper's test problems are of this kind: Section 4, logistic regression and a
 * correlated Gaussian): validates the descriptor, copies the data to the current
 * device in the layouts the kernels want.  STD_NORMAL needs no device.
 * Errors: INVALID_ARG (null/shape/kind/dtype, non-finite or non-positive scale),
 * DEVICE, ALLOC.  *out is set only on success. */
int nuts_create_target(const nuts_target_desc* desc, nuts_target** out);

/* Free a target and everything it owns (device data, cached workspace). NULL is allowed. */
int nuts_destroy_target(nuts_target* t);

/* The batched sampler itself: "the number of chains running in tandem" is the batch
 * size of Section 4.1, each chain is one batch member of Algorithm 2 with its own
 * program counter and stack.
 * Run n_iters NUTS iterations of n_chains chains (multinomial NUTS, one leapfrog
 * step per leaf, identity mass matrix, fixed step size; initial states
 * x0 ~ N(0, I) drawn from `seed`).  Every random number is a function of
 * (seed, chain, iteration, purpose, position) only, so results do not depend on
 * how chains are scheduled.
 *   out_states       DEVICE, dtype, [n_iters][n_chains][dim]: state after each iteration
 *   out_tree_depths  DEVICE, int32 [n_iters][n_chains]: doublings attempted (1..max_tree_depth)
 *   out_n_leapfrog   DEVICE, int32 [n_iters][n_chains]: leapfrog steps (= gradient evaluations
 *                    requested by the chain; the evaluation at x0 is not counted)
 * Any output may be NULL.  The caller owns the buffers.  The work is enqueued on
 * the stream given to nuts_set_stream (default: the null stream) and the call
 * returns without waiting; scratch memory is owned by the target and reused by
 * later calls, so calls on one target must not overlap.
 * Domain: n_chains >= 1, n_iters >= 1, step_size finite > 0, 1 <= max_tree_depth <= 20.
 * Errors: INVALID_ARG, DEVICE (no GPU / launch failure), ALLOC, UNSUPPORTED. */
int nuts_sample(const nuts_target* target, int64_t n_chains, int64_t n_iters, double step_size,
                int32_t max_tree_depth, uint64_t seed, void* out_states, int32_t* out_tree_depths,
                int32_t* out_n_leapfrog);

/* nuts_sample with options (initial states, global chain offset, kernel variant). */
int nuts_sample_ex(const nuts_target* target, int64_t n_chains, int64_t n_iters, double step_size,
                   int32_t max_tree_depth, uint64_t seed, const nuts_sample_options* options,
                   void* out_states, int32_t* out_tree_depths, int32_t* out_n_leapfrog);

/* nuts_sample_ex for callers that cannot allocate device memory while they call: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels, same
 * outputs bit for bit; but the call allocates and frees nothing.  Its workspace and counters live in a
 * static device array of NUTS_STATIC_SCRATCH_BYTES that is part of the library's code object (every GPU
 * the library runs on holds one copy until the process ends).
 *   - The target must have been created with a GPU present (creation is where device data, tables, counters
 *     and events are set up, and where the array's device address is looked up).
 *   - A run whose workspace does not fit is refused with NUTS_E_UNSUPPORTED and a message that states the bytes
 *     needed and the maximum; nothing is written.  (The workspace grows with the resident chain slots, the
 *     dimension and max_tree_depth: configuration 3, 4096 chains of logistic regression, needs 46 MB.)
 *   - Also refused: NUTS_VARIANT_GRID (it owns streams and pinned host memory and waits on the host), and
 *     NUTS_SCHEDULE_TRAJECTORY without out_states (it would need a carry buffer).
 *   - All calls on one GPU share that GPU's array, whatever the target or host thread: two calls that overlap
 *     in time on one GPU race, also on different streams.  The array keeps the last call's contents; the call
 *     clears what it needs at zero with a small kernel (no memset node, so it can be captured).
 * nuts_get_stats afterwards reports this call. */
#define NUTS_STATIC_SCRATCH_BYTES (64u << 20)
int nuts_sample_static(const nuts_target* target, int64_t n_chains, int64_t n_iters, double step_size,
                       int32_t max_tree_depth, uint64_t seed, const nuts_sample_options* options,
                       void* out_states, int32_t* out_tree_depths, int32_t* out_n_leapfrog);

/* Counters and kernel time of the last sampling call on `target`.  Waits for that
 * call to finish (synchronises on its stop event). */
int nuts_get_stats(const nuts_target* target, nuts_stats* out);

/* Stream (a hipStream_t) for subsequent nuts_sample* calls of this host thread. */
int nuts_set_stream(void* hip_stream);

/* Message for the last error on this host thread; valid until the next call. */
const char* nuts_last_error(void);

/* Host only (no device is touched): the operand stream that nuts_create_target lays out for the tile variant from a
 * binary64 logistic-regression data set (Section 4's logistic regression as the two GEMMs Z = X Theta, G = X' s on
 * 16-row tiles), for checking that layout without a GPU.  X is n x d row-major and y holds n labels (0 or not 0),
 * both host pointers.  `layout` is filled whenever the arguments and the shape are valid; the stream itself (layout->operand_doubles values) is copied to
 * `operands` if that is not NULL and `capacity` (in doubles) suffices, else INVALID_ARG when `operands` is not NULL.
 * Stream: per tile, operand pairs of 64 x 2 doubles; element (pair p, lane l, half h) is operand 2p + h as lane l
 * feeds it to v_mfma_f64_16x16x4: first GEMM operand s (0 .. ks1 - 1) holds X[16 t + l % 16][slot 4 s + l / 16],
 * second GEMM operand (u, s) (u < mt, s < 4; after the first GEMM's pairs, an odd ks1 leaves one half unused) holds
 * X[16 t + 4 s + l / 16][16 u + l % 16]; rows of y = 0 are negated unless a constant column stays out of the first
 * GEMM (const_col >= 0: then slot const_col carries feature d - 1 and slots from d - 1 on are zero). */
typedef struct {
    int32_t ks1, mt;             /* k-steps of the first GEMM, feature tiles of the second                */
    int32_t n_tiles;             /* row tiles that the kernel runs                                         */
    int32_t n_alloc_tiles;       /* row tiles in the stream (a multiple of 8)                              */
    int32_t const_col;           /* the constant column that is the first GEMM's initial value, or -1     */
    int32_t reserved;
    double const_val;            /* its value                                                              */
    int64_t n_pad;               /* rows of zeros that the kernel runs                                     */
    int64_t operand_doubles;     /* length of the stream                                                   */
} nuts_tile_layout;
int nuts_tile_pack(const double* X, const double* y, int64_t n, int64_t d, nuts_tile_layout* layout, double* operands,
                   int64_t capacity);

/* ---- Categorical models -------------------------------------------------------------------------------------------
 *
 * The logistic regression above has two classes, y in {0, 1}.  These operators are its parts for observations of one of
 * many classes (a word of a vocabulary, a group, a choice), for programs that put a log density of such a model and its
 * gradient together, or ask a fitted one for its answers: rows of a table by class and the gradient of that, the
 * log-probabilities of given classes, and their gradient.
 *
 * All pointers but the descriptors are DEVICE pointers.  The calls are enqueued on the stream of nuts_set_stream and
 * return; nothing is allocated, copied or kept, so they can be captured into a graph.  Sums, maxima and statistics are
 * binary32 whatever the element type, and each output is rounded once (the one exception is named at nuts_score_grad).  The order of
 * every sum is fixed by the descriptor and the classes: a call repeated gives the same bits.  Strides are in elements; rows
 * may begin at any address that suits an element, and outputs must not overlap inputs unless that is said.  A class
 * outside [0, n_classes) is no error: such a row has no class (a pad, an observation that does not count).
 * A workspace of the size that the *_workspace functions say may hold anything; it is the caller's again when the call's work
 * is done.  Alignment: workspaces 256 bytes.  Sizes of zero are allowed (n_ids, n_rows): nothing is read then. */

#define NUTS_CAT_MAX_TOP 64

typedef struct {
    int32_t dtype;        /* NUTS_F32, NUTS_BF16 or NUTS_F16: table, its gradient, rows                    */
    int32_t id_type;      /* NUTS_I32 or NUTS_I64                                                          */
    int64_t n_ids;        /* 0 .. 2^31 - 2                                                                 */
    int64_t n_classes;    /* rows of the table, 1 .. 2^31 - 2                                              */
    int64_t dim;          /* numbers in a row, 1 .. 2^24                                                   */
    int64_t table_stride; /* from one row of the table (or of its gradient) to the next, >= dim            */
    int64_t row_stride;   /* the same of the n_ids rows                                                    */
    double scale;         /* finite                                                                        */
    int32_t accumulate;   /* nuts_lookup_grad: 0 writes all of the gradient, 1 adds to what is there       */
    int32_t reserved;
} nuts_lookup_desc;

/* rows[i, :] = scale * table[ids[i], :]; zeros where ids[i] is no class. */
int nuts_lookup(const nuts_lookup_desc* desc, const void* table, const void* ids, void* rows);

/* grad_table[v, :] = scale * sum of grad_rows[i, :] over the i with ids[i] = v, zeros for a class that does not come
 * (accumulate: such rows are not touched, the others' sums are added to them and rounded once). */
int nuts_lookup_grad_workspace(const nuts_lookup_desc* desc, int64_t* bytes);
int nuts_lookup_grad(const nuts_lookup_desc* desc, const void* grad_rows, const void* ids, void* grad_table,
                     void* workspace, int64_t workspace_bytes);

typedef struct {
    int32_t dtype;          /* of the logits and their gradient                                            */
    int32_t id_type;        /* of the targets                                                              */
    int64_t n_rows;         /* 0 .. 2^31 - 2                                                               */
    int64_t n_classes;      /* 1 .. 2^31 - 2^18 - 1                                                        */
    int64_t row_stride;     /* of the logits, >= n_classes                                                 */
    int64_t allowed_stride; /* 32-bit words from one row of `allowed` to the next; 0: one row for all      */
    double scale;           /* z = scale * logits; finite, > 0 (a temperature is 1 / scale)                */
    int32_t n_top;          /* alternatives, 0 .. NUTS_CAT_MAX_TOP                                         */
    int32_t reserved;
} nuts_logits_desc;

/* For each row of z = scale * logits:
 *   lse = log sum_v e^(z_v);   logprob = z_target - lse, 0 if the row has no target (or `targets` is NULL);
 *   entropy = lse - sum_v p_v z_v, p = e^(z - lse);
 *   top_ids / top_logprobs [n_rows][n_top]: the n_top largest z in falling order, of equal ones the lower class first.
 * `allowed` (or NULL): class v may come if bit v % 32 of word v / 32 of the row is set; the others count as z = -infinity whatever
 * is there (NaN, too), and are no alternatives.  Where fewer classes than n_top may come, the rest is -1 and -infinity.
 * A row in which every z is -infinity has lse = -infinity, logprob = -infinity, entropy 0 and alternatives of
 * logprob -infinity.  A row with a NaN or +infinity that may come has NaN for all but its top_ids; NaN ranks above
 * everything.  Any output may be NULL. */
int nuts_logprobs_workspace(const nuts_logits_desc* desc, int64_t* bytes);
int nuts_logprobs(const nuts_logits_desc* desc, const void* logits, const void* targets, const uint32_t* allowed,
                  float* logprob, float* lse, float* entropy, int32_t* top_ids, float* top_logprobs,
                  void* workspace, int64_t workspace_bytes);

/* Gradient with respect to the logits of sum_rows grad_logprob * logprob + grad_lse * lse + grad_entropy * entropy (each
 * [n_rows] or NULL), from the forward pass's lse and entropy (entropy only with grad_entropy):
 *   scale * (grad_logprob ([v = target] - p_v) + grad_lse p_v - grad_entropy p_v (log p_v + entropy)),
 * where a row without a target has no grad_logprob; 0 for classes that may not come, and where p_v is 0 but for the target.
 * A row in which every z is -infinity has gradient 0.  Rows of grad_logits are grad_stride apart.  lse and entropy may be those
 * of a longer row that this one is a part of.  Where |lse| is above 64 (16-bit logits: 1024), p = e^(z - lse) would be off by lse's rounding:
 * such rows are read once more for their maximum and sum. */
int nuts_logprobs_grad(const nuts_logits_desc* desc, const void* logits, const void* targets, const uint32_t* allowed,
                       const float* lse, const float* entropy, const float* grad_logprob, const float* grad_lse,
                       const float* grad_entropy, void* grad_logits, int64_t grad_stride);

typedef struct {
    int32_t dtype;         /* NUTS_F32 or NUTS_BF16: x, weight and their gradients                         */
    int32_t id_type;       /* of the targets                                                               */
    int64_t n_rows;        /* 0 .. 2^20                                                                    */
    int64_t n_classes;     /* 1 .. 2^24                                                                    */
    int64_t dim;           /* 1 .. 2^20                                                                    */
    int64_t x_stride;      /* from row to row, >= dim; and so on                                           */
    int64_t weight_stride;
    int64_t logits_stride; /* >= n_classes                                                                 */
    int64_t grad_x_stride, grad_weight_stride;
    double scale;          /* z = scale * x weight'; finite, > 0                                           */
} nuts_score_desc;

/* nuts_logprobs of z = scale * x weight' [n_rows][n_classes], from the features x [n_rows][dim] and the classes' weights
 * [n_classes][dim]: the products are made tile by tile and reduced where they are made.  `logits`, if not NULL, receives z
 * itself in binary32 (for nuts_score_grad, or for nuts_logprobs with scale 1 to name alternatives).  Any output may
 * be NULL.  x and weight begin at multiples of 16 bytes (here and in nuts_score_grad).  Rows are read as they lie if their stride is a multiple
 * of 16 bytes, or of 4 while there are not many rows of x; others are copied to the workspace first. */
int nuts_score_workspace(const nuts_score_desc* desc, int64_t* bytes);
int nuts_score(const nuts_score_desc* desc, const void* x, const void* weight, const void* targets, float* logprob,
               float* lse, float* entropy, float* logits, void* workspace, int64_t workspace_bytes);

/* Gradients of sum_rows grad_logprob * logprob + grad_lse * lse + grad_entropy * entropy:
 *   grad_x = dz weight, grad_weight = dz' x, dz as in nuts_logprobs_grad.
 * `logits`: what nuts_score stored, or NULL, when z is computed again.  Either gradient may be NULL.  With bfloat16 features dz is
 * rounded to bfloat16, for the matrix instructions multiply nothing wider; the products' sums are binary32, and what the
 * entries of the rows' targets lose in that rounding is added to them.  Where probabilities are spread, that is nearly all that is lost;
 * another class that is nearly certain, and the parts of grad_lse and grad_entropy, keep it (2^-8 of each entry at most).  Features and
 * weights in binary32 have dz in binary32.  Rows with |lse| above 64 (bfloat16: 1024) have p from their own maximum and sum, and lse may
 * not be a longer row's there.  The workspace's size is that for the larger of both ways. */
int nuts_score_grad_workspace(const nuts_score_desc* desc, int64_t* bytes);
int nuts_score_grad(const nuts_score_desc* desc, const void* x, const void* weight, const void* targets,
                    const float* logits, const float* lse, const float* entropy, const float* grad_logprob,
                    const float* grad_lse, const float* grad_entropy, void* grad_x, void* grad_weight, void* workspace,
                    int64_t workspace_bytes);

/* ---- What a categorical model answers through and learns with ---------------------------------------------------------
 *
 * Logits are adjusted before a class is chosen from them (nuts_penalties, and its gradient for models that are trained
 * through that); all parameters of a model are moved at once along their gradients (nuts_adamw), as far as the gradients' common norm
 * lets them (nuts_norm).  What is said of the operators above holds here: streams, capture, workspaces, strides, ids that are no class,
 * sums in a fixed order, sizes of zero.  Tables of tensors are HOST arrays that are read during the call. */

#define NUTS_CAT_MAX_BIAS 1024

typedef struct {
    int32_t dtype;          /* NUTS_F32, NUTS_BF16 or NUTS_F16: logits, their gradients                    */
    int32_t id_type;        /* of the history and of bias_ids                                              */
    int64_t n_rows;         /* 0 .. 2^31 - 2                                                               */
    int64_t n_classes;      /* 1 .. 2^31 - 2^18 - 1                                                        */
    int64_t row_stride;     /* of the logits, >= n_classes                                                 */
    int64_t out_stride;     /* of what is written, >= n_classes                                            */
    int64_t allowed_stride; /* 32-bit words from one row of `allowed` to the next; 0: one row for all      */
    int64_t bias_stride;    /* of `bias`, >= n_classes; 0: one row for all                                 */
    int64_t history_len;    /* 0 .. 2^29 - 1: places in a row of the history                               */
    int64_t history_stride; /* >= history_len; 0: one row for all                                          */
    int64_t n_bias;         /* 0 .. 1024: single classes with a bias, in each row                          */
    double repetition;      /* what all rows have where the array of that name is NULL: finite, > 0        */
    double frequency, presence; /* finite                                                                  */
} nuts_penalties_desc;

/* A row's history is the first lengths[row] of its places (all of them where `lengths` is NULL; a length is taken as
 * the nearest in [0, history_len]), the first prompts[row] of which are not the model's own (NULL: none).  With seen_v = class v comes in it
 * and count_v = how often it comes behind the prompt, and z = logits_v,
 *   z = z > 0 ? z (1 / repetition) : z repetition   where seen_v;     z = z - (frequency count_v + presence [count_v > 0]);
 *   z = z + bias_v, then + the sum of the row's bias_values whose bias_ids are v, in their order;     z = -infinity where v is not allowed,
 * whatever was there (NaN, too).  The arrays repetition, frequency and presence are [n_rows], bias [n_classes] or rows of it, bias_ids and
 * bias_values [n_rows][n_bias]; each may be NULL, and `allowed` is that of nuts_logprobs.  All of it is binary32 and rounded once.
 * `out` may be `logits` itself, with the same stride: then 16 bytes (from a row's beginning on) in which nothing changes are neither read nor written, but a
 * row's last classes, where they are fewer than 16 bytes and there is a mask, are read and written as they were, NaNs as quiet ones. */
int nuts_penalties(const nuts_penalties_desc* desc, const void* logits, const void* history, const int32_t* lengths,
                   const int32_t* prompts, const float* repetition, const float* frequency, const float* presence,
                   const float* bias, const void* bias_ids, const float* bias_values, const uint32_t* allowed, void* out);

/* From grad_out, the gradient with respect to what nuts_penalties writes (rows grad_stride apart), that with respect to its logits,
 *   grad_logits_v = grad_out_v * (seen_v ? (logits_v > 0 ? 1 / repetition : repetition) : 1), 0 where v is not allowed,
 * and that with respect to a bias that all rows share, grad_bias_v = sum over the rows of grad_out_v where v is allowed.  Either may be
 * NULL.  grad_logits (rows out_stride apart) may be grad_out itself.  logits are those that nuts_penalties was given, and
 * are read where a class was seen. */
int nuts_penalties_grad_workspace(const nuts_penalties_desc* desc, int64_t* bytes);
int nuts_penalties_grad(const nuts_penalties_desc* desc, const void* grad_out, int64_t grad_stride, const void* logits,
                        const void* history, const int32_t* lengths, const float* repetition, const uint32_t* allowed,
                        void* grad_logits, float* grad_bias, void* workspace, int64_t workspace_bytes);

typedef struct {
    const void* data;  /* DEVICE; n numbers without gaps; NULL where n is 0                                */
    int64_t n;         /* 0 .. 2^40                                                                        */
    int32_t dtype;     /* NUTS_F32, NUTS_BF16 or NUTS_F16                                                  */
    int32_t reserved;
} nuts_tensor;

/* norm = square root of the sum of all squares, summed in binary64; factor = min(1, max_norm / norm), which times all
 * numbers keeps their norm to max_norm (finite, > 0), and NaN where the norm is not finite in binary64 (beyond binary32's range the norm is infinite and the
 * factor is not).  Either may be NULL; one number each. */
int nuts_norm_workspace(const nuts_tensor* tensors, int64_t n_tensors, int64_t* bytes);
int nuts_norm(const nuts_tensor* tensors, int64_t n_tensors, double max_norm, float* norm, float* factor, void* workspace,
              int64_t workspace_bytes);

typedef struct {
    void* param;       /* DEVICE pointers, each to n numbers without gaps                                  */
    const void* grad;  /* NULL: this tensor is left alone                                                  */
    void* copy;        /* NULL, or: receives the new parameters in copy_dtype                              */
    void* m;           /* float, or int8_t where state_bits is 8                                           */
    void* v;           /* float, or uint8_t                                                                */
    float* m_scale;    /* state_bits 8: one for each NUTS_STATE_BLOCK numbers of the tensor, the last ones together */
    float* v_scale;
    int64_t n;         /* 0 .. 2^40                                                                        */
} nuts_adamw_tensor;
#define NUTS_STATE_BLOCK 256

typedef struct {
    int32_t param_dtype;  /* NUTS_F32 or NUTS_BF16                                                         */
    int32_t grad_dtype;   /* NUTS_F32, NUTS_BF16 or NUTS_F16                                               */
    int32_t copy_dtype;   /* NUTS_BF16 or NUTS_F16                                                         */
    int32_t state_bits;   /* 32 or 8                                                                       */
    double lr;            /* finite                                                                        */
    double beta1, beta2;  /* [0, 1)                                                                        */
    double eps;           /* finite, >= 0                                                                  */
    double weight_decay;  /* finite                                                                        */
    double scale;         /* of the gradients; finite (-1: uphill)                                         */
    int64_t step;         /* >= 1: number of this step, the first is 1                                     */
    uint64_t seed;        /* of what is rounded at random                                                  */
} nuts_adamw_desc;

/* One step of AdamW (Loshchilov & Hutter, 2019) for every tensor:
 *   g = scale factor grad;   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2;
 *   param = param (1 - lr weight_decay) - lr m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps).
 * `step`, `lr` and `factor` are DEVICE scalars or NULL; the first two take the descriptor's place (a captured step that is replayed needs
 * them there; a step below 1 counts as 1), and where factor is NaN the call changes nothing.  No two things that are written may overlap, nor a gradient with them.
 *
 * Arithmetic is binary32 (the quotient, and with moments of 32 bits the root, are a unit or two in the last place off); where v is 0 in it and eps is 0, the
 * quotient is infinite or NaN.  Moments of 8 bits stand for powers of their codes, m = sign(c) c^2 m_scale (c = -127 .. 127), v = (c^2 v_scale)^2
 * (c = 0 .. 254); a block's largest has the last code.  What stands between two codes becomes one of them, at random so that
 * the mean is kept, but a v above 0 does not get the code 0 (in a block whose largest v is below 2^-118 the smallest codes stand for what binary32 has as 0), and a
 * block of m whose largest is below 2^-126 127^2 is zeros.  c = -128 and c = 255 are what is not finite and count as NaN.
 * Parameters of bfloat16 are rounded at random, too (a step is mostly less than half a unit in their last place, and to the nearest they would stay where they
 * are); the parameters' copies are rounded to the nearest.  The random bits of the four numbers from 4 q of tensor t on are the four words of
 * Philox4x32-10 with the key `seed` and the counter (q mod 2^32, 6 + 256 (q / 2^32), step mod 2^32, t): bits 0-9 of a word are m's, 10-19 v's,
 * 20-31 the parameter's. */
int nuts_adamw(const nuts_adamw_desc* desc, const nuts_adamw_tensor* tensors, int64_t n_tensors, const int64_t* step,
               const float* lr, const float* factor);

/* The moments of 8 bits as numbers: `param` receives m and `copy` v, in dtype (NUTS_F32, NUTS_BF16, NUTS_F16); either may
 * be NULL.  grad is not looked at.  What is written may not overlap, nor the moments. */
int nuts_adamw_values(const nuts_adamw_tensor* tensors, int64_t n_tensors, int32_t dtype);

#ifdef __cplusplus
}
#endif
#endif /* NUTS_H_ */
