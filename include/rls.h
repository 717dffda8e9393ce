/*
 * rls - adaptive-sampling hot path on one MI355X (gfx950): C ABI.
 *
 * The calls follow the paper's statement of the adaptive-sampling step
 * (Sec. 4.2, Algorithm 1) and of the cost-model query that precedes it
 * (Sec. 4.1, "Reward formulation" / "Learning procedure"):
 *
 *   rls_gbt_score       predicted fitness of every configuration of a trajectory
 *   rls_kmeans_sweep    k-means(s_Theta, k) for every k of a range: centroids, clusters, loss
 *   rls_pick_knee       the knee test on the loss curve (host, scalar)
 *   rls_kmeans_sweep_until_knee  the same loop with Algorithm 1's early exit at the knee
 *   rls_snap_to_valid   NextSamples = Centroids, as valid configurations
 *   rls_knob_modes      mode(s_Theta), dimension by dimension
 *   rls_replace_visited samples already in v_Theta give way to mode(s_Theta)
 *   rls_apply_actions   the search agent's configuration updater (producer of the trajectory)
 *
 * and, for the search agent itself (Sec. 4.1) and other models trained or sampled beside it:
 *
 *   rls_sample          a draw per row of logits: temperature, top-k, top-p, min-p, from given uniform numbers
 *   rls_linear_scan     the gated linear recurrence h_t = a_t h_{t-1} + b_t, and its backward pass
 *   rls_token_logprobs  log-probabilities of given entries of rows of logits, entropy, the best alternatives, and their gradient
 *   rls_distill_loss    the divergence of rows of logits from a teacher's best entries, and its gradient
 *   rls_gated_delta     the gated delta rule, a recurrence with a matrix per head for its state, and its backward pass
 *   rls_adamw_step      one AdamW step over all tensors of a model, moments in 32 or in 8 bits
 *
 * Conventions
 *   - Plain C. Every call returns an int32_t status: RLS_OK or a negative RLS_ERR_* code.
 *   - Pointers named *_dev are device (HBM) pointers owned by the caller; all others are host
 *     pointers.  The library never allocates or frees device memory: scratch space comes in
 *     through `workspace_dev`, sized by the matching *_workspace_bytes query.
 *   - `stream` is a hipStream_t passed as void*.  Calls enqueue kernels on it and return
 *     without synchronising; outputs are valid once the stream has drained.  The one exception,
 *     rls_kmeans_sweep_until_knee, says so.  Such a call may be recorded into a HIP graph by the
 *     caller (kernels only: nothing is allocated, copied to the host or cleared with a memset node;
 *     call it once outside the capture first, which sets the kernels' launch attributes).
 *   - Results do not depend on the run: labels, centroids, configurations and scores are exact or
 *     summed in a fixed order, and so are the reported losses.
 *   - Matrices are row-major fp32 with an explicit leading dimension in elements.
 *   - Argument errors are detected on the host before anything is enqueued.  Conditions that
 *     only the data can reveal (see rls_kmeans_sweep) are reported through `status_dev`.
 *   - Limits: 1 <= d <= RLS_MAX_D, k_max <= RLS_MAX_K, tree depth <= RLS_MAX_DEPTH,
 *     N <= RLS_MAX_N, batch <= RLS_MAX_BATCH; rls_kmeans_sweep also needs ldx <= RLS_MAX_LDX.
 */
#ifndef RLS_H
#define RLS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RLS_OK 0
#define RLS_ERR_INVALID_ARG (-1)   /* a size, range or limit is violated */
#define RLS_ERR_NULL (-2)          /* a required pointer is NULL */
#define RLS_ERR_SHAPE (-3)         /* shapes disagree (forest features vs d, ldx < d, ...) */
#define RLS_ERR_WORKSPACE (-4)     /* workspace missing, misaligned (256 B) or too small */
#define RLS_ERR_HIP (-5)           /* a HIP runtime call failed; see rls_last_hip_error() */
#define RLS_ERR_NOT_IMPLEMENTED (-6)

#define RLS_MAX_D 32
#define RLS_MAX_K 128
#define RLS_MAX_DEPTH 12
#define RLS_MAX_N (1LL << 26)
#define RLS_MAX_BATCH 1024
#define RLS_MAX_LDX (1 << 24)       /* leading dimension of X accepted by rls_kmeans_sweep (elements) */

/* bits of *status_dev written by rls_kmeans_sweep (0 = clean) */
#define RLS_STATUS_NONFINITE 1     /* X holds an infinity or NaN */
#define RLS_STATUS_RANGE 2         /* a feature column is too wide for exact fixed-point sums */

int32_t rls_version(void);
const char *rls_error_string(int32_t code);
/* hipError_t of the most recent failing HIP call on this thread (0 if none). */
int32_t rls_last_hip_error(void);

/*
 * Boosted-tree cost model (Sec. 4.1: the estimate of the cost model is the surrogate reward;
 * the whole trajectory is scored after each episode).  The paper names the model family only;
 * the layout here is: `n_trees` complete binary trees of depth `depth` in level order, node n
 * having children 2n+1 (taken when x[feat] < thr) and 2n+2 (otherwise, NaN included).
 * All three arrays are borrowed device pointers.
 */
typedef struct {
    int32_t n_trees;
    int32_t depth;             /* 1..RLS_MAX_DEPTH */
    int32_t n_features;        /* must equal d of the matrix scored */
    float base;                /* added before the first tree */
    const int32_t *feat_dev;   /* [n_trees][2^depth - 1] feature index of each internal node */
    const float *thr_dev;      /* [n_trees][2^depth - 1] threshold of each internal node */
    const float *leaf_dev;     /* [n_trees][2^depth] leaf values */
} rls_forest;

/*
 * score_dev[i] = base + sum_t leaf_t(walk_t(X[i])), added in fp32 in tree order t = 0, 1, ...
 *   X_dev      [N][ldx] fp32, first d columns used
 *   score_dev  [N] fp32 (written)
 * A feature index outside [0, d) is read as the nearest valid column (0 or d - 1): the forest lives in device
 * memory, which the host checks never read, and the walk must not leave the row.
 */
int32_t rls_gbt_score(const rls_forest *forest, const float *X_dev, int64_t N, int32_t d, int64_t ldx,
                      float *score_dev, void *stream);

/*
 * `batch` independent knob spaces, each with its own forest (host array of `batch` structs) and
 * its own N x d block of X: space b reads X_dev + b * x_batch_stride and writes score_dev + b * N.
 */
int32_t rls_gbt_score_batched(const rls_forest *forests, int32_t batch, const float *X_dev, int64_t N,
                              int32_t d, int64_t ldx, int64_t x_batch_stride, float *score_dev, void *stream);

/*
 * k-means++ seeding chain (D^2 sampling) of k_max centres drawn with the counter-based
 * generator SplitMix64(seed + (j+1) * 0x9E3779B97F4A7C15), top 53 bits as a uniform in [0,1).
 * The paper does not fix the initialisation of k-means; a run with k clusters starts from
 * the first k centres of this chain.
 *   init_idx_dev  [k_max] int64 row indices (written)
 *   workspace     rls_kmeans_sweep_workspace_bytes(N, d, k_max, k_max, 1) bytes suffice
 */
int32_t rls_kmeanspp_chain(const float *X_dev, int64_t N, int32_t d, int64_t ldx, int32_t k_max, uint64_t seed,
                           int64_t *init_idx_dev, void *workspace_dev, int64_t workspace_bytes, void *stream);

/*
 * Bytes of workspace (a multiple of 256) with which rls_kmeans_sweep[_batched] takes the form that its shape is fastest
 * in, or a negative RLS_ERR_* code.  For sweeps with much distance work that includes a copy of the points in spatial
 * order, and the value is up to 1.7 times the least one.
 */
int64_t rls_kmeans_sweep_workspace_bytes(int64_t N, int32_t d, int32_t k_min, int32_t k_max, int32_t batch);
/*
 * The least it needs.  With a workspace between the two the sweep takes the points as they come: slower as a rule, faster
 * where the rows have no structure at all (independent columns); labels, centroids and losses are the same to the last bit.
 */
int64_t rls_kmeans_sweep_least_workspace_bytes(int64_t N, int32_t d, int32_t k_min, int32_t k_max, int32_t batch);

/*
 * The loop over k of Algorithm 1 (Sec. 4.2) without its early break: Lloyd's k-means for
 * every k in [k_min, k_max], each run independent and started from the first k centres of
 * one seeding chain, `iters` rounds of (assign, update) and a final assignment.
 *   - distance: squared Euclidean on the fp32 rows as given; ties go to the lowest centroid index
 *   - centroid: fp32( fp64(exact sum of the members) / count ); a cluster without members keeps
 *     its centroid
 *   - loss (inertia): sum of squared distances to the assigned centroid, against the returned
 *     centroids, accumulated in fp64
 * Arguments
 *   X_dev             [N][ldx] fp32
 *   k_min..k_max      inclusive, 1 <= k_min <= k_max <= min(N, RLS_MAX_K)
 *   iters             >= 0
 *   seed              used only when init_idx_dev is NULL
 *   init_idx_dev      [k_max] int64 row indices of the initial centres, or NULL to draw the chain
 *   labels_dev        [n_k][N] int32 (n_k = k_max-k_min+1), or NULL
 *   centroids_dev     packed fp32: run k starts at element d * sum_{k_min <= k' < k} k'; sum(k)*d floats
 *   inertia_dev       [n_k] fp64
 *   inertia_trace_dev [n_k][iters+1] fp64 loss of assignment t against the centroids it used, or NULL
 *   status_dev        one int32 (written): 0, or RLS_STATUS_* bits when the data breaks a
 *                     precondition, in which case all other outputs are unspecified.  Exact sums
 *                     need, per feature column, the lowest set bit of every value to lie at most
 *                     79 binary places below the highest set bit of the column.
 *   workspace_dev     256-byte aligned, rls_kmeans_sweep_workspace_bytes(...) bytes, or fewer down to
 *                     rls_kmeans_sweep_least_workspace_bytes(...)
 */
int32_t rls_kmeans_sweep(const float *X_dev, int64_t N, int32_t d, int64_t ldx,
                         int32_t k_min, int32_t k_max, int32_t iters, uint64_t seed,
                         const int64_t *init_idx_dev, int32_t *labels_dev, float *centroids_dev,
                         double *inertia_dev, double *inertia_trace_dev, int32_t *status_dev,
                         void *workspace_dev, int64_t workspace_bytes, void *stream);

/*
 * rls_kmeans_sweep for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): same arguments, results and status bits, but the workspace is a fixed
 * array of RLS_STATIC_WORKSPACE_BYTES inside the library's device image (each GPU the library runs on holds its
 * own copy until the process ends).  The call allocates nothing and frees nothing.
 *   - RLS_ERR_WORKSPACE when rls_kmeans_sweep_least_workspace_bytes(N, d, k_min, k_max, 1) exceeds
 *     RLS_STATIC_WORKSPACE_BYTES (nothing is enqueued); that query tells beforehand whether a shape fits.
 *   - All calls on one GPU share that GPU's array: two such sweeps that overlap in time on one GPU (different
 *     streams or host threads) race.  Successive calls on one stream are fine; every call initialises the parts
 *     of the array it reads.
 */
#define RLS_STATIC_WORKSPACE_BYTES (64 << 20)
int32_t rls_kmeans_sweep_static(const float *X_dev, int64_t N, int32_t d, int64_t ldx,
                                int32_t k_min, int32_t k_max, int32_t iters, uint64_t seed,
                                const int64_t *init_idx_dev, int32_t *labels_dev, float *centroids_dev,
                                double *inertia_dev, double *inertia_trace_dev, int32_t *status_dev, void *stream);

/*
 * `batch` independent spaces of equal shape in one launch sequence.  Space b reads
 * X_dev + b * x_batch_stride, uses seeds[b] (host array) or init_idx_dev + b * k_max, and writes
 * block b of every output: labels [batch][n_k][N], centroids [batch][sum(k)*d], inertia [batch][n_k],
 * trace [batch][n_k][iters+1], status [batch].
 */
int32_t rls_kmeans_sweep_batched(int32_t batch, const float *X_dev, int64_t N, int32_t d, int64_t ldx,
                                 int64_t x_batch_stride, int32_t k_min, int32_t k_max, int32_t iters,
                                 const uint64_t *seeds, const int64_t *init_idx_dev, int32_t *labels_dev,
                                 float *centroids_dev, double *inertia_dev, double *inertia_trace_dev,
                                 int32_t *status_dev, void *workspace_dev, int64_t workspace_bytes, void *stream);

/*
 * Algorithm 1's loop as it is written: k-means for k = k_min, k_min + 1, ... until the knee test fires, then stop.
 * The k are taken k_wave at a time (one sweep per wave, its k side by side as in rls_kmeans_sweep); after each wave
 * this call SYNCHRONISES `stream`, copies the wave's losses to inertia_host and applies the test of rls_pick_knee in
 * k order.  The outputs for the k that were computed equal those of rls_kmeans_sweep over the whole range, and
 * *k_out equals rls_pick_knee on the whole curve: runs for different k do not depend on each other.
 *   k_wave        >= 1; a multiple of 8 keeps the MFMA tiles full.  The k of a wave share each read of the points, and
 *                 the waves of a call share the column statistics and the prepared copy of the points: larger waves
 *                 cost less per k, smaller ones stop closer behind the knee
 *   seed / init_idx_dev  as rls_kmeans_sweep (the chain is extended wave by wave)
 *   labels_dev    [k_max-k_min+1][N] or null; centroids_dev, inertia_dev as rls_kmeans_sweep; only the first
 *                 *n_done_out runs are written
 *   inertia_host  [k_max-k_min+1] fp64 (host), first *n_done_out entries written
 *   k_out         the chosen k (k_max when the test never fires; 0 when *status_dev != 0)
 *   n_done_out    how many k were computed (a whole number of waves, or all)
 * Workspace: rls_kmeans_sweep_until_knee_workspace_bytes; fewer bytes are taken as by rls_kmeans_sweep.
 */
int64_t rls_kmeans_sweep_until_knee_workspace_bytes(int64_t N, int32_t d, int32_t k_min, int32_t k_max, int32_t k_wave);
int32_t rls_kmeans_sweep_until_knee(const float *X_dev, int64_t N, int32_t d, int64_t ldx, int32_t k_min, int32_t k_max,
                                    int32_t k_wave, int32_t iters, uint64_t seed, const int64_t *init_idx_dev,
                                    double knee_const, int32_t *labels_dev, float *centroids_dev, double *inertia_dev,
                                    double *inertia_host, int32_t *k_out, int32_t *n_done_out, int32_t *status_dev,
                                    void *workspace_dev, int64_t workspace_bytes, void *stream);

/*
 * Knee of the loss curve (Algorithm 1): with PreviousLoss = infinity, walk k upward and stop at the
 * first k with knee_const * inertia[k] > PreviousLoss; that k (whose centroids Algorithm 1 has
 * already assigned when the test fires) is returned, or k_max when the test never fires.
 * Pure host function; inertia_host is [k_max-k_min+1] fp64.  The paper names the constant without
 * giving its value, so it is an argument.
 */
int32_t rls_pick_knee(const double *inertia_host, int32_t k_min, int32_t k_max, double knee_const, int32_t *k_out);

/*
 * Knob domains of one design space (Sec. 2.2: the space is the product of the knob domains):
 * knob j owns values_dev[offsets[j] .. offsets[j+1]) and reads feature column j.
 */
typedef struct {
    int32_t n_knobs;             /* 1..d */
    const int32_t *offsets_dev;  /* [n_knobs+1], strictly increasing */
    const float *values_dev;     /* [offsets[n_knobs]] */
} rls_knob_domains;

/*
 * NextSamples = Centroids (Algorithm 1): each centroid becomes a valid configuration by taking,
 * knob by knob, the index of the nearest domain value (|c - v| compared in fp64, ties to the lower index).
 *   centroids_dev [k][ldc] fp32;  cfg_dev [k][n_knobs] int32 domain indices (written)
 */
int32_t rls_snap_to_valid(const float *centroids_dev, int32_t k, int32_t d, int64_t ldc,
                          const rls_knob_domains *domains, int32_t *cfg_dev, void *stream);

/* Space b: centroids_dev + b * c_batch_stride, domains[b] (host array), cfg_dev + b * k * n_knobs. */
int32_t rls_snap_to_valid_batched(int32_t batch, const float *centroids_dev, int32_t k, int32_t d, int64_t ldc,
                                  int64_t c_batch_stride, const rls_knob_domains *domains, int32_t *cfg_dev,
                                  void *stream);

/*
 * mode(s_Theta) of Algorithm 1, which Sec. 4.2 describes as the configuration "generated from modes of each
 * dimension": for every knob j, the domain index that most rows of the trajectory take, a row's value in
 * knob j being the domain entry nearest to its coordinate j (same rule as rls_snap_to_valid: |x - v| in
 * fp64, ties to the lower index).  Equally frequent entries: the lower index.
 *   X_dev        [N][ldx] fp32, N <= 2^26
 *   mode_cfg_dev [n_knobs] int32 (written)
 *   hist_dev     [offsets[n_knobs]] int32 counts of every domain entry, laid out like values_dev; used as
 *                scratch and left holding the counts.  At most RLS_MAX_DOMAIN_VALUES entries in total.
 * domains->offsets_dev and values_dev are device arrays; n_total_values = offsets[n_knobs] is passed by the
 * caller (the library does not read device memory on the host).
 */
#define RLS_MAX_DOMAIN_VALUES 8192
int32_t rls_knob_modes(const float *X_dev, int64_t N, int32_t d, int64_t ldx, const rls_knob_domains *domains,
                       int32_t n_total_values, int32_t *mode_cfg_dev, int32_t *hist_dev, void *stream);

/*
 * The last loop of Algorithm 1: a sample that is already among the visited configurations v_Theta is
 * replaced by mode(s_Theta).  Configurations are rows of n_knobs domain indices.
 *   cfg_dev      [k][n_knobs] int32, updated in place; 1 <= k <= 65535
 *   visited_dev  [n_visited][n_knobs] int32 (may be null when n_visited == 0)
 *   mode_cfg_dev [n_knobs] int32
 *   replaced_dev [k] int32 (written): 1 where the row was replaced
 * The replacement is not checked against v_Theta again (the paper's loop does not).
 */
int32_t rls_replace_visited(int32_t *cfg_dev, int32_t k, int32_t n_knobs, const int32_t *visited_dev,
                            int64_t n_visited, const int32_t *mode_cfg_dev, int32_t *replaced_dev, void *stream);

/*
 * Configuration updater of the search agent (Sec. 4.1, "Action space", "Learning procedure"): an action is one
 * direction per dimension (-1 decrement, 0 stay, +1 increment); applying it to a configuration gives the next one
 * of the trajectory.  A step that would leave a knob's domain stays at the border (the paper does not say).
 *   cfg_dev      [m][n_knobs] int32 domain indices (values outside a domain are first brought to its border)
 *   action_dev   [m][n_knobs] int8 (values beyond +-1 count as +-1)
 *   cfg_out_dev  [m][n_knobs] int32 (written; may be cfg_dev)
 *   features_dev [m][ldf] fp32 or null: the first n_knobs columns receive the domain values of the new
 *                configurations, the form in which rls_gbt_score is queried for a whole trajectory
 */
int32_t rls_apply_actions(const int32_t *cfg_dev, const int8_t *action_dev, int64_t m, const rls_knob_domains *domains,
                          int32_t *cfg_out_dev, float *features_dev, int64_t ldf, void *stream);

/* Element types of arrays that come in several. */
#define RLS_F32 0
#define RLS_BF16 1
#define RLS_F16 2

/*
 * One draw per row of logits: the search agent's action in a knob (Sec. 4.1, "Action space"), a candidate out of a
 * trajectory's scores, an entry of a vocabulary.  For a row x with largest logit x_max:
 *   d_i = (x_i - x_max) * min(1 / temperature, largest fp32 number) in fp32, e_i = exp(d_i) in fp32 (0 beyond -100),
 *   w_i = e_i rounded to a multiple of 2^-38, as a whole number of them; sums of w are exact, whatever their order
 *   top-k:  the k first entries in the order of descending d, equal ones by ascending index
 *   top-p:  of these the ones before which, in that order, the sum of w is less than p times the sum over all of them
 *   min-p:  of these the ones with e_i >= min_p
 *   token:  the first kept i (by index) up to which the kept w add up to more than uniform * (sum of the kept w)
 *   logprob: d_token - log(sum of the kept w), the log-probability of the draw among what was kept, in fp32 (of the rounded weights: a
 *            weight is off by up to 2^-39 of the largest, so many small ones together move it against softmax's)
 * The first entry of the order is always kept.  Entries of -infinity (masked ones) and NaN are never drawn; a row without
 * any other gets token -1 and logprob -infinity.  Entries of +infinity share a draw among themselves.
 * Arguments
 *   logits_dev       [rows][ld_logits] of logits_type (RLS_F32, RLS_BF16, RLS_F16), first n_choices columns used
 *   uniform_dev      [rows] fp32 in [0, 1); NaN and less than 0 count as 0, 1 and more takes the last kept entry
 *   temperature_dev  [rows] fp32 or null (1); 0, less or NaN: the first entry of the order at temperature 1 (logprob 0)
 *   top_k_dev        [rows] int32 or null; less than 1: all
 *   top_p_dev        [rows] fp32 or null; 1, more or NaN: all
 *   min_p_dev        [rows] fp32 or null; 0, less or NaN: all; more than 1 counts as 1 (entries with e_i = 1: the largest, and equal ones)
 *   token_dev        [rows] int32 (written);  logprob_dev  [rows] fp32 (written) or null
 *   workspace_dev    rls_sample_workspace_bytes(rows, n_choices) bytes, 256-byte aligned (may be 0 bytes, and null then)
 * 1 <= rows <= RLS_MAX_N, 1 <= n_choices <= RLS_MAX_CHOICES.
 */
#define RLS_MAX_CHOICES (1LL << 24)
int64_t rls_sample_workspace_bytes(int64_t rows, int64_t n_choices);
int32_t rls_sample(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                   const float *uniform_dev, const float *temperature_dev, const int32_t *top_k_dev, const float *top_p_dev,
                   const float *min_p_dev, int32_t *token_dev, float *logprob_dev, void *workspace_dev,
                   int64_t workspace_bytes, void *stream);

/*
 * Log-probabilities of given entries, one per row of logits: of the actions that the search agent took (its policy loss), of the tokens of a
 * sequence.  With x_max the row's largest logit and inv = min(1 / temperature, 2e38), in fp32:
 *   d_i = (x_i - x_max) inv,  L = log(sum of exp(d_i)),  log p_i = d_i - L
 *   logprob = log p_token;  entropy = L - (sum of exp(d_i) d_i) / (sum of exp(d_i)), in nats;  norm = (x_max, L), which the gradients start from
 *   alternatives: the `top` first entries in the order of falling logits, equal ones by rising index, with their log p
 * Entries of -infinity (masked ones) and NaN have probability 0, as for rls_sample, and are no alternatives; +infinity counts as the largest fp32
 * number.  A row without any other: logprob -infinity, entropy 0, norm (-infinity, 0).  Alternatives beyond the entries that count are token -1
 * with log p -infinity.  A token outside 0 .. n_choices - 1 (a padded position) gets logprob 0 and no gradient by it.
 *   logits_dev       [rows][ld_logits] of logits_type, first n_choices columns used
 *   token_dev        [rows] int32;  logprob_dev [rows] fp32 (written); both null: only the others are wanted
 *   temperature_dev  [rows] fp32 or null (1); 0, less or NaN counts as 1 (the distribution that a greedy draw ignores)
 *   entropy_dev      [rows] fp32 (written) or null;  norm_dev [rows][2] fp32 (written) or null
 *   top              0 .. RLS_MAX_TOP;  top_logprob_dev, top_token_dev  [rows][top] fp32 and int32 (written), not looked at with top = 0
 *   workspace_dev    rls_token_logprobs_workspace_bytes(rows, n_choices, top) bytes, 256-byte aligned (may be 0 bytes, and null then)
 * 1 <= rows <= RLS_MAX_N, 1 <= n_choices <= RLS_MAX_CHOICES.  What is written must not lie in anything else (RLS_ERR_SHAPE).
 */
#define RLS_MAX_TOP 128
int64_t rls_token_logprobs_workspace_bytes(int64_t rows, int64_t n_choices, int32_t top);
int32_t rls_token_logprobs(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits, const int32_t *token_dev,
                           const float *temperature_dev, int32_t top, float *logprob_dev, float *entropy_dev, float *top_logprob_dev,
                           int32_t *top_token_dev, float *norm_dev, void *workspace_dev, int64_t workspace_bytes, void *stream);
/*
 * Gradient by the logits, from what the forward pass wrote (norm, and entropy where dentropy is given) and the gradients by logprob and entropy:
 *   dx_i = inv (dlogprob ([i = token] - p_i) - dentropy p_i (log p_i + entropy)),  0 where p_i is 0 (but for the token itself)  and at masked entries
 *   dlogprob_dev, dentropy_dev  [rows] fp32, either may be null (0)
 *   dlogits_dev      [rows][ld_dlogits] of logits_type (written, first n_choices columns); logits_dev itself, with ld_dlogits = ld_logits, or apart
 */
int32_t rls_token_logprobs_backward(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                                    const int32_t *token_dev, const float *temperature_dev, const float *norm_dev, const float *entropy_dev,
                                    const float *dlogprob_dev, const float *dentropy_dev, void *dlogits_dev, int64_t ld_dlogits, void *stream);
/*
 * Learning from a teacher of which only its best entries are kept (what rls_token_logprobs lists): per row
 *   p = the probabilities that the k given logits, or log-probabilities, have among themselves at the row's temperature
 *   loss = sum of p_j (log p_j - log q_token_j), with q the probabilities of all of the row's own logits at that temperature
 * A token outside 0 .. n_choices - 1, and a teacher's logit of -infinity or NaN, is no entry; a token may come more than once (its
 * probabilities add up in the gradient).  A row without an entry has loss 0 and no gradient; one whose entry of probability above 0 is masked
 * has loss +infinity.  The teacher is a constant: nothing is differentiated by it.
 *   teacher_token_dev  [rows][k] int32;  teacher_logits_dev [rows][k] of teacher_type;  1 <= k <= RLS_MAX_TOP
 *   loss_dev         [rows] fp32 (written);  norm_dev [rows][2] fp32 (written) or null, as above; the other arguments as above
 */
int64_t rls_distill_loss_workspace_bytes(int64_t rows, int64_t n_choices);
int32_t rls_distill_loss(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits, const int32_t *teacher_token_dev,
                         const void *teacher_logits_dev, int32_t teacher_type, int32_t k, const float *temperature_dev, float *loss_dev, float *norm_dev,
                         void *workspace_dev, int64_t workspace_bytes, void *stream);
/* Gradient by the logits: dx_i = inv dloss (q_i - sum of p_j over the entries with token_j = i);  dloss_dev [rows] fp32, dlogits as above. */
int32_t rls_distill_loss_backward(const void *logits_dev, int32_t logits_type, int64_t rows, int64_t n_choices, int64_t ld_logits,
                                  const int32_t *teacher_token_dev, const void *teacher_logits_dev, int32_t teacher_type, int32_t k,
                                  const float *temperature_dev, const float *norm_dev, const float *dloss_dev, void *dlogits_dev, int64_t ld_dlogits,
                                  void *stream);

/* A [batch][steps][channels] array: channels side by side, any strides (in elements) between steps and sequences.  Read-only
 * ones may repeat themselves (stride 0); written ones must not overlap themselves or anything else (RLS_ERR_SHAPE; views that lie between
 * each other's rows are fine if they are as far apart, and may be turned down if not). */
typedef struct {
    void *data_dev;
    int64_t batch_stride, step_stride;
} rls_sequence;

typedef struct {
    int64_t batch, steps, channels;
    int32_t type;              /* of b, h and their gradients: RLS_F32, RLS_BF16 or RLS_F16 */
    int32_t gate_type;         /* of a and its gradient: RLS_F32 or `type` */
    int32_t reverse;           /* != 0: time runs from the last step to the first (returns and advantages) */
} rls_scan_shape;

/*
 * The gated linear recurrence, sequence by sequence and channel by channel, in the direction of time:
 *   h_t = a_t h_{t-1} + b_t, in fp32; at a step whose reset byte is not 0 nothing is carried over: h_t = b_t
 * It is the search agent's discounted return or advantage (b the rewards or temporal differences, a the discount,
 * resets where an episode begins in the direction of time), and a recurrent layer over long sequences.
 *   h0_dev      [batch][channels] fp32, the state before the first step, or null (0)
 *   reset_dev   [batch][steps] bytes or null
 *   h           (written) every state, rounded to `type`;  h_last_dev [batch][channels] fp32 (written) or null, the state
 *               after the last step in fp32; it may be h0_dev's memory: with steps = 1 the step of a single token
 * steps = 0 leaves h alone and copies h0 (or 0) to h_last.
 * Gates may be anything: long sequences are cut into tiles that are composed, but where a product of gates, or what is added up under it, passes the
 * largest number the steps are taken one by one.  An input that is not finite makes every state from there on, up to the next reset, not
 * finite (infinite or NaN); after finite inputs whose states pass the largest number, later ones may be either.  A term smaller
 * than 2^-126 times the state that it comes from may be left out, also where later gates above 1 would bring it back.
 */
int64_t rls_linear_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t channels);
int32_t rls_linear_scan(const rls_scan_shape *shape, const rls_sequence *a, const rls_sequence *b, const float *h0_dev,
                        const uint8_t *reset_dev, const rls_sequence *h, float *h_last_dev, void *workspace_dev,
                        int64_t workspace_bytes, void *stream);
/*
 * Its backward pass, from the states h that the forward pass wrote and the gradients dh and dh_last (null: 0) by them:
 *   g_t = dh_t + a_{t+1} g_{t+1} (nothing from a step that was reset), dh_last added at the last step;
 *   db_t = g_t,  da_t = g_t h_{t-1} (0 at a reset),  dh0 = a_1 g_1 (0 where the first step is reset)
 * For a broadcast input the caller adds up the gradients along the broadcast axis.
 *   da, db      (written) of gate_type and type;  dh0_dev [batch][channels] fp32 (written) or null, may be dh_last_dev's memory
 */
int32_t rls_linear_scan_backward(const rls_scan_shape *shape, const rls_sequence *a, const rls_sequence *h, const rls_sequence *dh,
                                 const float *h0_dev, const uint8_t *reset_dev, const float *dh_last_dev, const rls_sequence *da,
                                 const rls_sequence *db, float *dh0_dev, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* A [batch][steps][heads][dim] array: dimensions side by side, any strides (in elements) between heads, steps and sequences.  Read-only ones may
 * repeat themselves (stride 0); written ones must not overlap themselves or anything else (RLS_ERR_SHAPE; arrays that reach into each other count as overlapping). */
typedef struct {
    void *data_dev;
    int64_t batch_stride, step_stride, head_stride;
} rls_heads;

typedef struct {
    int64_t batch, steps;
    int32_t heads;             /* of v, o, g, beta and the state */
    int32_t key_heads;         /* of q and k; heads is a multiple, and head h reads key head h / (heads / key_heads) */
    int32_t key_dim, value_dim;
    int32_t type;              /* of q, k, v, o and their gradients: RLS_F32, RLS_BF16 or RLS_F16 */
    float scale;               /* of the output */
} rls_delta_shape;

/*
 * The gated delta rule: a recurrent layer beside rls_linear_scan whose state is a matrix S [key_dim][value_dim] per sequence and head.  Per step
 *   S = exp(g_t) S;  y_t = v_t - S^T k_t;  S = S + beta_t k_t y_t^T;  o_t = scale S^T q_t,   all in fp32, o rounded to `type`
 * It replaces what the state answers to a key by the step's value, in part (beta) and after forgetting (g).
 *   g_dev       [batch][steps][heads] fp32, logarithms of the decay: 0 keeps everything, less than -87 (or -infinity) nothing
 *   beta_dev    [batch][steps][heads] fp32
 *   reset_dev   [batch][steps] bytes or null: where one is not 0 a sequence begins, and nothing is carried over from the step before
 *   state_dev   [batch][heads][key_dim][value_dim] fp32, before the first step, or null (0)
 *   o           (written);  last_dev as state_dev (written) or null, after the last step; it may be state_dev itself: a state kept in place
 * steps = 0 leaves o alone and copies the state.  Keys of length 1 and beta in 0 .. 1 (2) keep the state in bounds; others are computed
 * as they are.  What is not finite, an input or a state, makes not finite what follows from it step by step in its head, from there on up to the next
 * reset or gate that keeps nothing, and nothing else.  Steps are taken in chunks; a head whose state is not finite at the end of one of a call's
 * launches has that launch's steps taken one by one instead (some 1 to 4 us each), also where it was a product over a chunk that passed the largest number.
 * The workspace is bounded along the steps; it holds a chunk of every sequence and head at least (up to 0.2 MB with 128 x 128, 0.5 MB for the backward pass).
 * 1 <= key_dim <= RLS_MAX_KEY_DIM, 1 <= value_dim <= RLS_MAX_VALUE_DIM, batch * heads <= 2^17, batch * steps <= 2^30.
 */
#define RLS_MAX_KEY_DIM 128
#define RLS_MAX_VALUE_DIM 512
int64_t rls_gated_delta_workspace_bytes(const rls_delta_shape *shape, int32_t backward);
int32_t rls_gated_delta(const rls_delta_shape *shape, const rls_heads *q, const rls_heads *k, const rls_heads *v, const float *g_dev, const float *beta_dev,
                        const float *state_dev, const uint8_t *reset_dev, const rls_heads *o, float *last_dev, void *workspace_dev, int64_t workspace_bytes,
                        void *stream);
/*
 * Its backward pass, from the inputs (the states are computed again) and the gradients dout by o and dlast (null: 0) by the last state.
 *   dq, dk, dv  (written) as q, k, v, summed over the heads that share a key head;  dg_dev, dbeta_dev (written) as g, beta: dg is 0 where nothing is carried
 *   dstate_dev  (written) as state_dev, or null; may be dlast_dev's memory
 * What is not finite, a gradient or anything it meets in the recurrence, may make the gradients of its head between the resets or gates that keep nothing on both
 * sides of it not finite (with a key or query, those of all heads that share it), and no others; so may decays whose product over up to 64 steps passes the
 * largest number.
 */
int32_t rls_gated_delta_backward(const rls_delta_shape *shape, const rls_heads *q, const rls_heads *k, const rls_heads *v, const float *g_dev,
                                 const float *beta_dev, const float *state_dev, const uint8_t *reset_dev, const rls_heads *dout, const float *dlast_dev,
                                 const rls_heads *dq, const rls_heads *dk, const rls_heads *dv, float *dg_dev, float *dbeta_dev, float *dstate_dev,
                                 void *workspace_dev, int64_t workspace_bytes, void *stream);

/*
 * One AdamW step (Table 2's optimizer, with decoupled weight decay) over any number of tensors.  Per element, in fp32:
 *   g = grad * grad_scale;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g g
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * With a master array p is read from and written to it, and the parameter is its rounded copy.  NaN and infinite
 * gradients go into the element's parameter and moments as the arithmetic has it.
 * Moments in 8 bits (state_bits = 8): every 256 consecutive elements of a tensor share a scale, a power of two; m and sqrt(v)
 * are held as 8-bit floats (1-4-3, the format whose largest value is 448) times it.  They are rounded up or down at random, in
 * proportion: v moves by a thousandth a step, which rounding to nearest would lose every time.  The random bits come from
 * (seed, step, tensor, element) alone.  A v that is not 0 is never rounded to 0.
 */
typedef struct {
    int64_t n;                 /* elements, >= 0 */
    int32_t param_type;        /* RLS_F32, RLS_BF16, RLS_F16 */
    int32_t grad_type;         /* RLS_F32 or param_type */
    void *param_dev;           /* [n] (updated) */
    const void *grad_dev;      /* [n] */
    float *master_dev;         /* [n] fp32 weights (updated), or null: param itself is read */
    void *m_dev, *v_dev;       /* [n] fp32, or [n] 8-bit floats of m and sqrt(v) (updated) */
    float *m_scale_dev, *v_scale_dev;   /* [(n + 255) / 256] fp32 (updated); not read with state_bits = 32 */
} rls_adamw_tensor;
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;              /* >= 1: the number of this step */
    uint64_t seed;             /* of the rounding at random (state_bits = 8) */
    int32_t state_bits;        /* 32 or 8 */
    const float *grad_scale_dev;        /* one fp32 factor of all gradients (clipping, loss scaling), or null (1) */
} rls_adamw_options;
/* `tensors` is a host array, read before the call returns.  What a step updates must not overlap anything else that it reads or updates. */
int32_t rls_adamw_step(const rls_adamw_tensor *tensors, int32_t n_tensors, const rls_adamw_options *options, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* RLS_H */
