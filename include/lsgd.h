/*
 * lsgd.h - C boundary of the batched Leader-SGD step for one AMD MI355X (gfx950).
 *
 * A population of W workers lives on one GPU as a row-major fp32 matrix
 * x[W, ld] (row i = parameters of worker i, P <= ld used columns).  Workers are
 * partitioned into n contiguous groups (Eq. 2 of arXiv 1905.10395: n groups of
 * l workers, each with a local leader, plus one global leader).  One step is
 *
 *   1. lsgd_grad_loss       g_i, loss_i of every worker on its own minibatch
 *                           (Section 2: stochastic gradient g_t^{j,i}; Section
 *                           3.1.3: one loss sample per worker)
 *   2. lsgd_select_leaders  segmented argmin of the losses (Eq. 1 / Eq. 2;
 *                           the leader-picking steps of Algorithm 1)
 *   3. lsgd_pull_update     x_i <- x_i - eta*(g_i + lam_L (x_i - z_local)
 *                                              + lam_G (x_i - z_global))
 *                           (supplement B.1; Eq. 3), optional momentum
 *   lsgd_step               1-3 on the population's stream, no host sync.
 *
 * General rules
 *   - Pointers marked "device" are device memory owned by the caller for the
 *     life of the handle; the library never allocates, frees or resizes them.
 *     Pointers marked "host" are read during the call only.
 *   - Every call validates its arguments first; a failing call enqueues no
 *     device work.  Calls return an lsgd_status and never abort or throw;
 *     lsgd_last_error() gives a message for the last failure on this thread.
 *   - All device work is enqueued on the stream given at creation.  Only
 *     lsgd_get_leaders / lsgd_get_losses synchronise that stream.
 *   - Worker indices returned are global, in [0, W).
 */
#ifndef LSGD_H
#define LSGD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lsgd_population lsgd_population; /* opaque host object */

typedef enum {
    LSGD_OK = 0,
    LSGD_ERR_INVALID_ARG = 1, /* NULL where a pointer is required, bad enum, non-finite scalar */
    LSGD_ERR_SHAPE = 2,       /* W<=0, ld<P, offsets not covering [0,W], sizes not matching P  */
    LSGD_ERR_STATE = 3,       /* call order: pull with lam>0 before any selection, missing buffer */
    LSGD_ERR_UNSUPPORTED = 4, /* shape outside what the kernels implement                       */
    LSGD_ERR_HIP = 5,         /* a HIP runtime call failed                                      */
    LSGD_ERR_NOMEM = 6        /* workspace too small / host allocation failed                   */
} lsgd_status;

/* lsgd_config.flags */
enum {
    LSGD_NESTEROV = 1,            /* x <- x - eta*(d + mu*m) instead of x <- x - eta*m            */
    LSGD_LEADER_EXEMPT = 2,       /* a leader is not pulled to a (stale) copy of itself:
                                     supplement, lemma on leader descent                          */
    LSGD_PULL_UNSCALED_BY_ETA = 4,/* Eq. 3 as printed: pulls are not multiplied by eta            */
    LSGD_MOMENTUM_GRAD_ONLY = 8,  /* momentum buffer accumulates g only; pulls applied outside it */
    LSGD_WRITE_BF16_SHADOW = 16,  /* pull_update also writes bf16(x) to x_bf16 (MLP operands)     */
    LSGD_FUSED_MLP_UPDATE = 32    /* lsgd_step on LSGD_BATCH_MLP applies the update inside the
                                     backward kernels (the gradient never goes through memory):
                                     g is not written and holds unspecified values afterwards,
                                     x_bf16 is always kept current.  Same results as the
                                     three-call sequence up to fp32 rounding.  Needs z_snapshot
                                     when a lambda is non-zero.  Other batch kinds and the
                                     separate calls are unaffected.                              */
};

#define LSGD_MAX_WORKERS 32768
#define LSGD_MAX_GROUPS 1024

typedef struct {
    int32_t W;                    /* workers = rows                                              */
    int64_t P;                    /* parameters per worker                                       */
    int64_t ld;                   /* row stride in elements, ld >= P                             */
    int32_t n_groups;             /* n of Eq. 2                                                  */
    const int32_t* group_offsets; /* host [n_groups+1], strictly increasing, [0]=0, [n]=W;
                                     NULL: W % n_groups == 0 and equal contiguous groups          */
    float momentum;               /* mu; 0 disables the momentum buffer                          */
    int32_t flags;                /* LSGD_* bits above                                           */
    float weight_decay;           /* g <- g + wd*x inside the update; 0 = none                   */
} lsgd_config;

/* ---- minibatch descriptors (host structs; the arrays they point to are device memory) ---- */
typedef enum { LSGD_BATCH_EXTERNAL = 0, LSGD_BATCH_MC = 1, LSGD_BATCH_MLP = 2 } lsgd_batch_kind;

/* Gradient and losses were produced by the caller: g (given at creation) is
 * already filled; losses is device [W].                                        */
typedef struct {
    const float* losses; /* device [W] */
} lsgd_external_batch;

/* Low-rank matrix completion on observed entries (the problem family of the
 * paper's motivating example and supplement, rectangular form).  Worker row =
 * [U (m x r, row-major) | V (n x r, row-major)], P = (m+n)*r.  For each batch
 * entry k = (a_k, b_k, M_k): e_k = <U[a_k],V[b_k]> - M_k;
 * loss = c*sum e_k^2; dU[a] = 2c*sum_{a_k=a} e_k V[b_k]; dV[b] likewise.
 * Entries drawn more than once count each time.                                */
typedef struct {
    int32_t row, col; /* a, b                                                       */
    float val;        /* M_ab                                                       */
    int32_t reserved; /* keeps the record at 16 bytes                               */
} lsgd_mc_entry;

typedef struct {
    int32_t m, n, r;
    const int32_t* rows;      /* device [n_obs] row index a of each observed entry  */
    const int32_t* cols;      /* device [n_obs] column index b                      */
    const float* vals;        /* device [n_obs] observed value M_ab                 */
    int64_t n_obs;
    const int32_t* batch_idx; /* device [W, B] indices into the observed list, or
                                 NULL: every worker uses all n_obs entries (batch
                                 gradient, "LGD")                                   */
    int64_t B;                /* entries per worker when batch_idx != NULL          */
    float c;                  /* loss normalisation                                 */
    const lsgd_mc_entry* entries; /* device [n_obs], optional: the same observed list with
                                 one 16-byte record per entry (see lsgd_mc_pack_entries).
                                 When non-NULL it is read instead of rows/cols/vals:
                                 one random access per batch element instead of three */
} lsgd_mc_batch;

/* Fully connected ReLU classifier with softmax cross-entropy, mean over the
 * batch.  Worker row = [W_1 (d1 x d0 row-major) | b_1 | W_2 | b_2 | ...].
 * Matrix operands (inputs, weights, stored activations, back-propagated
 * deltas) are bf16, accumulation and everything else fp32.                     */
typedef struct {
    int32_t n_layers;    /* number of weight matrices                              */
    const int32_t* dims; /* host [n_layers+1]: d0 (input) ... d_L (classes)        */
    const void* X;       /* device [W, B, d0]: bf16 bit patterns (uint16), or fp32
                            values when x_is_fp32 (rounded to bf16, to nearest even,
                            on the way in: a copy in the workspace)                */
    const int32_t* y;    /* device [W, B] class labels in [0, d_L)                 */
    int32_t B;           /* samples per worker                                     */
    int32_t x_is_fp32;   /* 0: X holds bf16 bit patterns; 1: X holds fp32 values   */
} lsgd_mlp_batch;

typedef struct {
    int32_t kind;     /* lsgd_batch_kind                                            */
    const void* desc; /* host pointer to the matching struct above                  */
} lsgd_batch;

/* Bytes of device workspace lsgd_create_population needs for this population
 * and for gradient calls shaped like `largest` (NULL: selection and update
 * only).  Returns 0 on invalid arguments (see lsgd_last_error).               */
size_t lsgd_workspace_bytes(const lsgd_config* cfg, const lsgd_batch* largest);

/* Binds caller-owned device buffers into a population handle.
 *   x, g       device [W, ld] fp32, required
 *   m          device [W, ld] fp32, required iff cfg->momentum != 0; the caller zeroes it
 *   z_snapshot device [(n_groups+1), ld] fp32 leader copies kept between
 *              communications (Algorithm 1; supplement B.1).  NULL is allowed
 *              when every update follows a full refresh.
 *   x_bf16     device [W, ld] bf16, required for LSGD_BATCH_MLP and for
 *              LSGD_WRITE_BF16_SHADOW, else NULL
 *   workspace  device, >= lsgd_workspace_bytes(...), 256-byte aligned
 *   hip_stream a hipStream_t (NULL = default stream)
 * The fast update path needs x, g, m, z_snapshot 16-byte aligned and ld % 4 == 0;
 * other layouts take a scalar path.                                            */
lsgd_status lsgd_create_population(const lsgd_config* cfg, float* x, float* g, float* m,
                                   float* z_snapshot, uint16_t* x_bf16, void* workspace,
                                   size_t workspace_bytes, void* hip_stream,
                                   lsgd_population** out);

/* Frees the host object only. */
lsgd_status lsgd_destroy_population(lsgd_population* pop);

/* Writes g[W, ld] (unused padding columns zeroed) and losses (device [W]; NULL =
 * the population's own loss buffer, the one lsgd_step uses).  For
 * LSGD_BATCH_EXTERNAL copies the given losses into the population's buffer when
 * `losses` is NULL, otherwise into `losses`.  For LSGD_BATCH_MC gradients and
 * losses are sums in no fixed order (losses in double, rounded once): equal
 * calls can differ in the last bit, and workers of equal rows on equal entries
 * need not tie.                                                                */
lsgd_status lsgd_grad_loss(lsgd_population* pop, const lsgd_batch* batch, float* losses);

/* Objective values only: losses[i] = f_i(x_i) on worker i's part of the batch at
 * the current parameters (device [W]; NULL = the population's own loss buffer);
 * g is neither read nor written.  This is what choosing a leader costs (Section
 * 3.1.3: the leader is the worker whose estimate of the objective, one draw per
 * worker, is smallest; Algorithm 1 determines the best workers after the local
 * step, at the parameters that step produced, on the sample of the iteration
 * that follows).  lsgd_step and
 * lsgd_step_alg1 select from the losses of their own gradient pass, i.e. at the
 * parameters before the step; the printed order is
 *   lsgd_step_alg1(..., comm = 0); lsgd_loss(next batch, NULL);
 *   lsgd_select_leaders(NULL, mask, global); lsgd_leader_pull(lambda, lambda_G).
 * Same batch kinds, checks and workspace as lsgd_grad_loss.  For LSGD_BATCH_MC
 * the squared residuals are summed in another order than in lsgd_grad_loss, so
 * the two values can differ in the last bits; for LSGD_BATCH_MLP it is the
 * forward pass of lsgd_grad_loss (bit-identical losses).                        */
lsgd_status lsgd_loss(lsgd_population* pop, const lsgd_batch* batch, float* losses);

/* Segmented argmin.  For each group j with refresh_local[j] != 0 (host
 * [n_groups]; NULL = all) the local leader becomes the lowest index attaining the
 * group's minimum loss; if refresh_global the global leader becomes the lowest
 * index attaining the minimum over all workers.  NaN counts as +infinity.  The
 * leaders refreshed here are captured (copied from x before any row changes) by
 * the next lsgd_pull_update; the others keep their stored copies.
 * losses: device [W]; NULL = the population's own buffer (LSGD_ERR_STATE if
 * nothing has written it yet).                                                  */
lsgd_status lsgd_select_leaders(lsgd_population* pop, const float* losses,
                                const uint8_t* refresh_local, int refresh_global);

/* d = g + wd*x + lam_L (x - z_local) + lam_G (x - z_global);
 * mu = 0: x <- x - eta*d;  mu > 0: m <- mu*m + d, x <- x - eta*m (flags modify).
 * In place on x and m; every row is computed from pre-update values.  A term
 * whose coefficient is exactly 0 is skipped and its leader copy is neither read
 * nor written.  LSGD_ERR_STATE if a needed leader was never selected, or a kept
 * copy is needed and z_snapshot is NULL.  A leader re-selected since the last
 * update whose coefficient is 0 in this call is not captured; its kept copy is
 * then no longer valid (LSGD_ERR_STATE for a later update that would need it
 * before the next selection).                                                   */
lsgd_status lsgd_pull_update(lsgd_population* pop, float eta, float lambda_L, float lambda_G);

/* grad_loss -> select_leaders -> pull_update with the population's own loss
 * buffer.  The first step of a population must refresh everything.  With
 * LSGD_FUSED_MLP_UPDATE and an LSGD_BATCH_MLP batch the same three stages run as
 * forward pass + losses -> select_leaders -> kept copies brought up to date ->
 * backward pass that applies the update (see the flag); the state afterwards is
 * the same up to fp32 rounding, except that g is left unspecified.             */
lsgd_status lsgd_step(lsgd_population* pop, const lsgd_batch* batch, float eta, float lambda_L,
                      float lambda_G, const uint8_t* refresh_local, int refresh_global);

/* Communication pull of Algorithm 1 (its two blocks that pick the best
 * workers and move everyone towards them): captures every leader
 * re-selected since the last update (copied from x before any row changes, and
 * written to z_snapshot when it exists, also when its coefficient is 0), then
 *   groups whose local leader was re-selected:  x <- x - lambda_L (x - z_local)
 *   if the global leader was re-selected:        x <- x - lambda_G (x - z_global)
 * in that order, element-wise, with no gradient, learning rate or momentum
 * involved.  Groups (or the global term) with nothing re-selected are left
 * alone.  LSGD_ERR_STATE if nothing was re-selected since the last update.     */
lsgd_status lsgd_leader_pull(lsgd_population* pop, float lambda_L, float lambda_G);

/* lsgd_step_alg1.comm bits */
enum {
    LSGD_COMM_LOCAL = 1,  /* local communication at this step  (n l tau   divides the iteration count) */
    LSGD_COMM_GLOBAL = 2  /* global communication at this step (n l tau_G divides the iteration count) */
};

/* One iteration of Algorithm 1 for every worker at once:
 *   grad_loss;  x <- x - eta g - gamma_L (x - z_local) - gamma_G (x - z_global)
 *   with the kept leader copies (gamma_L = gamma/tau, gamma_G = gamma_G/tau_G,
 *   not multiplied by eta; momentum, weight decay and flags of the population
 *   apply to the gradient part as in lsgd_pull_update);
 *   then, when comm has LSGD_COMM_LOCAL / LSGD_COMM_GLOBAL: select_leaders from
 *   this iteration's losses (comm_local_mask: host [n_groups] choosing the
 *   groups that communicate, NULL = all) followed by lsgd_leader_pull.
 * Before the first iteration the caller initialises the leaders (the
 * initialisation block of Algorithm 1): grad_loss, select_leaders(all), lsgd_leader_pull(0, 0).
 * Needs z_snapshot.  eta must be non-zero when a gamma is.                      */
lsgd_status lsgd_step_alg1(lsgd_population* pop, const lsgd_batch* batch, float eta, float gamma_L,
                           float gamma_G, float lambda_L, float lambda_G, int comm,
                           const uint8_t* comm_local_mask);

/* Selection loss averaged over the last K minibatches (Section 4.1: leaders are
 * determined from the average training loss over the last 10 or 64 batches).
 *   window device [K, W] fp32 ring owned by the caller; slot t % K receives the
 *          new losses (no initialisation needed: only filled slots are read)
 *   t      0-based count of calls so far on this ring
 *   losses device [W] new losses; NULL = the population's own buffer
 *   out    device [W] mean over the min(t+1, K) newest slots, summed in slot
 *          order in double; NULL = the population's own buffer (so that a
 *          following lsgd_select_leaders(pop, NULL, ...) uses it); may alias losses. */
lsgd_status lsgd_smooth_losses(lsgd_population* pop, float* window, int32_t K, int64_t t,
                               const float* losses, float* out);

/* Center variable (Section 4.1: the model reported at test time is the average
 * of all workers' parameters): out[p] = (1/W) sum_i x[i, p], summed over i in
 * order in double and rounded once.  out: device [P] (16-byte aligned for the
 * fast path), must not overlap x.                                              */
lsgd_status lsgd_center(lsgd_population* pop, float* out);

/* Elastic averaging (EAGD / EASGD), the method the paper compares with, as a variant of the same update
 * (supplement, "Low-Rank Matrix Completion Experiments": both methods are X+ = (1 - eta lam) X + eta lam Z -
 * eta grad, with Z the leader for LGD and the center for EAGD):
 *   center+ = (1 - W eta lam) center + W eta lam * (1/W) sum_i x_i       (mean in double, rounded once)
 *   x_i+    = x_i - eta (g_i + lam (x_i - center))                        for every worker,
 * both from the values before the call; momentum, weight decay and the Nesterov / grad-only flags of the
 * population apply to the workers' step as in lsgd_pull_update; no leaders are involved.
 *   center device [ld] fp32 owned by the caller (16-byte aligned for the fast path), updated in place; the
 *          caller initialises it (the paper does not say how; e.g. with lsgd_center)
 * The pre-update center is kept in the global row of z_snapshot during the call, which therefore must exist
 * and afterwards no longer holds a global leader copy.  LSGD_ERR_STATE while a leader selection is pending.
 * lsgd_easgd_step = lsgd_grad_loss into the population's own buffers, then lsgd_easgd_update.            */
lsgd_status lsgd_easgd_update(lsgd_population* pop, float* center, float eta, float lambda);
lsgd_status lsgd_easgd_step(lsgd_population* pop, const lsgd_batch* batch, float* center, float eta, float lambda);

/* Builds the 16-byte-record form of an observed-entry list (device to device, on
 * hip_stream): out[k] = {rows[k], cols[k], vals[k], 0}.  The list of observed
 * entries is fixed across steps (the paper's M and its observed set), so this is
 * done once by the caller.  All pointers device, [n_obs].                          */
lsgd_status lsgd_mc_pack_entries(const int32_t* rows, const int32_t* cols, const float* vals,
                                 int64_t n_obs, lsgd_mc_entry* out, void* hip_stream);

/* Recomputes the whole bf16 shadow from x (after the caller changed x). */
lsgd_status lsgd_sync_shadow(lsgd_population* pop);

/* Synchronise the stream and read back.  local_leaders: host [n_groups];
 * global_leader: host [1]; either may be NULL.  Leaders never selected read -1. */
lsgd_status lsgd_get_leaders(lsgd_population* pop, int32_t* local_leaders, int32_t* global_leader);
/* Restores leader indices read earlier with lsgd_get_leaders (checkpoint / resume: the state of a run is
 * x, m, z_snapshot and these G+1 indices; x_bf16 is rebuilt from x by the next gradient call).  The rows of
 * z_snapshot are taken to be the copies that belong to these leaders, no re-selection is pending afterwards.
 * local_leaders: host [n_groups], each a row of its group or -1 (never selected); global_leader: a row or -1.
 * Synchronises the stream.                                                                                */
lsgd_status lsgd_set_leaders(lsgd_population* pop, const int32_t* local_leaders, int32_t global_leader);
/* losses_host: host [W], the population's own loss buffer. */
lsgd_status lsgd_get_losses(lsgd_population* pop, float* losses_host);

/* For callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  One leader selection over all groups and
 * the global leader followed by one pull update, i.e. what lsgd_step does for an
 * LSGD_BATCH_EXTERNAL batch with a full refresh, without a population handle or workspace:
 * the group table, leader indices and re-selection flags that the handle keeps in the
 * caller's workspace live in a static device array inside the library (38 KB per GPU, held
 * until the process ends), and the call itself allocates nothing on the host or the device.
 *   W <= LSGD_STATIC_MAX_WORKERS, n_groups <= LSGD_STATIC_MAX_GROUPS: larger shapes are
 *            rejected with LSGD_ERR_SHAPE
 *   group_offsets host [n_groups+1] or NULL (equal groups), as in lsgd_config
 *   x, g, m  device [W, ld] fp32 as in lsgd_create_population (m may be NULL when
 *            momentum == 0); updated in place exactly as lsgd_pull_update does
 *   losses   device [W]
 *   leaders  device [n_groups+1] int32 or NULL: receives the local leaders and, last, the
 *            global leader
 *   flags    LSGD_NESTEROV | LSGD_LEADER_EXEMPT | LSGD_PULL_UNSCALED_BY_ETA |
 *            LSGD_MOMENTUM_GRAD_ONLY
 * Every leader is re-selected at every call, so no leader copies are kept.  Work is enqueued
 * on hip_stream of the current device; nothing synchronises.  All calls on one GPU share
 * that GPU's array: calls that may overlap there (different streams, different threads)
 * race and must be ordered by the caller.  Every word a call reads it writes first, so the
 * contents left by an earlier call never matter.                                          */
#define LSGD_STATIC_MAX_WORKERS 1024
#define LSGD_STATIC_MAX_GROUPS 64
lsgd_status lsgd_select_pull_static(int32_t W, int64_t P, int64_t ld, int32_t n_groups,
                                    const int32_t* group_offsets, float* x, const float* g, float* m,
                                    const float* losses, int32_t* leaders, float eta, float lambda_L,
                                    float lambda_G, float momentum, float weight_decay, int32_t flags,
                                    void* hip_stream);

/* Measurement aid, not part of the method: one pass of a plain stream over n floats per buffer, in
 * memory order, so that a benchmark can report what the memory system at hand gives the access
 * shapes the update uses, beside the update's own rate.
 *   LSGD_PROBE_READ    reads a                              (4 n bytes)
 *   LSGD_PROBE_COPY    b <- a                               (8 n bytes)
 *   LSGD_PROBE_UPDATE  c <- 0.9 c + b ; a <- a - 1e-3 c     (20 n bytes: the momentum update without
 *                      leader rows, 3 reads and 2 writes per element)
 * a, b, c: device [n] fp32, 8-byte aligned, n even (c may be NULL except for LSGD_PROBE_UPDATE).     */
enum { LSGD_PROBE_READ = 0, LSGD_PROBE_COPY = 1, LSGD_PROBE_UPDATE = 2 };
lsgd_status lsgd_stream_probe(int32_t kind, float* a, float* b, float* c, int64_t n, void* hip_stream);

/* ---- Operators of token models ------------------------------------------------------------------
 * What a population of models over tokens needs around its blocks' matrix products and for its step.  As everywhere,
 * worker w's parameters and gradients are columns of row w of fp32 matrices (x, g), so a pointer into row 0 and the
 * row stride ld name a parameter tensor of all workers.  None of these needs a population handle; each takes its stream,
 * device pointers and workspace from the caller, allocates nothing on the device and does not synchronise (except
 * lsgd_adamw_create).  Strides count elements.  bf16 data are bit patterns; sums, norms and moments' arithmetic are fp32. */

/* Embedding lookup: out[w,t,:] = scale * table_w[tokens[w,t], :], the fp32 product, rounded again to bf16 if out is; zeros
 * where the token lies outside [0, V) (padding: such a place is never looked up).
 *   table  device, worker w's [V, D] at table + w*ld_table (fp32 or bf16; ld_table = 0: one table for all workers)
 *   tokens device int32, worker w's [T] at tokens + w*ld_tokens (0: the same for all workers)
 *   out    device, worker w's [T, D] at out + w*ld_out (fp32 or bf16); must not overlap the inputs
 * T = 0 is allowed.  T <= 2^24, V < 2^30, D <= 2^20, and T * ceil(D/8) below 2^34 (T * ceil(D/4) from fp32 to fp32). */
lsgd_status lsgd_embed_lookup(int32_t W, int32_t T, int32_t V, int32_t D, const void* table, int64_t ld_table, int32_t table_is_bf16,
                              const int32_t* tokens, int64_t ld_tokens, float scale, void* out, int64_t ld_out, int32_t out_is_bf16,
                              void* hip_stream);

/* Its gradient: dtable_w[v,:] = scale * sum over t with tokens[w,t] = v of dout[w,t,:], summed in fp32 in an order that
 * depends on the tokens alone (equal calls give equal bits).
 *   accumulate 0: every row of the table is written, zeros where no token names it; 1: the sum is added to what is there
 *              (tied weights, several batches a step) and rows that no token names are not touched
 *   dout       device, worker w's [T, D] at dout + w*ld_dout (fp32 or bf16; 0: the same for all workers)
 *   dtable     device fp32, worker w's [V, D] at dtable + w*ld_dtable, ld_dtable >= V*D; must not overlap the inputs
 *   workspace  device, >= lsgd_embed_grad_workspace_bytes, 256-byte aligned; not kept; may be NULL up to
 *              LSGD_EMBED_GRAD_ONE_LAUNCH tokens a worker, which take one launch and none                          */
#define LSGD_EMBED_GRAD_ONE_LAUNCH 8192
size_t lsgd_embed_grad_workspace_bytes(int32_t W, int32_t T, int32_t V, int32_t D); /* 0 on invalid arguments */
lsgd_status lsgd_embed_grad(int32_t W, int32_t T, int32_t V, int32_t D, const void* dout, int64_t ld_dout, int32_t dout_is_bf16,
                            const int32_t* tokens, int64_t ld_tokens, float scale, int32_t accumulate, float* dtable, int64_t ld_dtable,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* Activations [W, T, D] with dense rows: token t of worker w at data + w*worker_stride + t*token_stride. */
typedef struct {
    void* data; /* device; NULL: absent */
    int64_t worker_stride, token_stride;
} lsgd_rows;

/* Norms after and before a block, fused with its gate and residual sum, D <= 16384:
 *   r_out = r + scale * sigmoid(gate) o (q_post y o w_post)   q_post = (mean_d y^2 + eps)^-1/2     (when y is given)
 *   n     = q_pre r_out o w_pre                               q_pre  = (mean_d r_out^2 + eps)^-1/2  (when n is given)
 * With y absent the second line takes r in r_out's place (a model's first norm); with n absent only the sum is made (its
 * last).  gate absent: 1.  post_norm = 0: q_post = 1 (blocks without a norm behind them; w_post then scales channels).
 * n is computed from r_out before that is rounded to its type.  r_out may be r, and n may be y or gate, element for
 * element; no other overlaps.                                                                              */
typedef struct {
    int32_t W, T, D;
    int32_t is_bf16;              /* type of r, y, gate, r_out, n: 0 fp32, 1 bf16                    */
    int32_t post_norm;
    float scale, eps;             /* eps > 0                                                         */
    lsgd_rows r, y, gate, r_out, n;
    const float *w_post, *w_pre;  /* device fp32, worker w's [D] at w_post + w*ld_w_post; NULL: ones */
    int64_t ld_w_post, ld_w_pre;
    float *q_post, *q_pre;        /* device fp32 [W, T], what the gradient needs; NULL: not wanted   */
} lsgd_block_norm_args;
lsgd_status lsgd_block_norm(const lsgd_block_norm_args* args, void* hip_stream);

/* Its gradients from dn (of n; absent: there was no norm before the next block) and dr_out (what reaches r_out past it;
 * absent: nothing), given what the forward call read and gave:
 *   dr (of r), dy, dgate     [W, T, D] of the activations' type
 *   dw_post, dw_pre          device fp32, worker w's [D] at dw + w*ld; NULL: not wanted; accumulate = 1 adds to them
 * r_out and q_pre are needed with dn, q_post with a post-norm.  dr may be dr_out or dn, dy may be y, dgate may be gate,
 * element for element.  Sums over tokens are made in an order that depends on the sizes alone.
 *   workspace  device, >= lsgd_block_norm_grad_workspace_bytes, 256-byte aligned; may be NULL when no dw is wanted   */
typedef struct {
    int32_t W, T, D;
    int32_t is_bf16, post_norm, accumulate;
    float scale;
    lsgd_rows dn, dr_out, r_out, y, gate, dr, dy, dgate;
    const float *w_post, *w_pre;
    int64_t ld_w_post, ld_w_pre;
    const float *q_post, *q_pre;
    float *dw_post, *dw_pre;
    int64_t ld_dw_post, ld_dw_pre;
} lsgd_block_norm_grad_args;
size_t lsgd_block_norm_grad_workspace_bytes(int32_t W, int32_t T, int32_t D); /* 0 on invalid arguments */
lsgd_status lsgd_block_norm_grad(const lsgd_block_norm_grad_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Activations [B, T, H, D] of attention with dense columns: head h of token t of entry b (a worker, or one of its sequences) at
 * data + b*batch_stride + t*token_stride + h*head_stride.  Parts of one projection's columns are such tensors.        */
typedef struct {
    void* data; /* device; NULL: absent */
    int64_t batch_stride, token_stride, head_stride;
} lsgd_heads;

/* Queries and keys before attention: each head's norm and its rotation by the token's position, D <= 256:
 *   z = x o w / sqrt(mean_d x^2 + eps)       (norm = 0: z = x o w)
 *   out = z with pair i of its first R columns turned by 2 pi * position * turns[i] and multiplied by magnitude; pairs are columns
 *         (i, i + R/2), or, interleaved = 1, (2i, 2i + 1); columns from R on are z's
 * The entries are workers; q [W, T, Hq, D], k [W, T, Hk, D] (Hk = 0: no keys; keys alone are passed as q).
 *   turns      device fp64 [R/2]: turns per position of each pair; a context is stretched by making them smaller.  The product with
 *              the position is made in 64 bits.  R = 0: no rotation.
 *   positions  device int32, worker w's [T] at positions + w*ld_positions (0: the same for all workers); any values; NULL: 0 .. T-1
 *   w_q, w_k   device fp32, worker w's [D] at w + w*ld (0: the same for all workers), shared by its heads; NULL: ones
 *   stats      device fp32 [W, T, Hq + Hk]: the norms' factors, which the gradient needs; NULL: not wanted
 * q_out may be q and k_out may be k, element for element; no other overlaps.  T <= 2^24, Hq and Hk <= 1024.               */
typedef struct {
    int32_t W, T, Hq, Hk, D, R;
    int32_t is_bf16;              /* type of q, k and the results: 0 fp32, 1 bf16 */
    int32_t norm, interleaved;
    float eps, magnitude;         /* eps > 0                                     */
    lsgd_heads q, k, q_out, k_out;
    const int32_t* positions;
    int64_t ld_positions;
    const double* turns;
    const float *w_q, *w_k;
    int64_t ld_w_q, ld_w_k;
    float* stats;
} lsgd_qk_rotary_args;
lsgd_status lsgd_qk_rotary(const lsgd_qk_rotary_args* args, void* hip_stream);

/* Its gradients from dq_out, dk_out (of the results), given what the forward call read and gave:
 *   dq, dk      of q and k; dq may be dq_out or q, dk may be dk_out or k, element for element
 *   dw_q, dw_k  device fp32, worker w's [D] at dw + w*ld; NULL: not wanted; accumulate = 1 adds to them
 * q, k may be absent where there is no norm and their dw is not wanted.  Sums over tokens and heads are made in an order that depends
 * on the sizes and alignment alone.
 *   workspace  device, >= lsgd_qk_rotary_grad_workspace_bytes, 256-byte aligned; may be NULL when no dw is wanted          */
typedef struct {
    int32_t W, T, Hq, Hk, D, R;
    int32_t is_bf16, norm, interleaved, accumulate;
    float magnitude;
    lsgd_heads dq_out, dk_out, q, k, dq, dk;
    const int32_t* positions;
    int64_t ld_positions;
    const double* turns;
    const float *w_q, *w_k;
    int64_t ld_w_q, ld_w_k;
    const float* stats;
    float *dw_q, *dw_k;
    int64_t ld_dw_q, ld_dw_k;
} lsgd_qk_rotary_grad_args;
size_t lsgd_qk_rotary_grad_workspace_bytes(int32_t W, int32_t T, int32_t Hq, int32_t Hk, int32_t D, int32_t R, int32_t is_bf16); /* 0 on invalid arguments */
lsgd_status lsgd_qk_rotary_grad(const lsgd_qk_rotary_grad_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Attention, D <= 128: out[b,t,h,:] = sum_j p_j v[b,j,h',:], p = softmax over the seen keys j of scale * q[b,t,h,:] . k[b,j,h',:]
 * with h' = h / (Hq / Hk) (Hk divides Hq: query heads that share a key head are adjacent).
 *   seen        j < k_lens[b]; causal = 1: and j <= t + k_lens[b] - q_lens[b], that is both sequences end together (a new token sees
 *               its whole cache)
 *   q_lens, k_lens  device int32 [B], read on the device and taken as within [0, Tq], [0, Tk]; NULL: all Tq, all Tk
 *   lse         device fp32 [B, Hq, Tq]: log of the sum of exp(scale q.k), which the gradient needs; NULL: not wanted
 * A query that sees no key, or behind q_lens[b], has out = 0 and lse = -inf.  What lies in memory at such queries and at keys from
 * k_lens[b] on does not matter (NaN neither); a key that is merely not seen yet must be finite, or queries beside may get NaN from it.
 * NaN in a query, or in keys that it sees, makes its results NaN, and in their values those columns.  Infinities there make them
 * infinite or NaN; a score of -inf counts nothing, or makes them NaN.  fp32 elements above the largest bf16 (3.39e38) count as infinite.
 * Scores, softmax and sums are fp32; sums of p v before their division reach 2^8 Tk max|v|, which must be finite.  With bf16 data p is
 * rounded to bf16 before the product with v.  out must not overlap the inputs.
 *   workspace  device, >= lsgd_attention_workspace_bytes, 256-byte aligned, not kept; may be NULL where that says 256, which it does up
 *              to LSGD_ATTENTION_ONE_LAUNCH keys.  Few queries and longer keys are split over the keys, and the parts joined from there. */
#define LSGD_ATTENTION_ONE_LAUNCH 1024
typedef struct {
    int32_t B, Tq, Tk, Hq, Hk, D;
    int32_t is_bf16;              /* type of q, k, v, out: 0 fp32, 1 bf16 */
    int32_t causal;
    float scale;                  /* within [1e-30, 1e30]                 */
    lsgd_heads q, k, v, out;
    const int32_t *q_lens, *k_lens;
    float* lse;
} lsgd_attention_args;
size_t lsgd_attention_workspace_bytes(int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t is_bf16); /* 0 on invalid arguments */
lsgd_status lsgd_attention(const lsgd_attention_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its gradients dq, dk, dv from dout, given what the forward call read and gave (out, lse): sums over queries, and over the heads that
 * share a key head, in an order that depends on the sizes and lengths alone.  Zeros at queries that see nothing, at queries from q_lens
 * and keys from k_lens on; what lies there (in dout, q, out, k, v) does not matter.  With bf16 data p and its gradient are rounded to
 * bf16 before their products.  NaN or infinities at a query that sees some key, or at a key that is seen, may reach gradients of keys
 * and queries of its entry that do not see each other.  dq, dk, dv must not overlap the inputs or each other.
 *   workspace  device, >= lsgd_attention_grad_workspace_bytes, 256-byte aligned, not kept                                  */
typedef struct {
    int32_t B, Tq, Tk, Hq, Hk, D;
    int32_t is_bf16, causal;
    float scale;
    lsgd_heads dout, q, k, v, out, dq, dk, dv;
    const int32_t *q_lens, *k_lens;
    const float* lse;
} lsgd_attention_grad_args;
size_t lsgd_attention_grad_workspace_bytes(int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t is_bf16); /* 0 on invalid arguments */
lsgd_status lsgd_attention_grad(const lsgd_attention_grad_args* args, void* workspace, size_t workspace_bytes, void* hip_stream);

/* AdamW over a list of tensors, one launch a step.
 *   m <- b1 m + (1-b1) c g;  v <- b2 v + (1-b2) (c g)^2
 *   x <- x (1 - lr lr_mult wd) - lr lr_mult/(1-b1^t) * m / (sqrt(v)/sqrt(1-b2^t) + eps)
 * A tensor is a [rows, n] part of matrices (for a population: rows = W, n = the tensor's elements in a worker's row, the
 * strides those of x and g); one row stands for any dense tensor.  Tensors must not overlap.
 * x_bf16 is what the step leaves: whoever changes x afterwards leaves the copy behind.  With a population over the same x
 * and x_bf16, its updates and pulls write the copy too under LSGD_WRITE_BF16_SHADOW, else lsgd_sync_shadow brings it up to date
 * (as it does for the population after a step of tensors without x_bf16).
 * state_bits 32: m, v fp32.  8: m int8 and v uint8 codes with one fp32 scale for every LSGD_ADAMW_BLOCK elements of a
 * row (the last block may be shorter): m = sign(q) q^2 m_scale, v = (q^2 v_scale)^2; all zeros is the state before the
 * first step.  Which of the two codes around a value is stored follows from a threshold that the step number sets, so
 * that slow changes are kept on average; scales are the block's largest value's, and a block whose largest is below about
 * 2^-100 q_max^2 is held as zeros.  A moment that is not finite is held as the block's largest finite one.            */
#define LSGD_ADAMW_BLOCK 256
typedef struct {
    float* x;                     /* device [rows, n], updated                                         */
    const void* g;                /* device [rows, n], fp32 or bf16 (the same for all tensors)         */
    void *m, *v;                  /* device [rows, n] moments, updated                                 */
    float *m_scale, *v_scale;     /* device [rows, ceil(n / LSGD_ADAMW_BLOCK)]; 8 bits only            */
    float *m_values, *v_values;   /* device [rows, n], where lsgd_adamw_moments writes; NULL: nowhere  */
    uint16_t* x_bf16;             /* device [rows, n], kept equal to bf16(x); NULL: none               */
    int64_t rows, n;
    int64_t ld_x, ld_g, ld_state, ld_scale, ld_values, ld_bf16; /* row strides (ld_state: m and v)     */
    double weight_decay, lr_mult;
} lsgd_adamw_tensor;
typedef struct lsgd_adamw lsgd_adamw; /* opaque host object */

/* Bytes of the tables a handle keeps in its workspace; 0 on invalid arguments. */
size_t lsgd_adamw_workspace_bytes(const lsgd_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, int32_t g_is_bf16);
/* Binds caller-owned buffers into a handle; workspace is device memory, 256-byte aligned, owned by the caller for the
 * life of the handle.  Copies the tables there and synchronises the stream, which later calls use until
 * lsgd_adamw_set_stream names another.                                                                            */
lsgd_status lsgd_adamw_create(const lsgd_adamw_tensor* tensors, int32_t n_tensors, int32_t state_bits, int32_t g_is_bf16, void* workspace,
                              size_t workspace_bytes, void* hip_stream, lsgd_adamw** out);
lsgd_status lsgd_adamw_destroy(lsgd_adamw* opt); /* frees the host object only */
/* Later calls run on this stream; the caller orders it behind what earlier ones left on another. */
lsgd_status lsgd_adamw_set_stream(lsgd_adamw* opt, void* hip_stream);
/* step counts from 1; grad_scale is the c above.  All are values of this call: a captured call repeats them. */
lsgd_status lsgd_adamw_step(lsgd_adamw* opt, double lr, double beta1, double beta2, double eps, int64_t step, double grad_scale);
/* 8 bits: writes what the stored codes stand for to m_values and v_values of the tensors that have them. */
lsgd_status lsgd_adamw_moments(lsgd_adamw* opt);

/* Message for the last failing call on this thread ("" if none).  Static storage. */
const char* lsgd_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LSGD_H */
