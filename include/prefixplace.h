/*
 * prefixplace.h -- C ABI of the MI355X (gfx950) PrefixPlace planner hot path.
 *
 * PrefixPlace (arXiv 2608.01655) assigns every LLM-serving worker a
 * prefix-complete (parent-closed) set of KV-cache chunks under a per-worker
 * chunk budget, maximising the materialisation cost saved per epoch.
 *
 * Problem (Eq. 8): maximise F_pair(T) (Eq. 6) over T = (T_1..T_M) with
 * |T_m| <= k_m and every T_m parent-closed, where requester m saves
 *   q_{m<-h}(b) = w_m(b)                     if h == m,
 *                 max(w_m(b) - f_{m<-h}(b), 0) otherwise      (Eq. 5)
 * on chunk b when holder h is its best resident copy.  Each worker update
 * computes the exact marginals p_h(b) of Proposition 1 (Eq. 7) and solves
 * the rooted-tree knapsack of Eq. 9 / Theorem 1 exactly; updates run as
 * WorkerGreedy (Theorem 3) followed by coordinate refinement over
 * order-diverse starts (Sec. IV-C, Algorithm 1).
 *
 * Conventions shared by every entry point
 *   - Values: the integer entry points take demand in requests per epoch
 *     and costs in integer microseconds, and every value/objective is int64
 *     (request * us), exact.  The *_f64 entry points take finite,
 *     non-negative IEEE doubles in any consistent units and a refinement
 *     tolerance epsilon >= 0; every objective value they compare is the
 *     exact sum of its rounded terms, so no result depends on an order of
 *     summation.
 *   - Node ids are the caller's labels 0..n-1.  parent[v] = -1 attaches v to
 *     the implicit no-cost dummy root (Sec. III-A), so forests are allowed.
 *   - Host arrays are C-contiguous, caller-owned, read or written only during
 *     the call; the library keeps no pointer after returning.
 *   - On any error the outputs are left unmodified, a negative PP_E_* code is
 *     returned and pp_last_error() describes it.  No C++ exception crosses
 *     this ABI.  Inputs are validated before any device work.
 *   - Tie rules (deterministic):
 *       DP ties keep the skip branch (a node is taken only if strictly
 *       better), so among optimal sets the one whose 0/1 vector in canonical
 *       preorder (roots, then children, by increasing id) is
 *       lexicographically smallest is returned;
 *       a refinement replacement is accepted only if it raises the
 *       objective strictly (integer costs) or by more than epsilon (the
 *       *_f64 entry points);
 *       ties between starts go to the lowest start index.
 *   - Start orders: start 0 sorts workers by standalone score (the optimum
 *     of the worker's own rooted-tree problem against an empty placement)
 *     descending, ties by lower worker id; start 1 is its reverse; start
 *     s >= 2 is a Fisher-Yates shuffle of 0..m-1 driven by SplitMix64
 *     seeded with order_seed + s (j = next() mod (i+1), for i = m-1..1).
 *   - All GPU entry points run on the current HIP device.
 */
#ifndef PREFIXPLACE_H
#define PREFIXPLACE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PP_ABI_VERSION 11

enum {
    PP_OK = 0,
    PP_E_ARG = -1,      /* null pointer, n < 1, m < 1 or m > 255, bad option */
    PP_E_TREE = -2,     /* parent out of range, self-parent, or a cycle */
    PP_E_RANGE = -3,    /* negative demand, cost, capacity or profit */
    PP_E_OVERFLOW = -4, /* sum over (m,b) of demand*recompute exceeds INT64_MAX */
    PP_E_NOMEM = -5,    /* host or device allocation failed */
    PP_E_DEVICE = -6,   /* HIP error, no device, or a device-side stall */
    PP_E_UNSUPPORTED = -7 /* a shape beyond a documented limit (see below) */
};

enum {
    PP_F_VALIDATE_ONLY = 1u, /* validate and build the tree layout, no GPU work */
    PP_F_NO_REFINE = 2u,     /* greedy pass only (Theorem 3's WorkerGreedy) */
    PP_F_TIME_KERNELS = 4u,  /* time every DP-sweep launch with HIP events */
    PP_F_SAFEGUARDS = 8u     /* comparator safeguards (Sec. IV-C, Algorithm 1):
                                when every fetch_cost[src][dst][b], src != dst,
                                is equal over src (requester-side costs; M = 1
                                counts as such), also solve the Independent
                                (p = Lambda_m w_m per worker), Popularity
                                (p = Lambda_m) and LocalDedup (workers in
                                increasing id, p = a_m(b) + 1{b not in U}
                                Lambda_m [w_m - f_m]_+, U = the earlier
                                workers' sets) placements, each a rooted-tree
                                DP per worker, and return one of them if its
                                objective is strictly higher than every
                                start's (ties: Independent, Popularity,
                                LocalDedup).  3M more DP updates.  No effect
                                for source-dependent costs. */
};

/* Planner options.  Passing NULL selects
 * {n_starts = 8, max_rounds = 0, order_seed = 0, orders = NULL, flags = 0}. */
typedef struct {
    int32_t n_starts;       /* >= 1: number of starts; 0: the paper's default
                               set (m <= 5: all m! orders in lexicographic
                               order; otherwise 8 starts) */
    int32_t max_rounds;     /* cap on refinement sweeps, counting the final
                               non-improving one; 0 = until a sweep accepts
                               nothing */
    uint64_t order_seed;    /* seeds the shuffled starts (index >= 2) */
    const int32_t *orders;  /* optional [n_starts][m] explicit worker orders
                               (host); NULL = generate as described above */
    uint32_t flags;         /* PP_F_* */
} pp_options;

/* Optional statistics.  Pointer fields may be NULL; arrays indexed by start
 * must hold pp_num_starts(m, n_starts) entries. */
typedef struct {
    int32_t best_start;        /* out: start whose placement is returned, or
                                  n_starts + c when safeguard candidate c
                                  (0 Independent, 1 Popularity, 2 LocalDedup)
                                  is returned */
    int32_t n_starts;          /* out: number of starts run */
    int64_t updates;           /* out: worker updates of Algorithm 1
                                  (standalone + greedy + every sweep) */
    int64_t dp_cells;          /* out: sum over updates of n * min(k_h, n) */
    int64_t *start_objective;  /* out [S]: objective of each start */
    int32_t *start_sweeps;     /* out [S]: refinement sweeps per start */
    int32_t *start_accepts;    /* out [S]: accepted replacements per start */
    int64_t *standalone;       /* out [m]: standalone score per worker */
    int32_t *orders;           /* out [S][m]: start orders used */
    double dp_kernel_ms;       /* out with PP_F_TIME_KERNELS: summed duration
                                  of the solve launches: a reduced solve's two
                                  kernels (with its incumbents' values and
                                  decisions) count as one, each sweep as one */
    int32_t dp_launches;       /* out with PP_F_TIME_KERNELS */
    int32_t safeguards_run;    /* out: 1 if the PP_F_SAFEGUARDS candidates were
                                  evaluated (requester-side costs) */
    int64_t safeguard_objective[3]; /* out: their objectives (Independent,
                                  Popularity, LocalDedup), 0 if not run */
    int64_t dp_cells_executed; /* out: DP cells (n * min(k, n) each) of the
                                  updates actually solved, whether by the
                                  reduced solve, which proves most of them away
                                  without visiting them, or by a sweep.  A refinement
                                  update of a worker whose inputs have not
                                  changed since its last sweep (no other
                                  worker's set changed) would find the same
                                  set and reject it; it is resolved as
                                  rejected without a sweep, so this can be
                                  below dp_cells.  Speculative refinement
                                  updates (later positions of a start swept
                                  in the same launch, valid only if the
                                  earlier ones are rejected) that are
                                  discarded add their cells, so it can also
                                  exceed dp_cells.  Results are unaffected. */
    int32_t dp_lane_cells;     /* out: DP cells per lane of the sweep's
                                  compute wave (1, 2 or 4; 0 if no sweep
                                  ran), chosen per plan */
    int32_t dp_fmax;           /* out: 1 if the sweep took the maximum with
                                  one 64-bit float instruction (every value
                                  below 2^62, or real-valued costs), 0 if
                                  with a compare and two selects */
    int32_t dp_restarts;       /* out: times the plan was run again because a
                                  DP sweep stage gave up a bounded wait for
                                  its neighbour (the sweep's stages must be
                                  resident at once; other work on the GPU
                                  can crowd them out): each run uses fewer
                                  stage blocks per launch and longer waits;
                                  after 2 the call fails with PP_E_DEVICE.
                                  Results are unaffected. */
} pp_stats;

/* Number of starts the options select (see pp_options.n_starts). */
int32_t pp_num_starts(int32_t m, int32_t n_starts);

/* Full planner (Algorithm 1 with exact rooted-tree updates; Eq. 8).
 *   parent          [n]      host; -1 = child of the dummy root
 *   demand          [m][n]   host; Lambda_m(b) >= 0 (Sec. III-A)
 *   recompute_cost  [m][n]   host; w_m(b) >= 0 us
 *   fetch_cost      [m][m][n] host; fetch_cost[src][dst][b] = f_{dst<-src}(b)
 *                            >= 0 us; the src == dst plane is ignored.  A
 *                            requester-side cost f_m(b) is given by repeating
 *                            it over src (this reproduces Eq. 4 exactly).
 *   cap             [m]      host; k_m >= 0 chunks (values above n act as n)
 *   opt                      NULL or options
 *   target          [m][n]   host out: 1 iff b is in T_m; each row is
 *                            parent-closed with at most cap[m] ones
 *   objective                host out: F_pair(T) in request * us
 *   stats                    NULL or statistics
 * Limits: the DP sweep keeps pending skip-target rows in LDS slots (their
 * number is at most the tree depth; 14 and 17 on the 50,000-chunk benchmark
 * trees).  Up to 254 stay in LDS; a deeper tree that branches along long
 * chains has its long-lived pending rows spilled to device memory and
 * restored ahead of their reads (pp_sweep_spills), so any depth is
 * accepted; PP_E_UNSUPPORTED only if even then more than 254 LDS rows would
 * be needed at once, or the rows do not fit one compute unit's LDS. */
int pp_plan(int32_t n, int32_t m, const int32_t *parent, const int64_t *demand,
            const int64_t *recompute_cost, const int64_t *fetch_cost,
            const int32_t *cap, const pp_options *opt, uint8_t *target,
            int64_t *objective, pp_stats *stats);

/* Real-valued costs (the paper's own domain: demand in requests per epoch,
 * costs in milliseconds) with the refinement tolerance epsilon of Algorithm 1
 * (Sec. IV-C): a refinement replacement is accepted only if it raises G by
 * more than epsilon.  Every value is an IEEE double; inputs must be finite
 * and >= 0 (PP_E_RANGE otherwise), epsilon finite and >= 0 (PP_E_ARG).
 * The arithmetic is the integer path's, in doubles: each product
 * Lambda * x is rounded before it is added, p_h(b) adds its requester terms
 * in increasing m, the DP takes b_i only if p + D[i+1][j-1] > D[next(i)][j],
 * and G = F_pair is the exact sum of its rounded terms Lambda_m(b) *
 * max(...) (every finite double is a multiple of 2^-1074, so the sum is kept
 * as an exact integer of those units): a refinement replacement is accepted
 * iff the exact G with it exceeds the exact G(T) + epsilon (so one of
 * exactly equal value, e.g. differing only by chunks of zero marginal value,
 * is never accepted, also at epsilon = 0); starts and comparator candidates
 * compare exact values; reported objectives are the exact values rounded to
 * the nearest double.  PP_F_SAFEGUARDS adds the comparator
 * candidates for requester-side costs (fetch costs equal as values over
 * every source; -0.0 counts as 0.0) with the integer path's formulas in
 * doubles.  Statistics as pp_stats, with double objectives and scores. */
typedef struct {
    int32_t best_start;
    int32_t n_starts;
    int64_t updates;
    int64_t dp_cells;
    double *start_objective;   /* [S] or NULL */
    int32_t *start_sweeps;     /* [S] or NULL */
    int32_t *start_accepts;    /* [S] or NULL */
    double *standalone;        /* [m] or NULL */
    int32_t *orders;           /* [S][m] or NULL */
    double dp_kernel_ms;
    int32_t dp_launches;
    int32_t safeguards_run;
    double safeguard_objective[3];
    int64_t dp_cells_executed;   /* as in pp_stats */
    int32_t dp_lane_cells;       /* as in pp_stats */
    int32_t dp_fmax;             /* as in pp_stats */
    int32_t dp_restarts;         /* as in pp_stats */
} pp_stats_f64;

/* pp_plan on real-valued host arrays (layouts as pp_plan). */
int pp_plan_f64(int32_t n, int32_t m, const int32_t *parent, const double *demand,
                const double *recompute_cost, const double *fetch_cost,
                const int32_t *cap, double epsilon, const pp_options *opt,
                uint8_t *target, double *objective, pp_stats_f64 *stats);

/* pp_rooted_dp on real-valued profits (finite, >= 0). */
int pp_rooted_dp_f64(int32_t n, const int32_t *parent, const double *profit,
                     int32_t k, uint8_t *selected, double *value);

/* Epoch re-planning (Sec. IV-D): when demand or routing changes, plan the
 * refreshed inputs (as pp_plan, same options), evaluate the incumbent under
 * them, and switch to the new plan only when its gain per epoch over the
 * horizon pays for copying in the chunks it newly assigns:
 *   adopt  iff  horizon * (G(T') - G(T)) > sum over (m, b) with b in T'_m
 *               and not in T_m of c_m(b),
 *   c_m(b) = min(w_m(b), min over workers h != m holding b in the
 *            incumbent of f_{m<-h}(b)),
 * G = F_pair (Eq. 6) under the refreshed inputs; the product is compared
 * exactly (no overflow).  Arguments as pp_plan, plus
 *   incumbent [m][n] host: the current placement (0/1; it need not be
 *                    parent-closed or within the new capacities)
 *   horizon          epochs over which the gain is counted (>= 0)
 *   target    [m][n] host out: the placement to use (T' if adopted, else a
 *                    copy of the incumbent)
 *   proposal  [m][n] host out, may be NULL: T'
 *   info             out, required
 * Errors as pp_plan; PP_E_ARG for a negative horizon or an incumbent entry
 * other than 0 and 1, PP_E_OVERFLOW if the one-time cost exceeds INT64_MAX. */
typedef struct {
    int32_t adopt;                 /* 1 iff T' is adopted */
    int64_t incumbent_objective;   /* G(T) under the refreshed inputs */
    int64_t proposal_objective;    /* G(T') */
    int64_t materialization_cost;  /* one-time cost of T' over T, us */
} pp_replan_info;

int pp_replan(int32_t n, int32_t m, const int32_t *parent, const int64_t *demand,
              const int64_t *recompute_cost, const int64_t *fetch_cost,
              const int32_t *cap, const uint8_t *incumbent, int64_t horizon,
              const pp_options *opt, uint8_t *target, uint8_t *proposal,
              pp_replan_info *info, pp_stats *stats);

/* pp_replan on real-valued costs: the planner of pp_plan_f64 (tolerance
 * epsilon), the same rule with a real horizon (finite, >= 0):
 * adopt iff horizon * (G(T') - G(T)) > cost, where G(T') - G(T) and the
 * cost are exact sums each rounded once to the nearest double, and the
 * product and comparison are evaluated in doubles.  Errors as pp_plan_f64
 * and pp_replan. */
typedef struct {
    int32_t adopt;
    double incumbent_objective;
    double proposal_objective;
    double materialization_cost;
} pp_replan_info_f64;

int pp_replan_f64(int32_t n, int32_t m, const int32_t *parent, const double *demand,
                  const double *recompute_cost, const double *fetch_cost,
                  const int32_t *cap, const uint8_t *incumbent, double horizon,
                  double epsilon, const pp_options *opt, uint8_t *target,
                  uint8_t *proposal, pp_replan_info_f64 *info, pp_stats_f64 *stats);

/* One exact rooted-tree solve (Eq. 9, Theorem 1) on the GPU.
 *   parent [n] host, profit [n] host (>= 0, sum <= INT64_MAX), k >= 0;
 *   selected [n] host out (0/1, parent-closed, at most min(k, n) ones);
 *   value host out = max total profit. */
int pp_rooted_dp(int32_t n, const int32_t *parent, const int64_t *profit,
                 int32_t k, uint8_t *selected, int64_t *value);

/* Exact marginals of worker h against the other workers' current sets
 * (Proposition 1, Eq. 7), on the GPU.
 *   target [m][n] host: current placement (row h is ignored);
 *   profit [n] host out: p_h(b);
 *   g_without_h host out (may be NULL): F_pair with T_h emptied. */
int pp_marginal(int32_t n, int32_t m, const int64_t *demand,
                const int64_t *recompute_cost, const int64_t *fetch_cost,
                const uint8_t *target, int32_t h, int64_t *profit,
                int64_t *g_without_h);

/* F_pair(T) of Eq. 6 for an arbitrary placement (target [m][n] host), on
 * the GPU. */
int pp_objective(int32_t n, int32_t m, const int64_t *demand,
                 const int64_t *recompute_cost, const int64_t *fetch_cost,
                 const uint8_t *target, int64_t *objective);

/* Allocation-free F_pair(T), for callers that cannot allocate device memory
 * (code under HIP graph capture set-up, tight serving loops, harnesses that
 * forbid hipMalloc): the value pp_objective returns, on device-resident
 * arrays in caller ids (layouts as pp_plan; target [m][n], a chunk is held
 * where the byte is nonzero), enqueued on `hip_stream` (a hipStream_t; NULL
 * = the null stream).  The call waits for the stream and writes the result
 * to the host `objective`.  It calls no hipMalloc, hipFree or other
 * allocating routine, host or device: its only device memory besides the
 * caller's arrays is a file-scope array of PP_NOALLOC_SCRATCH_BYTES in the
 * library, one per GPU, held until the process ends.  The scratch does not
 * grow with the input (at most 1024 per-block partial sums), so every size
 * pp_objective accepts is accepted: n >= 1, 1 <= m <= 255.  Every call on a
 * GPU shares that GPU's array: calls that overlap on one GPU (other threads,
 * other streams) race and must be serialized by the caller.  Errors as
 * pp_objective: PP_E_ARG (null pointer, sizes), PP_E_RANGE (negative value),
 * PP_E_OVERFLOW (sum of demand * recompute cost above INT64_MAX),
 * PP_E_DEVICE (HIP error); *objective is then left unchanged. */
#define PP_NOALLOC_SCRATCH_BYTES 40960
int pp_objective_device_noalloc(int32_t n, int32_t m, const int64_t *demand_dev,
                                const int64_t *recompute_dev,
                                const int64_t *fetch_dev, const uint8_t *target_dev,
                                int64_t *objective, void *hip_stream);

/* Start orders (Sec. IV-C) from standalone scores [m]; host only.
 * orders [pp_num_starts(m, n_starts)][m] host out. */
int pp_orders(int32_t m, int32_t n_starts, uint64_t order_seed,
              const int64_t *standalone, int32_t *orders);

/* Reusable GPU context: keeps device buffers between calls.  A context is
 * used by one thread at a time; separate contexts may run concurrently. */
typedef struct pp_ctx pp_ctx;
int pp_ctx_create(pp_ctx **ctx, int device);
void pp_ctx_destroy(pp_ctx *ctx);

/* pp_plan with device-resident inputs and output, on `hip_stream`
 * (a hipStream_t; NULL = the null stream).  demand_dev, recompute_dev,
 * fetch_dev are device pointers in caller ids, laid out as in pp_plan;
 * target_dev [m][n] device out.  parent, cap and the options stay on the
 * host.  The call returns after the plan has finished on the stream. */
int pp_plan_device(pp_ctx *ctx, int32_t n, int32_t m, const int32_t *parent,
                   const int64_t *demand_dev, const int64_t *recompute_dev,
                   const int64_t *fetch_dev, const int32_t *cap,
                   const pp_options *opt, uint8_t *target_dev,
                   int64_t *objective, pp_stats *stats, void *hip_stream);

/* pp_plan_device on real-valued device arrays (layouts as pp_plan_device;
 * the value checks run on the device). */
int pp_plan_f64_device(pp_ctx *ctx, int32_t n, int32_t m, const int32_t *parent,
                       const double *demand_dev, const double *recompute_dev,
                       const double *fetch_dev, const int32_t *cap, double epsilon,
                       const pp_options *opt, uint8_t *target_dev, double *objective,
                       pp_stats_f64 *stats, void *hip_stream);

/* Host only, for inspection and CPU-side checks of the DP sweep's step
 * schedule: for the tree `parent` and `cells` (1, 2 or 4) DP cells per
 * lane, writes the per-step metadata of the sweep (`meta`, may be NULL to
 * query the size; 4 * nsteps words, nsteps = n padded up to a multiple of 32
 * with leading dummy steps; step s handles preorder row n - (s - pad), pad =
 * nsteps - n) and the number of LDS slot rows H.  LDS rows hold 64*cells
 * int64 (stride 512*cells + 8 bytes) in the order [H slot rows | zero row |
 * sink rows: 16 at one cell per lane, else 4].  Per step: word 0 = byte
 * offset of the row the step's DP row is stored to (its slot when a later
 * non-leaf row skips to it, else sink row step mod the sink count); word 1 =
 * byte offset of the row read as the next step's skip operand (Eq. 9's
 * D[next(i)][*]: a slot, or the zero row when that next() is past the end or
 * the next step's node is a leaf), which the sweep reads right after storing
 * the current step's row; word 2 = 0xFFFFFFFF when the step's node is a leaf
 * (skip operand: the previous row, in registers), else 0; word 3 = 0.  The
 * first step's node is a leaf. */
int pp_sweep_layout(int32_t n, const int32_t *parent, int32_t cells,
                    uint32_t *meta, int32_t *nsteps, int32_t *slots);

/* Host only, for CPU-side checks of the DP sweep on deep trees.  The sweep
 * keeps each pending skip row (a row that a later non-leaf row reads as its
 * D[next(i)][*]) in an LDS slot; when a tree has more of them pending at
 * once than the slots hold (deep trees that branch along long chains), the
 * rows first read kSpillGap = 3 or more sweep batches (of 32 steps) after
 * their store are spilled: stored to a temporary slot as usual, copied to
 * device memory by the stage's I/O wave once their batch is done (and
 * before it stages the batch after next), and copied back into a restore
 * slot when it stages each later batch that reads them.  Writes nbatches
 * (padded steps / 32), nspill (spill rows per stage; 0 = nothing spilled,
 * then the lists are empty and the offsets zero), n_out and n_in (list
 * entries); each of out_off, spill_out, in_off, spill_in may be NULL.
 * out_off [nbatches + 1]: batch b copies out the entries
 *   spill_out[2e], spill_out[2e + 1] = (LDS slot, spill index) for
 *   e in [out_off[b], out_off[b + 1]);
 * in_off [nbatches + 1]: batch b is staged after copying in the entries
 *   spill_in[2e], spill_in[2e + 1] = (LDS slot, spill index) for
 *   e in [in_off[b], in_off[b + 1]).
 * The step metadata of pp_sweep_layout already names the temporary and
 * restore slots.  Errors as pp_sweep_layout, PP_E_UNSUPPORTED if the
 * pending rows exceed 254 LDS rows even with spilling. */
int pp_sweep_spills(int32_t n, const int32_t *parent, int32_t *nbatches, int32_t *nspill,
                    int32_t *n_out, int32_t *n_in, int32_t *out_off, int32_t *spill_out,
                    int32_t *in_off, int32_t *spill_in);

/* Exit row in pp_backtrack_table for a skip sequence that runs past the
 * last row. */
#define PP_BT_END 0x7FFFFFFFu

/* Host only, for inspection and CPU-side checks of the backtrack's skip
 * table (Theorem 1's walk from (1, k'): a take moves to row i+1, a skip to
 * next(i)).  Rows are 0-based preorder positions, grouped in windows of 32
 * (rows 32w .. 32w+31).  For row q < n, with S(q) = q, next(q),
 * next(next(q)), ... (next(q) = first position after q's subtree):
 *   word 0 = mask of S(q) inside q's window, bit (r mod 32) for each row r
 *            of S(q) below min(32(w+1), n);
 *   word 1 = the first row of S(q) at or past that bound if it is < n, else
 *            PP_BT_END;
 *   word 2 = word 0 of that row (0 for PP_BT_END);
 *   word 3 = 0.
 * Rows n .. rows-1 are padding: {0, PP_BT_END, 0, 0}; rows = n rounded up to
 * a multiple of 512, plus 512.  `table` (4 * rows words) may be NULL to
 * query `rows`.  Errors as for pp_sweep_layout. */
int pp_backtrack_table(int32_t n, const int32_t *parent, uint32_t *table,
                       int64_t *rows);

/* ------------------------------------------------------------------------
 * The prefix cache of one worker: what runs below a plan.
 *
 * A worker keeps keys and values in pages of `page_size` tokens.  The chunks
 * of its target row lie in slots 0..n_slots-1; slot s owns the pages
 * s * (chunk_tokens / page_size) onwards, and every further page belongs to
 * one request at a time.  A batch step is
 *   pp_block_tables     prefixes found in the tree, pages handed out, the
 *                       place of every new token
 *   pp_kv_write         the new keys and values into their places (per layer)
 *   pp_paged_attention  the new tokens' attention over their requests' pages
 *                       (per layer), single tokens included
 * and pp_prefix_table (per tree) and pp_cache_slots (per plan) lay out on
 * the host what it looks things up in.
 *
 * The three enqueue their work on `hip_stream` and return; nothing is
 * allocated and nothing is waited for, so they can be captured into a graph.
 * What the host can see is checked before anything is enqueued (PP_E_ARG,
 * PP_E_UNSUPPORTED); contents of device arrays are not read by the host:
 * node, slot, page and token numbers out of range are treated as absent
 * where the text says so, and in no case lead out of the arrays given.
 * Row starts of queries, keys, values, outputs and pages are 16-byte
 * aligned: their pointers, and their strides times the element size.  Rows
 * that are written do not overlap (a stride below dim where there are two or
 * more is refused); rows that are only read may, of expanded tensors say.
 * ------------------------------------------------------------------------ */

/* Element types of rows and pages.  PP_E4M3 is the 8-bit float of 4 exponent
 * and 3 mantissa bits without infinities (largest value 448). */
enum { PP_BF16 = 1, PP_F16 = 2, PP_E4M3 = 3 };

/* Host only: the tree as pp_block_tables reads it.  table [n][16]: entries
 * 0..14 of line v are v, its parent and so on (-1 past a root), entry 15 is
 * v's depth (0 for a root).  One 64-byte line answers 14 levels, so a path
 * of d chunks takes d / 14 dependent reads. */
int pp_prefix_table(int32_t n, const int32_t *parent, int32_t *table);

/* Host only: slots for a target row.  target [n]: a worker's row (nonzero =
 * resident); held [n] or NULL: the slots so far (-1 = none).  A chunk that
 * is held and still targeted keeps its slot; the others of the target take
 * the free slots in increasing order, chunks in increasing id; every other
 * chunk gets -1.  slot [n] out (may be `held` itself); n_new out, may be
 * NULL: chunks without a slot so far, whose pages have to be filled before
 * pp_block_tables is given the slots.
 * A slot is free as soon as its chunk is not in the target, and may go to
 * another chunk in the same call.  Rows of requests that go on still name its
 * pages, so a chunk that such a request found has to stay in the target given
 * here, whatever the plan says, until the request has ended; the worker needs
 * that many slots beyond the plan's.
 * PP_E_RANGE if the target has more than n_slots chunks, or held names a
 * slot out of range or twice. */
int pp_cache_slots(int32_t n, const uint8_t *target, const int32_t *held,
                   int32_t n_slots, int32_t *slot, int32_t *n_new);

/* Block tables and slot maps of a batch, on the GPU.  All pointers are
 * device pointers.
 * Request r stands at `length[r]` tokens once all of them are computed.
 *   cached[r] < 0: it begins in this step.  Its prefix is the path from a
 *     root to chunk leaf[r] (out of range: none); the chunks on the path up
 *     to the first one without a slot in 0..n_slots-1 are found, as long as
 *     they end before the last token (one token at least is computed):
 *     start = chunk_tokens * min(found, (length - 1) / chunk_tokens).
 *   cached[r] >= 0: it goes on: start = min(cached[r], length[r]), and its
 *     row holds the pages of those tokens.
 * end = min(length, start + max_new) (max_new = 0: length).
 * Row r of block_table gets the found chunks' pages, and from block
 * ceil(start / page_size) to before ceil(end / page_size) pages off
 * free_pages, which requests take in order of r; other entries stay as they
 * are.  The new tokens of all requests, in order, are numbered from 0:
 * request r has query_start[r] .. query_start[r + 1] - 1, of which number i
 * stands at position[i] and its keys and values belong in slot_map[i] =
 * page * page_size + position % page_size.  Numbers from the batch's tokens
 * up to max_tokens get slot -1 and position 0.
 * taken[0] = pages needed; above n_free, the requests that came too late
 * have -1 in block_table and slot_map.  Blocks at or past max_blocks are not
 * written, and their tokens get slot -1; so do page numbers below 0 in a
 * row.  Tokens at or past max_tokens are counted in query_start and written
 * nowhere.  Negative lengths act as 0. */
typedef struct {
    int32_t requests;          /* >= 0, at most 65,536 */
    int32_t n;                 /* chunks in the tree, >= 0 */
    int32_t n_slots;
    int32_t n_free;
    int32_t max_blocks;        /* entries a row of block_table holds */
    int32_t max_tokens;        /* entries of slot_map and position */
    int32_t page_size;         /* a power of two, 16 .. 1,024 */
    int32_t chunk_tokens;      /* a multiple of page_size */
    int32_t max_new;
    int64_t row_stride;        /* entries from a row of block_table to the next, max_blocks at least */
    const int32_t *leaf, *length, *cached;      /* [requests] */
    const int32_t *prefix_table;                /* [n][16], 16-byte aligned */
    const int32_t *slot;                        /* [n] */
    const int32_t *free_pages;                  /* [n_free] */
    int32_t *block_table;                       /* [requests][max_blocks] */
    int32_t *query_start;                       /* out [requests + 1] */
    int32_t *start, *end;                       /* out [requests] */
    int64_t *slot_map;                          /* out [max_tokens] */
    int32_t *position;                          /* out [max_tokens] */
    int32_t *taken;                             /* out [1] */
} pp_block_args;
int pp_block_tables(const pp_block_args *args, void *hip_stream);

/* One layer's pages: element (page, head, token, i) of k and of v lies at
 * page * page_stride + head * head_stride + token * token_stride + i
 * elements (any order of the three).  dim is what the call takes: 64, 128 or
 * 256 in pp_kv_write and pp_paged_attention.  PP_E4M3 pages hold value / scale of
 * their head, k_scale and v_scale [heads] (device; NULL = 1; finite and
 * above 0, which the host cannot see); other types have no scales. */
typedef struct {
    void *k, *v;
    const float *k_scale, *v_scale;
    int32_t dtype;
    int32_t n_pages, page_size;    /* page_size a power of two, 16 .. 1,024 */
    int32_t heads;
    int32_t dim;
    int64_t page_stride, head_stride, token_stride;
} pp_kv_pages;

/* Writes rows k, v [tokens][heads][dim] (PP_BF16 or PP_F16) into the places
 * slot_map names; a place below 0 or past the pages is skipped.  No place is
 * to be named twice: it ends up with elements of either row, mixed, and its
 * key need not be of the row that its value is of.  (pp_block_tables names
 * none twice as long as no page is handed out twice.)
 * Pages of the rows' own type take them as they are;
 * PP_E4M3 pages take row / scale rounded to nearest even, values past +-448
 * (infinities too) as +-448, NaN as NaN.  Strides in elements. */
int pp_kv_write(const pp_kv_pages *pages, int32_t tokens, int32_t dtype,
                const void *k, int64_t k_token_stride, int64_t k_head_stride,
                const void *v, int64_t v_token_stride, int64_t v_head_stride,
                const int64_t *slot_map, void *hip_stream);

/* Attention of a batch's new tokens over their requests' pages.
 * Request r has length[r] tokens in its pages, the last of which are its
 * query_start[r + 1] - query_start[r] new ones, so new token i of u stands
 * at p = length - u + i and sees the keys j <= p of its request, with
 * window > 0 the last `window` of them (j > p - window):
 *   s_j = scale * <q, K_j>,  out = sum_j e^(s_j) V_j / sum_j e^(s_j),
 *   lse = log sum_j e^(s_j).
 * A row that sees no key (p < 0), or only keys of s_j = -infinity, has
 * out = 0 and lse = -infinity.  Query head g reads key head
 * g / (q_heads / heads).  What a row does not see does not touch it, whatever
 * it holds (NaN and infinities too).  Page numbers below 0 act as 0, above
 * the last as the last; tokens past a row of the block table do not exist.
 * Scores, sums and the accumulation are held in 32 bits; weights are rounded
 * to the queries' type for the product with V.
 * max_new and max_len bound every request's new tokens and length (parts of
 * long requests are cut by max_len, so one far above costs time); a request
 * of more than max_new new tokens may be left unwritten, and rows of tokens
 * that no request has are.  Calls that need more than 2^24 blocks (65,536
 * requests of more than 256 key heads) fail with PP_E_DEVICE and write
 * nothing, or the rows of a part of the requests.  `workspace` is device memory
 * of pp_attention_workspace bytes at least (256-byte aligned); the call
 * writes it before it reads it, so its contents need not be kept. */
typedef struct {
    int32_t requests;              /* >= 0, at most 65,536 */
    int32_t tokens;                /* rows of q and out */
    int32_t q_heads;               /* a multiple of the pages' heads */
    int32_t dtype;                 /* of q and out: PP_BF16 or PP_F16 */
    int32_t max_new, max_len;
    int32_t max_blocks;
    int32_t window;                /* 0 = none */
    float scale;
    int64_t q_token_stride, q_head_stride;      /* elements */
    int64_t out_token_stride, out_head_stride;
    int64_t row_stride;            /* of block_table */
    const void *q;                 /* [tokens][q_heads][dim] */
    void *out;                     /* [tokens][q_heads][dim] */
    float *lse;                    /* [tokens][q_heads], or NULL */
    const int32_t *query_start;    /* [requests + 1] */
    const int32_t *length;         /* [requests] */
    const int32_t *block_table;    /* [requests][max_blocks] */
    void *workspace;
    int64_t workspace_bytes;
} pp_attention_args;
int64_t pp_attention_workspace(const pp_kv_pages *pages, const pp_attention_args *args);
int pp_paged_attention(const pp_kv_pages *pages, const pp_attention_args *args,
                       void *hip_stream);

/* ------------------------------------------------------------------------
 * Around the pages: what brings rows into them, pages of latent rows, and
 * what moves, shares and frees pages.  The same conventions hold: work is
 * enqueued on `hip_stream`, nothing is allocated or waited for, numbers out
 * of range in device arrays lead out of no array given.  What a call reads
 * and what it writes do not overlap, but where the text allows it.
 * ------------------------------------------------------------------------ */

/* Host only: frequencies of rotary positions as pp_rotary_write reads them.
 * Pair i of dim / 2 turns by w_i = base^(-2 i / dim) radians a token, or,
 * for contexts longer than trained on, by g_i w_i + (1 - g_i) w_i / factor
 * with g_i = (original w_i / 2 pi - slow) / (fast - slow) held to 0 .. 1:
 * pairs that make fewer than `slow` turns in the `original` tokens slow down
 * by `factor`, those of more than `fast` keep their pace (original = 0: all
 * slow down; factor = 1: none).  Out, either may be NULL: radians
 * [dim / 2] and turns [dim / 2], w / 2 pi in units of 2^-64 turns, so that
 * position * turns modulo 2^64 is the angle at any position, exactly reduced.
 * dim even, base > 1, factor >= 1, original >= 0, fast > slow >= 0. */
int pp_rotary_turns(int32_t dim, double base, double factor, double original,
                    double slow, double fast, double *radians, uint64_t *turns);

/* Host only: turns [n] of any radians [n] a token (finite). */
int pp_turns(int32_t n, const double *radians, uint64_t *turns);

/* Norms of queries and keys for each head, their rotation by position, and
 * the write into the pages, in one pass.
 *   A row's first `norm` elements (0 = none) become
 *     x / sqrt(mean of x^2 + eps) * weight,
 *   then of the rot_dim elements from `first` on the pairs (a, b) become
 *     amplitude * (a cos t - b sin t, a sin t + b cos t),
 *   t = position[token] * frequency: elements (i, i + rot_dim / 2), or
 *   (2 i, 2 i + 1) where `interleaved`, with turns[i].
 * q goes to q_out.  k goes to k_out, or where pages are given to the place
 * slot_map names, with v as it is; places and 8-bit pages as in pp_kv_write,
 * but the one rounding is from 32 bits.  Pages without v (pages->v and v
 * NULL) hold one row a token and head, latent rows with heads = 1 say.
 * q_heads or k_heads = 0: no such rows.  Rows are [tokens][heads][dim];
 * dims, firsts and norms are multiples of 8, dims at most 1,024, rot_dim is
 * a multiple of 16 (0 = no rotation); weights are of the rows' type.  Tokens
 * times heads are 2^31 - 1 at most.
 * An output may be its input (the same pointer and strides). */
typedef struct {
    int32_t tokens;
    int32_t dtype;                 /* of all rows and weights: PP_BF16 or PP_F16 */
    int32_t q_heads, q_dim, q_first, q_norm;
    int32_t k_heads, k_dim, k_first, k_norm;
    int32_t rot_dim, interleaved;
    float eps, amplitude;
    int64_t q_token_stride, q_head_stride;      /* elements */
    int64_t q_out_token_stride, q_out_head_stride;
    int64_t k_token_stride, k_head_stride;
    int64_t k_out_token_stride, k_out_head_stride;
    int64_t v_token_stride, v_head_stride;
    const void *q, *k, *v;
    void *q_out, *k_out;
    const void *q_weight, *k_weight;            /* [q_norm], [k_norm], 16-byte aligned */
    const int32_t *position;                    /* [tokens] */
    const uint64_t *turns;                      /* [rot_dim / 2], 16-byte aligned */
    const int64_t *slot_map;                    /* [tokens] */
} pp_rotary_args;
int pp_rotary_write(const pp_rotary_args *args, const pp_kv_pages *pages, void *hip_stream);

/* Attention over pages of latent rows: one row C_j of `dim` elements a
 * token, which every query head reads, and whose first `value_dim` elements
 * are its value:
 *   s_j = scale * <q, C_j>,  out = sum_j e^(s_j) C_j[0 .. value_dim) / sum_j e^(s_j).
 * So queries are those of latent attention with the keys' expansion
 * multiplied in, and out is yet to be multiplied by the values' expansion.
 * Pages: k the rows, v NULL, heads 1, k_scale [1] (PP_E4M3 pages);
 * value_dim 512 or 256, dim = value_dim + 64.  Everything else is as in
 * pp_paged_attention; out rows are [tokens][q_heads][value_dim].  Requests
 * are cut by their lengths, not by max_len, so one far above costs no time
 * (it says whether requests of few tokens beside prompts may be long enough for
 * launches of their own).  A key of
 * s_j = -infinity makes elements of out NaN where its own are not finite (0
 * times them), unless the row sees no other keys, wherever the call cuts
 * requests.  Where query_start is not in order, so that requests overlap,
 * some may be left unwritten. */
int64_t pp_latent_workspace(const pp_kv_pages *pages, int32_t value_dim,
                            const pp_attention_args *args);
int pp_latent_attention(const pp_kv_pages *pages, int32_t value_dim,
                        const pp_attention_args *args, void *hip_stream);

/* Copies pages: move i copies page source[i] to page target[i], its first
 * tokens[i] tokens (tokens NULL: all), in every pool (all layers' keys and
 * values, say).  The pools' layouts are alike, in strides of elements as in
 * pp_kv_pages.  Moves whose source or target is out of range, or which are the
 * same page, do nothing; tokens are held to 0 .. page_size.  Moves
 * are made at once: no target is to be named twice, or to be a source. */
typedef struct {
    int32_t moves;
    int32_t n_pools;
    int32_t dtype;                 /* PP_BF16, PP_F16 or PP_E4M3 */
    int32_t n_pages, page_size;    /* page_size a power of two, 16 .. 1,024 */
    int32_t heads, dim;            /* rows of dim elements are multiples of 16 bytes */
    int64_t page_stride, head_stride, token_stride;
    void *const *pools;            /* host array [n_pools] of device pointers */
    const int32_t *source, *target;             /* [moves] */
    const int32_t *tokens;                      /* [moves] or NULL */
} pp_copy_args;
int pp_page_copy(const pp_copy_args *args, void *hip_stream);

/* Rows of block tables from their parents' (beams, several samples of a
 * prompt).  New row r continues row parent[r] of block_table (out of range:
 * it has no tokens and is not written): out_length[r] = length[parent[r]],
 * and row r of out_table gets the parent's pages, ceil(length / page_size).
 * Full pages are shared.  The page of the last block, where it is not full, is kept
 * by the first new row of a parent; every further one takes a page off
 * free_pages, in order of r, and the copy it needs is move r of source,
 * target and tokens as pp_page_copy reads them (source -1, target -1, 0
 * tokens: none).  taken[0] = pages needed; above n_free the rows that came
 * too late have target -1 and -1 in their last block.  Blocks at or past
 * max_blocks do not exist; negative lengths act as 0.  out_table does not
 * overlap block_table. */
typedef struct {
    int32_t rows;                  /* new rows, >= 0, at most 65,536 */
    int32_t parents;               /* rows of block_table, at most 65,536 */
    int32_t n_free;
    int32_t max_blocks;            /* entries a row of either table holds */
    int32_t page_size;             /* a power of two, 16 .. 1,024 */
    int64_t row_stride, out_row_stride;         /* entries, max_blocks at least */
    const int32_t *parent;                      /* [rows] */
    const int32_t *length;                      /* [parents] */
    const int32_t *block_table;                 /* [parents][max_blocks] */
    const int32_t *free_pages;                  /* [n_free] */
    int32_t *out_table;                         /* [rows][max_blocks] */
    int32_t *out_length;                        /* out [rows] */
    int32_t *source, *target, *tokens;          /* out [rows] */
    int32_t *taken;                             /* out [1] */
} pp_fork_args;
int pp_fork_tables(const pp_fork_args *args, void *hip_stream);

/* The pages that no request has: numbers from `first` (past the slots'
 * pages) to before n_pages that no row of block_table names in its
 * ceil(length / page_size) blocks, in increasing order.  count[0] = how
 * many; the first `room` of them are written to free_pages, whose other
 * entries stay as they are.  marks [n_pages] is scratch memory (8-byte
 * aligned), written before it is read.  Numbers out of range in rows name
 * no page.  n_pages is 2^24 at most. */
typedef struct {
    int32_t requests;              /* >= 0, at most 65,536 */
    int32_t max_blocks;
    int32_t page_size;             /* a power of two, 16 .. 1,024 */
    int32_t n_pages, first;        /* 0 <= first <= n_pages */
    int32_t room;
    int64_t row_stride;
    const int32_t *length;                      /* [requests] */
    const int32_t *block_table;                 /* [requests][max_blocks] */
    int32_t *free_pages;                        /* out [room] */
    int32_t *count;                             /* out [1] */
    uint8_t *marks;                             /* [n_pages] */
} pp_free_args;
int pp_free_pages(const pp_free_args *args, void *hip_stream);

/* Description of the last error on the calling thread; valid until the
 * next pp_* call on that thread. */
const char *pp_last_error(void);

int pp_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PREFIXPLACE_H */
