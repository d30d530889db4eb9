/*
 * harp.h - C ABI of the MI355X planner-search library.
 *
 * The library evaluates, on one GPU, a batch of candidate pipeline layouts for the inter-operator
 * planner of HARP (paper section 5.2).  A planning problem is an ordered sequence of L operators
 * with profiled per-GPU-type compute times and byte sizes, and a cluster of G homogeneous device
 * groups with intra- and inter-group link bandwidths (section 5.2.1, 5.2.3).  A candidate is an
 * ordered list of S stage slots; slot s is a submesh of tp_s devices of group g_s (the ordered
 * subclusters of section 5.2.1 together with the submesh choice of section 5.2.2, hoisted out of
 * the DP into the batch dimension).  For every candidate the library finds the partition of the
 * operators into S contiguous non-empty stages with the smallest feasible bottleneck t_max
 * (section 5.2.3, constraints (i)-(iii); the lower end t_S of the cap range of section 5.2.4 (2)) and
 * scores it with the iteration-time model of section 5.2.2 (eq. gpipe_cost_model).
 *
 * All quantities are integers: times in microseconds, sizes in bytes, bandwidths in bytes per
 * microsecond.  With segment [j, i) of operators on slot s = (g, tp), t = group_type[g]:
 *
 *   time(s; j, i) = ceil(sum_{j<=l<i} (fwd_us[t][l] + bwd_us[t][l]) / tp)
 *                   + sum_{j<=l<i} ceil(ar_count * 2 (tp-1) * act_bytes[l] / (tp * bw[g][g]))
 *                                                                   (second term 0 when tp == 1)
 *   comm(s; i)    = ceil(act_bytes[i-1] / bw[g_s][g_{s+1}])  for s < S-1,   0 for s == S-1
 *   fits(s; j, i) = sum param_bytes + N_s * sum stash_bytes <= tp * type_mem_bytes[t],
 *                   N_s = min(S - s, M)     (classic 1F1B in-flight microbatches, section 2.1;
 *                                            eq. mem_cons of section 5.2.3)
 *   bottleneck    = min over partitions with every stage fitting of
 *                   max_s max(time_s, comm_s)
 *   iter_time     = sum_s time_s + 2 sum_{s<S-1} comm_s + (M - 1) * bottleneck
 *
 * Among partitions of equal bottleneck the reported one is fixed by the recurrence
 *   D[s+1][i] = min_j max(D[s][j], time(s;j,i), comm(s;i))  over fitting j, lowest j on ties,
 * followed back from (S, L).
 *
 * Built on the same tables and cost model, further down in this header: the exact optimum of the
 * iteration-time model per candidate (harp_plan_exact_batch, section 5.2.4 (2)); the capped
 * recurrence with the warm-up counts of the H-1F1B scheduler in the memory constraint and as an
 * output (harp_plan_h1f1b_batch, harp_score_h1f1b; sections 4.1 and 5.2.3), and its search over
 * the cap (harp_plan_h1f1b_sweep_batch); the planner over ORDERINGS of device groups that chooses
 * every stage's devices inside the recurrence (harp_plan_mesh_batch, harp_plan_mesh_exact_batch,
 * harp_plan_mesh_h1f1b_batch; eq. dp_general's device index) and the paper's search in full around
 * it (harp_plan_mesh_h1f1b_sweep_batch); and the selection of the best plan of a batch
 * (harp_argmin_batch).
 *
 * Conventions.  Pointers marked DEVICE are device memory of the context's GPU, pointers marked
 * HOST are ordinary host memory.  The caller owns every buffer; the library allocates no device
 * memory.  Calls enqueue work on the given HIP stream (NULL = the default stream) and return
 * without waiting unless stated; outputs are valid once the stream has been synchronised.  Every
 * function returning int returns HARP_OK or a negative error code; harp_last_error gives the
 * message.  A context must not be used from two host threads at once.  No call falls back to the
 * CPU: without a usable GPU harp_create fails.
 */
#ifndef HARP_H
#define HARP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct harp_ctx harp_ctx;       /* opaque; host-side state of one GPU */
typedef struct harp_tables harp_tables; /* opaque host-side view of a caller-lent table buffer */

enum {
    HARP_OK = 0,
    HARP_ERR_INVALID_ARG = -1, /* null pointer, value out of range, malformed problem */
    HARP_ERR_SHAPE = -2,       /* sizes that do not fit together or exceed a stated limit */
    HARP_ERR_WORKSPACE = -3,   /* lent buffer too small or misaligned */
    HARP_ERR_HIP = -4,         /* a HIP runtime call failed */
    HARP_ERR_OVERFLOW = -5,    /* problem magnitudes outside the range the library guarantees */
    HARP_ERR_UNIMPLEMENTED = -6
};

/* per-candidate status written by harp_plan_batch and harp_score_1f1b */
enum { HARP_CAND_OK = 0, HARP_CAND_INFEASIBLE = 1, HARP_CAND_INVALID = 2 };

/* harp_plan_batch kernel selection (harp_set_plan_path).  Every path gives identical results. */
enum {
    HARP_PATH_AUTO = 0,    /* fastest path the tables allow */
    HARP_PATH_GENERIC = 1, /* int64 dense recurrence, one wave per DP cell; any degree, any size */
    HARP_PATH_FAST32 = 2   /* 32-bit times, bounded scan; needs harp_tables_fast32() != 0 */
};

#define HARP_INF INT64_MAX
#define HARP_MAX_TP_DEGREES 8
#define HARP_MAX_L_PLAN 65535

/* Creates the context for GPU `hip_device_ordinal`.  HARP_ERR_HIP when the device is missing. */
int harp_create(harp_ctx **out, int hip_device_ordinal);
void harp_destroy(harp_ctx *ctx);
/* Message of the last failed call on this context; owned by the context, never NULL. */
const char *harp_last_error(const harp_ctx *ctx);

/* The planning problem (paper section 5.2.2-5.2.3: layer sequence, profiled costs, subclusters).
 * All arrays row-major and contiguous. */
typedef struct {
    int32_t L;        /* operators, >= 1 */
    int32_t T;        /* GPU types, >= 1 */
    int32_t G;        /* device groups (homogeneous subclusters), >= 1 */
    int32_t M;        /* microbatches per iteration (the paper's B), >= 1 */
    int32_t ar_count; /* tensor-parallel all-reduces per operator per forward+backward, >= 0 */
    int32_t flags;    /* must be 0 */
    int32_t n_tp;     /* 1 .. HARP_MAX_TP_DEGREES */
    const int32_t *tp_degrees;     /* HOST   [n_tp] ascending, first == 1 */
    const int64_t *fwd_us;         /* DEVICE [T][L] forward time per operator and GPU type */
    const int64_t *bwd_us;         /* DEVICE [T][L] backward time */
    const int64_t *param_bytes;    /* DEVICE [L] parameters and buffers */
    const int64_t *stash_bytes;    /* DEVICE [L] activation kept per in-flight microbatch */
    const int64_t *act_bytes;      /* DEVICE [L] bytes crossing a cut placed right after l */
    const int32_t *group_type;     /* DEVICE [G] GPU type of each group */
    const int32_t *group_ndev;     /* DEVICE [G] devices in each group, >= 1 */
    const int64_t *type_mem_bytes; /* DEVICE [T] memory of one device */
    const int64_t *bw_bytes_per_us;/* DEVICE [G][G] symmetric, >= 1; diagonal = link inside a group */
} harp_problem;

/* Bytes of device memory the caller must lend to harp_build_segment_costs (0 on a malformed
 * problem).  Depends on L, T, G, n_tp only. */
size_t harp_tables_bytes(const harp_problem *problem);

/* Segment-cost tables (the stored stage costs that the search of section 5.2.3 looks up):
 * running sums over operators of compute time per GPU type, parameter bytes, stash bytes and
 * all-reduce time per (group, degree), so that any segment's time and memory is two lookups;
 * plus, when magnitudes allow, the 32-bit rows and per-link cut times of the fast path.
 * Also validates the device-resident problem (signs, ranges, magnitudes).
 *
 * table_buf: DEVICE, 256-byte aligned, at least harp_tables_bytes(problem) bytes; the returned
 * view aliases it and the problem's act_bytes, group_type, group_ndev, type_mem_bytes and
 * bw_bytes_per_us arrays, all of which must stay alive and unchanged until harp_tables_release.
 * Enqueues on `hip_stream` and returns; the verdict on the problem's values is collected by
 * harp_tables_finalize. */
int harp_build_segment_costs(harp_ctx *ctx, const harp_problem *problem, void *table_buf,
                             size_t table_bytes, harp_tables **out, void *hip_stream);

/* Waits for the build on its stream and returns its verdict: HARP_OK, HARP_ERR_INVALID_ARG
 * (negative input, bandwidth < 1, group type out of range, group without devices) or
 * HARP_ERR_OVERFLOW (sums that could leave int64, a stage or transfer time >= 2^47 us, or an
 * iteration time that could leave int64).  Idempotent.  harp_plan_batch and harp_score_1f1b call
 * it themselves on first use of a view. */
int harp_tables_finalize(harp_ctx *ctx, harp_tables *tables);

/* 1 when the finalized tables allow the 32-bit fast path (all degrees powers of two, every time
 * below 2^31 us, L <= 4096, per-link cut table within 256 MiB), else 0.  A batch runs on it when
 * its feasibility index (two tables of min(S_max, M, L) * T * n_tp rows of L + 1 16-bit entries)
 * stays within 256 MiB as well.  The min-max planner and the exact search use it for every such L;
 * the H-1F1B planner and the submesh planners, whose 32-bit kernels keep whole rows of several
 * arrays in LDS, use it up to L = 1024 and run on the int64 path beyond.  Tables with other degrees
 * have the 32-bit rows and cut times as well (and their share of harp_tables_bytes and of the build):
 * harp_plan_batch, harp_plan_exact_batch and harp_plan_h1f1b_batch take them there by themselves, everything
 * else runs in int64, and this stays 0. */
int harp_tables_fast32(const harp_tables *tables);

/* DEVICE pointers into the table buffer, for inspection: running sums indexed [row][i],
 * i = 0..L, row pitch in elements returned through `pitch`.  PF [T], PP [1], PS [1],
 * PR [G * n_tp] (row g * n_tp + k for degree tp_degrees[k]). */
const int64_t *harp_tables_pf(const harp_tables *tables, size_t *pitch);
const int64_t *harp_tables_pp(const harp_tables *tables);
const int64_t *harp_tables_ps(const harp_tables *tables);
const int64_t *harp_tables_pr(const harp_tables *tables, size_t *pitch);

/* Frees the host-side view only. */
void harp_tables_release(harp_tables *tables);

/* A batch of candidates. */
typedef struct {
    int32_t C;     /* candidates, >= 0 */
    int32_t S_max; /* row length of the slot arrays, >= 1 */
    const int32_t *cand_S;     /* DEVICE [C]        stages of each candidate */
    const int32_t *cand_group; /* DEVICE [C][S_max] group of each slot (entries beyond S ignored) */
    const int32_t *cand_tp;    /* DEVICE [C][S_max] devices of each slot */
} harp_candidates;

/* Plans, all DEVICE, caller-allocated.  For a candidate whose status is not HARP_CAND_OK:
 * splits and dev_first all -1, bottleneck = iter_time = HARP_INF. */
typedef struct {
    int32_t *splits;     /* [C][S_max+1] cut positions b_0 = 0 < ... < b_S = L, rest -1 */
    int32_t *dev_first;  /* [C][S_max]   first global device id of each stage, rest -1; groups
                            number their devices consecutively in group order, a group's slots
                            take its devices in slot order */
    int64_t *bottleneck; /* [C] */
    int64_t *iter_time;  /* [C] */
    int32_t *status;     /* [C] HARP_CAND_* */
} harp_plans;

/* Chooses the kernel of harp_plan_batch for this context (HARP_PATH_*); for tests and
 * measurements.  HARP_ERR_INVALID_ARG on an unknown value. */
int harp_set_plan_path(harp_ctx *ctx, int path);

/* Bytes of DEVICE workspace that harp_plan_batch, harp_plan_exact_batch and harp_plan_h1f1b_batch need for this
 * batch, the most of the three (0 on malformed arguments). */
size_t harp_plan_workspace_bytes(harp_ctx *ctx, const harp_tables *tables,
                                 const harp_candidates *cands);

/* The search itself (section 5.2.3 recurrence per candidate, back-pointers, backtrack, and the
 * score of section 5.2.2), one wavefront or workgroup per candidate.  A candidate is HARP_CAND_INVALID when
 * S is outside 1..S_max, a group id or degree is not allowed, a group's slots are not adjacent
 * or use more devices than the group has; HARP_CAND_INFEASIBLE when S > L or no partition fits
 * in memory.  workspace: DEVICE, 256-byte aligned, >= harp_plan_workspace_bytes; contents are
 * scratch.  Needs L <= HARP_MAX_L_PLAN.  Asynchronous on `hip_stream`, except that the first use
 * of a view finalizes it. */
int harp_plan_batch(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                    const harp_plans *out, void *workspace, size_t workspace_bytes,
                    void *hip_stream);

/* harp_plan_batch for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs,
 * outputs, statuses and kernel selection as harp_plan_batch; the planner workspace is a static
 * device array of HARP_STATIC_SCRATCH_BYTES inside the library (every GPU the library is used on
 * holds its own copy until the process ends; harp_create looks up its address).  The call
 * allocates and frees nothing, on the device or through any library.  It runs with as many
 * wavefronts (32-bit path, in fours) or workgroups (int64 path) as the array has room for, so large
 * batches are slower than with harp_plan_batch; a batch whose lists and reachability bands (about
 * 4 (S_max + 3) bytes per candidate), feasibility index (4 min(S_max, M, L) T n_tp (L + 1) bytes)
 * and the back-pointer slices of four wavefronts or one workgroup exceed the array is refused with
 * HARP_ERR_WORKSPACE and nothing is launched.  The tables must have been finalized (harp_tables_finalize) if the call is to stay
 * free of host waits.  Every call on one GPU uses the same array: calls that overlap on one GPU
 * (two streams, two contexts, two host threads) race; calls queued on one stream do not.  The
 * array keeps the previous call's contents; the kernels clear the counters they rely on. */
#define HARP_STATIC_SCRATCH_BYTES (32u << 20)
int harp_plan_batch_static(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                           const harp_plans *out, void *hip_stream);

/* Measurement support: harp_plan_batch with the work it does counted (an instrumented build of the
 * same kernel; slower, same outputs).  work: DEVICE [4], receives the number of transitions
 * (s, i, j) whose value max(D[s][j], time, comm) the kernel evaluated, the DP cells (s, i) it filled,
 * the groups of four previous cuts it read, and the candidates that reached the recurrence (the
 * others were rejected by the memory bounds of the pre-pass).  32-bit path only
 * (HARP_ERR_UNIMPLEMENTED otherwise).  Everything else as harp_plan_batch. */
int harp_plan_batch_count_work(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                               const harp_plans *out, void *workspace, size_t workspace_bytes,
                               uint64_t *work, void *hip_stream);

/* The exact optimum of eq. gpipe_cost_model per candidate: the sweep over the stage-time cap t_max
 * of section 5.2.4 (2), between t_S (the smallest feasible cap, found by the min-max search of
 * harp_plan_batch, which this call runs first) and t_E = ceil(T(t_S) / B), with the capped
 * least-sum recurrence of section 5.2.3 at each cap.  Outputs as for harp_plan_batch, except that
 * splits is the partition of least iteration time (ties: the smaller bottleneck, then the lowest
 * previous cut at every stage of the capped recurrence), bottleneck its largest stage or transfer
 * time and iter_time its iteration time; statuses are those of harp_plan_batch.
 * n_passes: DEVICE [C] or NULL; receives the number of capped recurrences run for the candidate
 * (0 when it has no plan or a single stage).
 * Kernel selection as for harp_plan_batch (harp_set_plan_path; identical results on every path);
 * workspace as for harp_plan_batch.  Asynchronous on `hip_stream`, except that the first use of a view
 * finalizes it. */
int harp_plan_exact_batch(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                          const harp_plans *out, int32_t *n_passes, void *workspace,
                          size_t workspace_bytes, void *hip_stream);

/* A batch of group orderings for harp_plan_mesh_batch: candidate c runs S = ord_S[c] stages on the
 * groups ord_group[c][0 .. ord_G[c]-1], in that order; the planner decides how each group's
 * devices are cut into stages. */
typedef struct {
    int32_t C;      /* orderings, >= 0 */
    int32_t G_max;  /* row length of ord_group, 1..1024 */
    int32_t S_max;  /* row length of the per-stage outputs, >= every ord_S */
    const int32_t *ord_S;     /* DEVICE [C] */
    const int32_t *ord_G;     /* DEVICE [C] groups listed, 1..G_max */
    const int32_t *ord_group; /* DEVICE [C][G_max] distinct group ids (entries beyond ord_G ignored) */
} harp_orderings;

/* Bytes of DEVICE workspace harp_plan_mesh_batch needs (0 on malformed arguments; finalizes the
 * view, because the size depends on the number of devices in the problem). */
size_t harp_plan_mesh_workspace_bytes(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders);

/* The search with the submesh of every stage chosen inside the recurrence (section 5.2.3, the third
 * index of eq. dp_general): state = (stages placed, operators placed, devices used across the
 * ordered groups).  A stage takes tp devices of the group its device offset falls in, tp an
 * allowed degree that does not reach beyond that group; the cut behind a stage that exhausts its
 * group crosses to the next group's link.  Every device of every listed group is used.  Min-max
 * form with the classic 1F1B counts, exactly the definitions of harp_plan_batch; ties: lowest
 * previous cut, then smallest degree.  The result for an ordering equals the best harp_plan_batch
 * result over all slicings of its groups into S stages.
 * out as for harp_plan_batch (rows of length S_max + 1 / S_max); stage_group, stage_tp: DEVICE
 * [C][S_max], the slicing found (-1 beyond S or without a plan).  HARP_CAND_INVALID: S outside
 * 1..S_max, ord_G outside 1..G_max, a group id out of range or listed twice; HARP_CAND_INFEASIBLE:
 * S > L, S < ord_G, S > devices, or no plan fits in memory.  At most 65535 devices, and
 * (devices + 1) x (L + 1) below 2^31 (HARP_ERR_SHAPE otherwise; also for the other entry points
 * with a device index).
 * Asynchronous on `hip_stream`, except that the first use of a view finalizes it. */
int harp_plan_mesh_batch(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders,
                         const harp_plans *out, int32_t *stage_group, int32_t *stage_tp,
                         void *workspace, size_t workspace_bytes, void *hip_stream);

/* The paper's full search for every ordering (sections 5.2.3 and 5.2.4 (2)): the capped least-sum
 * table of eq. dp_general with its device index, swept over the cap t_max between t_S (what
 * harp_plan_mesh_batch finds) and t_E = ceil(T(t_S) / B).  Outputs as harp_plan_mesh_batch, except
 * that the plan is the one of least iteration time over every slicing and partition (ties: smaller
 * bottleneck, then lowest previous cut and smallest degree at every stage of the capped table),
 * bottleneck its largest stage or transfer time and iter_time its iteration time.  n_passes: DEVICE
 * [C] or NULL, capped tables filled per ordering.  Workspace as for harp_plan_mesh_batch. */
int harp_plan_mesh_exact_batch(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders,
                               const harp_plans *out, int32_t *stage_group, int32_t *stage_tp,
                               int32_t *n_passes, void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/* The paper's recurrence in full for one cap per ordering (section 5.2.3): eq. dp_general with its
 * device index and the H-1F1B warm-up count of eq. dp_ni in the state, suffix direction, the memory
 * constraint eq. mem_cons with that count; delta, the cap on counts and the tie rule as for
 * harp_plan_h1f1b_batch (ties: lowest end cut, then smallest degree); device model as for
 * harp_plan_mesh_batch.  t_max: DEVICE [C].  Outputs: out as for harp_plan_mesh_batch with
 * bottleneck = the plan's own largest time and iter_time = least sum + (M - 1) t_max[c];
 * stage_group, stage_tp, warmup: DEVICE [C][S_max].  With single-device groups this is
 * harp_plan_h1f1b_batch on the one slicing there is.  Workspace as for harp_plan_mesh_batch. */
int harp_plan_mesh_h1f1b_batch(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders,
                               const int64_t *t_max, const harp_plans *out, int32_t *stage_group,
                               int32_t *stage_tp, int32_t *warmup, void *workspace,
                               size_t workspace_bytes, void *hip_stream);

/* The search of section 5.2.4 (2) around that recurrence, per ordering: the cap t_max is swept over
 * the sorted, distinct candidate values, from the smallest feasible one up to t_E = ceil(T / B), and
 * harp_plan_mesh_h1f1b_batch's recurrence is evaluated at every one of them.  Candidate values of an
 * ordering: every stage time of a listed group, an allowed degree not above the group's device
 * count and an operator range [j, i), 0 <= j < i <= L; and every transfer time of a cut
 * 1 <= i <= L - 1 on the links the ordering can use (inside each listed group, and from each
 * listed group to the one after it).  The sweep starts at the bottleneck harp_plan_mesh_batch
 * finds (no smaller cap admits a plan, and H-1F1B's counts are never below the classic ones), takes
 * the values in increasing order, fixes t_E from the T of the first cap that has a plan, and ends
 * past t_E, when the values run out, or after max_caps (>= 1) caps.  The answer is the plan with
 * the smallest T = least sum + (M - 1) cap, the lower cap on equal T.  Outputs as
 * harp_plan_mesh_h1f1b_batch at that cap; t_max_out: DEVICE [C], the cap of the answer (INT64_MAX
 * when there is none); n_caps: DEVICE [C] or NULL, caps tried.  HARP_CAND_INFEASIBLE when no tried
 * cap has a plan.  n_caps counts the values the sweep covers; with 32-bit rows most of them are ruled out
 * by bounds and get no pass of their own, otherwise the work per ordering is caps tried x one
 * harp_plan_mesh_h1f1b_batch pass.  Where the work on one ordering is long, several workgroups share its
 * caps (same results).  Workspace: harp_plan_mesh_sweep_workspace_bytes (the slices of the resident
 * workgroups plus up to 33 kept plans per ordering), 256-byte aligned, contents irrelevant. */
size_t harp_plan_mesh_sweep_workspace_bytes(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders);
int harp_plan_mesh_h1f1b_sweep_batch(harp_ctx *ctx, harp_tables *tables, const harp_orderings *orders,
                                     int32_t max_caps, const harp_plans *out, int32_t *stage_group,
                                     int32_t *stage_tp, int32_t *warmup, int64_t *t_max_out,
                                     int32_t *n_caps, void *workspace, size_t workspace_bytes,
                                     void *hip_stream);

/* The same search for candidates, whose slicing is fixed: the cap swept over the candidate values
 * from the bottleneck harp_plan_batch finds up to t_E = ceil(T / B), harp_plan_h1f1b_batch's
 * recurrence at every one of them.  Candidate values of a candidate: every stage time of one of
 * its slots (its group, its degree) over an operator range [j, i), 0 <= j < i <= L, and every
 * transfer time of a cut 1 <= i <= L - 1 on the link between two consecutive slots.  Order of the
 * sweep, t_E, the answer, max_caps, t_max_out and n_caps as for harp_plan_mesh_h1f1b_sweep_batch;
 * out and warmup as for harp_plan_h1f1b_batch at the cap of the answer; statuses as for
 * harp_plan_batch, and HARP_CAND_INFEASIBLE when no tried cap has a plan.  A workgroup searches for
 * one candidate at a time: meant for batches of moderate size.  With 32-bit rows most values are ruled
 * out by bounds; without them every one is tried.  Workspace: harp_plan_h1f1b_sweep_workspace_bytes,
 * 256-byte aligned, contents irrelevant. */
size_t harp_plan_h1f1b_sweep_workspace_bytes(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands);
int harp_plan_h1f1b_sweep_batch(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                                int32_t max_caps, const harp_plans *out, int32_t *warmup,
                                int64_t *t_max_out, int32_t *n_caps, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* The capped recurrence under the H-1F1B scheduler (sections 4.1 and 5.2.3): for candidate c and
 * the cap t_max[c] on every stage and transfer time (constraints (i), (ii)), the suffix recurrence
 * of eq. dp_general with the warm-up launch count carried in the state (eq. dp_ni) and used by the
 * memory constraint (eq. mem_cons):
 *   delta(c_cut; t_max) = 1 if 2 c_cut <= floor(t_max / 64), else 1 + ceil((2 c_cut - floor(t_max / 64)) / t_max)
 *   N(last stage) = 1,  N(stage s) = min(M, delta(cut behind s) + N(stage s + 1))        (eq. Ni)
 *   a state keeps the continuation of least sum (lowest end cut among equal sums) and its N.
 * t_max: DEVICE [C] (negative: no plan; above min(2^47 - 1, INT64_MAX / (3 L + M)), beyond which
 * sum + (M - 1) t_max could leave int64: the candidate is HARP_CAND_INVALID; the same bound holds
 * for every entry point that takes a cap).  warmup: DEVICE [C][S_max], receives N per stage, -1 beyond
 * S and for candidates without a plan.  out as for harp_plan_batch, with bottleneck = the plan's own
 * largest stage or transfer time (<= t_max[c]) and iter_time = least sum + (M - 1) t_max[c], the
 * T(t_max) of section 5.2.3; HARP_CAND_INFEASIBLE when no partition satisfies (i)-(iii) under the
 * cap.  Kernel selection, workspace and asynchrony as for harp_plan_batch. */
int harp_plan_h1f1b_batch(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                          const int64_t *t_max, const harp_plans *out, int32_t *warmup,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/* Warm-up counts and iteration time of caller-chosen partitions under H-1F1B with the cap
 * t_max[c] (section 4.1, eq. Ni; delta as above): splits DEVICE [C][S_max+1], t_max DEVICE [C];
 * outputs DEVICE: warmup [C][S_max], bottleneck (the partition's own), iter_time = sum of
 * (t + 2c) + (M - 1) t_max[c], status.  HARP_CAND_INVALID for a malformed candidate or cuts,
 * HARP_CAND_INFEASIBLE when a stage or transfer time exceeds the cap or a stage does not fit in
 * memory with its count (then warmup is -1 and the times HARP_INF). */
int harp_score_h1f1b(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                     const int32_t *splits, const int64_t *t_max, int32_t *warmup,
                     int64_t *bottleneck, int64_t *iter_time, int32_t *status, void *hip_stream);

/* Scores caller-chosen partitions with eq. gpipe_cost_model (section 5.2.2):
 * splits DEVICE [C][S_max+1].  Status HARP_CAND_INVALID when the candidate is malformed or its
 * cuts are not strictly increasing from 0 to L; HARP_CAND_INFEASIBLE when a stage does not fit
 * in memory; times are HARP_INF unless the status is HARP_CAND_OK.  Kernel selection as for
 * harp_plan_batch (harp_set_plan_path; the kernel for the 32-bit rows takes S_max <= 64, larger
 * batches run on the int64 one; identical results; HARP_ERR_UNIMPLEMENTED when HARP_PATH_FAST32 is
 * set and the tables have no 32-bit rows). */
int harp_score_1f1b(harp_ctx *ctx, harp_tables *tables, const harp_candidates *cands,
                    const int32_t *splits, int64_t *bottleneck, int64_t *iter_time,
                    int32_t *status, void *hip_stream);

/* Final selection over the batch (the min over evaluated candidates of section 5.2.3): smallest
 * iter_time among candidates with status HARP_CAND_OK, lowest index on ties.  best_time and
 * best_index are DEVICE scalars; -1 and HARP_INF when no candidate qualifies. */
int harp_argmin_batch(harp_ctx *ctx, int32_t C, const int64_t *iter_time, const int32_t *status,
                      int64_t *best_time, int32_t *best_index, void *hip_stream);

/* Measurement support for the roofline of the planner kernels (which are bound by integer vector
 * arithmetic, not by a contraction or by memory): launches `blocks` workgroups of 256 threads in
 * which every lane issues iters * 16 32-bit integer vector operations (8 independent chains of one
 * add and one max).  The caller times the launch; lane-operations = blocks * 256 * iters * 16.
 * sink: DEVICE [1], written only in a case that practically never occurs (it keeps the arithmetic
 * alive).  Asynchronous on `hip_stream`. */
int harp_measure_valu_int32(harp_ctx *ctx, int32_t blocks, int32_t iters, uint32_t *sink,
                            void *hip_stream);

/* ------------------------------------------------------------------------------------------------
 * Operators of a stage's training step.
 *
 * What a plan assigns to a stage is a run of operators, each described by the time and the memory it
 * takes on one device.  The calls below are the operators of a transformer's MLP block as they run on
 * an MI355X, forward, backward and optimizer step, so that the rows of a problem (fwd_us, bwd_us,
 * param_bytes, stash_bytes) can be taken on the card instead of being assumed:
 *   harp_linear_*   a matrix product with bias, activation and residual in its epilogue, its gradients
 *   harp_norm_*     the norm after a block, its gate and residual scale, the residual sum, the norm
 *                   before the next block, and their gradients
 *   harp_adamw_*    one AdamW step over many tensors, with moments in 32 bits or in 8
 * and those of its attention operator and of a gated MLP:
 *   harp_rotary*    rotary positions of queries and keys, and their gradients
 *   harp_attention_*  softmax attention to keys of the same or of another length, and its gradients
 *   harp_gated_*    two projections, an activation and a product, and the way back through them
 *
 * Matrices are row-major; a leading dimension (ld) is the distance between rows in elements, at least
 * the number of columns.  Pointers inside the structs are DEVICE; a NULL pointer to something optional
 * leaves it out.  All sums, statistics and moments are held in 32 bits; a result of 16 bits is rounded
 * once, to the nearest, when it is stored.  Infinities and NaN go where the formulas take them.
 * Calls are asynchronous on `hip_stream`, allocate nothing, give the same bits for the same inputs on
 * every call, and can be captured in a graph, whose replays repeat the call with the arguments and scalars
 * that it was captured with (harp_adamw_plan, which waits, cannot).  Outputs must not overlap inputs
 * unless stated.
 * ------------------------------------------------------------------------------------------------ */
enum { HARP_F32 = 0, HARP_BF16 = 1, HARP_F16 = 2 };
enum {
    HARP_ACT_NONE = 0,
    HARP_ACT_RELU = 1,      /* max(z, 0); its derivative at 0 is 0 */
    HARP_ACT_GELU = 2,      /* z (1 + erf(z / sqrt 2)) / 2 */
    HARP_ACT_GELU_TANH = 3, /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
    HARP_ACT_SILU = 4       /* z / (1 + exp(-z)) */
};
enum { HARP_NORM_NONE = 0, HARP_NORM_RMS = 1, HARP_NORM_LAYER = 2 };
enum { HARP_GATE_LINEAR = 0, HARP_GATE_SIGMOID = 1 };
enum { HARP_STATE_F32 = 32, HARP_STATE_8BIT = 8 };

/* Z = X W^T + bias,  Y = act(Z) + residual.  X [M][K], W [N][K], Y, Z and residual [M][N], bias [N], all
 * of `type`, HARP_BF16 or HARP_F16 (what the matrix instructions multiply at full rate).  Z NULL: not
 * stored.  residual may be Y itself.  0 <= M < 2^31, 1 <= N, K < 2^22. */
typedef struct {
    int64_t M, N, K;
    int32_t type, act;
    const void *X;
    int64_t ldx;
    const void *W;
    int64_t ldw;
    const void *bias;
    const void *residual;
    int64_t ldr;
    void *Y;
    int64_t ldy;
    void *Z;
    int64_t ldz;
} harp_linear;

/* dX = (dY W) * act'(Z) + residual: the gradient of the product's input, taken back through the
 * activation that made this input of Z [M][K] (act HARP_ACT_NONE: Z unused), plus the gradient that
 * reaches the same tensor another way.  dY [M][N], W [N][K], dX, Z and residual [M][K], all of `type`.
 * residual may be dX itself. */
typedef struct {
    int64_t M, N, K;
    int32_t type, act;
    const void *dY;
    int64_t lddy;
    const void *W;
    int64_t ldw;
    const void *Z;
    int64_t ldz;
    const void *residual;
    int64_t ldr;
    void *dX;
    int64_t lddx;
} harp_linear_input;

/* dW = dY^T X, dbias = column sums of dY; accumulate not 0: added to what dW and dbias hold (the sum
 * over a pipeline's micro-batches).  dY [M][N] and X [M][K] of `type`, dW [N][K] of `type` or HARP_F32
 * (dw_type), dbias [N] in 32 bits or NULL.  M == 0 gives zeros, or leaves the sums as they are. */
typedef struct {
    int64_t M, N, K;
    int32_t type, dw_type, accumulate;
    const void *dY;
    int64_t lddy;
    const void *X;
    int64_t ldx;
    void *dW;
    int64_t lddw;
    float *dbias;
} harp_linear_weight;

/* Bytes of DEVICE workspace, 256-byte aligned, that any of the three calls needs for these sizes,
 * whatever its strides and alignment (0 on sizes out of range). */
size_t harp_linear_workspace_bytes(harp_ctx *ctx, int64_t M, int64_t N, int64_t K);
int harp_linear_forward(harp_ctx *ctx, const harp_linear *args, void *workspace, size_t workspace_bytes,
                        void *hip_stream);
int harp_linear_grad_input(harp_ctx *ctx, const harp_linear_input *args, void *workspace,
                           size_t workspace_bytes, void *hip_stream);
int harp_linear_grad_weight(harp_ctx *ctx, const harp_linear_weight *args, void *workspace,
                            size_t workspace_bytes, void *hip_stream);
/* dZ = dY * act'(Z) over [M][N]: for an activation whose output goes elsewhere than into a product
 * (there harp_linear_grad_input's epilogue does it).  type HARP_F32, HARP_BF16 or HARP_F16; dZ may be
 * dY or Z. */
int harp_act_grad(harp_ctx *ctx, int64_t M, int64_t N, int32_t type, int32_t act, const void *dY,
                  int64_t lddy, const void *Z, int64_t ldz, void *dZ, int64_t lddz, void *hip_stream);

/* Between two blocks, per row r of `cols` channels:
 *   t = after(y)                               the norm after the block, HARP_NORM_NONE: t = y
 *   h = x + scale * gate(r / rows_per_gate) * t
 *   z = before(h)                              the norm before the next block
 *   RMS:   a / sqrt(mean(a^2) + eps) * w + b       LAYER: the same of a - mean(a)
 * y NULL: h = x, only the norm before (h is not written); x NULL: h = scale * gate * t (at least one of
 * the two is there); before HARP_NORM_NONE: no z.  z is taken of h before it is rounded.  gate_act says
 * whether gate holds the factor itself or what a sigmoid makes it from; gate row r / rows_per_gate, so
 * rows_per_gate = 1 is a gate of its own for every row, `rows` one for all; scale is one vector.
 * x, y, h, z, gate, and the gradients of x, y and gate are of `type` (any); w, b, scale and their
 * gradients [cols] are in 32 bits.  w and b may be NULL (1 and 0).  1 <= cols <= HARP_NORM_MAX_COLS. */
#define HARP_NORM_MAX_COLS 8192
typedef struct {
    int64_t rows;
    int32_t cols, type;
    int32_t after, before;
    float eps_after, eps_before;
    const float *w_after, *b_after, *w_before, *b_before;
    const float *scale;
    const void *gate;
    int64_t ldgate, rows_per_gate;
    int32_t gate_act;
} harp_norm;

/* h may be x or y, z may be y; h NULL: not stored. */
int harp_norm_forward(harp_ctx *ctx, const harp_norm *norm, const void *x, int64_t ldx, const void *y,
                      int64_t ldy, void *h, int64_t ldh, void *z, int64_t ldz, void *hip_stream);

/* The gradients of that, given dh and dz (one may be NULL: zero), h as the forward pass stored it (x where
 * y was NULL) and y:  with D = dh + the gradient of `before` at h,  dx = D,  dy = the gradient of `after`
 * at y of scale * gate * D, and the sums over rows.  dx, dy, and every sum may be NULL: not wanted.
 * dgate [ceil(rows / rows_per_gate)][cols], ld lddgate.  accumulate not 0: the sums in 32 bits (not
 * dgate) are added to what they hold.  dx may be dh or dz, dy may be y. */
typedef struct {
    const void *dh, *dz, *h, *y;
    int64_t lddh, lddz, ldh, ldy;
    void *dx, *dy, *dgate;
    int64_t lddx, lddy, lddgate;
    float *dw_after, *db_after, *dw_before, *db_before, *dscale;
    int32_t accumulate;
} harp_norm_grads;
size_t harp_norm_workspace_bytes(harp_ctx *ctx, const harp_norm *norm);
int harp_norm_backward(harp_ctx *ctx, const harp_norm *norm, const harp_norm_grads *grads,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/* One tensor of an AdamW step.  m and v: float [n], or uint8_t [n] with one exponent byte per block of
 * 256 elements, [ceil(n / 256)].  8 bits stand for
 *   m: sign, 4 bits e, 3 bits f    v: 5 bits e, 3 bits f,   value = (e ? (8 + f) 2^(e-1) : f) 2^(E-129-R),
 * R = 15 for m, 31 for v, E the block's exponent byte: that of the block's largest value as a float,
 * after rounding up to 3 bits of fraction, kept in 64..254 (a byte below 64 counts as 64); 255 marks a block that holds an infinity or
 * NaN and stands for NaN throughout.  A value between two codes goes up with the probability of the part
 * cut off, by a hash of hyper.seed and the element's place: moving averages whose increments are under
 * half a step would stand still otherwise.  A v below its first code that is not zero has that code: with
 * zero the step of an m beside it would be m / eps.  A state of zeros is zero bytes throughout. */
typedef struct {
    int64_t n;
    int32_t state;        /* HARP_STATE_F32 or HARP_STATE_8BIT */
    int32_t grad_type;    /* HARP_F32, HARP_BF16 or HARP_F16 */
    int32_t copy_type;    /* HARP_BF16 or HARP_F16, of copy */
    int32_t flags;        /* must be 0 */
    float *p;             /* [n] master weights, updated */
    const void *grad;     /* [n] */
    void *copy;           /* [n] or NULL: receives the new weights rounded to copy_type */
    void *m, *v;          /* [n] moments, updated */
    uint8_t *m_exp, *v_exp;
    void *m_seen, *v_seen;/* [n] bfloat16 or NULL: where harp_adamw_read_state puts the values */
    double weight_decay;
} harp_adamw_tensor;
typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;             /* 1 for the first */
    uint64_t seed;            /* of the rounding to 8 bits; another one every step */
    const float *grad_scale;  /* DEVICE scalar that gradients are multiplied by, or NULL */
    const int32_t *skip;      /* DEVICE scalar, or NULL: not 0 leaves everything as it is */
} harp_adamw_hyper;
typedef struct harp_adamw harp_adamw;   /* opaque host-side view of a caller-lent plan buffer */

/* Bytes of DEVICE memory for the plan of these tensors (0 on malformed arguments). */
size_t harp_adamw_plan_bytes(const harp_adamw_tensor *tensors /* HOST */, int32_t n_tensors);
/* Writes the plan (the tensors' places and how the work is split) into plan_buf, DEVICE, 256-byte aligned,
 * and waits for `hip_stream`; the tensors and the buffer must stay where they are until
 * harp_adamw_release.  HARP_ERR_INVALID_ARG while `hip_stream` is being captured. */
int harp_adamw_plan(harp_ctx *ctx, const harp_adamw_tensor *tensors, int32_t n_tensors, void *plan_buf,
                    size_t plan_bytes, harp_adamw **out, void *hip_stream);
/* For every tensor:  g = grad_scale * grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps).
 * What `hyper` holds is taken at the call, what its two pointers point to when the kernel runs: replays of a
 * captured step all have its lr, its step's corrections and, with moments in 8 bits, its random bits, so that
 * a program whose steps are to differ in these makes the call itself. */
int harp_adamw_step(harp_ctx *ctx, const harp_adamw *plan, const harp_adamw_hyper *hyper, void *hip_stream);
/* The values that the 8-bit states stand for (exact in bfloat16), into m_seen and v_seen. */
int harp_adamw_read_state(harp_ctx *ctx, const harp_adamw *plan, void *hip_stream);
void harp_adamw_release(harp_adamw *plan);

/* Rotary positions.  A head's first `turned` channels are pairs (a, b) of channels i and i + turned / 2 (HARP_ROTARY_HALF) or
 * 2 i and 2 i + 1 (HARP_ROTARY_INTERLEAVED); of token t at position p, pair i becomes
 *   a' = magnitude (a cos(p f_i) - b sin(p f_i)),   b' = magnitude (b cos(p f_i) + a sin(p f_i)),
 * its other channels stay.  inverse not 0: the angle the other way round, which is the gradient of that.
 * X and Y of `type` (any), element (t, h, c) at t * token + h * step + c; Y may be X (then with the same distances).  positions:
 * p of every token, or NULL: first + t, with period > 0 first + t % period.  frequency: f_i, radians per position; angles are
 * taken in 64 bits, so that they are as exact at position 10^6 as at 1.  Y's elements must not overlap one another; in X a
 * distance may be 0.
 * 0 <= tokens < 2^31, 1 <= heads < 2^16, 2 <= turned <= head < 2^16, turned even. */
enum { HARP_ROTARY_HALF = 0, HARP_ROTARY_INTERLEAVED = 1 };
typedef struct {
    int64_t tokens;
    int32_t heads, head, turned;
    int32_t type, layout, inverse;
    float magnitude;
    const void *X;
    int64_t x_token, x_step;
    void *Y;
    int64_t y_token, y_step;
    const double *frequency;  /* DEVICE [turned / 2] */
    const int64_t *positions; /* DEVICE [tokens] or NULL */
    int64_t first, period;
} harp_rotary_args;
int harp_rotary(harp_ctx *ctx, const harp_rotary_args *args, void *hip_stream);

/* The frequencies of `turned` channels, base^(-2 i / turned), and what they become where contexts are longer than those
 * trained on, by `factor` >= 1:
 *   LINEAR    f / factor
 *   NTK       the base times factor^(turned / (turned - 2)): the last pair as LINEAR, the first as it was
 *   BY_PARTS  f ((1 - g) / factor + g), g = (r - low) / (high - low) kept in 0 .. 1, r = original f / (2 pi): pairs that turn more
 *             than `high` times in `original` positions stay, those of fewer than `low` turns are as LINEAR; magnitude
 *             0.1 ln(factor) + 1 (else 1)
 * frequency: HOST [turned / 2]; magnitude: HOST, or NULL.  Host code: no device is touched. */
enum { HARP_SCALING_NONE = 0, HARP_SCALING_LINEAR = 1, HARP_SCALING_NTK = 2, HARP_SCALING_BY_PARTS = 3 };
int harp_rotary_frequencies(int32_t turned, double base, int32_t scaling, double factor, double original, double low,
                            double high, double *frequency, float *magnitude);

/* Softmax attention.  Per sequence b, head h, query i and key j of the sequence's, with kv head h / (heads / kv_heads):
 *   s_ij = scale q_i . k_j over the keys that i sees,  lse_i = log(sum of exp(s_ij)),  o_i = sum of exp(s_ij - lse_i) v_j
 * Sequence b has queries q_begin[b] .. q_begin[b + 1] - 1 of tokens_q, and keys k_begin[b] .. k_begin[b + 1] - 1 of tokens_k, of
 * which it uses the first k_count[b] (NULL: all).  Where a begin is NULL the sequences have tokens / batch each.  With Lq
 * queries and Lk used keys, i sees all of them, or with causal not 0 those j <= i + Lk - Lq: the last query sees all.  A query
 * that sees no key has o = 0, lse = -infinity, and no part in any gradient, whatever it holds.  One whose scores are all -infinity
 * has o = 0, lse = -infinity and dQ = 0, and where it, its row of dO and a key and value are finite no part in their gradients.
 * Gradients of a key or value that is not finite may be NaN.  Keys that are not used are not read into any result, whatever they
 * hold.  A key or value that is not finite and hidden by the causal order alone may make results of a query that sees other keys
 * NaN, and a query that is not finite, or whose row of dO is not, the gradients of keys hidden from it.
 * What a pass writes lies over nothing else that it reads or writes.
 * Q and O [tokens_q][heads][head], K and V [tokens_k][kv_heads][head], of `type` (HARP_BF16 or HARP_F16), element (t, h, c) at
 * t * token + h * step + c.  lse: float [heads][tokens_q], or NULL in the forward pass.  0 < scale < 2^127.
 * Begins and counts are DEVICE int32, read when the kernels run, so that a captured call takes those of each replay; begins rise
 * and end within tokens; whatever they hold, nothing outside the tensors is touched.  Work is dealt out by what the host knows,
 * tokens / batch: sequences much longer than that take their time alone.  Rows of no sequence are left as they were.
 * Scores, weights' sums and all sums over keys or queries are in 32 bits; weights and their gradients are rounded to `type`
 * where they are multiplied with V, K, Q and dO (what the matrix instructions take; in HARP_F16 weights times 2^12, so that
 * those below 2^-37 of a row's largest are lost, and their gradients times a power of two that keeps them from both ends of its range).
 * head a multiple of 8, at most HARP_ATTENTION_MAX_HEAD; heads a multiple of kv_heads, heads <= 2^14;
 * 0 <= tokens < 2^30, tokens_q * heads / kv_heads < 2^30; 1 <= batch <= 2^20. */
#define HARP_ATTENTION_MAX_HEAD 128
typedef struct {
    int64_t tokens_q, tokens_k;
    int32_t batch, heads, kv_heads, head;
    int32_t type, causal;
    float scale;
    const int32_t *q_begin, *k_begin; /* DEVICE [batch + 1] or NULL */
    const int32_t *k_count;           /* DEVICE [batch] or NULL */
    const void *Q, *K, *V;
    int64_t q_token, q_step, k_token, k_step, v_token, v_step;
    void *O;                          /* the backward pass reads it */
    int64_t o_token, o_step;
    float *lse;                       /* the backward pass reads it */
} harp_attention;
/* Bytes of DEVICE workspace, 256-byte aligned, that both passes need for these tokens, batch, heads, kv_heads and head
 * (0 on sizes out of range). */
size_t harp_attention_workspace_bytes(harp_ctx *ctx, const harp_attention *args);
int harp_attention_forward(harp_ctx *ctx, const harp_attention *args, void *workspace, size_t workspace_bytes,
                           void *hip_stream);
/* With P = exp(s - lse) and D_i = sum over channels of dO_i O_i:  dV = P^T dO,  dS = P (dO V^T - D),  dQ = scale dS K,
 * dK = scale dS^T Q, a kv head's gradients summed over the heads that share it.  dO and dQ like Q, dK and dV like K.  Keys of a
 * sequence that it does not use get zeros.  All three are written (none is added to), each may be NULL: not wanted. */
typedef struct {
    const void *dO;
    int64_t do_token, do_step;
    void *dQ, *dK, *dV;
    int64_t dq_token, dq_step, dk_token, dk_step, dv_token, dv_step;
} harp_attention_grads;
int harp_attention_backward(harp_ctx *ctx, const harp_attention *args, const harp_attention_grads *grads, void *workspace,
                            size_t workspace_bytes, void *hip_stream);

/* The first half of a gated MLP block:  Z = X W^T + bias,  H = act(Z's first F columns) * Z's last F columns.
 * X [M][K], W [2 F][K]: rows 0 .. F - 1 make the gate, the others what it is multiplied with; bias [2 F], H [M][F], Z [M][2 F], all of
 * `type`, HARP_BF16 or HARP_F16.  Z NULL: not stored (the backward pass wants it).  H is taken of Z before it is rounded.
 * 0 <= M < 2^31, 1 <= F, K < 2^21. */
typedef struct {
    int64_t M, F, K;
    int32_t type, act;
    const void *X;
    int64_t ldx;
    const void *W;
    int64_t ldw;
    const void *bias;
    void *H;
    int64_t ldh;
    void *Z;
    int64_t ldz;
} harp_gated;
/* Bytes of DEVICE workspace, 256-byte aligned, that harp_gated_forward (X [M][K]) and harp_gated_grad (dY [M][K]) need, whatever
 * the strides and alignment (0 on sizes out of range). */
size_t harp_gated_workspace_bytes(harp_ctx *ctx, int64_t M, int64_t F, int64_t K);
int harp_gated_forward(harp_ctx *ctx, const harp_gated *args, void *workspace, size_t workspace_bytes,
                       void *hip_stream);
/* The way back through the product behind the block, Y = H W^T with W [N][F], and through the gate:
 *   dH = dY W,   dZ's first F columns = dH * Z's last F * act'(Z's first F),   its last F = dH * act(Z's first F)
 * and H again, for that product's weight gradient, so that it need not be kept (H NULL: not wanted).  W NULL: dY [M][F] is dH (N
 * unused).  Then harp_linear_grad_input and harp_linear_grad_weight of dZ with the block's W [2 F][K] and X give the rest.
 * dY [M][N], Z and dZ [M][2 F], H [M][F] of `type`; dZ may be Z (then lddz is ldz). */
typedef struct {
    int64_t M, F, N;
    int32_t type, act;
    const void *dY;
    int64_t lddy;
    const void *W;
    int64_t ldw;
    const void *Z;
    int64_t ldz;
    void *dZ;
    int64_t lddz;
    void *H;
    int64_t ldh;
} harp_gated_grads;
int harp_gated_grad(harp_ctx *ctx, const harp_gated_grads *args, void *workspace, size_t workspace_bytes,
                    void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HARP_H */
