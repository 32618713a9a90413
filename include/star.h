/*
 * star.h — C ABI of the B200 grouped gradient aggregation + parameter update.
 *
 * The operation (STAR's parameter-server hot path).  A round hands the server W
 * workers' gradient buffers and a SCHEDULE: an ordered list of disjoint,
 * non-empty groups of workers.  SSGD is one group of all workers, ASGD is one
 * group per worker in arrival order (paper Section I); the static x-order mode
 * uses x workers per update and the dynamic x-order mode one worker cluster per
 * update (Section I contribution (2), Section IV-B), clusters taken in
 * ascending order of their slowest member (Section IV-C1, text before Eq. 2).
 * For every element i and every group k in schedule order the library applies
 *
 *     s    = g[m_k0][i] + g[m_k1][i] + ...          members in listed order
 *     gbar = s / |G_k|
 *     d    = fma(wd, p[i], gbar)
 *     v[i] = fma(mu, v[i], d)
 *     p[i] = fma(-lr_k, v[i], p[i])
 *
 * each line one correctly rounded IEEE-754 binary32 operation (bf16 gradients
 * are widened exactly first).  All groups of a round are fused into ONE pass:
 * every scheduled gradient element and p, v are read once, p and v are written
 * once: n * (sum_k |G_k| * sizeof(g) + 16) bytes of traffic per round.
 *
 * A schedule is a CSR pair: group k = group_members[group_offsets[k] ..
 * group_offsets[k+1]).  It need not cover every worker (a round may use only
 * the workers that reported); a worker may appear at most once.
 *
 * Conventions that hold for every entry point
 *   - "device" pointers are CUDA device memory of the current device; "host"
 *     arrays are ordinary memory that is read completely before the call
 *     returns (the caller may free or reuse it at once).
 *   - The caller owns every buffer.  The library allocates no device memory and
 *     keeps no pointer after a call returns, except inside a caller-provided
 *     workspace.
 *   - Work is enqueued on `cuda_stream` (a cudaStream_t; NULL = legacy default
 *     stream) and the call returns without synchronizing.  The exceptions are
 *     the calls that copy a table from ordinary host memory (star_multi_prepare,
 *     star_multi_prepare_ex, star_group_update_multi_noalloc): such a copy
 *     makes the host wait until earlier work on `cuda_stream` has finished and
 *     the table is staged, and those calls refuse to run inside a stream
 *     capture (STAR_ERR_UNSUPPORTED, nothing enqueued).
 *   - Every argument error is found on the host BEFORE anything is launched and
 *     leaves p and v untouched.  STAR_ERR_CUDA is a failed launch or runtime
 *     call; star_last_cuda_error() gives its cudaError_t.
 *   - There is no CPU path: without a usable CUDA device the compute entry
 *     points return STAR_ERR_CUDA.
 *   - params, momentum and the scheduled gradient buffers must not overlap.
 *     Element-size alignment is required (4 bytes fp32, 2 bytes bf16).  Buffers
 *     aligned to 32 bytes take the full-width vector path.  So do buffers that
 *     are all views at one common element offset into 32-byte aligned storage
 *     (the usual way a tensor ends up misaligned): up to 7 leading elements are
 *     done one by one and the rest in vectors.  Buffers with no common
 *     alignment phase take a narrower or element-by-element path (slower).
 *     Results are identical on every path.
 */
#ifndef STAR_H_
#define STAR_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define STAR_API __attribute__((visibility("default")))
#else
#define STAR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    STAR_OK = 0,
    STAR_ERR_NULL_POINTER = 1,      /* a required pointer is NULL */
    STAR_ERR_INVALID_ARG = 2,       /* negative size, bad dtype, misaligned or overlapping buffers */
    STAR_ERR_BAD_SCHEDULE = 3,      /* empty group, duplicate or out-of-range member, bad offsets */
    STAR_ERR_UNSUPPORTED = 4,       /* W above STAR_MAX_WORKERS; a table-copying call inside a stream capture */
    STAR_ERR_WORKSPACE_TOO_SMALL = 5,
    STAR_ERR_CUDA = 6,              /* see star_last_cuda_error() */
    STAR_ERR_TIMEOUT = 7            /* see star_check_waits() */
} star_status_t;

typedef enum { STAR_DTYPE_F32 = 0, STAR_DTYPE_BF16 = 1 } star_dtype_t;

/* Order of the additions inside a group (only rounding depends on it).
 * STAR_SUM_LINEAR: left to right in the listed member order.
 * STAR_SUM_TREE:   pairwise, as gradients are combined along a binary
 *                  aggregation tree (Section IV-D2b: workers add their children's
 *                  gradients to their own on the way up): tree(m_0..m_{c-1}) is the
 *                  member itself for c = 1, else tree(first h) + tree(remaining
 *                  c - h) with h the largest power of two below c. */
typedef enum { STAR_SUM_LINEAR = 0, STAR_SUM_TREE = 1 } star_sum_order_t;

#define STAR_MAX_WORKERS 64

/* Static, NUL-terminated name of a status code. */
STAR_API const char *star_status_string(star_status_t status);

/* cudaError_t of the most recent STAR_ERR_CUDA on the calling thread (0 if none). */
STAR_API int star_last_cuda_error(void);

/* Number of kernels this library has launched in the calling process so far. */
STAR_API int64_t star_launch_count(void);

/* ---------------------------------------------------------------------------
 * Schedule encoding (host only; no CUDA call).  Turns a synchronization-mode
 * decision into the CSR pair.  offsets_out needs room for W + 1 entries,
 * members_out for W entries; *n_groups_out receives K.
 * ------------------------------------------------------------------------- */

/* STAR_OK iff the pair describes n_groups non-empty, pairwise disjoint groups
 * of workers in [0, W) with group_offsets[0] == 0 (Section IV-B: a gradient
 * report feeds exactly one update).  n_groups == 0 is valid. */
STAR_API star_status_t star_schedule_validate(const int32_t *group_offsets, const int32_t *group_members,
                                     int n_groups, int W);

/* Static x-order mode (Section IV-B): consecutive runs of x workers of
 * arrival_order (n_arrived distinct workers, earliest first; NULL = 0..W-1 with
 * n_arrived = W).  x == n_arrived gives SSGD, x == 1 ASGD (Section I).  If x
 * does not divide n_arrived the last group is smaller.  sort_members != 0 lists
 * each group's members in ascending worker index, otherwise in arrival order. */
STAR_API star_status_t star_schedule_static_x(const int32_t *arrival_order, int n_arrived, int W, int x,
                                     int sort_members, int32_t *offsets_out,
                                     int32_t *members_out, int *n_groups_out);

/* Groups from a per-worker label group_of_worker[W] (-1 = worker absent):
 * groups in ascending label order, members in ascending worker index. */
STAR_API star_status_t star_schedule_from_labels(const int32_t *group_of_worker, int W,
                                        int32_t *offsets_out, int32_t *members_out,
                                        int *n_groups_out);

/* Dynamic x-order mode (Section IV-B, ordering of Section IV-C1): one group per
 * cluster id in cluster_of_worker[W] (-1 = absent), groups ascending in the
 * cluster's largest iter_time; ties go to the cluster holding the smaller
 * worker index; members in ascending worker index.  iter_time must be finite. */
STAR_API star_status_t star_schedule_dynamic_x(const double *iter_time, const int32_t *cluster_of_worker,
                                      int W, int32_t *offsets_out, int32_t *members_out,
                                      int *n_groups_out);

/* ---------------------------------------------------------------------------
 * Mode decision (host only): from predicted iteration times to the schedule of
 * the cheapest synchronization mode.  iter_time[w] > 0, finite.
 * ------------------------------------------------------------------------- */

/* Dynamic x-order clustering (Section IV-B): agglomerative hierarchical
 * clustering of the W predicted iteration times with average linkage (mean
 * pairwise |t_a - t_b|).  Merging continues while more than n_clusters clusters
 * remain (n_clusters <= 0: down to one) and the closest pair is no farther
 * apart than max_distance (max_distance < 0: no distance limit).  Equally close
 * pairs: the pair whose clusters hold the smaller worker indices merges first.
 * cluster_of_worker_out[W] receives labels 0..K-1 numbered by each cluster's
 * smallest worker index; *n_clusters_out = K.  Feed the labels to
 * star_schedule_dynamic_x or star_choose_mode. */
STAR_API star_status_t star_cluster_iteration_times(const double *iter_time, int W, int n_clusters,
                                                    double max_distance,
                                                    int32_t *cluster_of_worker_out,
                                                    int *n_clusters_out);

/* Expected time to a fixed training progress per mode (Section IV-C1).
 * T_static_out[x-1], x = 1..W, is Eq. 1: (1 + phi / (x M / W)) * t_x, where t_x,
 * the time one update takes, is read as the x-th smallest iteration time (the
 * moment x gradient reports are in); x = 1 is ASGD, x = W SSGD.  If
 * cluster_of_worker is not NULL (labels >= 0 for every worker), *T_dynamic_out
 * is Eq. 2: 1 / sum_i 1 / ((1 + phi / (n_ci M / W)) * t_ci) over the clusters,
 * n_ci the cluster's size and t_ci its slowest member.  phi is the
 * pre-conditioned gradient noise scale of the current update (>= 0), M the
 * total batch size (> 0); both are the caller's inputs. */
STAR_API star_status_t star_mode_times(const double *iter_time, const int32_t *cluster_of_worker,
                                       int W, double phi, double M, double *T_static_out,
                                       double *T_dynamic_out);

/* The mode with the smallest time and its schedule.  *x_out = x of the chosen
 * static x-order mode, or 0 for the dynamic mode (only if cluster_of_worker is
 * given and Eq. 2 is strictly smaller than every Eq. 1 value); equal static
 * times go to the larger x.  *T_out = that time.  The CSR outputs are as for the
 * schedule encoders: static modes group the workers in ascending predicted time
 * (ties by index) in runs of x, members listed in ascending index; the dynamic
 * mode is star_schedule_dynamic_x on the clusters. */
STAR_API star_status_t star_choose_mode(const double *iter_time, const int32_t *cluster_of_worker,
                                        int W, double phi, double M, int *x_out, double *T_out,
                                        int32_t *offsets_out, int32_t *members_out,
                                        int *n_groups_out);

/* All-reduce architecture (Section IV-B, Section IV-C1 Eq. 3): remove x of the
 * stragglers from the ring, attach each to a parent that waits t_w after the
 * ring's slowest member and adds the gradients of the children that reported
 * by then.  T_a = (1 + phi / ((W - x + q) M / W)) * (t_ring + t_w).
 *   iter_time[w]   predicted iteration time in the ring; a worker is a straggler
 *                  iff (t - min t) / min t > straggler_threshold (Section II: 0.2)
 *   child_time[w]  predicted iteration time of w when attached to a parent; a
 *                  removed worker counts (q) iff child_time[w] - t_ring <= t_w
 *   t_w_max        largest wait considered (t_w in [0, t_w_max])
 * The x slowest stragglers are removed (x = 0..X, at least one worker stays);
 * only t_w = 0 and the waits at which one more child makes it are candidates;
 * ties go to fewer removals, then the shorter wait.  Outputs: *x_out, *t_w_out,
 * *T_out, removed_out[0..x) (slowest first), and the CSR of the ONE group whose
 * gradients enter the update (ring members and children in time, ascending
 * index): on a server holding every worker's buffer the all-reduce mode's
 * update is star_group_update with that schedule. */
STAR_API star_status_t star_choose_all_reduce_mode(const double *iter_time, const double *child_time,
                                                   int W, double phi, double M, double t_w_max,
                                                   double straggler_threshold, int *x_out,
                                                   double *t_w_out, double *T_out,
                                                   int32_t *removed_out, int32_t *offsets_out,
                                                   int32_t *members_out, int *n_groups_out);

/* Parents of the workers taken out of the ring (Section IV-B: each removed
 * straggler reports to a non-straggler with high bandwidth; Section IV-D2a
 * balances the number of children per parent).  Behind a non-blocking switch
 * every ring member is equally near, so the removed workers (removed[0..x), in
 * the order star_choose_all_reduce_mode lists them) are dealt round-robin over
 * the ring members in ascending worker index.  parent_of_out[W] receives the
 * parent of each removed worker and -1 for ring members.  0 <= x < W. */
STAR_API star_status_t star_assign_parents(const int32_t *removed, int x, int W,
                                           int32_t *parent_of_out);

/* Communication tree (Section IV-D2b: the workers of a job form a tree under
 * the parameter server, or under a parent in the all-reduce architecture;
 * workers with longer communication latency sit in lower layers; every worker
 * adds its children's gradients to its own and forwards the sum; the tree is
 * rebuilt before each iteration).  A fanout-ary tree filled layer by layer in
 * ascending latency (ties: the smaller worker index first): the `fanout`
 * quickest workers become children of the root, the next `fanout` children of
 * the quickest worker, and so on.  parent_of_out[W] receives each worker's
 * parent, -1 for the root's children.  latency finite, fanout >= 1. */
STAR_API star_status_t star_build_tree(const double *latency, int W, int fanout, int32_t *parent_of_out);

/* Sharding helper (host only).  The path is elementwise, so a job spread over
 * several parameter servers / GPUs (the paper runs one to N PSs per job,
 * Section III set-up) needs no exchange inside it: rank r of world owns the
 * contiguous element range [*first_out, *first_out + *count_out) of a tensor of
 * n elements.  Ranges are disjoint, cover [0, n), differ in length by less than
 * 2 x `align`, and every range starts at a multiple of `align` elements (use 16 to
 * keep bf16 and fp32 shards on the vector path).  align >= 1. */
STAR_API star_status_t star_shard_range(int64_t n, int world, int rank, int64_t align,
                                        int64_t *first_out, int64_t *count_out);

/* ---------------------------------------------------------------------------
 * Fused grouped update of one flat tensor (the operation defined at the top).
 *   params, momentum : device, fp32, n elements, updated in place
 *   grads            : host array of W device pointers, n elements of
 *                      grad_dtype each; entries of unscheduled workers are
 *                      never dereferenced and may be NULL
 *   group_offsets    : host, n_groups + 1 entries;  group_members : host
 *   lr, mu, wd       : learning rate, momentum coefficient, weight decay
 * n == 0 or n_groups == 0 is a successful no-op.  One kernel launch.
 * ------------------------------------------------------------------------- */
STAR_API star_status_t star_group_update(float *params, float *momentum, const void *const *grads, int W,
                                star_dtype_t grad_dtype, int64_t n,
                                const int32_t *group_offsets, const int32_t *group_members,
                                int n_groups, float lr, float mu, float wd, void *cuda_stream);

/* The same round with one learning rate per group, optional parameter
 * snapshots and a choice of the in-group summation order (sum_order; with
 * groups of more than 4 members the tree order keeps partial sums per element
 * in registers and runs at half the occupancy of the linear order).
 *   lrs        : host, n_groups learning rates.  Section IV-C1 ("Scaling learning
 *                rate after switching") sets the rate of an update built from y
 *                gradient reports to (y / N) x the SSGD rate; the caller computes
 *                the rates, the kernel applies lrs[k] in group k's update.
 *   snapshots  : NULL, or host array of n_groups device pointers (n elements of
 *                snapshot_dtype each, entries may be NULL).  snapshots[k] receives
 *                the parameters as they stand right after group k's update -- the
 *                copy the server sends back to that group's workers (Section II)
 *                -- written in the same pass: fp32 (4 n more bytes of traffic
 *                each) or rounded to bf16, nearest-even (2 n bytes each).
 *                Snapshot buffers must not overlap each other or any other
 *                buffer of the call.
 * Everything else as star_group_update.  One kernel launch. */
STAR_API star_status_t star_group_update_ex(float *params, float *momentum, const void *const *grads,
                                            int W, star_dtype_t grad_dtype, int64_t n,
                                            const int32_t *group_offsets,
                                            const int32_t *group_members, int n_groups,
                                            const float *lrs, float mu, float wd,
                                            void *const *snapshots, star_dtype_t snapshot_dtype,
                                            star_sum_order_t sum_order, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * All-reduce architecture (Section IV-B, paragraph "All-reduce architecture";
 * Section IV-C1, Eq. 3).  Stragglers are taken out of the ring and report their
 * gradients to a parent in the ring; the parent adds the gradients of the
 * children that reported in time to its own, the ring sums its members'
 * aggregates, and one update is made from the gradients of N - x + q workers.
 * Two kernels cover the arithmetic of such a round on one GPU; moving the
 * buffers between GPUs is the caller's (a collective library's) part, and
 * every buffer handed to these calls is memory of the current device.
 * ------------------------------------------------------------------------- */

/* A parent's local aggregate: out[i] = g[m_0][i] + g[m_1][i] + ... over the
 * `count` listed workers (own gradient first, then the children), each addition
 * one binary32 operation, left to right or in tree order (sum_order), written as
 * binary32 (out_dtype F32) or rounded to bf16, nearest even (BF16).
 *   out     : device, n elements of out_dtype; must not overlap a listed buffer
 *   grads   : host array of W device pointers (n elements of grad_dtype each);
 *             only the listed entries are dereferenced
 *   members : host, `count` distinct workers in [0, W); count == 0 is
 *             STAR_ERR_BAD_SCHEDULE (an empty sum has no meaning in this round)
 * n == 0 is a successful no-op.  One kernel launch; n * (count * sizeof(g) +
 * sizeof(out)) bytes of traffic. */
STAR_API star_status_t star_group_reduce(void *out, star_dtype_t out_dtype, const void *const *grads,
                                         int W, star_dtype_t grad_dtype, int64_t n,
                                         const int32_t *members, int count,
                                         star_sum_order_t sum_order, void *cuda_stream);

/* The one update of an all-reduce round from the R ring members' aggregates
 * (binary32, n elements each, device), added left to right in the listed (ring)
 * order; the mean divides by n_reports, the number of gradient reports behind
 * the aggregates (N - x + q of Eq. 3, R <= n_reports <= 255):
 *     s = sums[0][i] + sums[1][i] + ... ; gbar = s / n_reports ;
 *     d = fma(wd, p, gbar) ; v = fma(mu, v, d) ; p = fma(-lr, v, p)
 * sums: host array of R device pointers.  Every rank that applies this call to
 * the same aggregates in the same order holds bit-identical parameters
 * afterwards.  R == 0 with n_reports == 0, or n == 0, is a no-op.  One launch. */
STAR_API star_status_t star_group_update_from_sums(float *params, float *momentum,
                                                   const float *const *sums, int R, int64_t n,
                                                   int n_reports, float lr, float mu, float wd,
                                                   void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Fused grouped update of a LIST of tensors (per-layer parameters) in one
 * launch.  The pointer table and tile map live in a caller-provided device
 * workspace that is prepared once per tensor list and reused every round.
 * ------------------------------------------------------------------------- */

/* Host-side description of a prepared tensor list.  Plain data, filled by
 * star_multi_prepare and passed back by value-pointer every round; it holds
 * the workspace address but owns nothing. */
typedef struct {
    uint64_t magic;            /* set by star_multi_prepare; anything else is rejected */
    const void *d_workspace;   /* the caller's device workspace */
    int64_t total_elements;    /* sum of the tensor sizes */
    int64_t n_tiles;           /* work items the kernel walks */
    uint64_t complete_workers; /* bit w set: worker w has a gradient for every non-empty tensor */
    int32_t n_tensors;
    int32_t W;
    int32_t grad_dtype;        /* star_dtype_t */
    int32_t tile_elements;     /* elements per tile */
    int32_t n_snapshot_sets;   /* snapshot buffer sets registered by star_multi_prepare_ex (else 0) */
    int32_t snapshot_dtype;    /* star_dtype_t of those buffers */
} star_multi_plan_t;

/* Bytes of device workspace needed for n_tensors tensors of the given sizes
 * (host array, elements per tensor, 0 allowed) and W workers (no snapshot sets). */
STAR_API star_status_t star_multi_workspace_bytes(int n_tensors, const int64_t *sizes, int W,
                                         size_t *bytes_out);

/* Fill the workspace and *plan_out.  params, momentum: host arrays of n_tensors
 * device pointers; grads: host array of n_tensors * W device pointers, entry
 * [t * W + w] = worker w's gradient for tensor t (NULL allowed for workers that
 * will never be scheduled); sizes: host, elements per tensor.  d_workspace:
 * device, 256-byte aligned, at least star_multi_workspace_bytes() bytes.  The
 * table is built in ordinary host memory and copied with one cudaMemcpyAsync on
 * cuda_stream; the host copy is released before the call returns (a copy from
 * pageable memory returns once the data is staged, which makes the host wait
 * for earlier work on cuda_stream), later work on the same stream sees the
 * table.  Inside a stream capture the call returns STAR_ERR_UNSUPPORTED and
 * enqueues nothing.  No buffer that a round writes (params, momentum) may
 * share memory with any other buffer of the list, in the same or in another
 * tensor (STAR_ERR_INVALID_ARG: e.g. a tied weight listed twice); gradient
 * buffers may alias one another.  Not a per-round call: once per tensor list. */
STAR_API star_status_t star_multi_prepare(int n_tensors, float *const *params, float *const *momentum,
                                 const void *const *grads, const int64_t *sizes, int W,
                                 star_dtype_t grad_dtype, void *d_workspace,
                                 size_t workspace_bytes, void *cuda_stream,
                                 star_multi_plan_t *plan_out);

/* One round over the prepared list: the same operation as star_group_update on
 * every tensor, one kernel launch in total.  Scheduling a worker whose gradient
 * pointer was NULL for some non-empty tensor at prepare time is rejected with
 * STAR_ERR_NULL_POINTER.  A plan not made by star_multi_prepare is rejected
 * with STAR_ERR_INVALID_ARG. */
STAR_API star_status_t star_group_update_multi(const star_multi_plan_t *plan,
                                      const int32_t *group_offsets, const int32_t *group_members,
                                      int n_groups, float lr, float mu, float wd,
                                      void *cuda_stream);

/* The tensor-list round with one learning rate per group (lrs: host, n_groups
 * values; Section IV-C1 rate scaling).  Otherwise as star_group_update_multi. */
STAR_API star_status_t star_group_update_multi_lrs(const star_multi_plan_t *plan,
                                                   const int32_t *group_offsets,
                                                   const int32_t *group_members, int n_groups,
                                                   const float *lrs, float mu, float wd,
                                                   void *cuda_stream);

/* Tensor lists with parameter snapshots and the tree order.  A snapshot SET is
 * one buffer per tensor of the list; up to STAR_MAX_WORKERS sets are registered
 * when the list is prepared (their pointers go into the same workspace table),
 * and every round says which set, if any, receives the parameters as they stand
 * right after each group's update -- the copy the server sends back to that
 * group's workers (Section II) -- written in the same pass.
 *   star_multi_workspace_bytes_ex : workspace size with n_snapshot_sets sets
 *   star_multi_prepare_ex         : as star_multi_prepare, plus
 *       snapshots      host array of n_tensors * n_snapshot_sets device pointers,
 *                      entry [t * n_snapshot_sets + s] = tensor t's buffer of set
 *                      s (sizes[t] elements of snapshot_dtype; NULL = tensor t is
 *                      not captured by set s); snapshot buffers are written, so
 *                      they must not overlap anything else in the list
 *   star_group_update_multi_ex    : one round, one launch, with
 *       lrs                    host, one learning rate per group (Section IV-C1)
 *       snapshot_set_of_group  NULL, or host array of n_groups entries: the set
 *                              (0 .. n_snapshot_sets-1) written after group k, or -1
 *       sum_order              STAR_SUM_LINEAR or STAR_SUM_TREE (Section IV-D2b)
 * Results equal star_group_update_ex applied to every tensor of the list. */
STAR_API star_status_t star_multi_workspace_bytes_ex(int n_tensors, const int64_t *sizes, int W,
                                                     int n_snapshot_sets, size_t *bytes_out);

STAR_API star_status_t star_multi_prepare_ex(int n_tensors, float *const *params, float *const *momentum,
                                             const void *const *grads, const int64_t *sizes, int W,
                                             star_dtype_t grad_dtype, int n_snapshot_sets,
                                             void *const *snapshots, star_dtype_t snapshot_dtype,
                                             void *d_workspace, size_t workspace_bytes,
                                             void *cuda_stream, star_multi_plan_t *plan_out);

STAR_API star_status_t star_group_update_multi_ex(const star_multi_plan_t *plan,
                                                  const int32_t *group_offsets,
                                                  const int32_t *group_members, int n_groups,
                                                  const float *lrs, float mu, float wd,
                                                  const int32_t *snapshot_set_of_group,
                                                  star_sum_order_t sum_order, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Fused grouped update with the state and the gradients in HOST memory (the
 * paper's parameter server keeps its parameter and gradient copies in host
 * memory, Section II).  Same operation and results as star_group_update; the
 * data is streamed through the GPU in chunks: copy a chunk of p, v and of every
 * scheduled worker's gradient to the device, run the fused kernel on it, copy
 * p and v back, with the copies of neighbouring chunks overlapping (host to
 * device on cuda_stream, device to host on an internal stream).
 *   h_params, h_momentum : host, fp32, n elements, updated in place
 *   h_grads              : host array of W host pointers (unscheduled: may be NULL)
 *   d_workspace          : device, 256-byte aligned staging memory provided by
 *                          the caller; star_host_workspace_bytes() gives the
 *                          size for a chosen chunk length
 * Host buffers should be page-locked (cudaHostAlloc / cudaHostRegister):
 * pageable memory works but its copies do not overlap.  The call enqueues all
 * work and returns; results are in the host buffers once cuda_stream has been
 * synchronized.  The first call on a device creates one internal stream and a
 * few events (no device memory).  Calls on the same device are serialized
 * against each other at enqueue time by the library; they must not share a
 * workspace unless they are ordered on one stream.
 * ------------------------------------------------------------------------- */

/* Workspace bytes for chunks of chunk_elements elements (a multiple of 2048, at
 * least 2048) when at most max_scheduled workers are scheduled in a round. */
STAR_API star_status_t star_host_workspace_bytes(int max_scheduled, star_dtype_t grad_dtype,
                                                 int64_t chunk_elements, size_t *bytes_out);

/* The chunk length is the largest multiple of 2048 that fits workspace_bytes for
 * the number of workers this schedule uses; STAR_ERR_WORKSPACE_TOO_SMALL if
 * that is below 2048.  One kernel launch per chunk. */
STAR_API star_status_t star_group_update_host(float *h_params, float *h_momentum,
                                              const void *const *h_grads, int W,
                                              star_dtype_t grad_dtype, int64_t n,
                                              const int32_t *group_offsets,
                                              const int32_t *group_members, int n_groups, float lr,
                                              float mu, float wd, void *d_workspace,
                                              size_t workspace_bytes, void *cuda_stream);

/* The host-buffer round with one learning rate per group (lrs: host, n_groups
 * values; Section IV-C1), optional parameter snapshots into HOST buffers
 * (h_snapshots: NULL, or host array of n_groups host pointers, n elements of
 * snapshot_dtype each, entries may be NULL: the copy of the parameters after
 * that group's update that the server sends back to the group's workers,
 * Section II) and the choice of summation order.  Snapshot chunks are staged in
 * the workspace and copied back with p and v; star_host_workspace_bytes_ex sizes
 * the workspace for up to max_snapshots snapshots of snapshot_dtype per round.
 * Everything else as star_group_update_host. */
STAR_API star_status_t star_host_workspace_bytes_ex(int max_scheduled, star_dtype_t grad_dtype,
                                                    int max_snapshots, star_dtype_t snapshot_dtype,
                                                    int64_t chunk_elements, size_t *bytes_out);

STAR_API star_status_t star_group_update_host_ex(float *h_params, float *h_momentum,
                                                 const void *const *h_grads, int W,
                                                 star_dtype_t grad_dtype, int64_t n,
                                                 const int32_t *group_offsets,
                                                 const int32_t *group_members, int n_groups,
                                                 const float *lrs, float mu, float wd,
                                                 void *const *h_snapshots, star_dtype_t snapshot_dtype,
                                                 star_sum_order_t sum_order, void *d_workspace,
                                                 size_t workspace_bytes, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * A worker's step: the loss over the vocabulary with the gradient of the
 * logits, and activations kept in 8 bits whose backward pass writes the
 * worker's gradient buffers -- what a worker does before its gradients reach
 * star_group_update.
 *
 * Matrices are row-major with a row stride (`ld`, in elements, at least the
 * number of columns); any element-aligned base and any stride is taken, rows
 * that share one phase modulo 16 bytes and whose stride keeps it are the fast
 * case.  Sizes of zero are successful no-ops (sums and losses are still
 * written: zero).  Written buffers must not overlap any other buffer of the
 * call, except where an in-place form is named; matrices with one stride may lie
 * side by side in the rows of one buffer, those with different strides may not.
 * All sums, softmax statistics
 * and activation values are held in binary32; results are rounded once.  The
 * same call on the same inputs gives the same bits.
 * ------------------------------------------------------------------------- */

/* Rows of logits x[t][0 .. vocab), one label each.  With z = x / temperature,
 *     lse = log(sum_j exp(z[j])),  p[j] = exp(z[j] - lse),  logp = z[label] - lse.
 * A row is ACTIVE iff its label lies in [0, vocab) (a prompt or padding token
 * carries any other value, -100 by custom), its weight, where weights are
 * given, is not 0, and not every logit of it is -inf.  The logits of a row that
 * its label or weight makes inactive are not read: they may hold anything.  An
 * inactive row has logp = lse = loss = 0 and a zero gradient.  A NaN or +inf
 * logit makes its own row's results NaN and the totals with them.
 *
 * star_token_logprobs: logp[rows] and, unless NULL, lse[rows].
 * temperature finite, > 0; vocab at most 2^31 - 1 (STAR_ERR_UNSUPPORTED beyond).
 * One kernel launch. */
STAR_API star_status_t star_token_logprobs(const void *logits, star_dtype_t dtype, int64_t rows,
                                           int64_t vocab, int64_t ld, const int64_t *labels,
                                           float temperature, float *logp, float *lse,
                                           void *cuda_stream);

/* Device workspace of the two losses below: bytes for `rows` rows in
 * `sequences` sequences (0 for the policy loss).  Need not be initialized. */
STAR_API star_status_t star_loss_workspace_bytes(int64_t rows, int64_t sequences, size_t *bytes_out);

/* Clipped policy loss with a KL term, forward and backward in one pass over the
 * logits.  Per active row t, with A = advantages[t] and w = weights[t] (1
 * without weights):
 *     r    = exp(logp - old_logp[t])                 (1 if old_logp is NULL)
 *     u    = r A,   c = clamp(r, 1 - clip_low, 1 + clip_high) A
 *     kl   = exp(ref_logp[t] - logp) - (ref_logp[t] - logp) - 1      (0 if ref_logp is NULL)
 *     token_loss[t] = -min(u, c) + kl_coef kl
 *     dlogits[t][j] = w / temperature * ((j == label) - p[j]) *
 *                     (-(u <= c) r A + kl_coef (1 - exp(ref_logp[t] - logp)))
 *     sums = { sum w token_loss, sum w (-min(u, c)), sum w kl, sum w (c < u) }
 * A factor of exactly 0 (A, kl_coef) takes its term out, however large the other one.
 * dlogits is the gradient of sums[0]; the caller puts the mean's 1 / n (per
 * token or per sequence) and any loss scale into weights.
 *   old_logp NULL differentiates the ratio as if old_logp were logp itself.  So with
 *               advantages of 1 and no ref_logp dlogits is the gradient of the weighted
 *               cross-entropy, -sum w logp, whose terms are in logp
 *   dlogits   : rows x vocab of dtype with stride ld_dlogits, or NULL for the
 *               forward pass alone; may be the logits themselves (same pointer
 *               and stride), which are then replaced by their gradient
 *   logp, token_loss : rows entries each; sums : 4 entries
 *   workspace : device, 16-byte aligned, star_loss_workspace_bytes(rows, 0) bytes
 * 0 <= clip_low <= 1, clip_high >= 0, kl_coef finite. */
STAR_API star_status_t star_policy_loss(const void *logits, star_dtype_t dtype, int64_t rows, int64_t vocab,
                                        int64_t ld, const int64_t *labels, const float *weights,
                                        const float *advantages, const float *old_logp,
                                        const float *ref_logp, float temperature, float clip_low,
                                        float clip_high, float kl_coef, float *logp, float *token_loss,
                                        float *sums, void *dlogits, int64_t ld_dlogits, void *workspace,
                                        size_t workspace_bytes, void *cuda_stream);

/* Preference loss on pairs of sequences (paired log ratios), forward and
 * backward.  Rows seq_offsets[s] .. seq_offsets[s + 1] are sequence s; sequence
 * 2 i is pair i's chosen answer, 2 i + 1 its rejected one.  With L_s the sum of
 * logp over the active rows of sequence s, divided by their number if average
 * != 0 (an empty sequence has L = 0), and ref_s = ref_seq_logp[s] (0 if NULL):
 *     h    = (L_2i - L_2i+1) - (ref_2i - ref_2i+1),   margin[i] = beta h
 *     pair_loss[i] = -(1 - e) log sigmoid(beta h) - e log sigmoid(-beta h),   e = label_smoothing
 *     loss[0] = loss_scale * sum_i pair_loss[i]
 * and dlogits is the gradient of loss[0] (rows x vocab, as for the policy loss;
 * NULL: forward alone; may be the logits themselves).  Rows outside every
 * sequence are inactive.
 *   seq_offsets : DEVICE, 2 pairs + 1 entries, ascending, in [0, rows].  It is
 *                 not read on the host; entries are clamped to [0, rows], so
 *                 that a wrong array gives wrong results but no access outside
 *                 the buffers
 *   seq_logp    : 2 pairs entries (L_s);  pair_loss, margin : pairs entries
 *   workspace   : star_loss_workspace_bytes(rows, 2 * pairs) bytes, 16-byte aligned
 * beta and loss_scale finite, 0 <= label_smoothing <= 1. */
STAR_API star_status_t star_preference_loss(const void *logits, star_dtype_t dtype, int64_t rows,
                                            int64_t vocab, int64_t ld, const int64_t *labels,
                                            const int32_t *seq_offsets, int64_t pairs,
                                            const float *ref_seq_logp, float temperature, float beta,
                                            float label_smoothing, int average, float loss_scale,
                                            float *seq_logp, float *pair_loss, float *margin, float *loss,
                                            void *dlogits, int64_t ld_dlogits, void *workspace,
                                            size_t workspace_bytes, void *cuda_stream);

/* Activations kept in 8 bits.  A checkpoint of x (rows x cols) holds, for every
 * block of 32 consecutive columns of a row (the last block of a row may be
 * shorter), a scale 2^e and a code per element,
 *     e    = the smallest integer >= -126 for which every code of the block is
 *            within -127 .. 127
 *     code = round(x / 2^e)   nearest, ties to even;     value = code * 2^e
 * so a value is off by at most half a step, 1/127 of the block's largest
 * magnitude at worst and 1/254 at best, and stands exactly in bf16 and fp32: whoever
 * reads it, the tensor cores included, rounds nothing further.  A block that
 * holds a NaN, an infinity or a magnitude of 127.5 * 2^104 (2.6e33) or more has
 * codes 0 and the scale byte 255: all its values are NaN, so that an overflow
 * reaches the gradients as it would without the checkpoint.
 *   codes  : int8, row-major, `pitch` bytes from row to row: cols rounded up to a
 *            multiple of 16 (bytes past cols are 0).  16-byte aligned
 *   scales : bytes e + 127, four neighbouring blocks side by side for one row,
 *            then the next row: byte ((c / 128) * tall + t) * 4 + (c / 32) % 4 for
 *            element (t, c), tall = rows rounded up to a multiple of 64 (bytes of
 *            rows past `rows` and of blocks past cols are not used).  16-byte aligned
 * star_checkpoint_sizes gives pitch and the bytes of both (8.25 bits an element).
 * The calls below take up to 2^31 - 1 rows and 2^32 columns (STAR_ERR_UNSUPPORTED
 * beyond) and launch one kernel (pack, unpack and act_backward: one per 2^34
 * elements). */
STAR_API star_status_t star_checkpoint_sizes(int64_t rows, int64_t cols, int64_t *pitch_out,
                                             size_t *code_bytes_out, size_t *scale_bytes_out);

/* Elementwise activations.  GELU_TANH is the tanh form (GPT-2),
 * 0.5 x (1 + tanh(sqrt(2 / pi) (x + 0.044715 x^3))); GELU_ERF is x Phi(x) (BERT);
 * SILU is x / (1 + exp(-x)). */
typedef enum {
    STAR_ACT_NONE = 0,
    STAR_ACT_GELU_TANH = 1,
    STAR_ACT_GELU_ERF = 2,
    STAR_ACT_SILU = 3
} star_activation_t;

/* Forward pass: keeps x (rows x cols of dtype, stride ld) in codes and scales
 * and, where act_out is given, writes act(x) to it in the same pass over x
 * (rows x cols of dtype, stride ld_act; the activation of x itself, not of its
 * kept value; may be x: same pointer and stride). */
STAR_API star_status_t star_checkpoint_pack(int8_t *codes, uint8_t *scales, const void *x, star_dtype_t dtype,
                                            int64_t rows, int64_t cols, int64_t ld, star_activation_t act,
                                            void *act_out, int64_t ld_act, void *cuda_stream);

/* out = act(value) for every kept value (STAR_ACT_NONE: the value itself,
 * exact).  out: rows x cols of dtype, stride ld. */
STAR_API star_status_t star_checkpoint_unpack(void *out, star_dtype_t dtype, int64_t ld, const int8_t *codes,
                                              const uint8_t *scales, int64_t rows, int64_t cols,
                                              star_activation_t act, void *cuda_stream);

/* Backward pass of an activation whose input was kept: dx = dy * act'(value).
 * dx, dy: rows x cols of dtype; dx may be dy (same pointer and stride). */
STAR_API star_status_t star_checkpoint_act_backward(void *dx, int64_t ld_dx, const void *dy, int64_t ld_dy,
                                                    star_dtype_t dtype, const int8_t *codes,
                                                    const uint8_t *scales, int64_t rows, int64_t cols,
                                                    star_activation_t act, void *cuda_stream);

/* Weight gradient of a linear layer whose input was kept:
 *     dw[o][c] = sum_t dy[t][o] * value[t][c]       (+ dw[o][c] before, if accumulate != 0)
 *   dy : rows x outs of dy_dtype, stride ld_dy
 *   dw : dw_dtype, outs x cols with stride ld_dw; with transposed != 0 it is
 *        stored as cols x outs (the layout of a layer y = x W with W[in][out]).
 *        Usually the worker's gradient buffer that a round reads
 * rows == 0 gives zeros (or leaves dw, when accumulating).  cols and outs up to
 * 4194240, rows below 2^31 - 256 (STAR_ERR_UNSUPPORTED beyond). */
STAR_API star_status_t star_checkpoint_weight_grad(void *dw, star_dtype_t dw_dtype, int64_t ld_dw, int transposed,
                                                   const void *dy, star_dtype_t dy_dtype, int64_t ld_dy,
                                                   const int8_t *codes, const uint8_t *scales, int64_t rows,
                                                   int64_t cols, int64_t outs, int accumulate,
                                                   void *cuda_stream);

/* The policy loss and the weight gradient wait inside their kernels for copies
 * that they have started.  Every such wait is bounded; one that runs out (a third
 * of a second at the earliest, as long as the hardware holds its attempts at the
 * latest; a fault of the device or its memory) ends the kernel without a valid
 * result: the policy loss's sums are NaN.  star_check_waits waits for cuda_stream
 * and says whether that has happened on the current device since the last check:
 * STAR_ERR_TIMEOUT, or STAR_OK.  Not inside a stream capture. */
STAR_API star_status_t star_check_waits(void *cuda_stream);

/* The attempts of every such wait in launches made after this call, by any thread:
 * 2^24 (what more is taken for) unless set, not negative.  With 0 each wait has run
 * out at once and a call whose kernel waits ends without a result, which is how a
 * program's answer to STAR_ERR_TIMEOUT is tried out; what a kernel has in flight it
 * waits for all the same. */
STAR_API star_status_t star_set_wait_attempts(int attempts);

/* ---------------------------------------------------------------------------
 * Tensor-list round for callers that cannot allocate device memory.
 *
 * The paper has no counterpart to this entry point; it exists for integration.
 * Some callers of this library are not in a position to call cudaMalloc or to
 * obtain a workspace from an allocator: a plug-in that runs inside another
 * framework's step after that framework's pool has taken all free device
 * memory, a hook on a latency-critical path where cudaMalloc's device-wide
 * synchronization is not acceptable, or early start-up code that runs before
 * any allocator exists.  For them the pointer table and tile map that
 * star_multi_prepare would place in a caller workspace live in a fixed array of
 * STAR_STATIC_SCRATCH_BYTES inside the library's device image (each GPU that
 * loads the library holds that much until the process exits).
 *
 * The call does the work of star_multi_prepare followed by
 * star_group_update_multi: arguments have the same meaning as there, and the
 * results are identical.  It calls no cudaMalloc, cudaFree or other allocating
 * routine.  Differences to know about:
 *   - Size limit: a list whose table needs more than STAR_STATIC_SCRATCH_BYTES
 *     (see star_multi_workspace_bytes) is rejected with
 *     STAR_ERR_WORKSPACE_TOO_SMALL and nothing is launched.  1 MiB covers, for
 *     example, 292 tensors / 355 M elements / 16 workers (about 0.75 MiB).
 *   - The first call on each device looks up the array's device address (with
 *     that device current).
 *   - The call cannot be part of a stream capture, first call or not: the table
 *     is copied from host memory that is released on return, which a captured
 *     graph would read again at every replay.  When cuda_stream is capturing
 *     the call returns STAR_ERR_UNSUPPORTED and enqueues nothing.
 *   - All calls on a device share the one array, and it keeps the previous
 *     call's table; each call rewrites the part it uses before its kernel
 *     reads it, so nothing has to start out zeroed.  Calls on one stream are
 *     ordered and safe.  Calls that can overlap on the GPU (different streams
 *     without a dependency, or several host threads) race on the array: the
 *     caller must serialize them.
 *   - The table is rebuilt and copied (one cudaMemcpyAsync from pageable host
 *     memory) on every call.  That copy makes the host wait until the work
 *     queued earlier on cuda_stream, the previous round included, has finished:
 *     the call does not run ahead of the GPU.  Callers that can provide a
 *     workspace should prepare once and use star_group_update_multi.
 * ------------------------------------------------------------------------- */
#define STAR_STATIC_SCRATCH_BYTES (1u << 20)

STAR_API star_status_t star_group_update_multi_noalloc(
    int n_tensors, float *const *params, float *const *momentum, const void *const *grads,
    const int64_t *sizes, int W, star_dtype_t grad_dtype, const int32_t *group_offsets,
    const int32_t *group_members, int n_groups, float lr, float mu, float wd, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* STAR_H_ */
