/*
 * cpeval -- batched evaluation of the weighted critical path of a data-flow DAG
 * under many candidate device partitions, on one AMD MI355X (gfx950).
 *
 * Model (paper, section 2): a DAG G=(V,E) with n vertices and m edges, vertex
 * complexity c(v) >= 0, edge volume t(e) >= 0, k devices of speed s[i] >= 1 and a
 * k x k bandwidth matrix B (row = device of the edge's source vertex, column =
 * device of its target; the diagonal is never read).  A partition p: V -> D is
 * one row of `assignments`.  Costs are integer ticks, each term rounded up on
 * its own:
 *
 *   w(v)  = ceil(c(v) / s[p(v)])                             (section 2: time = complexity / speed)
 *   x(e)  = 0 if p(u) == p(v), else ceil(t(e) / B[p(u)][p(v)])   for e = (u -> v)   (section 4.1)
 *   b(v)  = w(v) + max over out-edges (x(e) + b(head)), empty max = 0
 *           (section 4.1, the PCT equation; a sink's value is its own execution time)
 *   tl(v) = max over in-edges (tl(tail) + w(tail) + x(e)), empty max = 0
 *           (section 3.2, the downward rank without the vertex's own term)
 *   CP    = max_v b(v)     (section 2: the start time of a zero-cost final sink
 *                           joined to every sink by zero-cost edges)
 *   mask(v) = [tl(v) + b(v) == CP]    (the union of all critical paths, section 3.2.2)
 *
 * Multi-edges are allowed (the costlier one decides), c = 0 and t = 0 are allowed,
 * m = 0 is allowed.  B need not be symmetric.
 *
 * Calling convention: plain C, no exceptions, no aborts.  Every function returns
 * CP_OK (0) or a negative CP_ERR_* code.  "host" pointers are ordinary memory that
 * is only read during the call; "device" pointers are HIP device memory owned by
 * the caller.  The library never allocates or frees device memory.  `stream` is
 * a hipStream_t passed as void* (NULL = the default stream).
 */
#ifndef CPEVAL_H
#define CPEVAL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- error codes (return values) ---- */
#define CP_OK              0
#define CP_ERR_NULL       (-1)   /* a required pointer is NULL */
#define CP_ERR_SIZE       (-2)   /* n < 1, m < 0, L < 1, batch < 1, k < 1 or k > 255 */
#define CP_ERR_CSR        (-3)   /* non-monotone ptr, index out of range, succ/pred mismatch */
#define CP_ERR_LEVELS     (-4)   /* level index is not a partition of V, or an edge does not go to a higher level */
#define CP_ERR_NEGATIVE   (-5)   /* c(v) < 0 or t(e) < 0 */
#define CP_ERR_SPEED      (-6)   /* s[i] < 1 */
#define CP_ERR_BANDWIDTH  (-7)   /* off-diagonal B[i][j] < 1 */
#define CP_ERR_OVERFLOW   (-8)   /* longest raw path >= 2^62, or 32-bit ticks asked for but not provably safe */
#define CP_ERR_WORKSPACE  (-9)   /* workspace or blob too small or misaligned */
#define CP_ERR_HIP        (-10)  /* a HIP runtime call failed */
#define CP_ERR_STATE      (-11)  /* graph not uploaded yet, or profile slot out of range */
#define CP_ERR_ARG        (-12)  /* unknown enum value, or an output requested without the outputs it depends on */
#define CP_ERR_ALLOC      (-13)  /* host allocation failed */

/* ---- value written to *status_out by the device ---- */
#define CP_STATUS_OK             0
#define CP_STATUS_BAD_DEVICE_ID  1   /* some assignments entry is >= k: the call's outputs are meaningless
                                        (the entry was replaced by a valid device so that no access leaves its table) */
#define CP_STATUS_BAD_CONSTRAINT  4   /* cp_validate: a constraint names a vertex >= n or a device >= k; it was skipped */
#define CP_STATUS_B_OUT_OF_RANGE 2   /* cp_pct_order: some b lies outside [0, max_b]: the order is meaningless;
                                        status values are bit flags and may be or-ed */
#define CP_STATUS_BAD_TIE        8   /* cp_simulate: tie is not a permutation of 0 .. n-1: nothing was simulated */
#define CP_STATUS_INCOMPLETE     16  /* cp_simulate: a partition ended with vertices that never started (cannot
                                        happen on a graph that cp_graph_create accepted) */
#define CP_STATUS_BAD_TOKEN      32  /* cp_token_logprobs: a token >= vocab; it counts as one that is to be ignored */
#define CP_STATUS_BAD_SEQUENCE   64  /* cp_recurrence: seq_ptr does not rise from 0 to rows: the outputs are meaningless */
#define CP_STATUS_BAD_SLOT       128 /* cp_recurrence_step: a slot >= num_slots; its row was left out */
#define CP_STATUS_BAD_SAMPLING   256 /* cp_token_sample: a row's own setting is out of range: the row got no tokens */

/* ---- enums ---- */
#define CP_TICK_I32  4   /* b-level / t-level stored as int32 (only if the graph's bound allows) */
#define CP_TICK_I64  8   /* stored as int64 */

#define CP_ASSIGN_PARTITION_MAJOR 0   /* assignments[batch][n] */
#define CP_ASSIGN_VERTEX_MAJOR    1   /* assignments[n][batch] */

/* Layout of the per-vertex outputs.  Vertex-major suits consumers that look at one
 * vertex across partitions (and is what the wave-column plan produces natively);
 * partition-major gives every partition one contiguous row (what the resident-window
 * plan, the priority lists and the critical-path walk work on natively).  Every plan
 * honours either choice. */
#define CP_OUT_VERTEX_MAJOR       0   /* b, tl [n][batch]; mask [n][ceil(batch/64)], bit = partition */
#define CP_OUT_PARTITION_MAJOR    1   /* b, tl [batch][n]; mask [batch][ceil(n/64)], bit = vertex */

#define CP_PLAN_AUTO             0
#define CP_PLAN_WAVE_COLUMN      1   /* one wavefront = one vertex x 64 partitions; one launch per level */
#define CP_PLAN_RESIDENT_WINDOW  2   /* one workgroup = one partition; recent levels kept in LDS; one launch per sweep, or
                                        one for both sweeps where a workgroup of each fits a compute unit side by side
                                        or all workgroups of both sweeps find room on the chip at once */
#define CP_PLAN_SHARED_WINDOW_2  3   /* as 2, but one workgroup = 2 partitions behind one graph stream */
#define CP_PLAN_SHARED_WINDOW_4  4   /* ... 4 partitions */
#define CP_PLAN_STREAMED_WINDOW  6   /* as 2, but the compute wavefronts fetch the graph themselves, two ticks ahead, into
                                        registers; LDS holds only what depends on the partition */
#define CP_PLAN_LANE_WINDOW      7   /* as 2, but one workgroup = 4 or 8 partitions in the lanes of its wavefronts, both
                                        sweeps in one launch; CP_PLAN_AUTO takes it in place of the plan it resolves to
                                        where it is faster for the call (see cp_eval_choose_plan) */
#define CP_PLAN_COLUMN_SLICE     5   /* the wave-column layout, but one persistent workgroup owns 64 partitions and
                                        walks all levels in one launch per sweep (never chosen by CP_PLAN_AUTO) */
#define CP_PLAN_CHAIN            8   /* only told by cp_profile_plan, never accepted: what CP_PLAN_AUTO may run for up to 64
                                        partitions of a graph of many levels.  One workgroup = one sweep of one partition,
                                        behind a launch that writes what every edge costs under it */
#define CP_PLAN_WHOLE            9   /* only told by cp_profile_plan as well: CP_PLAN_AUTO's way with small graphs.  One workgroup =
                                        4 or 8 partitions, all values in LDS; a call is one launch, or two */

/* stages of one cp_eval call, in the order they run; also the index into cp_profile_read's output */
#define CP_STAGE_PREP    0   /* clear outputs, cost tables, assignment transpose */
#define CP_STAGE_BLEVEL  1   /* b-level sweep, last level to first */
#define CP_STAGE_CP      2   /* critical-path length per partition */
#define CP_STAGE_TLEVEL  3   /* t-level sweep, first level to last */
#define CP_STAGE_MASK    4   /* critical-vertex mask */
#define CP_NUM_STAGES    5

typedef struct cp_graph cp_graph;
typedef struct cp_profile cp_profile;

typedef struct cp_graph_info {
    int32_t n, L;
    int64_t m;
    int32_t max_out_degree, max_in_degree, max_level_width;
    int32_t num_sources, num_sinks;
    int64_t max_c, max_t;
    int64_t raw_path_bound;      /* U0: longest path with w = c and x = t; every tick value is <= U0 */
    int32_t min_tick_bytes;      /* 4 if U0 < 2^31, else 8 */
    int32_t window_ok;           /* 1 if the resident-window plan can run this graph */
    int32_t window_slots_b;      /* LDS slots the b-level sweep needs under that plan */
    int32_t window_slots_t;      /* ... and the t-level sweep */
    int32_t window_packet_bytes_b;   /* largest per-level packet of that plan, b-level sweep */
    int32_t window_packet_bytes_t;   /* ... and t-level sweep */
    int32_t window_far_b;        /* far reads per tick of that plan's b-level sweep (neighbours too far back for the
                                    LDS ring are read from the output array); 0 = none */
    int32_t window_far_t;        /* ... and t-level sweep */
    int32_t window_ticks_b;      /* barriers of that plan's b-level sweep: a level is cut into ticks of at most 8 slices
                                    of 64 vertices */
    int32_t window_ticks_t;      /* ... and t-level sweep */
    int32_t window_slices_b;     /* slices of the widest tick, b-level sweep */
    int32_t window_slices_t;     /* ... and t-level sweep */
    int32_t auto_plan;           /* plan CP_PLAN_AUTO resolves to for a batch of 256, in cp_eval_choose_plan's sense (the
                                    choice is made per call) */
    int32_t uploaded;            /* 1 after cp_graph_upload */
    uint64_t blob_bytes;
} cp_graph_info;

/*
 * Validate a graph and pack it (host work only; no GPU is touched).
 *
 *   succ_ptr[n+1], succ_idx[m], succ_t[m]   successor CSR: out-edges of v are
 *       succ_ptr[v] .. succ_ptr[v+1]-1, succ_idx = head vertex, succ_t = t(e)
 *   pred_ptr[n+1], pred_idx[m], pred_eid[m] predecessor CSR: pred_idx = tail vertex,
 *       pred_eid = position of the same edge in the successor arrays
 *   c[n]                                    vertex complexity
 *   level_ptr[L+1], level_vtx[n]            vertices grouped by topological level;
 *       any grouping in which every edge goes to a strictly higher level is accepted
 *
 * All arrays are host memory, borrowed for the call.  succ_idx, succ_t, pred_idx,
 * pred_eid may be NULL when m == 0.  On success *out owns a host object to be
 * released with cp_graph_destroy.
 * Errors: CP_ERR_NULL, CP_ERR_SIZE, CP_ERR_CSR, CP_ERR_LEVELS, CP_ERR_NEGATIVE,
 * CP_ERR_OVERFLOW (longest raw path >= 2^62), CP_ERR_ALLOC.
 */
int cp_graph_create(int32_t n, int64_t m, int32_t L,
                    const int32_t *succ_ptr, const int32_t *succ_idx, const int64_t *succ_t,
                    const int32_t *pred_ptr, const int32_t *pred_idx, const int32_t *pred_eid,
                    const int64_t *c,
                    const int32_t *level_ptr, const int32_t *level_vtx,
                    cp_graph **out);

/* Facts about a created graph. */
int cp_graph_get_info(const cp_graph *g, cp_graph_info *out);

/*
 * Copy the packed graph into caller-owned device memory (>= info.blob_bytes bytes,
 * 256-byte aligned) and wait for the copy.  The memory must stay valid and
 * unmodified until cp_graph_destroy.  Errors: CP_ERR_NULL, CP_ERR_WORKSPACE, CP_ERR_HIP.
 */
int cp_graph_upload(cp_graph *g, void *device_blob, size_t blob_bytes, void *stream);

/* Release the host object (the device blob stays the caller's).  NULL is accepted. */
void cp_graph_destroy(cp_graph *g);

/*
 * Bytes of device workspace cp_eval needs for this batch size, device count,
 * assignment layout, plan (CP_PLAN_AUTO allowed), output layout and tick type.
 * For up to 64 partitions of a graph of 256 levels or more CP_PLAN_AUTO also asks for what
 * CP_PLAN_CHAIN works on, 18 bytes or more a vertex and partition (36 where the volumes do not
 * keep every cost below 2^16) and never more than 512 MB: such a call may ask for more than one of
 * 65 partitions.  With less it runs all the same, in more rounds or under another plan, where
 * there is room for what that takes.
 */
int cp_eval_workspace_bytes(const cp_graph *g, int32_t batch, int32_t k, int assign_layout,
                            int plan, int out_layout, int tick_dtype, size_t *out_bytes);

/*
 * The plan CP_PLAN_AUTO resolves to for this batch and cost model on the current
 * device (a caller may want to know it to ask for the layout that plan produces
 * directly, or whether CP can be had without b).  Where the lane-window plan is faster for
 * the call at hand, which depends on its outputs, layouts and workspace, AUTO runs that one in
 * its place, with the same results and the same refusals: it is never the answer here, and
 * cp_profile_plan tells what a call ran; the same holds for CP_PLAN_CHAIN and CP_PLAN_WHOLE.  Errors: as cp_eval's argument checks.
 */
int cp_eval_choose_plan(const cp_graph *g, int32_t batch, int32_t k, const int64_t *speeds,
                        const int64_t *bandwidth, int tick_dtype, int *plan_out);

/*
 * Evaluate `batch` partitions.  Only enqueues work on `stream`; it does not wait (with more
 * than 64 devices the cost tables, up to 1 MB, go through eight pinned host buffers shared
 * by the process: the ninth such call in flight waits for the first to have copied its tables).
 *
 *   assignments   device, uint8, [batch][n] or [n][batch] per assign_layout; entries < k
 *   speeds        host, int64 [k], each >= 1
 *   bandwidth     host, int64 [k][k], row = source vertex's device; off-diagonal >= 1
 *   workspace     device, >= cp_eval_workspace_bytes, 256-byte aligned; contents are scratch.
 *                 Two calls that may overlap in time need distinct workspaces.
 *   cp_out        device int64 [batch], or NULL
 *   blevel_out    device ticks, or NULL.  CP_OUT_VERTEX_MAJOR: [n][batch], partition j of vertex v at
 *                 v*batch + j; CP_OUT_PARTITION_MAJOR: [batch][n], at j*n + v
 *   tlevel_out    device ticks, same shape, or NULL
 *   mask_out      device uint64, or NULL.  CP_OUT_VERTEX_MAJOR: [n][ceil(batch/64)], bit i of word w of
 *                 row v is partition 64w+i; CP_OUT_PARTITION_MAJOR: [batch][ceil(n/64)], bit i of word w
 *                 of row j is vertex 64w+i.  Bits past the last partition / vertex are 0.
 *   tick_dtype    CP_TICK_I32 or CP_TICK_I64: element type of blevel_out / tlevel_out
 *   out_layout    CP_OUT_VERTEX_MAJOR or CP_OUT_PARTITION_MAJOR
 *   plan          CP_PLAN_AUTO, or force one (CP_ERR_ARG if it cannot run this graph / cost model)
 *   status_out    device int32, required: CP_STATUS_* after the stream has drained
 *   profile       NULL, or a profile whose next slot receives this call's stage timestamps
 *
 * Dependencies between outputs: mask_out needs cp_out, blevel_out and tlevel_out; cp_out needs
 * blevel_out unless a window plan (2, 3, 4, 6) runs on a graph without far reads (info.window_far_b
 * == 0), or the lane-window plan is asked for by name: these keep a running maximum, so CP alone costs
 * no output traffic (CP_PLAN_AUTO goes by the plan that cp_eval_choose_plan names).  CP_ERR_ARG otherwise.
 * Errors: CP_ERR_NULL, CP_ERR_SIZE, CP_ERR_SPEED, CP_ERR_BANDWIDTH, CP_ERR_OVERFLOW
 * (CP_TICK_I32 with a bound >= 2^31), CP_ERR_WORKSPACE, CP_ERR_STATE, CP_ERR_ARG, CP_ERR_HIP.
 */
int cp_eval(const cp_graph *g, int32_t batch, int32_t k,
            const uint8_t *assignments, int assign_layout,
            const int64_t *speeds, const int64_t *bandwidth,
            void *workspace, size_t workspace_bytes, void *stream,
            int64_t *cp_out, void *blevel_out, void *tlevel_out, uint64_t *mask_out,
            int tick_dtype, int out_layout, int plan, int32_t *status_out, cp_profile *profile);

/*
 * cp_eval for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, results and errors as cp_eval without `workspace`, `workspace_bytes` and
 * `profile`.  The scratch memory is a fixed array of CP_STATIC_SCRATCH_BYTES bytes that is
 * part of the library's device code (every GPU the library runs on holds one until the
 * process ends), and the cost tables travel as kernel arguments, so the call allocates
 * nothing, copies nothing through the copy engine and records no memset.  (The array's
 * device address is looked up on the first call on a device; make that call outside a
 * capture.)
 *
 * Limits: k <= CP_STATIC_MAX_K (CP_ERR_SIZE) and a workspace need of at most
 * CP_STATIC_SCRATCH_BYTES (CP_ERR_WORKSPACE).  The need is the cost tables
 * ((2k^2 + k) * 8 bytes) plus, depending on how the call goes: n * batch bytes when the
 * wave-column plan reads partition-major assignments; 2 * n * batch ticks more when it
 * writes partition-major outputs; the device ids in sweep order (about n * batch bytes per
 * sweep) when the resident-window plan cannot read them straight from the caller's rows
 * (vertex-major assignments, rows not 16-byte aligned, or a graph whose levels are
 * scattered over the vertex numbers); the same and the copies of far reads for the lane-window plan, and
 * what every edge costs (8 to 20 bytes for up to four of a vertex and sweep) for CP_PLAN_CHAIN, which
 * CP_PLAN_AUTO runs on fewer partitions at a time, or leaves aside, where they do not fit.  A resident-window call on aligned partition-major
 * rows needs the tables only.
 *
 * All calls on one GPU share that GPU's array: calls that may overlap in time on one GPU
 * (different streams or threads) race; serialise them or use cp_eval with distinct
 * workspaces.  Nothing in the array has to survive between calls.
 */
#define CP_STATIC_SCRATCH_BYTES (32u << 20)
#define CP_STATIC_MAX_K         64
int cp_eval_static(const cp_graph *g, int32_t batch, int32_t k,
                   const uint8_t *assignments, int assign_layout,
                   const int64_t *speeds, const int64_t *bandwidth, void *stream,
                   int64_t *cp_out, void *blevel_out, void *tlevel_out, uint64_t *mask_out,
                   int tick_dtype, int out_layout, int plan, int32_t *status_out);

/*
 * One critical path per partition (paper, section 3.2.2 "compute the critical path";
 * the paper leaves ties open).  Among all source-to-sink paths whose cost equals CP the
 * one with the lexicographically smallest vertex sequence is returned: it starts at the
 * lowest-numbered vertex without predecessors whose b-level equals CP and always moves
 * to the lowest-numbered successor u of v with b(v) = w(v) + x(v->u) + b(u).
 * Only enqueues work on `stream`.
 *
 *   assignments, assign_layout, speeds, bandwidth   as for cp_eval (same values as the
 *                 call that produced blevel and cp)
 *   blevel        device ticks laid out per b_layout (CP_OUT_*), cp device int64 [batch]: outputs of cp_eval
 *   workspace     device, 256-byte aligned, >= the 12 k (2 k + 1) bytes, rounded up to 256, of the tables, which
 *                 cp_eval_workspace_bytes never falls short of.  Graphs of 256 levels and more, of up to 1,024 vertices
 *                 each and up to five edges a vertex, are walked faster, with the same result, where it holds 64 bytes
 *                 a vertex behind them (fewer than 32 partitions: where vertices and edges are few enough to repay
 *                 writing these); a larger workspace may be handed over
 *   max_len       row length of path_out, >= the graph's number of levels L
 *   path_out      device int32 [batch][max_len]; unused tail = -1
 *   len_out       device int32 [batch]: vertices on the path
 *   status_out    device int32, as for cp_eval
 * Errors: CP_ERR_NULL, CP_ERR_SIZE (also max_len < L), CP_ERR_ARG, CP_ERR_STATE,
 * CP_ERR_OVERFLOW, CP_ERR_WORKSPACE, CP_ERR_SPEED, CP_ERR_BANDWIDTH, CP_ERR_HIP.
 */
int cp_critical_path(const cp_graph *g, int32_t batch, int32_t k,
                     const uint8_t *assignments, int assign_layout,
                     const int64_t *speeds, const int64_t *bandwidth,
                     const void *blevel, const int64_t *cp, int tick_dtype, int b_layout,
                     void *workspace, size_t workspace_bytes, void *stream,
                     int32_t max_len, int32_t *path_out, int32_t *len_out, int32_t *status_out);

/*
 * PCT priority lists (paper, section 4.1: every device runs, among its executable
 * vertices, the one with the highest PCT; PCT is computed once after partitioning and
 * the schedule is reused).  Per partition, the static priority list of every device:
 * its vertices by descending PCT = b, equal values by ascending vertex number.
 * order_out[j] lists the vertices of device 0, then of device 1, ...;
 * seg_out[j][d] .. seg_out[j][d+1] is device d's range.  Only enqueues work on `stream`.
 *
 *   assignments, assign_layout   as for cp_eval
 *   blevel      device ticks laid out per b_layout (CP_OUT_*): output of cp_eval for these assignments
 *   max_b       an upper bound on every b (for instance the largest CP of the batch); 0 = the
 *               graph's raw path bound.  A tighter bound means fewer sorting passes.  A b
 *               outside [0, max_b] sets CP_STATUS_B_OUT_OF_RANGE.
 *   workspace   device, 256-byte aligned, >= cp_pct_order_workspace_bytes (same batch, k, max_b)
 *   order_out   device int32 [batch][n]
 *   seg_out     device int32 [batch][k+1]
 *   status_out  device int32: CP_STATUS_* flags after the stream has drained
 * Errors: CP_ERR_NULL, CP_ERR_SIZE (also batch * ceil(n / 4096) >= 2^31), CP_ERR_ARG
 * (max_b < 0), CP_ERR_STATE, CP_ERR_OVERFLOW (device bits + bits of max_b > 64, or 32-bit
 * ticks asked for a graph that needs 64), CP_ERR_WORKSPACE, CP_ERR_HIP.
 */
int cp_pct_order_workspace_bytes(const cp_graph *g, int32_t batch, int32_t k, int64_t max_b,
                                 size_t *out_bytes);
int cp_pct_order(const cp_graph *g, int32_t batch, int32_t k,
                 const uint8_t *assignments, int assign_layout,
                 const void *blevel, int tick_dtype, int b_layout, int64_t max_b,
                 void *workspace, size_t workspace_bytes, void *stream,
                 int32_t *order_out, int32_t *seg_out, int32_t *status_out);

/*
 * Validity of `batch` partitions under the placement constraints of the problem
 * statement (paper, section 2, the collocation and the device constraint equations):
 * every collocation pair (v_i, v_j) must share a device, every device constraint
 * (v_i, d_j) must have p(v_i) = d_j.  Needs no graph.  Only enqueues work on `stream`.
 *
 *   n, k          vertices, devices
 *   assignments   device uint8, laid out per assign_layout (CP_ASSIGN_*)
 *   pairs         device int32 [num_pairs][2]; may be NULL when num_pairs = 0
 *   pins          device int32 [num_pins][2] = {vertex, device}; may be NULL when num_pins = 0
 *   valid_out     device uint8 [batch]: 1 if the partition meets every constraint
 *   violations_out  device int32 [batch] or NULL: constraints the partition breaks
 *   status_out    device int32: CP_STATUS_BAD_CONSTRAINT if an index is out of range
 * Errors: CP_ERR_NULL, CP_ERR_SIZE (n < 1, batch < 1, k < 1 or > 255, a negative count), CP_ERR_ARG, CP_ERR_HIP.
 */
int cp_validate(int32_t n, int32_t batch, int32_t k, const uint8_t *assignments, int assign_layout,
                int64_t num_pairs, const int32_t *pairs, int64_t num_pins, const int32_t *pins,
                void *stream, uint8_t *valid_out, int32_t *violations_out, int32_t *status_out);

/* ---- scheduling policies of cp_simulate ---- */
#define CP_POLICY_FIFO 0   /* the vertex that became executable first (paper, section 5.1) */
#define CP_POLICY_PCT  1   /* the vertex with the largest path computation time b (paper, section 4.1) */

/*
 * List-scheduling simulation of one iteration under each of `batch` partitions: the
 * execution time the paper's evaluation plots (section 5).  The scheduling criteria of
 * section 4 are read as follows, in the integer ticks of cp_eval:
 *   - a device runs its own vertices one at a time, without interruption, w(v) ticks each;
 *   - the tensor of an edge (u -> v) is at v's device x(u -> v) ticks after u finishes;
 *     transfers occupy no device and do not compete (section 2 models a rate per device
 *     pair and nothing else);
 *   - v is executable once all its input tensors are there (time 0 without inputs);
 *   - a free device that owns an executable vertex starts one at once, otherwise it waits
 *     for the first of its vertices to become executable;
 *   - CP_POLICY_FIFO takes the vertex that became executable first; among equals the paper
 *     draws at random, here the caller passes the draw: the smaller tie[v] wins;
 *     CP_POLICY_PCT takes the largest b(v), the smaller vertex number among equals.
 * Every vertex must cost at least one tick (c(v) >= 1 for all v, else CP_ERR_ARG): then
 * devices that decide at the same time cannot influence each other and the schedule is
 * unique.  All times must stay below 2^31: the summed execution times on the slowest device plus
 * the longest chain of transfers (bounded by the graph's raw path bound and by L - 1 transfers
 * at the lowest rate), which no makespan exceeds, else CP_ERR_OVERFLOW.
 * One wavefront simulates one partition, one lane per device: k <= 64.
 * Only enqueues work on `stream`.
 *
 *   assignments   device uint8, laid out per assign_layout (CP_ASSIGN_*)
 *   speeds, bandwidth  host, as for cp_eval
 *   policy        CP_POLICY_*
 *   blevel        CP_POLICY_PCT: device ticks as cp_eval wrote them for these assignments
 *                 (tick_dtype, b_layout = CP_OUT_*); values outside [0, 2^31) set
 *                 CP_STATUS_B_OUT_OF_RANGE.  Ignored (may be NULL) under CP_POLICY_FIFO.
 *   tie           CP_POLICY_FIFO: device int32 [n], a permutation of 0 .. n-1 (else
 *                 CP_STATUS_BAD_TIE and makespan -1), or NULL for tie[v] = v.  Ignored under PCT.
 *   workspace     device, 256-byte aligned, >= cp_simulate_workspace_bytes (28 bytes per
 *                 vertex and partition under PCT, 20 under FIFO, plus the cost tables)
 *   makespan_out  device int64 [batch]: the largest finish time; -1 for a partition with a
 *                 device id >= k (CP_STATUS_BAD_DEVICE_ID)
 *   start_out     device int32 [batch][n] (partition-major) or NULL: start time of every vertex
 *   status_out    device int32: CP_STATUS_* flags after the stream has drained
 * Errors: CP_ERR_NULL, CP_ERR_SIZE (k > 64), CP_ERR_ARG, CP_ERR_STATE, CP_ERR_SPEED,
 * CP_ERR_BANDWIDTH, CP_ERR_OVERFLOW, CP_ERR_WORKSPACE, CP_ERR_ALLOC, CP_ERR_HIP.
 */
int cp_simulate_workspace_bytes(const cp_graph *g, int32_t batch, int32_t k, int policy, int with_tie,
                                size_t *out_bytes);
int cp_simulate(const cp_graph *g, int32_t batch, int32_t k,
                const uint8_t *assignments, int assign_layout,
                const int64_t *speeds, const int64_t *bandwidth, int policy,
                const void *blevel, int tick_dtype, int b_layout, const int32_t *tie,
                void *workspace, size_t workspace_bytes, void *stream,
                int64_t *makespan_out, int32_t *start_out, int32_t *status_out);

/*
 * The paper's Critical Path partitioning strategy (section 3.2.2), e.g. as the start of
 * cp_search: the critical path of the ranks (vertex cost c, no devices, no transfers;
 * section 3.2's rank equations) goes to the fastest device (largest s, lowest number on
 * ties); every other vertex, in increasing vertex number, goes to the device d with the
 * smallest load(d) + ceil(c(v) / s[d]) (lowest number on ties), load(d) being the summed
 * execution times of the vertices already on d, the path included (the strategy's load
 * equation in integer ticks).  Memory capacities are not modelled.  The load rule is a
 * chain of n dependent choices on one wavefront: 0.037 microseconds a vertex with 16 devices or fewer, 0.046 with up
 * to 32 and 0.067 with up to 64; about twice that where 64 vertices may part the loads by more than 28, 27 or 26 bits,
 * 0.30 to 0.38 from 32 bits on, and 0.46 to 0.54 where c or speeds have no multiply-shift constants (cp_cost_magic).
 * Only enqueues work on `stream`.
 *
 *   k <= 64, speeds host int64 [k]
 *   workspace       device, 256-byte aligned, >= cp_seed_workspace_bytes
 *   assignment_out  device uint8 [n]
 *   status_out      device int32 (CP_STATUS_OK unless the inner evaluation reports otherwise)
 * Errors: CP_ERR_NULL, CP_ERR_SIZE (k < 1 or k > 64), CP_ERR_STATE, CP_ERR_WORKSPACE,
 * CP_ERR_SPEED, CP_ERR_HIP.
 */
int cp_seed_workspace_bytes(const cp_graph *g, size_t *out_bytes);
int cp_seed_partition(const cp_graph *g, int32_t k, const int64_t *speeds, void *workspace, size_t workspace_bytes,
                      void *stream, uint8_t *assignment_out, int32_t *status_out);

/*
 * Critical-path move search: a descent over partitions built from the paper's own
 * pieces.  Section 3.2 places the critical path first because it decides the running
 * time; here, from a start partition, every single move of a vertex of the current
 * critical path (cp_critical_path's path) to another device is a candidate; candidate
 * number i * (k-1) + r moves path vertex number i to the r-th device other than its own.
 * Every candidate's CP is what cp_eval would return for it (it is computed from both levels
 * of the current partition: only paths through the moved vertex change); candidates that break a
 * placement constraint (section 2, as in cp_validate) are left out; the candidate with
 * the smallest CP (lowest number on ties) is taken if it is smaller than the current CP,
 * and the step repeats; otherwise, or after max_moves moves, the search stops.
 * The call blocks: it waits on `stream` between steps.
 *
 *   assignment   device uint8 [n]: in the start partition, out the result
 *   pairs, pins  device, as for cp_validate (NULL with a count of 0)
 *   chunk        >= 1; has no effect on the result or the time (all candidates of a step are
 *                compared at once)
 *   workspace    device, 256-byte aligned, >= cp_search_workspace_bytes(g, k, chunk)
 *   cp_trace     host int64 [max_moves + 1]: CP of the start, then after each move
 *   moves        host int32 [max_moves][2] = {vertex, new device}, or NULL
 *   num_moves    host: moves made
 *   evaluated    host: candidates evaluated, or NULL
 * Errors: CP_ERR_NULL, CP_ERR_SIZE, CP_ERR_STATE, CP_ERR_WORKSPACE, CP_ERR_ARG (a device id
 * >= k in the start), CP_ERR_SPEED, CP_ERR_BANDWIDTH, CP_ERR_HIP.
 */
int cp_search_workspace_bytes(const cp_graph *g, int32_t k, int32_t chunk, size_t *out_bytes);
int cp_search(const cp_graph *g, int32_t k, const int64_t *speeds, const int64_t *bandwidth,
              uint8_t *assignment, int64_t num_pairs, const int32_t *pairs, int64_t num_pins,
              const int32_t *pins, int32_t max_moves, int32_t chunk, void *workspace, size_t workspace_bytes,
              void *stream, int64_t *cp_trace, int32_t *moves, int32_t *num_moves, int64_t *evaluated);

/*
 * The device-free ranks of section 3.2: upRank (equation for the upward rank), downRank
 * (equation for the downward rank) and totalRank = upRank + downRank (section 3.2.1).
 * Both rank equations add the vertex's own c, so upRank is the b-level and downRank the
 * t-level plus c of the evaluation with a single device of speed 1, which is how they
 * are computed: one cp_eval with batch = 1, k = 1, then one elementwise kernel.
 * Only enqueues work on `stream`.
 *
 *   workspace   device, 256-byte aligned, >= cp_ranks_workspace_bytes
 *   up_out, down_out, total_out   device int64 [n] each; any may be NULL, not all
 * Errors: CP_ERR_NULL, CP_ERR_STATE (graph not uploaded), CP_ERR_WORKSPACE, CP_ERR_HIP.
 */
int cp_ranks_workspace_bytes(const cp_graph *g, size_t *out_bytes);
int cp_ranks(const cp_graph *g, void *workspace, size_t workspace_bytes, void *stream,
             int64_t *up_out, int64_t *down_out, int64_t *total_out);

/*
 * ---- Operators of a learned placement policy ----
 *
 * A policy that learns where to place a graph's vertices reads them in topological order as a
 * sequence and gives each a row of logits over the devices; partitions are drawn from the rows,
 * cp_eval rates them, and the gradient of their log probabilities, weighted by the ratings,
 * trains the policy.  The entry points below are its sequence layers (cp_recurrence and
 * cp_linear_attention), the joint between its blocks (cp_norm_gate) and its head
 * (cp_token_logprobs), each with its gradient, and the draw of tokens from its rows
 * (cp_token_sample); the matrix products between them are left to the caller's library.
 *
 * Common to them: all arrays are device memory; matrices have rows of contiguous elements and
 * a distance ld between rows, in elements, at least the row's length.  Element types are
 * CP_TYPE_*; vectors of parameters, states and statistics are float where nothing else is said.
 * States, sums and statistics are formed in 32 bits or more and a result is rounded once, to its
 * type.  Results share no memory with inputs or with each other (CP_ERR_ARG) except where it is
 * said; the rows of slices of one buffer may lie between each other.  The calls only enqueue work
 * on `stream`, allocate nothing and record no memset or copy, so that they may be captured into a
 * graph; results do not depend on the order in which workgroups run.  Workspaces are scratch,
 * 256-byte aligned; two calls that may overlap in time need distinct ones.
 */
#define CP_TYPE_F32  0
#define CP_TYPE_BF16 1
#define CP_TYPE_F16  2

#define CP_RECURRENCE_CHUNK      128
#define CP_RECURRENCE_MAX_WIDTH  65536
#define CP_RECURRENCE_MAX_DISTANCE (1 << 24)   /* elements from a row to the next */
#define CP_RECURRENCE_MAX_PACKED 0x7ffffc00    /* sequences that seq_ptr can cut the rows into */

/*
 * Gated linear recurrence along `rows` rows of `width` channels, for each channel on its own:
 *     a_t = sigmoid(f_t + bias),   h_t = a_t h_{t-1} + (1 - a_t) x_t
 *
 *   num_seq, seq_ptr   the rows are cut into num_seq sequences: seq_ptr int32 [num_seq + 1], rising
 *                 from 0 to rows (sequences may be empty), or NULL: num_seq equal parts (rows is a
 *                 multiple of num_seq)
 *   type          CP_TYPE_* of f, x and h
 *   reverse       0: from each sequence's first row to its last, 1: from the last to the first
 *   bias          [width], or NULL (0)
 *   h0            [num_seq][width], the state that each sequence begins with, or NULL (0)
 *   h             [rows][width]
 *   last          [num_seq][width], the state that each sequence ends in (h0's where it is empty), or NULL
 *   carry         [ceil(rows / CP_RECURRENCE_CHUNK)][width] for the backward pass, or NULL
 *   status_out    device int32, required with seq_ptr: CP_STATUS_BAD_SEQUENCE after the stream has
 *                 drained where seq_ptr is not what it has to be (no access leaves the arrays)
 * Errors: CP_ERR_ARG (type, reverse), CP_ERR_SIZE (rows < 0 or >= 2^31, width, num_seq < 1 or, with
 * seq_ptr, above CP_RECURRENCE_MAX_PACKED, rows no multiple of num_seq without seq_ptr, a distance below
 * width or above CP_RECURRENCE_MAX_DISTANCE), CP_ERR_NULL, CP_ERR_WORKSPACE, CP_ERR_HIP.  An infinite
 * x or state makes its channel NaN from the next row to the sequence's end; nothing passes from one sequence
 * or channel to another.
 */
int cp_recurrence_workspace_bytes(int64_t rows, int32_t width, int backward, size_t *out_bytes);
int cp_recurrence(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse,
                  const void *f, int64_t ldf, const void *x, int64_t ldx, const float *bias, const float *h0,
                  void *h, int64_t ldh, float *last, float *carry, void *workspace, size_t workspace_bytes,
                  void *stream, int32_t *status_out);

/*
 * Gradient of cp_recurrence: dh [rows][width] and dlast [num_seq][width] (or NULL) are the gradients
 * of h and last; carry and the inputs are those of the forward call.  df, dx [rows][width] of the
 * element type; dbias [width] and dh0 [num_seq][width] float, or NULL.  h is not read: it is computed
 * again from the states in carry.  Errors as cp_recurrence's; carry is required from more than
 * CP_RECURRENCE_CHUNK rows on.
 */
int cp_recurrence_backward(int64_t rows, int32_t width, int32_t num_seq, const int32_t *seq_ptr, int type, int reverse,
                           const void *dh, int64_t lddh, const float *dlast, const void *f, int64_t ldf,
                           const void *x, int64_t ldx, const float *bias, const float *h0, const float *carry,
                           void *df, int64_t lddf, void *dx, int64_t lddx, float *dbias, float *dh0,
                           void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out);

/*
 * One more row of each of num_seq sequences: state [num_slots][width] is updated in place and
 * h [num_seq][width] gets the new states.  slots int32 [num_seq]: the state row of each sequence, all
 * different, or NULL (row i for sequence i); a negative slot leaves its sequence out (its h is 0).
 * h may take the place of f or x.
 * status_out: device int32, required with slots (CP_STATUS_BAD_SLOT).  Errors as cp_recurrence's.
 */
int cp_recurrence_step(int32_t num_seq, int32_t width, int type, const void *f, int64_t ldf, const void *x, int64_t ldx,
                       const float *bias, float *state, int32_t num_slots, const int32_t *slots, void *h, int64_t ldh,
                       void *stream, int32_t *status_out);

#define CP_ATTENTION_MAX_WIDTH 256
#define CP_ATTENTION_MAX_HEADS 1024
#define CP_ATTENTION_MAX_DISTANCE (1 << 28)            /* elements from a row to the next */
#define CP_ATTENTION_MAX_HEAD_DISTANCE (1ll << 40)     /* from a head to the next */

/*
 * Linear attention with a decay for each head, along `rows` rows of `heads` heads: the recurrence whose state
 * is a width_k x width_v matrix a head,
 *     S_t = exp(log_decay) S_{t-1} + k_t^T v_t,   o_t = scale q_t S_t
 *
 *   num_seq, seq_ptr   as cp_recurrence's, but seq_ptr may end before rows: the rows behind the last sequence
 *                 are not looked at and their results left as they were
 *   heads, kv_heads   k and v have kv_heads heads, heads / kv_heads neighbouring heads share one
 *   type          CP_TYPE_* of q, k, v and o
 *   reverse       as cp_recurrence's
 *   q, k          [rows][heads or kv_heads][width_k], ldq (ldk) elements from row to row and hdq (hdk) from head to head, in
 *                 either order of rows and heads; of inputs either may be 0 (one row or head for all)
 *   v, o          [rows][kv_heads or heads][width_v]
 *   log_decay     [heads], at most 0 (above it, or NaN, its head becomes NaN), or NULL (0: no decay)
 *   h0            [num_seq][heads][width_k][width_v], the state that each sequence begins with, or NULL (0)
 *   last          as h0, the state that each sequence ends in (h0's where it is empty), or NULL
 *   carry         [cp_linear_attention_carry_states][heads][width_k][width_v] for the backward pass, or NULL
 *   status_out    device int32, required with seq_ptr: CP_STATUS_BAD_SEQUENCE where seq_ptr does not rise from 0 to at most
 *                 rows (no access leaves the arrays)
 * Products of 16-bit elements are exact, and summed in 32 bits.  States, scores and rows on their way to a state enter products with all
 * 24 bits (against fp16 elements but for what is below 2^-23 of a product).  An infinity or a NaN
 * makes what follows from it, from its row to its sequence's end and in its head (or those that share it), infinite or NaN, and
 * nothing else.
 * Errors: CP_ERR_ARG (type, reverse), CP_ERR_SIZE (rows < 0 or >= 2^31, widths, heads, num_seq < 1, num_seq * heads of equal
 * parts above 2^28, rows no multiple of num_seq without seq_ptr, distances; results whose rows or heads overlap),
 * CP_ERR_NULL, CP_ERR_WORKSPACE, CP_ERR_HIP.
 */
int cp_linear_attention_workspace_bytes(int64_t rows, int32_t num_seq, int packed, int32_t heads, int32_t kv_heads, int32_t width_k,
                                        int32_t width_v, int backward, size_t *out_bytes);
int cp_linear_attention_carry_states(int64_t rows, int32_t num_seq, int packed, int32_t heads, int32_t width_k, int32_t width_v, int64_t *out_states);
int cp_linear_attention(int64_t rows, int32_t num_seq, const int32_t *seq_ptr, int32_t heads, int32_t kv_heads, int32_t width_k,
                        int32_t width_v, int type, int reverse, const void *q, int64_t ldq, int64_t hdq, const void *k, int64_t ldk,
                        int64_t hdk, const void *v, int64_t ldv, int64_t hdv, const float *log_decay, float scale, const float *h0, void *o,
                        int64_t ldo, int64_t hdo, float *last, float *carry, void *workspace, size_t workspace_bytes, void *stream,
                        int32_t *status_out);

/*
 * Gradient of cp_linear_attention: d_o (of o) and dlast (of last, or NULL) in; dq, dk, dv of the element type out, each with
 * its own distances; dlog_decay [heads] and dh0 (as h0) float, or NULL.  The inputs and carry are those of the forward call; carry is
 * required where cp_linear_attention_carry_states is above 0.  Gradients of shared heads are summed in 32 bits; those
 * of inputs given with a distance of 0 are not (the results have rows and heads of their own).
 */
int cp_linear_attention_backward(int64_t rows, int32_t num_seq, const int32_t *seq_ptr, int32_t heads, int32_t kv_heads, int32_t width_k,
                                 int32_t width_v, int type, int reverse, const void *d_o, int64_t lddo, int64_t hddo, const float *dlast,
                                 const void *q, int64_t ldq, int64_t hdq, const void *k, int64_t ldk, int64_t hdk, const void *v, int64_t ldv,
                                 int64_t hdv, const float *log_decay, float scale, const float *h0, const float *carry, void *dq, int64_t lddq,
                                 int64_t hddq, void *dk, int64_t lddk, int64_t hddk, void *dv, int64_t lddv, int64_t hddv, float *dlog_decay,
                                 float *dh0, void *workspace, size_t workspace_bytes, void *stream, int32_t *status_out);

/*
 * One more row of each of num_seq sequences: state [num_slots][heads][width_k][width_v] is updated in place and o gets the new rows.
 * slots as cp_recurrence_step's; o of a sequence that is left out is 0.
 */
int cp_linear_attention_step(int32_t num_seq, int32_t heads, int32_t kv_heads, int32_t width_k, int32_t width_v, int type, const void *q,
                             int64_t ldq, int64_t hdq, const void *k, int64_t ldk, int64_t hdk, const void *v, int64_t ldv, int64_t hdv,
                             const float *log_decay, float scale, float *state, int32_t num_slots, const int32_t *slots, void *o, int64_t ldo,
                             int64_t hdo, void *stream, int32_t *status_out);

#define CP_GATE_NONE     0   /* the gate as it is */
#define CP_GATE_SIGMOID  1
#define CP_GATE_SILU     2
#define CP_NORM_MAX_WIDTH 16384

/*
 * The joint between two blocks: the norm behind the block that gave y, its gate, the residual
 * stream x and the norm in front of the next block, row by row of `width` values:
 *     u = y / rms(y) * w_post,   r = x + scale * act(gate) * u,   z = r / rms(r) * w_pre
 * with rms(v) = sqrt(mean(v^2) + eps).  z is formed from r before it is rounded.
 *
 *   stream_type   of x and r: `type`, or CP_TYPE_F32
 *   type          of y, gate and z
 *   weight_type   of w_pre and w_post, [width]
 *   gate_act      CP_GATE_*
 *   y             NULL: no block yet, z is the norm of x (gate, w_post NULL; r may be)
 *   gate          NULL: 1;   w_post NULL: u = y
 *   stats         [2][rows] for the backward pass (1 / rms of y and of r), or NULL
 * r and z may each take the place of an input whose elements are as wide (its address and distance).
 * Errors: CP_ERR_ARG, CP_ERR_SIZE (rows < 0, width, a distance below width), CP_ERR_NULL, CP_ERR_HIP.
 */
int cp_norm_gate(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int gate_act,
                 const void *x, int64_t ldx, const void *y, int64_t ldy, const void *gate, int64_t ldg,
                 const void *w_pre, const void *w_post, float scale, float eps,
                 void *r, int64_t ldr, void *z, int64_t ldz, float *stats, void *stream);

/*
 * Gradient of cp_norm_gate: dr (of r, or NULL: 0) and dz (of z) in; dx, dy, dgate, dw_pre, dw_post out,
 * each of the type of what it is the gradient of; dy is required with y, the last three may be
 * NULL.  The inputs and stats are those of the forward call; workspace is needed for dw_pre and dw_post.
 * dx, dy and dgate may each take the place of an input, as cp_norm_gate's r and z.
 */
int cp_norm_gate_backward_workspace_bytes(int64_t rows, int32_t width, size_t *out_bytes);
int cp_norm_gate_backward(int64_t rows, int32_t width, int stream_type, int type, int weight_type, int gate_act,
                          const void *dr, int64_t lddr, const void *dz, int64_t lddz,
                          const void *x, int64_t ldx, const void *y, int64_t ldy, const void *gate, int64_t ldg,
                          const void *w_pre, const void *w_post, float scale, const float *stats,
                          void *dx, int64_t lddx, void *dy, int64_t lddy, void *dgate, int64_t lddg,
                          void *dw_pre, void *dw_post, void *workspace, size_t workspace_bytes, void *stream);

#define CP_TOKEN_U8  1
#define CP_TOKEN_I32 4
#define CP_TOKEN_I64 8
#define CP_LOGPROBS_MAX_VOCAB (1 << 26)
#define CP_LOGPROBS_MAX_TOP   64
#define CP_LOGPROBS_IN_PLACE  256
#define CP_LOGPROBS_MAX_GIVEN 0x7ffffc00   /* tokens of a row */

/*
 * Log probabilities of given tokens, with the rows' entropy and their best alternatives, under
 * softmax(scale * logits) over the allowed places of each row.
 *
 *   logits        [rows][vocab] of `type`; scale > 0 (1 / temperature), so that scale / ln 2 is a finite float
 *   allow         uint64 [rows][ceil(vocab / 64)], bit i of word w = place 64 w + i may be taken, or NULL
 *                 (all).  What lies at a place that may not is not looked at.
 *   given, tokens `given` tokens of each row, at most CP_LOGPROBS_MAX_GIVEN: token g of row i at i * token_row_stride + g * token_stride, of
 *                 CP_TOKEN_*.  cp_eval's assignments of a batch of partitions are such tokens, in either
 *                 layout.  A negative token is ignored: its logp is 0 and it has no gradient.
 *   logp          [rows][given]; -inf at a place that is not allowed
 *   entropy       [rows]
 *   stats         [rows][3] for the backward pass
 *   top           alternatives of each row, at most CP_LOGPROBS_MAX_TOP: top_idx int32 [rows][top], by falling
 *                 logit, equal ones by rising place, and top_logp; -1 and -inf where fewer have a probability
 *   status_out    device int32, required: CP_STATUS_BAD_TOKEN after the stream has drained
 * A row with nothing allowed has entropy 0, logp -inf and no alternatives.  A NaN or +inf at an allowed
 * place makes its row's results NaN; a NaN is no alternative.
 * Errors: CP_ERR_ARG (type, token_type, scale), CP_ERR_SIZE (rows, vocab, given, top, ld < vocab),
 * CP_ERR_NULL, CP_ERR_WORKSPACE, CP_ERR_HIP.
 */
int cp_token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top, size_t *out_bytes);
int cp_token_logprobs(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, float scale,
                      const uint64_t *allow, int32_t given, const void *tokens, int token_type,
                      int64_t token_row_stride, int64_t token_stride, float *logp, float *entropy, float *stats,
                      int32_t top, float *top_logp, int32_t *top_idx, void *workspace, size_t workspace_bytes,
                      void *stream, int32_t *status_out);

/*
 * Gradient of cp_token_logprobs with respect to the logits, [rows][vocab] of their type: dlogp is the
 * gradient of logp, at i * dlogp_row_stride + g * dlogp_stride (a stride of 0: the same for all rows or
 * tokens), dentropy that of entropy at i * dentropy_stride, or NULL; stats are the forward call's.  Tokens
 * that are ignored, out of range or without a probability pass nothing on; places that are not allowed
 * or hold -inf and rows with nothing allowed get 0, whatever flows in.  The alternatives have no gradient.  Of up to CP_LOGPROBS_IN_PLACE
 * places a row, dlogits may take the place of the logits.
 */
int cp_token_logprobs_backward(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, float scale,
                               const uint64_t *allow, int32_t given, const void *tokens, int token_type,
                               int64_t token_row_stride, int64_t token_stride, const float *stats,
                               const float *dlogp, int64_t dlogp_row_stride, int64_t dlogp_stride,
                               const float *dentropy, int64_t dentropy_stride, void *dlogits, int64_t ldd, void *stream);

/*
 * Tokens drawn from softmax(scale * logits) over what top_k, top_p and min_p leave of each row's allowed places, by given random
 * numbers.  With p_v the probabilities in units of the best place's, and the places in the order of falling logit (equal ones by rising
 * place), what is kept is of the first top_k places those in front of which less than top_p of these places' mass lies (the first
 * in any case), and of them those with p_v >= min_p.  A token is the first kept place, by place, up to and with which more than u of
 * the kept mass lies.
 *
 *   logits, allow as cp_token_logprobs's
 *   scale, top_k, top_p, min_p   for all rows: scale > 0 and finite (1 / temperature), top_k >= 0 (0: all), top_p and
 *                 min_p from 0 to 1; or for each row from scales, top_ks, top_ps, min_ps ([rows] on the device, or NULL).  A row whose
 *                 own setting is none of these gets no tokens, and CP_STATUS_BAD_SAMPLING
 *   given, u      random numbers of each row, number g of row i at i * u_row_stride + g * u_stride, from 0 to 1 (below 0 and NaN
 *                 count as 0, from 1 on as the last number below 1)
 *   tokens        of CP_TOKEN_* (CP_TOKEN_U8 for at most 255 places), token g of row i at i * token_row_stride + g *
 *                 token_stride: in either layout such as cp_eval takes as a batch of assignments
 *   logp          [rows][given], the logarithm of the token's share of the kept mass, or NULL
 *   status_out    device int32, required where a row has settings of its own
 * A row with nothing allowed, or with a NaN or +inf at an allowed place, gets tokens -1 (255 of CP_TOKEN_U8) and logp 0.
 * Probabilities and sums are formed in 64 bits.  workspace may be NULL where cp_token_sample_workspace_bytes says 0.
 * Errors: as cp_token_logprobs's; CP_ERR_SIZE where strides put two tokens in one place, or are above 2^28 (a row's where there are several
 * rows, a number's where there are several).
 */
int cp_token_sample_workspace_bytes(int64_t rows, int32_t vocab, int32_t given, size_t *out_bytes);
int cp_token_sample(int64_t rows, int32_t vocab, int type, const void *logits, int64_t ld, double scale, const float *scales,
                    const uint64_t *allow, int32_t top_k, const int32_t *top_ks, double top_p, const float *top_ps, double min_p,
                    const float *min_ps, int32_t given, const float *u, int64_t u_row_stride, int64_t u_stride, void *tokens, int token_type,
                    int64_t token_row_stride, int64_t token_stride, float *logp, void *workspace, size_t workspace_bytes, void *stream,
                    int32_t *status_out);

/*
 * Stage timing with HIP events recorded on the stream the kernels run on.
 * A profile holds `slots` sets of CP_NUM_STAGES+1 events; every cp_eval call that
 * is given the profile fills the next slot (CP_ERR_STATE when full).
 */
int cp_profile_create(int32_t slots, cp_profile **out);
int cp_profile_reset(cp_profile *p);                       /* next call fills slot 0 again */
int cp_profile_count(const cp_profile *p, int32_t *out);   /* slots filled so far */
/* Milliseconds per stage for one filled slot; the stream must have drained.
 * sweep_launches[0], [1] (may be NULL) receive the number of kernel launches the
 * b-level and t-level stages made; {1, 0} for a call that asked for both sweeps means one
 * launch ran both (its time is the b-level stage's). */
int cp_profile_read(const cp_profile *p, int32_t slot, float ms_out[CP_NUM_STAGES],
                    int32_t sweep_launches[2]);
/* CP_PLAN_* that the call in a filled slot ran. */
int cp_profile_plan(const cp_profile *p, int32_t slot, int *plan_out);
void cp_profile_destroy(cp_profile *p);

/*
 * Diagnostic: the 32-bit multiply-shift constants the kernels would use for
 * ceil(a / divisor) with 0 <= a <= max_dividend:
 *     ceil(a / divisor) == ((a + *dm1) * (uint64)*mul + (a + *dm1)) >> 32.
 * Returns 1 and fills mul, dm1 if that form is exact over the whole range, 0 if it
 * is not (the kernels then divide plainly), or a negative CP_ERR_* code.
 */
int cp_cost_magic(int64_t divisor, int64_t max_dividend, uint32_t *mul, uint32_t *dm1);

/*
 * Diagnostic: the 4-byte table entry some kernels use instead where every divisor of the
 * call is at most 256 and every weight below 2^24:
 *     ceil(a / divisor) == ((a + (e & 0xff)) * (uint64)(e | 0xff) + (a + (e & 0xff))) >> 32.
 * Returns 1 and fills *entry if that form is exact for 0 <= a <= max_dividend, 0 if not,
 * or a negative CP_ERR_* code.
 */
int cp_cost_compact(int64_t divisor, int64_t max_dividend, uint32_t *entry);

/*
 * Diagnostic: the workgroup shape the resident-window plan would launch with for one sweep
 * (tsweep = 0: b-levels, 1: t-levels) of this graph with k devices, on a compute unit with
 * 160 KB of LDS.  shape[0..7] = 16-byte loads per loader lane and tick, loader wavefronts, far
 * wavefronts, compute wavefronts, ticks of prefetch, partitions per workgroup, output stores one
 * compute wavefront issues per tick (1 or 2: the bound the far reads' ordering rests on), LDS
 * bytes per workgroup.  Host only.  Returns CP_OK, CP_ERR_NULL, CP_ERR_ARG (no such shape: the
 * plan does not apply to this graph, device count or tick type).
 */
int cp_window_shape(const cp_graph *g, int32_t k, int tick_dtype, int tsweep, int32_t shape[8]);

/* Human-readable text for a CP_ERR_* code (static storage). */
const char *cp_error_string(int code);

#ifdef __cplusplus
}
#endif
#endif /* CPEVAL_H */
