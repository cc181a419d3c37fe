/*
 * ink.h -- C ABI of the MI355X (gfx950) incremental GNN-inference library.
 *
 * The library keeps, on one GPU, the cached state of a k-layer message-passing GNN
 * (per layer: the messages m_l, the aggregated neighbourhoods alpha_l and, for min/max,
 * the per-dimension argmax/argmin neighbour ids) and updates it after a batch of edge
 * insertions and deletions by the event-driven incremental method of the paper
 * (Sec. 2.3 workflow; Sec. 2.4 events, grouping and propagation; Sec. 2.5 incremental
 * update, reset conditions and recompute).  The result equals plain inference on the
 * post-update snapshot (Abstract; Sec. 1, "No Accuracy Loss").
 *
 * Conventions for every entry point
 *   - Plain C types only.  Pointers are HOST pointers unless `ink_options.mem` says
 *     INK_MEM_DEVICE, in which case caller arrays (graph, features, weights, update
 *     batches) are device pointers on the current HIP device (`ink_options.batch_mem`
 *     can place only the update batches on the device).
 *   - The caller keeps ownership of everything it passes in; the library copies what it
 *     needs.  Buffers returned by the library are library-owned DEVICE memory, valid until
 *     the next ink_apply_updates / ink_full_infer / ink_destroy on the same context.
 *   - Every call returns an ink_status.  On an argument / range / state error nothing in
 *     the context has been modified.  INK_E_OOM or INK_E_DEVICE from a call that updates the
 *     context (ink_apply_updates, ink_apply_updates_affected, ink_update_features,
 *     ink_add_nodes) may leave the graph store or the cache half-written: the context is then
 *     unusable, every later call on it returns INK_E_STATE, and it must be destroyed.
 *     ink_last_error() gives a readable message.
 *   - One context = one HIP stream; calls on one context must not overlap.  All calls are
 *     synchronous: on return the work is complete, what was passed in is no longer read and results
 *     can be used on any stream.  A successful update ends with a record that the device writes to the
 *     host when everything else is done: its last kernel, which writes nothing after that record, may for
 *     a moment still show as running on the stream.  A call that returns an error leaves nothing running.
 *     The calling thread polls for such records: it keeps a host core busy for up to a millisecond per record
 *     and blocks only then.  A layer of an update has one to three records, small updates have one for all.
 *   - Node ids are int32 in [0, n_nodes); the graph is a simple directed graph without self
 *     loops.  Edge batches never change n_nodes (the paper's update stream holds edges only,
 *     Sec. 2.1); it grows only through ink_add_nodes, up to ink_options.node_capacity.
 *     Edge (u -> v) makes u an in-neighbour of v: v aggregates m_u.
 *   - At most 2^31 - 2^30 - 1 edges (event offsets are 32-bit); a batch that could take the graph
 *     past that is refused.
 *   - All matrices of a context are row-major float32.  Layer outputs are at most INK_MAX_OUT_DIM wide, layer
 *     inputs (the feature width in particular) at most INK_MAX_IN_DIM.
 */
#ifndef INK_H
#define INK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define INK_MAX_OUT_DIM 256
#define INK_MAX_IN_DIM 16384
#define INK_MAX_LAYERS 8
#define INK_MAX_CLASSES (1 << 27) /* ink_log_probs: classes of a row */
#define INK_MAX_TOP 16            /* ink_log_probs: alternatives asked for */
#define INK_ADAMW_BLOCK 128       /* ink_adamw: neighbouring elements whose 8-bit moments share a scale */

typedef struct ink_ctx ink_ctx; /* opaque; owns all device state */

typedef enum {
  INK_OK = 0,
  INK_E_ARG = 1,    /* null pointer, bad dimension, malformed CSR, unsupported combination */
  INK_E_STATE = 2,  /* ink_apply_updates / ink_get_layer before ink_full_infer */
  INK_E_OOM = 3,    /* device or host allocation failed; from an updating call: destroy the context */
  INK_E_DEVICE = 4, /* a HIP call failed; the context must be destroyed */
  INK_E_RANGE = 5   /* node id or layer index out of range */
} ink_status;

/* Model families of Sec. 3 (eqs. (1)-(6)). */
typedef enum { INK_MODEL_SAGE = 0, INK_MODEL_GCN = 1, INK_MODEL_GIN = 2 } ink_model_kind;

/* Aggregation function A of Sec. 2.1.  MAX / MIN are the paper's monotonic selections
 * (Sec. 2.2 item 1).  SUM / MEAN / GCN_SYM use the delta-accumulative update the paper names
 * as its extension (Sec. 7).  GCN_SYM = symmetric degree normalisation with self loop:
 * a_v = sum_{u in N(v)+{v}} h_u / sqrt(dhat_u dhat_v), dhat_x = indeg(x) + 1. */
typedef enum {
  INK_AGG_MAX = 0, INK_AGG_MIN = 1, INK_AGG_SUM = 2, INK_AGG_MEAN = 3, INK_AGG_GCN_SYM = 4
} ink_agg;

/* GELU (z times the normal distribution function) and SILU (z times the logistic function): ink_linear and
 * ink_gated only, a layer takes NONE or RELU. */
typedef enum { INK_ACT_NONE = 0, INK_ACT_RELU = 1, INK_ACT_GELU = 2, INK_ACT_SILU = 3 } ink_act;
typedef enum { INK_F32 = 0, INK_BF16 = 1, INK_F16 = 2, /* element types of an answer head's operators */
               INK_E4M3 = 3, /* 8 bits (4 of exponent, 3 of mantissa, largest number 448), where an operator says so */
               INK_NO_TYPE = -1 } ink_type;
typedef enum { INK_MEM_HOST = 0, INK_MEM_DEVICE = 1 } ink_mem;

/* In-neighbour CSR of the initial snapshot: row v lists the sources u of edges u -> v,
 * strictly ascending within a row (no duplicates), no self loops. */
typedef struct {
  int32_t n_nodes;
  int64_t n_edges;
  const int64_t *rowptr; /* [n_nodes + 1], rowptr[0] = 0, rowptr[n_nodes] = n_edges */
  const int32_t *col;    /* [n_edges] */
} ink_csr;

/* One GNN layer.  Weights are row-major [in][out]; a NULL pointer means "absent".
 *   SAGE: h' = act(W_neigh^T a + W_self^T h + bias)                          (eq. (4))
 *   GCN : h' = act(W_neigh^T a + bias)                                       (eq. (2))
 *   GIN : h' = act(W_mlp2^T relu(W_neigh^T ((1+eps) h + a) + bias) + bias_mlp2)  (eq. (6));
 *         W_neigh is [in_dim][mlp_hidden], W_mlp2 is [mlp_hidden][out_dim]. */
typedef struct {
  int32_t in_dim, out_dim, mlp_hidden;
  const float *W_neigh, *W_self, *bias;
  const float *W_mlp2, *bias_mlp2;
  int32_t act; /* ink_act applied at the end of the layer (Sec. 2.1) */
} ink_layer;

typedef struct {
  int32_t kind;    /* ink_model_kind */
  int32_t agg;     /* ink_agg; SAGE: MAX|MIN|SUM|MEAN, GIN: SUM|MAX|MIN|MEAN, GCN: GCN_SYM */
  float gin_eps;
  int32_t n_layers; /* 1 .. INK_MAX_LAYERS */
  const ink_layer *layers;
} ink_model;

typedef struct {
  int32_t mem;        /* ink_mem: where the caller's arrays live, for every call on the context */
  void *hip_stream;   /* hipStream_t to run on, or NULL for a stream the library creates */
  float slack_factor; /* extra capacity per edge block, as a fraction of its degree (default 0.25) */
  int32_t max_batch;  /* hint: largest update batch expected (sizes buffers up front); 0 = default */
  int32_t profile;    /* non-zero: time each kernel class with HIP events (see ink_stats) */
  float dense_threshold; /* a layer whose event count exceeds this fraction of the edge count
                            re-aggregates every node instead of grouping events (the dense
                            fallback Sec. 5.1 argues for when updates are not sparse);
                            0 = default: 0.75; for max and min, in layers of more than 4096 events,
                            0.45 (0.35 for rows of at most 64 floats) plus 2.5 events for every
                            node beyond 300 000 (for wider rows: in batches of edge updates), but
                            at most 0.75; negative = never */
  int32_t batch_mem;     /* ink_mem of the `updates` array of ink_apply_updates when it differs from
                            `mem` (e.g. host-built graph, device-resident update stream): the
                            effective location is device if either field says INK_MEM_DEVICE */
  int32_t small_batch_limit; /* update batches of at most this many entries take the short form of the
                                graph-store update (same result, fewer launches, one host read-back
                                instead of two); 0 = default 16384, which is also the largest value;
                                negative = never */
  int64_t pool_reserve;  /* free id slots kept behind the edge blocks of each direction for blocks
                            that outgrow their slack; when they run out the pool is re-allocated
                            at twice the size.  0 = default max(25 % of the pool, 2^20) */
  int64_t node_capacity; /* largest node count the context can grow to with ink_add_nodes; every
                            per-node table is allocated for it.  0 (or less than the graph's
                            node count) = the graph's node count, i.e. no growth */
} ink_options;

/* One streaming update (Sec. 2.1: Delta E holds inserted and removed edges). */
typedef struct {
  uint8_t op; /* 0 = insert, 1 = delete */
  uint8_t pad_[3];
  int32_t src, dst;
} ink_edge_update;

/* Result of one update batch (library-owned device buffers, see top comment). */
typedef struct {
  int64_t n_changed;          /* nodes whose final embedding h_k changed bitwise            */
  const int32_t *changed_ids; /* DEVICE [n_changed], ascending                                */
  const float *embeddings;    /* DEVICE [n_changed][out_dim of last layer], new h_k rows      */
  int64_t n_applied_ins, n_applied_del; /* edges whose presence differs between the snapshots */
  int64_t n_noop; /* list entries without net effect: duplicate insert, delete of an absent
                     edge, self loop, or an insert/delete pair that cancels within the batch */
} ink_update_result;

/* Kernels of a layer that are timed one by one (ink_layer_stats.ms_kernel). */
enum { INK_K_AGG_EVENTS = 0, /* incremental aggregation over the grouped events (Sec. 2.5)          */
       INK_K_AGG_EXPOSED,    /* recompute of the exposed rows of moderate length, one wave per row  */
       INK_K_AGG_LONG,       /* recompute of long rows: plan, chunk partials, combine               */
       INK_K_AGG_FULL,       /* recompute of every row (full inference, dense fallback), short rows */
       INK_K_SORT,           /* grouping: radix sort of the events by target                        */
       INK_K_XFORM,          /* dense combination (all linear maps of the layer)                    */
       INK_K_NKERNEL = 8 };

/* Per-layer counters and timings of the LAST ink_apply_updates (or ink_full_infer). */
typedef struct {
  int64_t n_sources;     /* |F_l|: nodes whose message m_l changed                         */
  int64_t n_events;      /* event records created (changed edges + propagated)   Sec. 2.4.2 */
  int64_t n_targets;     /* unique target nodes after grouping                    Sec. 2.4.1 */
  int64_t n_exposed;     /* targets recomputed from their whole neighbourhood    Sec. 2.5.1 */
  int64_t n_regather_nb; /* neighbour rows fetched by those recomputes                       */
  int64_t n_alpha_changed; /* targets whose alpha changed (not resilient)         Sec. 2.5.2 */
  int64_t n_transformed; /* rows through the dense combination                              */
  int64_t n_changed;     /* rows whose layer output changed: next layer's sources           */
  /* MAX / MIN only: how the targets that were NOT recomputed split over the conditions of
   * Sec. 2.5.1 (the distribution of Sec. 5.2); together with n_exposed they sum to n_targets.
   * Aggregated rows wider than 256 columns are processed in 256-column blocks: the condition
   * counters, n_exposed and n_alpha_changed then describe the first block of each target,
   * n_regather_nb counts the neighbour rows of every block. */
  int64_t n_no_deletion;        /* only additions arrived                                    */
  int64_t n_deletion_no_effect; /* something was cancelled but no dimension needed a reset   */
  int64_t n_covered;            /* resets, all covered by added messages                     */
  int32_t dense;         /* 1 if the layer fell back to re-aggregating every node           */
  int32_t pad_;
  int64_t n_regather_nb_long; /* the part of n_regather_nb fetched by the chunked long-row kernels */
  float ms_kernel[INK_K_NKERNEL]; /* GPU time of single kernels of this layer, HIP events (profile != 0) */
} ink_layer_stats;

enum { INK_T_GRAPH = 0, INK_T_EVENTS, INK_T_GROUP, INK_T_AGG, INK_T_COMPACT, INK_T_TRANSFORM,
       INK_T_NCLASS };

typedef struct {
  int32_t n_layers, pad_;
  ink_layer_stats layer[INK_MAX_LAYERS];
  float ms[INK_T_NCLASS];       /* GPU time per kernel class, HIP events (profile != 0), else 0 */
  int32_t launches[INK_T_NCLASS];
  float ms_total;               /* wall time of the call measured on the host                   */
  float pad2_;
} ink_stats;

/* Builds a context: copies graph, features ([n_nodes][feat_dim]) and weights to the device and
 * builds the device graph store (per-node in- and out-edge blocks with slack).  The method's
 * input is a completed full inference of the initial snapshot (Sec. 2): call ink_full_infer next.  Errors: INK_E_ARG (malformed input), INK_E_RANGE (column id outside
 * [0, n)), INK_E_OOM. */
ink_status ink_create(const ink_csr *graph, const float *features, int32_t feat_dim,
                      const ink_model *model, const ink_options *opts, ink_ctx **out);

/* Initial full-graph inference with caching (Sec. 2: the embedding before and after the
 * aggregation is saved for every node in every layer).  May be called again at any time to
 * rebuild the cache from the current graph. */
ink_status ink_full_infer(ink_ctx *ctx);

/* ink_full_infer for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid it): same arguments, same result, bit for bit, but
 * the call makes no hipMalloc / hipFree (nor any other allocating call).  The work memory that
 * ink_full_infer takes from the allocator -- the list of long rows, the first chunk of each and the
 * partial rows of the chunks, GIN's staging rows -- lies in one static device array of
 * INK_NOALLOC_SCRATCH_BYTES bytes per GPU, which that GPU holds until the process ends; the
 * per-kernel-class timing of ink_stats is off during the call.  Every context on a GPU shares
 * the array: calls of this entry point that overlap on one GPU race (calls on one context never
 * overlap anyway).  Nothing in the array is expected to be zero between calls.
 * Errors: INK_E_RANGE if the graph and model need more than the array holds -- the need is
 * 4 R + 4 (R + 1) + p w (E / 1024 + R) 4 bytes plus, for GIN, 4 n_nodes hidden (each in multiples of 256), with
 * E the edge count, R = min(node capacity, max(E / 256, 8192)) + 1 the bound on long rows, w the
 * widest aggregated row (at most 256) and p = 4 tables for MAX / MIN, 1 otherwise; then use
 * ink_full_infer.  Otherwise as ink_full_infer. */
#define INK_NOALLOC_SCRATCH_BYTES (64u << 20)
ink_status ink_full_infer_noalloc(ink_ctx *ctx);

/* Applies an ordered list of n updates and incrementally refreshes every layer (Sec. 2.3).
 * The post-update snapshot is the net effect of the list on the edge set.  `updates` is a host
 * or device array according to ink_options.mem.  n = 0 is allowed (empty result).
 * Errors: INK_E_STATE before ink_full_infer; INK_E_RANGE for an id outside [0, n_nodes);
 * INK_E_ARG for op > 1 or n < 0.  On error the graph and the cache are unchanged. */
ink_status ink_apply_updates(ink_ctx *ctx, const ink_edge_update *updates, int64_t n,
                             ink_update_result *out);

/* The result of the last call that returned one (ink_apply_updates, ink_apply_updates_affected, ink_update_features,
 * ink_apply_user_events, ink_add_nodes), copied to host memory: n ids and n rows of the last layer's width, n being that
 * result's n_changed.  For callers who want every result on the host: from the first such call on, and in a context
 * whose batches are in host memory from the start, modest results (INK_RESULT_HOST_BYTES) are written to pinned memory by the
 * kernel that gathers them, until one of them is not asked for.
 * Errors: INK_E_STATE if there is none or another call that changes the context (or tried to) has come since,
 * INK_E_ARG if n is another number. */
#define INK_RESULT_HOST_BYTES (1u << 20)
ink_status ink_copy_result(ink_ctx *ctx, int32_t *ids, float *embeddings, int64_t n);

/* Baseline for comparison, same arguments and result as ink_apply_updates: the "Affected" method
 * of Sec. 4.1 (inference on the theoretically affected area; Fig. "Inference on a streaming graph"
 * (b)).  Every node reached by a changed edge or by an affected node of the previous layer is
 * recomputed from its whole neighbourhood and re-transformed, and propagates whether or not it
 * changed.  The cache ends in the same state as after ink_apply_updates. */
ink_status ink_apply_updates_affected(ink_ctx *ctx, const ink_edge_update *updates, int64_t n,
                                      ink_update_result *out);

/* Vertex feature update (the input-side counterpart of an edge update; Sec. 2.6 lets callers
 * create and propagate events of their own next to the built-in ones, and this is the one such
 * event a fixed-function library can offer): x_v <- rows[i] for v = node_ids[i], then the same
 * layer-wise propagation as ink_apply_updates with F_1 = the nodes whose feature row changed
 * bitwise (Sec. 2.4: a node whose message changed sends its old and new message to its
 * out-neighbours; Sec. 3.2: its own next embedding depends on it too).  The graph is unchanged.
 *   node_ids : [n] distinct ids in [0, n_nodes), any order
 *   rows     : [n][feat_dim] fp32, row i belongs to node_ids[i]
 * Both arrays are host or device memory like the update batches (ink_options.batch_mem, else
 * ink_options.mem).  The result has the layout of ink_apply_updates' (n_applied_* are 0).
 * Errors: INK_E_STATE before ink_full_infer; INK_E_RANGE for an id outside [0, n_nodes);
 * INK_E_ARG for a repeated id, n < 0 or NULL arrays.  On error nothing is changed. */
ink_status ink_update_features(ink_ctx *ctx, const int32_t *node_ids, const float *rows, int64_t n,
                               ink_update_result *out);

/* User-defined events (Sec. 2.6: callers may create, group and apply events of their own next
 * to the built-in ones, and these are managed apart from them; Sec. 3.2 shows the use: a user_apply
 * step adds a caller-supplied per-node term to the tensor between the linear map and the
 * activation).  Every layer l has a user term u_l[v] of out_dim_l floats per node, zero until an
 * event touches it, and the layer computes h_l[v] = act(T_l(alpha_l[v], h_{l-1}[v]) + u_l[v])
 * (added to the fp32 result of the linear map and its bias, before the activation).  An event
 * names a layer (1 .. n_layers), a target node and an operation on that node's term. */
typedef enum { INK_USER_SET = 0,   /* u <- row          */
               INK_USER_ADD = 1,   /* u <- u + row, one fp32 addition per event */
               INK_USER_CLEAR = 2  /* u <- 0 (row ignored) */ } ink_user_op;
typedef struct {
  int32_t layer, target;
  int32_t op;      /* ink_user_op */
  int32_t pad_;
} ink_user_event;

/* Applies an ordered list of n user events: they are grouped by (layer, target), each group is
 * applied in list order to its node's term, and every node whose term changed bitwise is
 * re-transformed at its layer and, if its embedding changed, propagates to the deeper layers
 * like any changed node (Sec. 2.4.2).  The graph is unchanged; the terms stay in force for every
 * later call, ink_full_infer included.
 *   events : HOST array [n]
 *   rows   : HOST array [n][row_stride]; the first out_dim_layer floats of row i belong to event i
 * (both always host memory: user events are control input, not a data stream).  The first event
 * on a layer allocates that layer's term table (n_nodes capacity x out_dim floats).
 * The result has the layout of ink_apply_updates' (n_applied_* are 0).  Every model kind takes
 * them; for GCN the term joins the bias: h_l = act(normalised sum of layer l + b_l + u_l).
 * Errors: INK_E_STATE before ink_full_infer; INK_E_RANGE for a layer outside 1 .. n_layers or a
 * target outside [0, n_nodes); INK_E_ARG for an unknown op, row_stride below the width of a named
 * layer, n < 0 or NULL arrays.  On these errors nothing is changed. */
ink_status ink_apply_user_events(ink_ctx *ctx, const ink_user_event *events, const float *rows, int32_t row_stride,
                                 int64_t n, ink_update_result *out);

/* Node arrival (Sec. 1 names newly arriving nodes as one source of change; Sec. 2.1 defines the
 * update stream over edges only, so a node arrives without edges and its edges follow through
 * ink_apply_updates).  Appends n_new nodes with ids n_nodes .. n_nodes + n_new - 1 and the given
 * feature rows ([n_new][feat_dim], host or device like the update batches).  Their cached state
 * is that of a node with an empty neighbourhood (alpha = 0, argument -1; GCN: d-hat = 1) and
 * their embeddings are computed layer by layer from it; no other node changes.  The result lists
 * the new ids with their final embeddings.
 * Errors: INK_E_STATE before ink_full_infer; INK_E_RANGE if the node count would exceed
 * ink_options.node_capacity; INK_E_ARG for n_new < 0 or NULL features.  On error nothing changes. */
ink_status ink_add_nodes(ink_ctx *ctx, const float *features, int64_t n_new, ink_update_result *out);

/* Inspection for tests: copies rows [row0, row0 + nrows) of a cached table to dst (host or
 * device per dst_mem), densely packed [nrows][width].  layer in 0..n_layers.
 *   which = 0: h_layer, the output of layer `layer` (layer 0 = input features); it is the
 *              message m_{layer+1} of the aggregate-first models (Sec. 2.1).
 *   which = 1: alpha_layer, the aggregated neighbourhood of layer `layer` >= 1.  For SUM / MEAN
 *              it is the cached plain sum of the neighbours' messages; for GCN_SYM the cached
 *              sum over in-neighbours u of c_u (h_{layer-1} W_layer)_u with c = dhat^(-1/2)
 *              (the row-local factor c_v and the self term are applied when h is formed).
 *   which = 2: int32 argmax/argmin neighbour ids of layer `layer` >= 1 (MAX / MIN only).
 *   which = 3: MAX / MIN only: the cached bound on the best value among the neighbours other
 *              than the holder (>= it for MAX, <= it for MIN; -inf / +inf if there is none).  It is
 *              exact after a recompute and may be loose afterwards; it never affects results.
 *   which = 4: MAX / MIN only, int32: the neighbour other than the holder that has exactly the
 *              value of which = 3 (the lowest such id), or -1 where that is not known.
 *   which = 5: the user term u_layer of ink_apply_user_events (INK_E_ARG if no event ever named the layer).
 * width is returned in *width_out if not NULL. */
ink_status ink_get_layer(ink_ctx *ctx, int32_t layer, int32_t which, int64_t row0, int64_t nrows,
                         void *dst, int32_t dst_mem, int32_t *width_out);

/* Copies the current in-neighbour lists into caller HOST arrays: rowptr [n_nodes + 1] and, if
 * col is not NULL, col [n_edges] (each row ascending).  Pass col = NULL first to size it. */
ink_status ink_get_graph(ink_ctx *ctx, int64_t *rowptr, int32_t *col);

/* Turns the per-kernel-class HIP-event timing of ink_stats on or off (it costs a few event
 * records per layer, which matters for the latency of tiny batches). */
ink_status ink_set_profiling(ink_ctx *ctx, int32_t on);

/* Copies min(bytes, sizeof(ink_stats)) bytes of the last call's statistics. */
ink_status ink_get_stats(ink_ctx *ctx, void *stats_out, size_t bytes);

/* ---------------------------------------------------------------- operators of an answer head
 *
 * What turns embeddings into answers, and re-fits that map while the graph changes: layer norm, root-mean-square norm, a
 * linear layer with its epilogue, a gated pair of projections, log probabilities of classes; each with its gradient; and a step of AdamW.  They need no context
 * and take rows from anywhere on the device, an update's result (ink_update_result) among them.
 *
 * Unlike the calls on a context these are ASYNCHRONOUS: a call enqueues its kernels on `hip_stream`
 * (NULL: the default stream) of the current device and returns; it allocates nothing, keeps nothing and never waits, so
 * it can be captured into a graph.  Every pointer is DEVICE memory that has to stay valid, unchanged
 * and ready on that stream until the work is done; outputs must overlap neither inputs nor each other.  Where a call
 * needs `work` memory, its ..._work function says how many bytes (0: none, NULL will do); a
 * work buffer serves one call at a time.  The same call on the same inputs gives the same bits.
 *
 * Matrices are row-major, of ink_type elements, row i at i * ld elements.  ld is any number from the
 * row's length up; a matrix that is read may also have ld = 0, one row for all.  Pointers need the alignment of an
 * element only, work memory that of 16 bytes.  rows may be 0 (sums over the rows are then zeros).  Sums and statistics are kept in 32 bits
 * (but for ink_gated's 16-bit results of 8-bit rows), outputs are rounded once, to nearest even.  NaN and infinities go where the formulas take them.
 * The order of a sum depends on the call's sizes: the same row in a call of other sizes may differ in the last bits.
 *
 * Errors: INK_E_ARG (NULL, misaligned or too little memory, sizes or types out of range, an unknown activation; nothing was
 * enqueued) and INK_E_DEVICE (a launch was refused); ink_last_error(NULL) has the message. */

/* y = (x - mean) * rstd * weight + bias, rstd = 1 / sqrt(var + eps), mean and (biased) variance of each row.
 *   x, y         [rows][cols] of `type`, cols 1 .. INK_MAX_IN_DIM
 *   weight, bias [cols] of `param_type` (`type` or INK_F32), or NULL: 1 and 0
 *   mean, rstd   [rows] float, written for the gradient, or NULL
 *   eps          > 0 */
ink_status ink_layer_norm(const void *x, int64_t ld_x, const void *weight, const void *bias, int64_t rows, int32_t cols,
                          int32_t type, int32_t param_type, float eps, void *y, int64_t ld_y, float *mean, float *rstd,
                          void *hip_stream);

/* Gradient of ink_layer_norm: dx [rows][cols] of `type`, dweight and dbias [cols] of `param_type`, summed over the rows; each
 * may be NULL (not wanted).  mean and rstd as the forward call wrote them. */
size_t ink_layer_norm_backward_work(int64_t rows, int32_t cols, int32_t type);
ink_status ink_layer_norm_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const float *mean,
                                   const float *rstd, const void *weight, int64_t rows, int32_t cols, int32_t type,
                                   int32_t param_type, void *dx, int64_t ld_dx, void *dweight, void *dbias, void *work,
                                   size_t work_bytes, void *hip_stream);

/* y = act(z) + residual, z = x W + bias.
 *   x            [rows][cols] of `type`; W [cols][out] and bias [out] (or NULL) of `type`; cols and out 1 .. INK_MAX_IN_DIM
 *   residual     [rows][out] of `out_type`, or NULL
 *   y, pre       [rows][out] of `out_type` (`type` or INK_F32: logits of 16-bit rows); pre, where not NULL, gets z for the gradient
 *   act          ink_act */
ink_status ink_linear(const void *x, int64_t ld_x, const void *weight, int64_t ld_w, const void *bias, const void *residual,
                      int64_t ld_res, int64_t rows, int32_t cols, int32_t out, int32_t type, int32_t out_type, int32_t act,
                      void *y, int64_t ld_y, void *pre, int64_t ld_pre, void *hip_stream);

/* Gradient of ink_linear (that of the residual is dy itself): dz = dy * act'(pre), dx = dz W^T [rows][cols], dweight = x^T dz
 * [cols][out], dbias [out] = sum of dz over the rows, all of `type`; each may be NULL (not wanted).
 *   dy, pre      [rows][out] of `dy_type` (`type`, or INK_F32 with INK_BF16); pre is not read for INK_ACT_NONE
 * With 16-bit rows dz is rounded to `type` before the two products. */
size_t ink_linear_backward_work(int64_t rows, int32_t cols, int32_t out);
ink_status ink_linear_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const void *weight, int64_t ld_w,
                               const void *pre, int64_t ld_pre, int64_t rows, int32_t cols, int32_t out, int32_t type,
                               int32_t dy_type, int32_t act, void *dx, int64_t ld_dx, void *dweight, int64_t ld_dw, void *dbias,
                               void *work, size_t work_bytes, void *hip_stream);

/* For each row of logits, with z = scale * logit and p = softmax(z):
 *   logp      [rows] log p of the row's target; 0 for a row without one (a target outside [0, classes), or targets NULL)
 *   entropy   [rows] -sum p log p
 *   lse       [rows] log sum exp z
 *   top_ids   [rows][top] the classes of the `top` largest logits, largest first; equal logits by the lower class, NaN
 *             first of all; top_logp [rows][top] their log p.  top 0 .. min(classes, INK_MAX_TOP)
 * Each output may be NULL.  targets: int32 (target_bytes 4) or int64 (8).  A class at -inf is masked.  In a row of masked
 * classes lse and every log p is -inf and the entropy 0; a NaN or +inf among the logits makes lse, entropy and log p NaN.  Finite
 * logits are numbers like others, a type's lowest among them, but for one further below its row's largest than a float can
 * say (masked).  log p is formed of differences of logits and has its digits however far from zero these lie; where lse passes
 * the range of float it is the largest finite number of its sign.
 *   scale     > 0, at most 2.3e38 (1 / temperature);  classes 1 .. INK_MAX_CLASSES */
size_t ink_log_probs_work(int64_t rows, int64_t classes, int32_t type, int32_t top);
ink_status ink_log_probs(const void *logits, int64_t ld, const void *targets, int32_t target_bytes, int64_t rows, int64_t classes,
                         int32_t type, float scale, int32_t top, float *logp, float *entropy, float *lse, int32_t *top_ids,
                         float *top_logp, void *work, size_t work_bytes, void *hip_stream);

/* Gradient of sum_r g_logp[r] logp[r] + g_entropy[r] entropy[r] by the logits, [rows][classes] of `type` (not that of lse or
 * top_logp).  Either of g_logp and g_entropy may be NULL; lse and entropy as the forward call wrote them (entropy
 * is read with g_entropy only).  A row without a target takes no part in g_logp; a row of masked classes has gradient 0.
 * Where lse lies beyond -256 .. 256 the row's sum is formed anew: a float near that size does not hold log p. */
ink_status ink_log_probs_backward(const void *logits, int64_t ld, const void *targets, int32_t target_bytes, const float *lse,
                                  const float *entropy, const float *g_logp, const float *g_entropy, int64_t rows, int64_t classes,
                                  int32_t type, float scale, void *dlogits, int64_t ld_out, void *hip_stream);

/* Root-mean-square norm of rows after the addition of a residual: t = x + residual, rounded to `type`;
 * y = t * rstd * weight, rstd = 1 / sqrt(mean of t^2 + eps).
 *   x, residual  [rows][cols] of `type`; residual NULL: t is x
 *   weight       [cols] of `param_type` (`type` or INK_F32), or NULL: 1
 *   y            [rows][cols] of `out_type`, `type` or INK_E4M3: then scale[r] = max |y| of the row / 448 and y holds the numbers y / scale, each
 *                rounded to nearest even.  A row whose largest |y| is below 448 * 2^-126 has scale 0 and zeros, one with a NaN or an
 *                infinity scale and codes NaN
 *   total        [rows][cols] of `type`, gets t where residual is not NULL (for the next block and the gradient)
 *   rstd         [rows] float, written for the gradient, or NULL;  scale [rows] float, for INK_E4M3 only
 *   eps          > 0
 * The squares are summed in 32 bits: a row whose sum passes their range (elements beyond 10^19) has rstd 0. */
ink_status ink_rms_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_res, const void *weight, int64_t rows, int32_t cols,
                        int32_t type, int32_t param_type, float eps, int32_t out_type, void *y, int64_t ld_y, float *scale, void *total,
                        int64_t ld_total, float *rstd, void *hip_stream);

/* Gradient of ink_rms_norm with y of `type`: dx (of x and of the residual alike) [rows][cols] of `type`, dweight [cols] of `param_type`,
 * summed over the rows; each may be NULL (not wanted).  total is t (x where there was no residual), rstd as the forward call wrote it;
 * d_total, the gradient that arrives at t from elsewhere, is added to dx (NULL: none). */
size_t ink_rms_norm_backward_work(int64_t rows, int32_t cols, int32_t type);
ink_status ink_rms_norm_backward(const void *dy, int64_t ld_dy, const void *total, int64_t ld_total, const float *rstd, const void *weight,
                                 const void *d_total, int64_t ld_dt, int64_t rows, int32_t cols, int32_t type, int32_t param_type, void *dx,
                                 int64_t ld_dx, void *dweight, void *work, size_t work_bytes, void *hip_stream);

/* The gated pair of projections, h = act(x Wg) * (x Wu).
 *   x            [rows][cols] of `type`;  w_gate (Wg), w_up (Wu) [cols][hidden] of `type`;  cols and hidden 1 .. INK_MAX_IN_DIM
 *   h            [rows][hidden] of `out_type`, which is `type`
 *   act          ink_act
 * Of 8-bit rows (type INK_E4M3, ink_rms_norm's): row r of x is x_scale[r] times its numbers; the weights lie column by column,
 * [hidden][cols], and column c of Wg is gate_scale[c] times its numbers, of Wu up_scale[c] times; out_type is any of the other three.  The
 * scales are float and not read for other types; x_scale[r] * gate_scale[c] is formed in 32 bits and should be a normal number.
 * The sums of 8-bit numbers are those of 32 bits with out_type INK_F32 alone.  For 16-bit results of each eight neighbouring products of a sum (k = 8 i .. 8 i + 7)
 * what lies below 2^-13 of the largest is dropped: less than 2^-13 of the largest max(|x|, 2^-6) * max(|w|, 2^-6) of the eight, for each of seven.  Typically that
 * is 1.4e-5 of the result, less than its rounding; where large products cancel it can be more than what is left. */
ink_status ink_gated(const void *x, int64_t ld_x, const float *x_scale, const void *w_gate, int64_t ld_gate, const void *w_up,
                     int64_t ld_up, const float *gate_scale, const float *up_scale, int64_t rows, int32_t cols, int32_t hidden, int32_t type,
                     int32_t out_type, int32_t act, void *h, int64_t ld_h, void *hip_stream);

/* Gradient of ink_gated (not of 8-bit rows), with g = x Wg and u = x Wu formed anew: dg = dh u act'(g), du = dh act(g), dx = dg Wg^T + du Wu^T
 * [rows][cols], dw_gate = x^T dg and dw_up = x^T du [cols][hidden], all of `type`; each may be NULL (not wanted).  With 16-bit rows
 * dg and du are rounded to `type` before the products, but for a few rows; those of float16 rows with powers of two beside them, so that they may lie
 * beyond float16's range where the results do not.  The work memory does not grow with the rows beyond 2.1 GB, or
 * 1.1 GB and a matrix of [cols][2 hidden] floats where that has more; with dw_gate and dw_up NULL ink_gated_backward_work_dx bytes do, up to 1.1 GB. */
size_t ink_gated_backward_work(int64_t rows, int32_t cols, int32_t hidden, int32_t type);
size_t ink_gated_backward_work_dx(int64_t rows, int32_t hidden, int32_t type);
ink_status ink_gated_backward(const void *dh, int64_t ld_dh, const void *x, int64_t ld_x, const void *w_gate, int64_t ld_gate,
                              const void *w_up, int64_t ld_up, int64_t rows, int32_t cols, int32_t hidden, int32_t type, int32_t act, void *dx,
                              int64_t ld_dx, void *dw_gate, int64_t ld_dg, void *dw_up, int64_t ld_du, void *work, size_t work_bytes,
                              void *hip_stream);

/* One step of AdamW over n_tensors tensors, in place: with g = grad * grad_scale (times *grad_scale_at where that is not NULL) and t the step,
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps).
 *   tensors      HOST array, read before the call returns; what its entries point to is DEVICE memory.  What the step changes must
 *                not overlap, nor hold a gradient, step_at or grad_scale_at (INK_E_ARG; INK_E_OOM without host memory to look for that)
 *   param_type   INK_F32 or INK_BF16;  grad_type any;  copy_type INK_BF16 or INK_F16 with INK_F32 parameters, or INK_NO_TYPE
 *   moment_bits  32: m and v are float arrays.  8: m and v are INK_E4M3 arrays, and of each INK_ADAMW_BLOCK neighbouring elements m is
 *                m_scale times the number of its code, sqrt(v) v_scale times that of its code; zeros everywhere are the moments at the start
 *   step         t, from 1; or step_at, one int64 on the device that holds it (a captured call reads it at every replay; below 1 counts as 1)
 *   seed         of the random numbers that round 8-bit moments and INK_BF16 parameters: up or down, in proportion, so that the expectation of
 *                a parameter, of m and of sqrt(v) is what was to be rounded (that of v is larger by the variance); but a root that is not 0 and
 *                below 2^-9 of its block's scale, 1/229376 of the block's largest, is held at 2^-9 of it, and its element's step is smaller by
 *                that much.  The numbers depend on seed, t, the tensor's id and the element, and on nothing else
 *   lr and weight_decay 0 .. 1e18;  betas in [0, 1);  eps > 0
 * A gradient that is NaN or infinite makes its element NaN, with 8-bit moments the moments of its block; so does, with 8-bit moments, one
 * whose square is beyond a float (with 32-bit ones its element stays where it is, but for the decay). */
typedef struct {
  void *param;
  const void *grad;
  void *copy;                /* gets the new parameters, rounded to nearest; with copy_type only */
  void *m, *v;
  float *m_scale, *v_scale;  /* 8 bits only: [(n + INK_ADAMW_BLOCK - 1) / INK_ADAMW_BLOCK] */
  int64_t n;                 /* elements; 0: nothing is done */
  int64_t id;                /* its low 32 bits tell the tensor's random numbers from those of others */
} ink_adamw_tensor;
ink_status ink_adamw(const ink_adamw_tensor *tensors, int32_t n_tensors, int32_t param_type, int32_t grad_type, int32_t copy_type,
                     int32_t moment_bits, double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                     const int64_t *step_at, double grad_scale, const float *grad_scale_at, uint64_t seed, void *hip_stream);

/* Message of the last failing call on this context ("" if none).  ctx may be NULL: then the
 * message of the last failing ink_create or operator of an answer head on this thread. */
const char *ink_last_error(const ink_ctx *ctx);

void ink_destroy(ink_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* INK_H */
