/*
 * gnn.h -- C ABI of the GB300 interaction-network edge classifier.
 *
 * The library scores candidate edges of a particle-detector hit graph with an
 * interaction network, the edge-classification stage of the GNN tracking
 * pipeline (paper Section 2.1: space points and the candidate edges built
 * between them go in; the interaction network gives every edge a score that
 * the connected-components step thresholds into track candidates).  The
 * paper's service boundary takes a 2-D array of space points (rows) by raw
 * features (columns) (Section 2.3); this ABI keeps that layout and adds the
 * candidate edges, and returns one score per edge.
 *
 * Network (fp32 model; every MLP is L x [Linear -> LayerNorm -> ReLU]):
 *   h_j  = MLP_node_encoder(x_j)            e_ij = MLP_edge_encoder(dr, dphi)
 *   T times: m_ij = MLP_edge([h_i, h_j, e_ij]);  e_ij = m_ij
 *            a_j  = sum over edges (i -> j) of m_ij
 *            h_j  = MLP_node([h_j, a_j])
 *   score_ij = sigmoid(w_o . MLP_classifier([h_i, h_j, e_ij]) + b_o)
 * with dr = x_j[0] - x_i[0] and dphi = x_j[1] - x_i[1] wrapped into (-1, 1]
 * (columns 0 and 1 hold r/1000 and phi/pi).
 *
 * Threading and streams: every call that takes a stream only enqueues work on
 * it (no host synchronisation) unless stated otherwise.  A context is not
 * safe for concurrent use from several streams or threads (it owns one
 * workspace); use one context per stream.
 *
 * Return codes: GNN_OK (0) or a negative gnn_status_code.  Errors found on
 * the host are returned at once; errors found by the kernels are recorded in
 * the context's device error word and returned by gnn_status().
 */
#ifndef GNN_GB300_H
#define GNN_GB300_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* gnn_stream_t; /* a cudaStream_t; NULL = legacy default stream */

/* The largest count any call accepts (nodes, edges, an output capacity): 2^31 - 1 - 8192, so that
 * the kernels' 32-bit row indices stay in range after rounding up to whole blocks and tiles.  A
 * larger count (or a negative one) is INVALID_ARG, returned before any device work. */
#define GNN_MAX_COUNT 2147475455

enum gnn_status_code {
  GNN_OK = 0,
  GNN_ERR_INVALID_ARG = -1,    /* null pointer, bad size or unsupported configuration */
  GNN_ERR_BAD_WEIGHTS = -2,    /* weight blob: wrong magic/version/size or config mismatch */
  GNN_ERR_OOM = -3,            /* device allocation failed */
  GNN_ERR_CUDA = -4,           /* a CUDA runtime call or kernel launch failed */
  GNN_ERR_INDEX_RANGE = -5,    /* device: an edge endpoint was outside [0, n_nodes) */
  GNN_ERR_DEVICE_TIMEOUT = -6, /* device: a pipeline wait expired; results are invalid */
  GNN_ERR_CAPACITY = -7,       /* device: an output buffer was too small (gnn_build_graph) */
};

enum gnn_precision {
  GNN_PRECISION_FP32 = 0,      /* fp32 weights and state; products as three bf16 pieces */
  GNN_PRECISION_BF16 = 1,      /* bf16 weights, activations and stored states (h, e, a); fp32
                                  accumulation and LayerNorm; the blob's values must be bf16 */
};

/* Model configuration (must equal the blob header). */
typedef struct gnn_config {
  int32_t version;             /* must be 1 */
  int32_t n_node_feat;         /* F_n: node feature columns, 2..16 (cols 0, 1 = r/1000, phi/pi) */
  int32_t n_edge_feat;         /* must be 2: (dr, dphi) */
  int32_t hidden;              /* H: 64 or 128 */
  int32_t n_iters;             /* T: message-passing iterations, 0..64 */
  int32_t mlp_layers;          /* L: Linear layers per MLP, 2..4 */
  int32_t precision;           /* enum gnn_precision */
  float ln_eps;                /* LayerNorm epsilon (1e-5) */
} gnn_config;

typedef struct gnn_ctx gnn_ctx;

/*
 * gnn_create -- build a context on the current CUDA device.
 *
 * weights_host: host pointer to a little-endian weight blob of weights_bytes
 * bytes: a header of eight int32 (magic 0x57474E47, version 1, n_node_feat,
 * n_edge_feat, hidden, n_iters, mlp_layers, precision), float32 ln_eps, int32
 * reserved, int64 float count; then float32 arrays.  For each MLP in the order
 * node_encoder, edge_encoder, edge_network, node_network, edge_classifier and
 * each of its L layers: W [H, in] row-major, b [H], gamma [H], beta [H]
 * (in = F_n, 2, 3H, 2H, 3H for layer 1, H afterwards; the 3H inputs are
 * ordered [h_src, h_dst, e] and the 2H input [h, a]); then w_o [H] and b_o [1].
 * The blob is copied and repacked; the caller may free it on return.
 * On success *out receives the context (free with gnn_destroy).
 * Errors: INVALID_ARG (null pointer, unsupported config), BAD_WEIGHTS, OOM,
 * CUDA.  Synchronous.
 */
int gnn_create(const gnn_config* cfg, const void* weights_host, size_t weights_bytes, gnn_ctx** out);

/*
 * gnn_reserve -- size the context's workspace for graphs up to max_nodes
 * nodes and max_edges edges, so that later gnn_infer calls of that size
 * allocate nothing.  Synchronous (device allocation).  Errors: INVALID_ARG,
 * OOM.
 */
int gnn_reserve(gnn_ctx* ctx, int64_t max_nodes, int64_t max_edges);

/*
 * gnn_infer -- score every edge of one graph (a single event, or several
 * events concatenated block-diagonally).
 *
 *   node_feats  device, float32 [n_nodes, n_node_feat] row-major, 16-byte aligned
 *   edge_index  device, int32 [2, n_edges] row-major: row 0 = source ids,
 *               row 1 = destination ids, any order; duplicates and
 *               self-loops are legal
 *   edge_scores device, float32 [n_edges]: score of edge k of the input order
 *
 * All three buffers are caller-owned and must stay valid until the stream
 * reaches this work; the library never frees them.  n_edges == 0 is a no-op;
 * n_nodes == 0 with n_edges > 0 and sizes above GNN_MAX_COUNT are
 * INVALID_ARG.  The workspace grows here (synchronous allocation) when the
 * graph is larger than any earlier one; call gnn_reserve first to avoid it.
 * An edge with an endpoint outside [0, n_nodes) gets a NaN score, takes no
 * part in any aggregation, and makes gnn_status report INDEX_RANGE.
 * Scores are deterministic: the same inputs give bitwise-identical outputs.
 */
int gnn_infer(gnn_ctx* ctx, const float* node_feats, const int32_t* edge_index, int64_t n_nodes,
              int64_t n_edges, float* edge_scores, gnn_stream_t stream);

/*
 * gnn_infer_host -- gnn_infer on HOST buffers (the form a serving backend
 * receives requests in): copies node_feats [n_nodes, n_node_feat] float32 and
 * edge_index [2, n_edges] int32 from host memory into the context's staging
 * buffers, scores on the device, copies the scores back into edge_scores
 * [n_edges] float32 (host), and synchronises `stream` before returning.
 * Pinned (page-locked) host memory makes the copies asynchronous DMA;
 * pageable memory also works.  Same argument rules and errors as gnn_infer,
 * plus the device status of this call (as gnn_status would return it).
 */
int gnn_infer_host(gnn_ctx* ctx, const float* node_feats, const int32_t* edge_index, int64_t n_nodes,
                   int64_t n_edges, float* edge_scores, gnn_stream_t stream);

/*
 * gnn_embed_load -- load the embedding MLP (paper Section 2.1: the first step maps every space
 * point's raw features into a latent space where hits of one track lie close together).  Network:
 * y = normalize(W_out . MLP_L(x) + b_out), L hidden layers Linear -> LayerNorm -> ReLU of the
 * context's hidden width, then a Linear to D outputs, scaled to unit length (a zero vector stays
 * zero).  Blob (little-endian, copied): eight int32 (magic 0x4D454E47 "GNEM", version 1,
 * n_node_feat, hidden, L (2..4), precision, D (1..16), reserved), float32 ln_eps, int32 reserved,
 * int64 float count, then per hidden layer W [H, in] row-major, b, gamma, beta (in = n_node_feat
 * for layer 1, H afterwards), then W_out [D, H], b_out [D].  n_node_feat, hidden and precision
 * must equal the context's.  A later call replaces it.  Errors: INVALID_ARG, BAD_WEIGHTS, OOM, CUDA.
 *
 * gnn_embed -- embedding of every hit: node_feats device float32 [n_nodes, n_node_feat] in,
 * embedding device float32 [n_nodes, D] out (caller-owned).  Enqueued on `stream`.  Errors:
 * INVALID_ARG (no embedding loaded, null pointer, bad size), CUDA.
 *
 * gnn_build_graph -- candidate edges by fixed-radius neighbours in the embedding space (Section
 * 2.1: the graph is built between hits closer than a radius in the latent space).  Every pair of
 * hits whose squared distance, summed over the emb_dim coordinates in order in fp32 with one
 * rounding per product and per sum, is below radius * radius (rounded to fp32) becomes one edge,
 * oriented from the hit with the smaller r (node_feats column 0; the smaller id on a tie).
 *   embedding  device float32 [n_nodes, emb_dim], emb_dim 1..16; unit vectors (as gnn_embed
 *              writes them) are searched on a grid over [-1, 1]^K (K = 4 for emb_dim >= 4,
 *              else 3), other values stay exact but
 *              crowd into the grid's edge cells
 *   node_feats device float32 [n_nodes, n_node_feat] (column 0 orients the edges)
 *   edge_index device int32 with room for [2, max_edges], output: contiguous [2, n_edges]
 *   n_edges    device int32 [1], output: the number of edges found
 * When n_edges exceeds max_edges nothing is written to edge_index, *n_edges still holds the
 * count (saturated at INT32_MAX), and gnn_status reports GNN_ERR_CAPACITY: call again with room
 * for that many.  The order of the edges is deterministic.  Uses a scratch buffer of the context
 * (grown on demand, synchronous then): besides the sorted copies, 128 bytes per hit for the partner
 * chains the counting pass keeps (see gnn_debug_graph_pool) and 64 (128 for emb_dim > 8) for the
 * pair filter; half of the former suffice, with a second search for hits with more than 15 partners,
 * and are made do with where memory does not hold all.  Errors: INVALID_ARG (radius <= 0, emb_dim out
 * of range, null pointer, bad sizes), OOM, CUDA.
 */
int gnn_embed_load(gnn_ctx* ctx, const void* weights_host, size_t weights_bytes);
int gnn_embed(gnn_ctx* ctx, const float* node_feats, int64_t n_nodes, float* embedding, gnn_stream_t stream);
int gnn_build_graph(gnn_ctx* ctx, const float* embedding, int emb_dim, const float* node_feats, int64_t n_nodes,
                    float radius, int64_t max_edges, int32_t* edge_index, int32_t* n_edges, gnn_stream_t stream);

/*
 * gnn_filter_load -- load the filtering MLP (paper Section 2.1: the step before the GNN scores every
 * candidate edge from the raw features of its two hits; applyFiltering then drops the edges below
 * a fixed threshold).  Network: s = sigmoid(w_o . MLP_L([x_src, x_dst]) + b_o), each of its L
 * layers Linear -> LayerNorm -> ReLU, in the context's precision and hidden width.
 * Blob (little-endian, copied; the caller may free it): eight int32 (magic 0x4C464E47 "GNFL",
 * version 1, n_node_feat, hidden, mlp_layers (2..4), precision, two reserved), float32 ln_eps,
 * int32 reserved, int64 float count, then float32 arrays: per layer W [H, in] row-major, b, gamma,
 * beta (in = 2 * n_node_feat for layer 1, H afterwards), then w_o [H], b_o [1].  n_node_feat,
 * hidden and precision must equal the context's.  A later call replaces the filter.
 * Errors: INVALID_ARG, BAD_WEIGHTS, OOM, CUDA.  Synchronous.
 *
 * gnn_filter_edges -- score every candidate edge with the filtering MLP and keep those with
 * score > threshold, in input order.
 *   node_feats  device float32 [n_nodes, n_node_feat]
 *   edge_index  device int32 [2, n_edges] (row 0 sources, row 1 destinations)
 *   edge_scores device float32 [n_edges], output: filter score of every input edge (NaN for an edge
 *               with an endpoint out of range, which is never kept; gnn_status then reports
 *               INDEX_RANGE)
 *   kept_index  device int32 with room for [2, n_edges], output: the kept edges as a contiguous
 *               [2, n_kept] edge index (row 1 starts at n_kept), ready for gnn_infer
 *   kept_id     device int32 [n_edges] or NULL, output: input id of every kept edge
 *   n_kept      device int32 [1], output
 * All buffers are caller-owned.  Enqueued on `stream`; uses the context's workspace (it may grow,
 * as in gnn_infer).  Errors: INVALID_ARG (no filter loaded, null pointer, bad sizes), OOM, CUDA.
 */
int gnn_filter_load(gnn_ctx* ctx, const void* weights_host, size_t weights_bytes);
int gnn_filter_edges(gnn_ctx* ctx, const float* node_feats, const int32_t* edge_index, int64_t n_nodes,
                     int64_t n_edges, float threshold, float* edge_scores, int32_t* kept_index, int32_t* kept_id,
                     int32_t* n_kept, gnn_stream_t stream);

/*
 * gnn_track_labels -- track candidates from scored edges: one integer label per hit.  The
 * edge-classification scores are thresholded and the weakly connected components of the kept
 * edges are the track candidates (paper Section 2.1, the step after the interaction network);
 * the service returns an integer label per space point (Section 2.3).
 *
 *   edge_scores device float32 [n_edges], input edge order (as gnn_infer writes them)
 *   edge_index  device int32 [2, n_edges]: row 0 sources, row 1 destinations
 *   threshold   an edge is kept when its score is > threshold (NaN scores are never kept)
 *   labels      device int32 [n_nodes], output: the smallest node id of the hit's component
 *               (a hit without kept edges is its own component); caller-owned
 *
 * Edges with an endpoint outside [0, n_nodes) are skipped.  The labels do not depend on thread
 * or edge order.  Enqueued on `stream`; uses no workspace (the labels array is the union-find
 * forest).  Every union and find loop gives up after 1 s of wall-clock time (%globaltimer) and
 * then records GNN_ERR_DEVICE_TIMEOUT in the context's device error word (see gnn_status); the
 * labels are then invalid.  Errors: INVALID_ARG (null pointer, negative sizes or sizes above
 * GNN_MAX_COUNT, n_nodes == 0 with edges), CUDA.
 */
int gnn_track_labels(gnn_ctx* ctx, const float* edge_scores, const int32_t* edge_index, int64_t n_nodes,
                     int64_t n_edges, float threshold, int32_t* labels, gnn_stream_t stream);

/*
 * gnn_profile_enable -- when on != 0, later gnn_infer / gnn_infer_host calls
 * record a CUDA event pair on their stream around every kernel group, so
 * gnn_profile_read can report device time per group.  Off by default.
 *
 * gnn_profile_read -- synchronise the recorded events and write, for each
 * group g < n_groups, the summed device milliseconds ms[g] and the number of
 * kernel launches launches[g]; then clear the records.  Groups: 0 CSR build
 * (all its kernels), 1 node encoder, 2 edge encoder, 3 edge update, 4 node
 * update, 5 classifier, 6 host<->device copies of gnn_infer_host, 7 message
 * aggregation, 8 filtering MLP, 9 embedding MLP.  Either output pointer may
 * be NULL.  Returns the number of groups (10) or an error.
 */
int gnn_profile_enable(gnn_ctx* ctx, int on);
int gnn_profile_read(gnn_ctx* ctx, double* ms, int64_t* launches, int n_groups);

/*
 * gnn_status -- synchronise `stream`, then return and clear the device error
 * word of the context: GNN_OK, GNN_ERR_INDEX_RANGE, GNN_ERR_DEVICE_TIMEOUT,
 * GNN_ERR_CAPACITY (gnn_build_graph) or GNN_ERR_CUDA (a failed synchronisation).
 */
int gnn_status(gnn_ctx* ctx, gnn_stream_t stream);

/* gnn_destroy -- wait for the device (cudaDeviceSynchronize: the context does not know which
 * streams used it, so other work on the device is waited for too) and free ctx and all its
 * device memory. NULL is a no-op. */
void gnn_destroy(gnn_ctx* ctx);

/* gnn_error_string -- static text for a status code. */
const char* gnn_error_string(int code);

/*
 * gnn_debug_copy -- test hook: copy an internal buffer of the last gnn_infer
 * into caller device memory `dst` of at least `bytes` bytes (enqueued on
 * `stream`).  which: 0 rowptr int32 [N+1], 1 perm int32 [E] (CSR slot ->
 * input edge id), 2 src_sorted int32 [E], 3 node state h, 4 edge state e (CSR
 * order).  The states are float32 (bfloat16 for GNN_PRECISION_BF16) in the row-tiled layout of the kernels:
 * R = rows rounded up to a multiple of 128, element (r, c) at index
 * ((r / 128) * (H / 16) + bp) * 2048 + (r % 128) * 16 + x, R * H floats, where
 * b = c / 8, bp = b / 2 and x = 4 * ((c % 8) / 2) + 2 * (b % 2) + c % 2.
 * Errors: INVALID_ARG when the buffer is unknown or `bytes` is too small.
 */
int gnn_debug_copy(gnn_ctx* ctx, int which, void* dst, size_t bytes, gnn_stream_t stream);

/*
 * Failure-injection hooks for tests (no paper counterpart).  Neither faults nor hangs a GPU.
 *
 * gnn_debug_fail_allocs -- the next n device allocations made by the library (context creation,
 * workspace growth, gnn_infer_host staging) fail as if the device were out of memory, so the
 * GNN_ERR_OOM paths can be exercised; n = 0 cancels.  Process-wide.  Errors: INVALID_ARG (n < 0).
 *
 * gnn_debug_wait_timeout -- enqueue on `stream` one kernel that waits, through the same bounded
 * wait every pipeline wait in the library uses, on an mbarrier that nothing completes; after
 * limit_ns nanoseconds (0 < limit_ns <= 2e9) the wait gives up and records GNN_ERR_DEVICE_TIMEOUT
 * in the context's device error word, which gnn_status then returns (and clears).  The context
 * stays usable.  Errors: INVALID_ARG, CUDA.
 */
int gnn_debug_fail_allocs(int n);
int gnn_debug_wait_timeout(gnn_ctx* ctx, int64_t limit_ns, gnn_stream_t stream);

/*
 * gnn_debug_graph_pool -- test hook for gnn_build_graph (no paper counterpart).  The counting pass
 * keeps every hit's partners in a chain of 15-entry chunks, the hit's own first chunk plus chunks
 * from a pool, and the writing pass copies them; a hit whose chain could not grow because the pool
 * was used up is searched again instead, with the same result.  This sets the pool size in chunks
 * for later calls on this context (0: every hit with more than 15 partners takes the search-again
 * path); a negative value restores the default of one pool chunk per hit.  Errors: INVALID_ARG
 * (null context).
 */
int gnn_debug_graph_pool(gnn_ctx* ctx, int64_t chunks);

/*
 * gnn_csr_build_noalloc -- the destination-keyed CSR of an edge list, built
 * without allocating any device memory.  (Library plumbing: the paper has no
 * counterpart.)  It is for callers that must not allocate: a serving backend
 * or host framework whose memory planner owns every device allocation and
 * forbids new ones after start-up, or code that must keep cudaMalloc and
 * cudaFree (and their implicit device synchronisation) off its request path.
 *
 * Scratch is one fixed, library-owned device array of
 * GNN_CSR_NOALLOC_SCRATCH_BYTES bytes, allocated when the library is loaded
 * on a device and held by every device that loads the library until the
 * process exits.  The caller provides only inputs and outputs:
 *   edge_index device int32 [2, n_edges] (row 0 sources, row 1 destinations)
 *   rowptr     device int32 [n_nodes + 1]: first sorted slot of each node
 *   perm       device int32 [n_edges]: input edge id of each sorted slot
 *   src_sorted device int32 [n_edges]: source of each sorted slot
 * The result is bit-identical to the CSR gnn_infer builds: edges stably
 * sorted by destination (ties keep input order).  Edges with an endpoint
 * outside [0, n_nodes) are placed after rowptr[n_nodes], in input order,
 * with source 0: rowptr[n_nodes] < n_edges is the only signal of them (this
 * call has no context, so no error word records them).
 * Limits: n_edges <= GNN_CSR_NOALLOC_MAX_EDGES and 0 <= n_nodes <= GNN_MAX_COUNT;
 * larger sizes, negative sizes or null pointers return GNN_ERR_INVALID_ARG
 * before any device work.  Every call looks up the scratch array's device
 * address in the current context (cudaGetSymbolAddress: it allocates and
 * enqueues nothing, and follows the array when a device reset or another
 * context gives it a new address); the first call in a context may load the
 * library's device code, so make that first call outside any stream capture.
 * All calls share the one array and it keeps the last
 * call's contents (nothing in it needs to start at zero); calls that overlap
 * on the GPU (several streams, or several host threads) race on it and must
 * be serialised by the caller.  Enqueued on `stream`; no host synchronisation.
 * Errors: INVALID_ARG, CUDA.
 */
#define GNN_CSR_NOALLOC_MAX_EDGES (1 << 20)
#define GNN_CSR_NOALLOC_SCRATCH_BYTES (5u * 4u * GNN_CSR_NOALLOC_MAX_EDGES + 4u * 256u * 256u)
int gnn_csr_build_noalloc(const int32_t* edge_index, int64_t n_nodes, int64_t n_edges, int32_t* rowptr,
                          int32_t* perm, int32_t* src_sorted, gnn_stream_t stream);

/*
 * Hits as a sequence.  An event's hits in order (of azimuth, or along a track) can be read as a
 * sequence: queries and keys of every hit are normalised for each head and rotated by their
 * positions, and a hit attends to a window of the order and to a few first tokens that stay
 * visible.  The calls below are those three steps, for a batch of whole events at once and for new
 * hits over a cache of earlier ones.  (Library operators: the paper has no counterpart.)  They need
 * no gnn_ctx.  Arrays and streams are those of the current device.
 *
 * gnn_heads -- a view of a device array [rows, n_heads, head_dim] of one of the types below: element
 * (r, h, d) at data + r * row_stride + h * head_stride + d, strides in elements, so that slices of a
 * packed projection and either order of rows and heads are views.  Strides are not negative.
 */
enum gnn_dtype {
  GNN_DTYPE_FP32 = 0,
  GNN_DTYPE_BF16 = 1,
  GNN_DTYPE_FP16 = 2,
};

typedef struct gnn_heads {
  void* data;
  int64_t row_stride, head_stride;
  int32_t n_heads;
  int32_t reserved;            /* 0 */
} gnn_heads;

/*
 * gnn_rotary_init -- the table of a rotation, computed on the host (no device work): frequencies
 * f_i = base^(-2 i / rot_dim), i < rot_dim / 2, in radians a position, scaled for positions beyond
 * those a model was made for:
 *   GNN_ROTARY_PLAIN    f_i
 *   GNN_ROTARY_LINEAR   f_i / factor
 *   GNN_ROTARY_BY_TURNS f_i (g + (1 - g) / factor), g = clamp((n_i - slow) / (fast - slow), 0, 1), with
 *                       n_i = length f_i / 2 pi the turns pair i makes over `length` positions: fast
 *                       pairs stay, slow ones are stretched
 * Pair i is the elements i and i + rot_dim / 2 of a head (GNN_ROTARY_HALF) or 2 i and 2 i + 1
 * (GNN_ROTARY_INTERLEAVED); elements from rot_dim on pass unrotated.  A pair (u, w) at position x
 * becomes amplitude * (u cos - w sin, w cos + u sin) of the angle x f_i.  The table is the caller's;
 * every field of it is read-only after this call.  Errors: INVALID_ARG (null pointer, rot_dim odd or
 * outside 2..256, unknown layout or scaling, base or factor not positive and finite, amplitude not finite,
 * by turns: length <= 0, slow < 0 or fast <= slow).
 */
enum gnn_rotary_layout { GNN_ROTARY_HALF = 0, GNN_ROTARY_INTERLEAVED = 1 };
enum gnn_rotary_scaling { GNN_ROTARY_PLAIN = 0, GNN_ROTARY_LINEAR = 1, GNN_ROTARY_BY_TURNS = 2 };

typedef struct gnn_rotary_config {
  int32_t rot_dim, layout, scaling;
  int32_t reserved;            /* 0 */
  double base, factor, length, slow, fast, amplitude;
} gnn_rotary_config;

typedef struct gnn_rotary {
  int32_t rot_dim, layout;
  float amplitude;
  int32_t magic;               /* set by gnn_rotary_init */
  uint64_t turn_fixed[128];          /* f_i / 2 pi, modulo 1, in units of 2^-64 */
  float turn_hi[128], turn_lo[128];  /* f_i / 2 pi as a sum of two floats */
} gnn_rotary;

int gnn_rotary_init(const gnn_rotary_config* cfg, gnn_rotary* out);

/*
 * gnn_rope -- rotate every head of x by its row's position.
 *   x, y       views of n_rows rows with the same n_heads; y may be x itself (same strides), otherwise
 *              they do not overlap
 *   positions  device, int32 [n_rows] or, with positions_float != 0, float32 [n_rows]; NULL: row number
 * head_dim 1..256, at least rot_dim, even.  Angles keep fp32 accuracy at any int32 position and at
 * float32 ones up to 2^24; the arithmetic is fp32, rounded once.  Enqueued on `stream`.  n_rows == 0 is a no-op.
 * Errors: INVALID_ARG (null pointer, table not made by gnn_rotary_init, unknown type, head_dim, n_heads < 1 or
 * unequal, negative stride, data not aligned to its elements, sizes above GNN_MAX_COUNT), CUDA.
 *
 * gnn_qk_norm_rope -- q and k of every row: x / sqrt(mean(x^2) + eps) over each head, times the gain of each
 * element, then the rotation, rounded once; v is copied.  One launch.
 *   q, k, v              input views of n_rows rows; v may be NULL (then v_out is NULL too); k and v have
 *                        the same n_heads
 *   q_gain, k_gain       device float32 [head_dim], or NULL: 1
 *   q_out, k_out, v_out  output views; each may be its input (rows == NULL, same strides), otherwise
 *                        outputs overlap nothing
 *   rows                 device int64 [n_rows], or NULL: row r of k and v goes to row rows[r] of k_out and
 *                        v_out (the rows of a cache), of which there are out_rows; a row outside [0, out_rows) is
 *                        not written; no two may be equal.  NULL: row r (out_rows is not read)
 * eps > 0.  positions, types, limits and errors as for gnn_rope.
 */
int gnn_rope(const gnn_rotary* rot, int dtype, int head_dim, const gnn_heads* x, const gnn_heads* y,
             const void* positions, int positions_float, int64_t n_rows, gnn_stream_t stream);
int gnn_qk_norm_rope(const gnn_rotary* rot, int dtype, int head_dim, float eps, const float* q_gain,
                     const float* k_gain, const gnn_heads* q, const gnn_heads* k, const gnn_heads* v,
                     const gnn_heads* q_out, const gnn_heads* k_out, const gnn_heads* v_out, const void* positions,
                     int positions_float, const int64_t* rows, int64_t out_rows, int64_t n_rows,
                     gnn_stream_t stream);

/*
 * gnn_attention_run -- attention with a sliding window and first tokens that stay visible, for n_seqs
 * sequences at once.  Sequence b has the query rows q_start[b] .. q_start[b + 1] - 1 and the kv_len[b] key
 * (and value) rows from kv_start[b] on.  Its queries are the last ones of the sequence: query i of nq stands at
 * position p = kv_len[b] - nq + i and sees key j when
 *   j <= p + right  and  (j >= p - left  or  j < sinks);      left, right < 0: no bound.
 * out = sum over the visible j of softmax_j(scale * q . k_j) v_j, head by head; query head h reads key head
 * h / (q.n_heads / k.n_heads).  A query that sees no key, or whose visible scores are all -inf, gets zeros.  A scale of 0
 * is taken as one too small to change a weight (a q . k_j of -inf weighs nothing then too).  An infinite value that a query
 * sees makes its result infinite or, where the value's weight rounds to zero, NaN.
 * Keys that a query does not see take no part in its result, whatever they hold (NaN and infinities too),
 * nor do rows outside the sequence.  A row that comes out not finite is computed again, key by key, which is slow: a NaN
 * that every query of a large event sees costs hundreds of times the call's time.
 *   dtype           GNN_DTYPE_BF16 or GNN_DTYPE_FP16, of q, k, v and out; scores, sums and outputs are held in
 *                   fp32, the weights that multiply v are rounded to dtype (their sum is not)
 *   head_dim        a multiple of 8, 8..128
 *   q, k, v, out    views of n_q_rows (q, out) and n_kv_rows (k, v) rows; data 16-byte aligned, strides
 *                   positive multiples of 8 elements below 2^39; q.n_heads a multiple of k.n_heads == v.n_heads,
 *                   at most 4096.
 *                   out overlaps no input
 *   q_start         device int32 [n_seqs + 1], not decreasing; rows before the first and from the last on are
 *                   not written
 *   kv_start, kv_len  device int32 [n_seqs]; both NULL: a sequence's keys are the rows of its queries
 *   max_q, max_kv   the most queries and keys of a sequence; 0: not known (n_q_rows, n_kv_rows).  A sequence with
 *                   more queries than max_q is INDEX_RANGE and its rows are undefined; max_kv only shapes the launch
 * Device arrays of offsets that point outside the views are cut to them and reported as INDEX_RANGE by
 * gnn_attention_status.  Enqueued on `stream`; only enqueues kernels (it can be captured).  The same inputs
 * give bitwise-identical outputs.
 * Errors: INVALID_ARG (null pointer, any limit above, scale not finite, sinks < 0, sizes above GNN_MAX_COUNT,
 * n_seqs above 2^28, 2^31 or more tiles of 128 queries for one key head, a handle of another device than the current
 * one), CUDA.
 *
 * gnn_attention_create -- a handle on the current device: the workspace of calls with few queries and the
 * device error word.  Synchronous.  One handle per stream: it is not safe for concurrent use.  Errors:
 * INVALID_ARG, OOM, CUDA.
 * gnn_attention_status -- synchronise `stream`, then return and clear the handle's error word: GNN_OK,
 * GNN_ERR_INDEX_RANGE, GNN_ERR_DEVICE_TIMEOUT or GNN_ERR_CUDA.
 * gnn_attention_destroy -- wait for the device and free the handle.  NULL is a no-op.
 */
typedef struct gnn_attention gnn_attention;

typedef struct gnn_attention_call {
  int32_t dtype, head_dim;
  gnn_heads q, k, v, out;
  const int32_t* q_start;
  const int32_t* kv_start;
  const int32_t* kv_len;
  int64_t n_q_rows, n_kv_rows;
  int32_t n_seqs, max_q, max_kv;
  int32_t left, right, sinks;
  float scale;
  int32_t reserved;            /* 0 */
} gnn_attention_call;

int gnn_attention_create(gnn_attention** out);
int gnn_attention_run(gnn_attention* att, const gnn_attention_call* call, gnn_stream_t stream);
int gnn_attention_status(gnn_attention* att, gnn_stream_t stream);
void gnn_attention_destroy(gnn_attention* att);

/*
 * Several hypotheses of a sequence.  A decoder that extends tracks hit by hit keeps a few hypotheses (beams) of each
 * event.  Their keys and values lie in pages, the event's own tokens once for all of them; the calls below append new
 * rows, attend over the event's rows and each hypothesis' own, choose the best continuations and move the states
 * to them.  (Library operators: the paper has no counterpart.)
 *
 * gnn_pages -- a cache in pages: position j of sequence b lies in row table[b * table_stride + j / page_size] * page_size
 * + j % page_size of k and v, views of n_pages * page_size rows.
 *   dtype, head_dim  of k and v
 *   page_size     a power of two, 16..1024
 *   table         device int32, n_seqs rows of table_width entries; entries that no position below kv_len uses are not
 *                 read.  Sequences may have pages in common
 *   kv_len        device int32 [n_seqs]: each sequence's positions, those of new rows among them
 *   status        device uint32, zero before the first call: where calls report what they find
 * Entries outside [0, n_pages), lengths below zero or past the table's, and offsets that fall or lie outside the views that a call
 * is given are reported as INDEX_RANGE, of whichever sequence; no such row is read or written, and the results of the sequences
 * that they belong to are undefined.  A cache is these arrays and nothing else: there is no handle, and calls on several streams may use one at once.
 *
 * gnn_paged_status -- read a status word behind the work of `stream` so far, clear it, and return what it said: GNN_OK,
 * GNN_ERR_INDEX_RANGE, GNN_ERR_DEVICE_TIMEOUT or GNN_ERR_CUDA.  Waits for `stream`.  Errors: INVALID_ARG (NULL, misaligned).
 */
typedef struct gnn_pages {
  gnn_heads k, v;
  int64_t n_pages;
  int32_t dtype, head_dim, page_size, table_width;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* kv_len;
  int32_t n_seqs;
  int32_t reserved;            /* 0 */
  uint32_t* status;
} gnn_pages;

int gnn_paged_status(uint32_t* status, gnn_stream_t stream);

/*
 * gnn_paged_append -- new rows of keys and values into their pages.  Rows q_start[b] .. q_start[b + 1] - 1 are the last
 * positions of sequence b, of kv_len[b] with them: each key is rotated (and normalised first, with eps > 0, as by
 * gnn_qk_norm_rope) and written to its place, values are copied, and so are queries, when given, to q_out.  One launch.
 *   rot              table of the rotation
 *   q, q_out         views of n_rows rows, or data NULL in both: no queries.  q_out may be q (same strides)
 *   k, v             views of n_rows rows with the cache's heads, which overlap no page
 *   q_gain, k_gain   device float32 [head_dim], or NULL: 1; only with eps > 0
 *   eps              0: no norms
 *   positions        device, of the rotation, int32 [n_rows] or, with positions_float != 0, float32 [n_rows]; NULL: those in
 *                    the sequences
 *   q_start          device int32 [n_seqs + 1], not decreasing; rows before the first and from the last on are skipped
 * The key and value of a row whose position is below zero (a sequence with fewer positions than rows) are not written; its query
 * is, to q_out.  No place may be that of two rows.  Types, head_dim and limits as for gnn_rope.  Enqueued on `stream`; n_rows == 0 or n_seqs == 0 is a no-op.
 * Errors: INVALID_ARG, CUDA.
 */
typedef struct gnn_append_call {
  gnn_heads q, k, v, q_out;
  const float* q_gain;
  const float* k_gain;
  const void* positions;
  const int32_t* q_start;
  int64_t n_rows;
  float eps;
  int32_t positions_float;
} gnn_append_call;

int gnn_paged_append(const gnn_pages* pages, const gnn_rotary* rot, const gnn_append_call* call, gnn_stream_t stream);

/*
 * gnn_paged_attend -- attention of new queries over a cache in pages.  Query i of the nq rows of sequence b stands at
 * position p = kv_len[b] - nq + i and sees its keys j <= p:
 *   out = sum over j of softmax_j(scale * q . k_j) v_j, head by head; query head h reads key head h / (q.n_heads /
 * k.n_heads).  A query that sees no key, or whose scores are all -inf, gets zeros.
 * Sequences group_start[g] .. group_start[g + 1] - 1 share their first shared_len[g] positions: those are read once for all
 * of them, through the pages of the first.  (The others' entries for them are not read.)  Sequences of no group share nothing.
 * What a query does not see takes no part in its result, whatever it holds.  An infinite or NaN value that a query sees
 * makes its result infinite or NaN.  A scale of 0 is taken as one too small to change a weight.
 *   pages            GNN_DTYPE_BF16 or GNN_DTYPE_FP16; head_dim a multiple of 8, 8..128; k, v: data 16-byte aligned,
 *                    strides positive multiples of 8 elements
 *   q, out           views of n_q_rows rows, in the same way; q.n_heads a multiple of the cache's heads, at most
 *                    4096, at most 128 query heads to a key head, and fewer than 2^32 query rows times heads.  out overlaps no
 *                    input
 *   q_start          device int32 [n_seqs + 1], not decreasing; rows before the first and from the last on are not written
 *   group_start      device int32 [n_groups + 1], not decreasing, and shared_len, device int32 [n_groups]; both NULL with
 *                    n_groups 0.  Groups may be empty
 *   max_q            the most queries of a sequence; 0: not known.  Short sequences are computed together only where it is known
 *                    (20,000 of up to 30 keys: 0.19 ms, else 1.2).  A sequence with more is INDEX_RANGE, its rows undefined
 *   workspace        device, 32-byte aligned, of at least the bytes that gnn_paged_workspace says for the same call; written
 *                    before it is read, so its contents need not be anything.  Calls that may overlap have one each.
 *                    Two parts of 4 (head_dim + 2) bytes for each query row and head, as many again with groups, up to 512
 *                    parts for each SM, and some 8 bytes for each sequence, group and key head: the call is for few new rows at a time,
 *                    not for whole prompts
 * Positions are below 2^30.  A sequence some of whose queries stand below its group's shared_len is computed row by row, which is
 * slow.  Scores, sums and outputs are held in fp32, the weights that multiply v are rounded to dtype (their sum is not).
 * Enqueued on `stream`; only enqueues kernels (it can be captured).  The same inputs give bitwise-identical outputs.
 * Errors: INVALID_ARG (any limit above, a workspace that is too small), CUDA.
 */
typedef struct gnn_paged_call {
  gnn_heads q, out;
  const int32_t* q_start;
  const int32_t* group_start;
  const int32_t* shared_len;
  int64_t n_q_rows;
  int32_t n_groups, max_q;
  float scale;
  int32_t reserved;            /* 0 */
  void* workspace;
  uint64_t workspace_bytes;
} gnn_paged_call;

int gnn_paged_workspace(const gnn_pages* pages, const gnn_paged_call* call, uint64_t* bytes);
int gnn_paged_attend(const gnn_pages* pages, const gnn_paged_call* call, gnn_stream_t stream);

/*
 * gnn_beam_select -- the best continuations of each group of `beams` hypotheses.  Hypothesis b (row b of logits, scores)
 * goes on with token t at
 *   value(b, t) = scores[b] + logits[b, t] - log(sum over t of exp(logits[b, t]))
 * and the `best` largest values of a group's hypotheses and tokens come out in order, ties to the lowest
 * (hypothesis, token): out_scores (value), out_parents (hypothesis, 0 .. beams - 1 within the group), out_tokens, each
 * [n_groups * best].  A hypothesis that has ended (ended[b] != 0) has one continuation: token end_token at scores[b]; its
 * logits are not read.  A value of -inf is no continuation; a row whose logits hold NaN or +inf, or whose score is
 * NaN, has none.  Where there are fewer than `best`, the rest is -inf, parent 0, token -1.  Logits may have any finite magnitude:
 * large negative numbers (masks) weigh nothing beside others, and a row of nothing else is an even choice.  (A value that is chosen
 * and lies below what fp32 holds comes out as -inf, with its parent and token.)
 * Values are held and compared to about 1e-7 (their order within a row is that of the logits, exactly).
 *   dtype, logits    of any gnn_dtype, device [n_groups * beams, vocab], row_stride elements apart, aligned to elements
 *   scores           device float32 [n_groups * beams];  ended  device uint8 [n_groups * beams], or NULL
 *   beams, best      1..64;  vocab 1..GNN_MAX_COUNT
 *   workspace        as for gnn_paged_attend, of the bytes that gnn_beam_workspace says
 * The same inputs give bitwise-identical outputs.  Enqueued on `stream`; n_groups == 0 is a no-op.
 * Errors: INVALID_ARG (n_groups * beams above GNN_MAX_COUNT too), CUDA.
 */
typedef struct gnn_beam_call {
  const void* logits;
  int64_t row_stride, n_groups;
  const float* scores;
  const uint8_t* ended;
  int32_t dtype, beams, vocab, best, end_token;
  int32_t reserved;            /* 0 */
  float* out_scores;
  int32_t* out_parents;
  int32_t* out_tokens;
  void* workspace;
  uint64_t workspace_bytes;
} gnn_beam_call;

int gnn_beam_workspace(const gnn_beam_call* call, uint64_t* bytes);
int gnn_beam_select(const gnn_beam_call* call, gnn_stream_t stream);

/*
 * gnn_beam_reorder -- states of hypotheses moved to those that continue them: in every group of `beams` slots, slot i of
 * each of n_states arrays gets what slot parents[i] of it held.
 *   parents          device int32 [n_groups * beams], 0 .. beams - 1 within the group; a slot whose parent is
 *                    outside that keeps its own
 *   states           host array; data has n_groups * beams rows of row_bytes bytes, `stride` bytes apart (stride >=
 *                    row_bytes); out: the same out_stride bytes apart, or data itself (same strides): in place.  Arrays
 *                    do not overlap otherwise; two states with one out are refused
 *   beams            1..64;  n_groups at most 2^26
 * Enqueued on `stream`; no workspace.  With n_groups == 0 the arguments are checked and nothing is done.  Errors: INVALID_ARG, CUDA.
 *
 * gnn_paged_reorder -- the same for caches in pages, whose sequences are the hypotheses: n_caches caches (of a model's
 * layers) that share one table and kv_len, n_seqs = n_groups * beams.  Views of keys or values that are the same (data, type, sizes and
 * strides) are moved once; such that have only the same data are refused, and views do not overlap otherwise.  In place: a slot's entries for its parent's full
 * pages become the parent's (such pages are shared from then on: append writes none of them), and the rows of the
 * page that the parent has begun are copied into the slot's own page of the same number.  So every slot has, from its first page
 * that is not full on, pages of its own.  kv_len is not written: the slots of a group have the same (a group whose
 * slots have not, or whose length is outside the table's, is INDEX_RANGE, in the first cache's status, whether any of its slots
 * moves or not, and is left as it is; so is one with slots that move where a slot's own page is outside the pages).
 * Types: any gnn_dtype.
 */
typedef struct gnn_beam_state {
  void* data;
  void* out;
  int64_t stride, out_stride, row_bytes;
} gnn_beam_state;

int gnn_beam_reorder(const int32_t* parents, int64_t n_groups, int32_t beams, const gnn_beam_state* states, int32_t n_states,
                     gnn_stream_t stream);
int gnn_paged_reorder(const gnn_pages* caches, int32_t n_caches, const int32_t* parents, int64_t n_groups, int32_t beams,
                      gnn_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* GNN_GB300_H */
