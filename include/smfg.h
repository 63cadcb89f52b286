/*
 * smfg - sampled mini-batch preparation for GNN training / inference on one AMD MI355X.
 *
 * C ABI of libsmfg.so.  The library computes, on the GPU, what the paper's batch-preparation
 * step computes on CPU cores (paper section 4.1 and Listing 1, lines 2-3):
 *
 *   1. node-wise neighbour sampling: for every destination node take at most d_h of its
 *      neighbours, uniformly, without replacement (section 2.2, "node-wise sampling";
 *      section 4.1, first paragraph), one fanout d_h per hop;
 *   2. construction of one bipartite block per hop with compact local node ids: destination
 *      nodes keep the first local ids in their given order, every other node gets the next id
 *      at its first appearance when scanning destinations in order and each destination's
 *      samples in slot order (the MFG construction algorithm, procedure OneHopMFG); hops are
 *      chained, the node list of hop h being the destination list of hop h+1 (section 4.1);
 *   3. the feature slice xs = x[ids] for the final node list (Listing 1).
 *
 * A fanout may also be SMFG_FANOUT_ALL: the full neighbourhood, as the paper's inference
 * experiments use it next to sampled fanouts (section 5, Table 6).
 *
 * Conventions fixed where the paper is silent:
 *   - fanouts[0] belongs to hop 0, whose destinations are the seeds;
 *   - a node with degree <= d_h contributes its whole CSR row in CSR order (no random draw);
 *     otherwise d_h distinct row positions are chosen by Floyd's subset algorithm, slot s
 *     holding the s-th pick;
 *   - random words come from Philox4x32-10 (Salmon et al., SC'11) with key = (low, high) 32-bit
 *     halves of rng_key and counter = (destination node, hop, s / 4, 0), word s % 4; a word r
 *     gives an index in [0, m) as floor(r * m / 2^32);
 *   - block h is a CSR keyed by destination: indptr[h] has n_h + 1 entries, indices[h] holds the
 *     local ids of the sampled source nodes; destination i and source i are the same node.
 * The result is a pure function of (graph, seeds, fanouts, rng_key).
 *
 * All "device" pointers are HIP device memory on the device that was current when the graph
 * handle was created.  The caller allocates and frees every input and output buffer; handles
 * own only their private scratch.  No function throws or aborts; every function returns SMFG_OK
 * or a negative SMFG_ERR_* code.  Conditions only the GPU can see are reported as a positive
 * SMFG_ST_* value in counts[2L+1]; outputs are then unspecified but nothing is written out of
 * bounds.
 */
#ifndef SMFG_H_
#define SMFG_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SMFG_MAX_LAYERS 8
#define SMFG_MAX_FANOUT 32         /* fanouts up to here take the fast path (one lane per slot)   */
#define SMFG_MAX_WIDE_FANOUT 1024  /* larger fanouts, up to here, take the wide path               */
#define SMFG_FANOUT_ALL (-1)       /* every neighbour (full neighbourhood, no draw); wide path     */
#define SMFG_MAX_BATCHES 16 /* batches per smfg_sample_mfg_many call */

/* host-detected errors (return values) */
#define SMFG_OK 0
#define SMFG_ERR_INVALID_ARG (-1)
#define SMFG_ERR_NULL_PTR (-2)
#define SMFG_ERR_BAD_FANOUT (-3)      /* d is neither SMFG_FANOUT_ALL nor in [1, SMFG_MAX_WIDE_FANOUT] */
#define SMFG_ERR_TOO_MANY_LAYERS (-4) /* L < 1 or L > SMFG_MAX_LAYERS */
#define SMFG_ERR_TOO_MANY_SEEDS (-5)  /* more seeds than the workspace / output was sized for */
#define SMFG_ERR_OOM (-6)             /* scratch allocation failed */
#define SMFG_ERR_CAPACITY (-7)        /* output capacities exceed what the workspace supports */
#define SMFG_ERR_BAD_GRAPH (-8)       /* smfg_graph_validate found a broken CSR array */
#define SMFG_ERR_HIP_BASE (-1000)     /* a HIP call failed: code = SMFG_ERR_HIP_BASE - hipError_t */

/* device-detected conditions (value of counts[2L+1]) */
#define SMFG_ST_OK 0
#define SMFG_ST_NODE_CAPACITY 1     /* more distinct nodes than out->node_capacity */
#define SMFG_ST_EDGE_CAPACITY 2     /* a block has more edges than out->edge_capacity[h] */
#define SMFG_ST_TABLE_FULL 3        /* dedup table exhausted (only if node capacity is too) */
#define SMFG_ST_SEED_OUT_OF_RANGE 4 /* a seed is < 0 or >= num_nodes */
#define SMFG_ST_DUPLICATE_SEED 5    /* the seed list holds a node twice */
#define SMFG_ST_INTERNAL 6          /* a kernel met a state its own invariants exclude (a defect, or
                                       scratch memory overwritten from outside during the call) */

typedef struct smfg_graph smfg_graph_t;         /* opaque; BORROWS the device arrays given to it */
typedef struct smfg_workspace smfg_workspace_t; /* opaque; OWNS the scratch of one in-flight batch */

/*
 * Input graph G and feature matrix X (section 2.1: X is n x f, row v the features of node v;
 * N(v) = {u : (u,v) in E}).  CSR row v = the neighbours N(v) of v; rows must not contain
 * duplicates (else "without replacement" holds for positions, not neighbours).
 *   d_indptr   device, int64 [num_nodes + 1], non-decreasing, d_indptr[0] = 0; each degree < 2^31
 *   d_indices  device, int32 [num_edges], values in [0, num_nodes)
 *              (both naturally aligned, like every typed pointer of this interface: a pointer that
 *              is not a multiple of its element size is refused with SMFG_ERR_INVALID_ARG)
 *   d_feat     device, row-major, row v at byte offset v * row_stride_bytes, the first
 *              feat_dim * elem_bytes bytes of a row are its features (any elem_bytes >= 1;
 *              rows are moved as opaque bytes, no conversion).  May be NULL: no gather then.
 * num_nodes < 2^31.  The arrays are not copied and must outlive the handle.
 */
int smfg_graph_create(smfg_graph_t **out, int64_t num_nodes, int64_t num_edges,
                      const int64_t *d_indptr, const int32_t *d_indices, const void *d_feat,
                      int32_t feat_dim, int32_t elem_bytes, int64_t row_stride_bytes);
int smfg_graph_destroy(smfg_graph_t *g);

/*
 * Optional check of the borrowed CSR arrays against the conditions above, for callers that do
 * not trust their input: the sampling calls themselves check seeds, not the graph, and follow a
 * bad offset or neighbour id out of bounds.  One streaming pass over d_indptr and d_indices on
 * hip_stream, then a synchronisation of that stream; allocates and frees 4 bytes of device memory
 * (not for use inside a stream capture).  Returns SMFG_OK, or SMFG_ERR_BAD_GRAPH with the OR of
 * the SMFG_BAD_* bits below in *h_flags (host, may be NULL).  Duplicates inside a row are not
 * looked for.
 */
#define SMFG_BAD_INDPTR_START 1u /* d_indptr[0] != 0 */
#define SMFG_BAD_INDPTR_ORDER 2u /* some d_indptr[v+1] < d_indptr[v], or a degree >= 2^31 */
#define SMFG_BAD_INDPTR_END 4u   /* d_indptr[num_nodes] != num_edges */
#define SMFG_BAD_INDEX_RANGE 8u  /* some d_indices[e] outside [0, num_nodes) */
int smfg_graph_validate(const smfg_graph_t *g, uint32_t *h_flags, void *hip_stream);

/*
 * Optional label vector y (Listing 1: ys = y[ids[:batch_size]], the labels of the seed nodes).
 * d_labels: device, num_nodes elements of elem_bytes (1, 2, 4 or 8) each, borrowed like the other
 * arrays; NULL removes it.  A batch whose output has a non-NULL `labels` buffer then receives
 * labels[i] = y[seed i], copied as opaque bytes.
 */
int smfg_graph_set_labels(smfg_graph_t *g, const void *d_labels, int32_t elem_bytes);

/*
 * Worst-case sizes (host only, pure).  With disjoint neighbourhoods (section 3 draft text on
 * neighbourhood expansion) n_{h+1} <= min(num_nodes, n_h (1 + d_h)) and E_h <= n_h d_h.
 *   max_nodes host [L + 1], max_edges host [L].  From the first hop with SMFG_FANOUT_ALL on, the
 * bounds are num_nodes nodes and -1 (unknown without the degrees) edges; E_h never exceeds the
 * graph's num_edges, because destinations are distinct.
 */
int smfg_bounds(int32_t num_seeds, int32_t L, const int32_t *fanouts, int64_t num_nodes,
                int64_t *max_nodes, int64_t *max_edges);

/*
 * Scratch for one batch in flight: per-sample and per-row state, scan partials and, by dedup
 * strategy (smfg_workspace_strategy), the records of a hop with their bucket counts and offsets,
 * or a dedup table (>= 2 slots per node of capacity).  Sized for up to max_seeds seeds, the given
 * fanouts (a later call may use the same or smaller fanouts / fewer hops) and node_capacity
 * distinct nodes (0 = the worst case of smfg_bounds).  Allocates device memory with hipMalloc,
 * zeroes part of it and synchronises the device once; not for use inside a stream capture.
 */
int smfg_workspace_create(smfg_workspace_t **out, const smfg_graph_t *g, int32_t max_seeds,
                          int32_t L, const int32_t *fanouts, int64_t node_capacity);
/*
 * The same with an explicit bound on the samples of a single hop (sample_capacity >= max_h E_h;
 * 0 = derive it from the fanouts as smfg_workspace_create does).  Needed when a fanout is
 * SMFG_FANOUT_ALL, or when the derived worst case (destinations x fanout) would exceed the 2^30
 * positions a hop can address.  A hop that draws more samples ends with SMFG_ST_EDGE_CAPACITY.
 * Calls whose fanouts are all <= SMFG_MAX_FANOUT address samples at padded positions
 * (destination x fanout + slot): for them the capacity must cover destinations x fanout of every
 * hop, else the call returns SMFG_ERR_CAPACITY.
 */
int smfg_workspace_create_sized(smfg_workspace_t **out, const smfg_graph_t *g, int32_t max_seeds,
                                int32_t L, const int32_t *fanouts, int64_t node_capacity,
                                int64_t sample_capacity);
int smfg_workspace_destroy(smfg_workspace_t *ws);
/* Bytes of device scratch the workspace holds (0 for NULL). */
int64_t smfg_workspace_bytes(const smfg_workspace_t *ws);
/*
 * How calls on this workspace remove duplicates and number new nodes (the global-to-local map of
 * procedure OneHopMFG); both give the same, serial-order result.
 *   SMFG_STRATEGY_PARTITION  the records of a hop (known nodes, samples) are grouped by node hash
 *                            and every group is settled in a hash table in on-chip memory: no
 *                            table in device memory, no device-wide atomics.  The default.
 *   SMFG_STRATEGY_TABLE      one open-addressing table in device memory per batch, claimed with
 *                            atomics.  Chosen when no hop of the planned size reaches 32768
 *                            records.
 * A call whose own hops all stay below that, on a workspace of either kind, reads all its records in every
 * one of a few blocks instead (one or two launches per hop and at most one before the first; such calls are launch bound): no table in
 * device memory, no atomics.  On partition workspaces the first hops of a larger call do so as well, unless
 * it is a set of more than four batches that leaves the gather to another call.  The result is the same again.
 * The environment variable SMFG_DEDUP=table or =partition, read when a workspace is created,
 * overrides the choice, for small calls as well (for measurements and tests).  Returns -1 for NULL.
 */
#define SMFG_STRATEGY_TABLE 0
#define SMFG_STRATEGY_PARTITION 1
int smfg_workspace_strategy(const smfg_workspace_t *ws);

/* Output of one batch.  Every pointer is a caller-owned DEVICE buffer. */
typedef struct {
  int32_t *indptr[SMFG_MAX_LAYERS];  /* hop h: [node_capacity + 1]; n_h + 1 entries are written   */
  int32_t *indices[SMFG_MAX_LAYERS]; /* hop h: [edge_capacity[h]]; E_h local source ids written   */
  int32_t *node_ids;                 /* [node_capacity] global ids; N_h = the first n_h entries   */
  void *features;                    /* [node_capacity x feat_dim*elem_bytes] dense rows, or NULL */
  int64_t *counts;                   /* [2L+2]: n_0..n_L, E_0..E_{L-1}, status                    */
  int64_t node_capacity;
  int64_t edge_capacity[SMFG_MAX_LAYERS];
  void *labels;                      /* [num_seeds x label elem_bytes], or NULL (needs graph labels) */
} smfg_output_t;

/*
 * sample_mfg(graph, seeds, fanouts, rng_key) -> per-hop MFG blocks + node ids + gathered features.
 * Enqueues all work on `hip_stream` (a hipStream_t, NULL = the default stream) and returns
 * without waiting; nothing is copied to the host.  d_seeds: device int32 [num_seeds], distinct,
 * in [0, num_nodes).  fanouts: host int32 [L].  `out` is read during the call only (the struct
 * itself is host memory).  The workspace must not be used by another call until this one has
 * finished on the GPU.  num_seeds = 0 is allowed (all counts 0).
 */
int smfg_sample_mfg(const smfg_graph_t *g, smfg_workspace_t *ws, const int32_t *d_seeds,
                    int32_t num_seeds, const int32_t *fanouts, int32_t L, uint64_t rng_key,
                    const smfg_output_t *out, void *hip_stream);

/*
 * smfg_sample_mfg for callers that cannot allocate device memory or hold a workspace handle: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs,
 * outputs and results as smfg_sample_mfg, but the scratch lives in a fixed array inside the
 * library (SMFG_STATIC_SCRATCH_BYTES per GPU, held from the library's load until the process
 * ends) and the call allocates and frees nothing.  The scratch needed grows with
 * out->node_capacity and the fanouts exactly as smfg_workspace_bytes reports for a workspace
 * created with (num_seeds, fanouts, out->node_capacity); a call that needs more than the array
 * holds returns SMFG_ERR_CAPACITY and launches nothing (pass a smaller out->node_capacity - a
 * batch that outgrows it ends with SMFG_ST_NODE_CAPACITY - or use a workspace).  Fanouts must be
 * in [1, SMFG_MAX_WIDE_FANOUT] (SMFG_FANOUT_ALL has no size bound without a workspace:
 * SMFG_ERR_INVALID_ARG).  All calls on one GPU share the array: two calls that overlap in time
 * on the same GPU, on any streams, race; order them (one stream, or events).
 */
#define SMFG_STATIC_SCRATCH_BYTES (64u << 20)
int smfg_sample_mfg_static(const smfg_graph_t *g, const int32_t *d_seeds, int32_t num_seeds,
                           const int32_t *fanouts, int32_t L, uint64_t rng_key,
                           const smfg_output_t *out, void *hip_stream);

/*
 * The same for num_batches (1..SMFG_MAX_BATCHES) independent batches in one set of launches:
 * batch b uses ws[b], d_seeds[b], num_seeds[b], rng_keys[b], outs[b]; all share the fanouts.
 * Batches are independent units (section 4.2), so this is how several are kept in flight.
 * Results are identical to num_batches separate smfg_sample_mfg calls.
 */
int smfg_sample_mfg_many(const smfg_graph_t *g, smfg_workspace_t *const *ws,
                         const int32_t *const *d_seeds, const int32_t *num_seeds,
                         const int32_t *fanouts, int32_t L, const uint64_t *rng_keys,
                         const smfg_output_t *outs, int32_t num_batches, void *hip_stream);

/*
 * Only the gather xs = x[ids] (Listing 1): out rows j < *d_num_rows (a device int64) are copied
 * from the graph's feature rows d_node_ids[j].  max_rows bounds the launch.  Asynchronous.
 * An id outside [0, num_nodes) yields a copy of row 0: never a read outside the feature matrix.
 */
int smfg_gather_rows(const smfg_graph_t *g, const int32_t *d_node_ids, const int64_t *d_num_rows,
                     int64_t max_rows, void *d_out, void *hip_stream);

/*
 * The gather stage of smfg_sample_mfg_many on its own, for callers that run it on another stream
 * than the sampling stages (a call with outs[b].features == NULL skips the gather; this function
 * does it later): for every batch b, rows j < counts[L] of outs[b].features are copied from the
 * feature rows outs[b].node_ids[j] (an id outside [0, num_nodes) reads row 0); a batch whose
 * status word is non-zero is skipped.  One launch for all batches.  The caller orders it after the sampling call (same stream, or an event).
 */
int smfg_gather_many(const smfg_graph_t *g, const smfg_output_t *outs, int32_t num_batches,
                     int32_t L, void *hip_stream);

/*
 * A consumer of one MFG block: the mean aggregation of a GraphSAGE layer (Appendix C, GraphSAGE
 * listing: x_target = x[:size[1]], conv((x, x_target), edge_index); equation 1 with agg = mean):
 *   out[i, :] = (1 / k_i) * sum over e in [indptr[i], indptr[i+1]) of float(x[indices[e], :]),
 * k_i = indptr[i+1] - indptr[i]; a destination without samples gets zeros.  i < *d_num_dst (a device
 * int64, e.g. &counts[h]); max_dst bounds the launch (d_indptr holds at least max_dst + 1 entries,
 * d_indices max_edges).  x: device, row-major [max_src x dim], dense, max_src >= 1,
 * elem_bytes 2 (IEEE half) or 4 (float); out: device float [max_dst x dim].  Offsets beyond
 * max_edges and source ids outside [0, max_src) - which only the unspecified arrays of a batch
 * that ended with a status can hold - are clamped (row 0 is read): no read leaves the buffers.  Sums run in float in
 * slot order, then one division: the error of an output is at most k_i * 2^-24 times the mean of
 * the magnitudes added (k_i - 1 rounded additions and one rounded division).  Asynchronous on
 * hip_stream.
 */
int smfg_mean_aggregate(const int32_t *d_indptr, const int32_t *d_indices, int64_t max_edges,
                        const int64_t *d_num_dst, int64_t max_dst, const void *d_x, int64_t max_src,
                        int32_t dim, int32_t elem_bytes, float *d_out, void *hip_stream);

/*
 * One whole GraphSAGE layer over a block, with the aggregation fused into the linear transform
 * (equation 1 with the choices section 2.1 names for GraphSAGE: agg = mean, upd = a linear layer
 * on the concatenation of the node's own representation and the mean; ReLU between layers as in
 * the model listing of Appendix C):
 *   out[i, j] = act(bias[j] + sum_c w[j, c] x[i, c] + sum_c w[j, dim + c] mean_i[c]),  i < *d_num_dst,
 * mean_i as in smfg_mean_aggregate, act = max(., 0) if relu != 0 else the identity.
 *   d_x     device, IEEE half, row-major [max_src x dim], dense, 16-byte aligned; dim a multiple of
 *           8, at most 256.  Destination i is source i, so row i is also the node's own row
 *           (destinations beyond max_src are not computed).
 *   w       IEEE half, row-major [out_dim x 2 dim] (a linear layer's weight: columns [0, dim)
 *           act on the own row, [dim, 2 dim) on the mean); out_dim >= 1.  The layer call takes
 *           it re-arranged for the matrix cores: smfg_sage_pack_weights writes that arrangement
 *           (smfg_sage_packed_bytes bytes, 0 for unsupported sizes; both buffers device, 16-byte
 *           aligned; asynchronous) once per set of weights.
 *   d_bias  device, float [out_dim], or NULL.
 *   d_out   device, row-major [max_dst x out_dim] of out_elem_bytes 2 (half, round to nearest) or
 *           4 (float).
 * Arithmetic: the mean is summed in float in slot order, divided once and rounded to half; the
 * products of halfs are exact and are added in float on the matrix cores in an unspecified order.
 * With S = |bias[j]| + sum_c |w||x| + sum_c |w| mean|x| the error of an output is at most
 * S * (2^-11 + (2 dim + k_i + 2) * 2^-24), plus half an ulp of the half result if out is half.
 * Offsets and source ids are clamped as in smfg_mean_aggregate.  Asynchronous on hip_stream.
 */
int64_t smfg_sage_packed_bytes(int32_t dim, int32_t out_dim);
int smfg_sage_pack_weights(const void *d_w, int32_t dim, int32_t out_dim, void *d_packed,
                           void *hip_stream);
int smfg_sage_layer(const int32_t *d_indptr, const int32_t *d_indices, int64_t max_edges,
                    const int64_t *d_num_dst, int64_t max_dst, const void *d_x, int64_t max_src,
                    int32_t dim, const void *d_w_packed, const float *d_bias, int32_t out_dim, int32_t relu,
                    void *d_out, int32_t out_elem_bytes, void *hip_stream);

/*
 * Operators of a training step over the prepared batches, for what the paper's training loop (Listing 1) leaves to its
 * framework: learned features of nodes that have none and their gradient, layer normalisation and its gradient, and the
 * clipping of all gradients by their global norm.  All are asynchronous on hip_stream, on the current device, allocate and
 * synchronise nothing, and can be captured.  As for the other consumers, the number of rows in use is a device int64 (e.g.
 * &counts[L]), read as at least 0 and at most the max_* that bounds the launch; rows of an output beyond it are not written.
 * Sums run in float or wider and a result is rounded to its type once.  The same inputs give the same bits.
 * Element types are SMFG_DTYPE_*; matrices are row-major with their rows `stride` elements apart (>= dim); dim is in
 * [1, SMFG_MAX_DIM].  Scratch is the caller's device memory of *_scratch_bytes bytes (host only, pure; -1 for sizes that
 * the call refuses), 256-byte aligned, not shared by calls that overlap in time; a call with less returns SMFG_ERR_CAPACITY.
 */
#define SMFG_DTYPE_F32 0  /* float */
#define SMFG_DTYPE_F16 1  /* IEEE half */
#define SMFG_DTYPE_BF16 2 /* bfloat16 */
#define SMFG_MAX_DIM (1 << 23)

/*
 * Embedding: out[i, :] = scale * table[ids[i], :], i < *d_num_ids; a row of zeros for an id outside [0, num_rows) (a padded
 * place): no read leaves the table.
 *   d_table  num_rows x dim, 1 <= num_rows < 2^31;  d_ids  int32 or int64 (id_bytes 4 or 8) [max_ids], max_ids < 2^31
 *   d_out    max_ids x dim, of the table's type, or of any type where the table is of float
 */
int smfg_embedding(const void *d_table, int64_t num_rows, int64_t table_stride, int32_t table_dtype, const void *d_ids,
                   int32_t id_bytes, const int64_t *d_num_ids, int64_t max_ids, int32_t dim, float scale, void *d_out,
                   int64_t out_stride, int32_t out_dtype, void *hip_stream);

/*
 * Its gradient: G[v, :] = scale * sum of dy[i, :] over i < *d_num_ids with ids[i] = v; ids outside [0, num_rows) have none.
 * The sum is made of partial sums over pieces of the sorted ids: a fixed order for given ids and max_ids, but not that of i, and not
 * that of the same tokens among other ids.  d_dy: max_ids x dim.  The gradient is of float or of dy's type.
 *   smfg_embedding_grad       the whole table's, num_rows x dim: rows that no id names are zeros; with accumulate != 0 it
 *                             is added to what d_grad holds, and those rows are not touched
 *   smfg_embedding_grad_rows  the touched rows alone: their number *d_num_unique, their ids ascending in d_row_ids [max_ids] and
 *                             their sums in d_grad (max_ids x dim); nothing is written past *d_num_unique
 * With S = |scale| * sum |dy| over the k summed values (and the value added to) the error of a float result is at most
 * (k + 2) * 2^-24 * S.
 */
int64_t smfg_embedding_grad_scratch_bytes(int64_t max_ids, int64_t num_rows, int32_t dim);
int smfg_embedding_grad(const void *d_ids, int32_t id_bytes, const int64_t *d_num_ids, int64_t max_ids, const void *d_dy,
                        int64_t dy_stride, int32_t dy_dtype, int32_t dim, float scale, void *d_grad, int64_t num_rows,
                        int64_t grad_stride, int32_t grad_dtype, int32_t accumulate, void *d_scratch, int64_t scratch_bytes,
                        void *hip_stream);
int smfg_embedding_grad_rows(const void *d_ids, int32_t id_bytes, const int64_t *d_num_ids, int64_t max_ids,
                             const void *d_dy, int64_t dy_stride, int32_t dy_dtype, int32_t dim, float scale,
                             int64_t num_rows, int32_t *d_row_ids, int64_t *d_num_unique, void *d_grad,
                             int64_t grad_stride, int32_t grad_dtype, void *d_scratch, int64_t scratch_bytes,
                             void *hip_stream);

/*
 * Layer norm of rows i < *d_num_rows:
 *   m_i = mean of x[i, :],  r_i = 1 / sqrt(mean of (x[i, :] - m_i)^2 + eps),  y[i, j] = (x[i, j] - m_i) r_i w[j] + b[j]
 *   d_x, d_y  of dtype; y may be x with the same stride.  d_w, d_b: [dim] of param_dtype, which is float or dtype; either
 *             may be NULL (ones, zeros).  eps >= 0.
 *   d_mean, d_rstd  float [max_rows] for the gradient, or NULL
 */
int smfg_layer_norm(const void *d_x, int64_t x_stride, int32_t dtype, const int64_t *d_num_rows, int64_t max_rows,
                    int32_t dim, const void *d_w, const void *d_b, int32_t param_dtype, float eps, void *d_y,
                    int64_t y_stride, float *d_mean, float *d_rstd, void *hip_stream);
/*
 * Its gradient, with h = (x - m) r and g = dy w:
 *   dx = r (g - mean(g) - h mean(g h)),  dw[j] = sum over rows of dy h,  db[j] = sum over rows of dy
 *   d_dy, d_x, d_dx  of dtype; dx may be dy or x with the same stride.  d_w as above.  d_dx NULL, or d_dw and d_db NULL (or one
 *   of them): not wanted.  d_dw, d_db: [dim] of param_dtype.
 */
int64_t smfg_layer_norm_grad_scratch_bytes(int64_t max_rows, int32_t dim);
int smfg_layer_norm_grad(const void *d_dy, int64_t dy_stride, const void *d_x, int64_t x_stride, int32_t dtype,
                         const int64_t *d_num_rows, int64_t max_rows, int32_t dim, const void *d_w, int32_t param_dtype,
                         const float *d_mean, const float *d_rstd, void *d_dx, int64_t dx_stride, void *d_dw, void *d_db,
                         void *d_scratch, int64_t scratch_bytes, void *hip_stream);

/*
 * Root-mean-square norm of rows i < *d_num_rows, with the addition of a residual before it and an output in 8 bits with scales:
 *   t_i = x_i + residual_i, rounded to dtype (t = x without a residual),  r_i = 1 / sqrt(mean of t_i^2 + eps),  y[i, j] = t[i, j] r_i w[j]
 * The norm is of the rounded sum, which is the one that the gradient reads.
 *   d_x, d_residual, d_total  of dtype; d_residual NULL: none; d_total: the sum t, or NULL (always without a residual).  d_total may be d_x or
 *             d_residual with the same stride.
 *   d_w       [dim] of param_dtype, which is float or dtype, or NULL (ones).  eps >= 0.
 *   d_y       of y_dtype: dtype (y may be x or the residual then, with the same stride), or
 *               SMFG_DTYPE_I8    y = s q, q a whole number in [-127, 127], s = (largest |y|) / 127
 *               SMFG_DTYPE_E4M3  y = s q, q a float of 8 bits (4 of exponent, 3 of mantissa, no infinities), s = (largest |y|) / 448
 *             for every `group` consecutive columns of a row (32, 64 or 128; 0: the whole row), q rounded to nearest even.  A largest value below
 *             2^-120 (e4m3: 2^-119) counts as 0: s = 0, q = 0.  With an infinity or a NaN among the values s is NaN and q = 0.
 *   d_scales  float, s of group k of row i at i * scales_stride + k; NULL if y is of dtype
 *   d_rstd    float [max_rows], r for the gradient, or NULL
 * Squares are added in float (in double in rows of over 16384 halfs or 8192 floats).
 */
#define SMFG_DTYPE_I8 3   /* outputs of smfg_rms_norm alone */
#define SMFG_DTYPE_E4M3 4 /* the same */
int smfg_rms_norm(const void *d_x, int64_t x_stride, int32_t dtype, const void *d_residual, int64_t residual_stride, void *d_total,
                  int64_t total_stride, const int64_t *d_num_rows, int64_t max_rows, int32_t dim, const void *d_w, int32_t param_dtype,
                  float eps, void *d_y, int64_t y_stride, int32_t y_dtype, float *d_scales, int64_t scales_stride, int32_t group,
                  float *d_rstd, void *hip_stream);
/*
 * Its gradient, with n = t r and g = dy w:
 *   dx = r (g - n mean(g n)) + dtotal,  dw[j] = sum over rows of dy n
 *   d_t       the sum (x without a residual).  d_dtotal: the gradient that reaches the sum from elsewhere, or NULL.  dx is the gradient of x and of
 *             the residual alike.
 *   d_dy, d_t, d_dtotal, d_dx  of dtype; dx may be any of the others with the same stride; NULL: not wanted.  d_dw: [dim] of param_dtype, or NULL.
 */
int64_t smfg_rms_norm_grad_scratch_bytes(int64_t max_rows, int32_t dim);
int smfg_rms_norm_grad(const void *d_dy, int64_t dy_stride, const void *d_t, int64_t t_stride, int32_t dtype, const void *d_dtotal,
                       int64_t dtotal_stride, const int64_t *d_num_rows, int64_t max_rows, int32_t dim, const void *d_w, int32_t param_dtype,
                       const float *d_rstd, void *d_dx, int64_t dx_stride, void *d_dw, void *d_scratch, int64_t scratch_bytes,
                       void *hip_stream);

/*
 * Softmax cross entropy over rows i < *d_num_rows of logits, and their gradient in the same pass:
 *   loss_i = log(sum over j of exp(x[i, j])) - x[i, y_i],  dx[i, j] = c (softmax(x_i)[j] - [j = y_i])
 * A row whose label is outside [0, classes) does not count: its loss is 0, its gradient zeros, whatever its logits are.
 *   d_logits, d_dlogits  of dtype, max_rows x classes; classes in [1, SMFG_MAX_DIM]; dlogits may be logits with the same stride; NULL: not wanted
 *   d_labels  int32 or int64 (label_bytes 4 or 8) [max_rows]
 *   reduction SMFG_LOSS_MEAN: *d_loss is the mean of the counted rows' losses (0 of none), c = scale / their number;
 *             SMFG_LOSS_SUM: their sum, c = scale.  scale (a loss scale, the share of a micro-batch) does not act on the loss.
 *   d_row_loss  float [max_rows], or NULL
 * A logit of -infinity has probability 0, and an infinite loss where it is the label's.  A counted row with a NaN, with +infinity or with -infinity alone
 * has a loss and a gradient of NaN.  Exponentials below 2^-126 of the row's largest are zeros.  Losses are added in double.
 */
#define SMFG_LOSS_MEAN 0
#define SMFG_LOSS_SUM 1
int64_t smfg_cross_entropy_scratch_bytes(int64_t max_rows, int32_t classes);
int smfg_cross_entropy(const void *d_logits, int64_t logits_stride, int32_t dtype, const void *d_labels, int32_t label_bytes,
                       const int64_t *d_num_rows, int64_t max_rows, int32_t classes, int32_t reduction, float scale, float *d_loss,
                       float *d_row_loss, void *d_dlogits, int64_t dlogits_stride, void *d_scratch, int64_t scratch_bytes, void *hip_stream);

/*
 * Global norm over any number of gradients, and clipping:
 *   N = sqrt(sum over all elements of (scale g)^2),  out = scale * min(1, max_norm / (N + 1e-6)) * g
 * scale undoes a loss scale or averages micro-batches; max_norm > 0, infinite: no clipping.  *d_norm = N (device float).  Squares
 * are added in double.  A NaN among the gradients makes N and all outputs NaN, whatever max_norm is.  An infinite one makes N infinite, so
 * finite ones 0; with an infinite max_norm nothing is clipped then either, and they are scaled alone.
 * Gradients that are clipped in place are not written again where scale and factor multiply to one.
 */
typedef struct {
  const void *grad;      /* device, numel contiguous elements of dtype */
  void *out;             /* device, of out_dtype: dtype, or float; NULL: in place */
  int64_t numel;         /* >= 0 */
  int32_t dtype, out_dtype;
  const int64_t *d_rows; /* device: only the first *d_rows rows of row_elems elements count (the d_num_unique of a */
  int64_t row_elems;     /* gradient of touched rows); NULL: all do */
} smfg_grad_t;
int64_t smfg_clip_grad_norm_scratch_bytes(const smfg_grad_t *grads, int32_t num_grads);
int smfg_clip_grad_norm(const smfg_grad_t *grads /* host */, int32_t num_grads, float scale, float max_norm, float *d_norm,
                        void *d_scratch, int64_t scratch_bytes, void *hip_stream);

/*
 * One step of AdamW over any number of tensors, in place:
 *   g' = f g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
 *   p = p - lr weight_decay p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps),  
 *   f = scale min(1, max_norm / (|scale| norm + 1e-6))
 * With d_norm, the norm of the gradients as they are (smfg_clip_grad_norm with scale 1, an infinite max_norm and no outputs finds it and writes nothing else),
 * they are clipped here, and not written; where *d_norm is not finite the step is not taken: nothing is written.  Without it f = scale, whatever max_norm is.
 * No two of the buffers written to share memory.
 * A tensor is of rows of row_elems elements (0: a single row of numel).  With d_row_ids the gradient's row i is that of row d_row_ids[i] of a table of
 * num_rows rows (param, m, v and copy), whose other rows are left as they are: the touched rows that smfg_embedding_grad_rows tells.  These ids are
 * distinct; one outside [0, num_rows) is left out.
 * m and v are of float (state_bits 32), or of 8 bits: every SMFG_STATE_BLOCK consecutive elements of a row (the last of a row may be fewer) share two floats,
 * A in m_scale and B in v_scale, of ceil(row_elems / SMFG_STATE_BLOCK) a row, and
 *   m = A (k / 127) |k / 127| with k int8,  v = (B (k / 255)^2)^2 with k uint8
 * are what is next to the value in k, A and B being the largest |m| and sqrt(v) of the elements; v > 0 is kept as k >= 1.  A below 2^-100 counts as 0, and v below 2^-126.
 * An infinity or a NaN in m or v makes the kept state of its block NaN.  Zeroed memory is the state of zeros, of either kind.  The step itself uses m
 * and v before they are rounded.
 * States of 8 bits are rounded to the nearest in each step, so that slow changes are lost: k moves only where a step changes it by a half or more, for m if about
 * (1 - beta1) |g' / m - 1| k > 1, for v if (1 - beta2) |g'^2 / v - 1| k > 2.  An element that does not move keeps its share of its block's largest, whatever its gradients do meanwhile.
 * With beta2 = 0.999 gradients that get smaller never lower a k of v, and it rises only where g'^2 > (1 + 2000 / k) v, so that steps are too small behind the former, and behind gradients that
 * get larger up to sqrt(1 + 2000 / k) times too large; with 0.99 the first holds for k up to 200, with 0.95 up to 40.  By a simulation with normal gradients of one size (256 blocks) sqrt(v) is
 * off by 5 % (rms) after 1000 steps and 15 % after 3000 with beta2 = 0.999, by 1.6 % with 0.99, by 0.8 % with 0.95; where half of a block's gradients become a quarter, theirs is 1.6 times too large
 * 1000 steps later and 4.3 times 6000 steps later with 0.999, 1 % with 0.99.  Where that matters: states of floats, or beta2 <= 0.99.
 * Parameters of half or bfloat16 that are not copies of float ones lose what a step changes by less than half their last digit: 2^-12 to 2^-11
 * of the value, or 2^-9 to 2^-8.
 */
#define SMFG_STATE_BLOCK 128
typedef struct {
  void *param;           /* device, of param_dtype */
  const void *grad;      /* device, numel elements of grad_dtype: float, or param_dtype, or any if the parameters are of float */
  void *m, *v;           /* device, as many elements as param */
  float *m_scale, *v_scale; /* device, for states of 8 bits */
  void *copy;            /* device, of copy_dtype (half or bfloat16): the new parameters, rounded, if these are of float; or NULL */
  int64_t numel;         /* of grad; >= 0 */
  int32_t param_dtype, grad_dtype, copy_dtype, state_bits;
  float weight_decay;    /* >= 0 */
  int64_t row_elems;     /* numel is a multiple */
  const int64_t *d_rows; /* device: only the first *d_rows rows of grad count; NULL: all do */
  const int32_t *d_row_ids; /* device, a row of the table for each row of grad; NULL: the same */
  int64_t num_rows;      /* of the table, with d_row_ids */
} smfg_param_t;
typedef struct {
  double lr, beta1, beta2, eps; /* beta1, beta2 in [0, 1), eps >= 2^-126 */
  double scale, max_norm;       /* max_norm > 0 */
  int64_t step;                 /* t = step + *d_step, 1 in the first step */
  const int64_t *d_step;        /* device, or NULL (0): for graphs, in which step is what it was when they were captured */
  const float *d_lr;            /* device, multiplies lr, or NULL (1): the same */
  const float *d_norm;          /* device, or NULL */
} smfg_adamw_t;
int smfg_adamw(const smfg_param_t *params /* host */, int32_t num_params, const smfg_adamw_t *hyper /* host */, void *hip_stream);
/* What states of 8 bits stand for, as numel values of out_dtype: m's (second 0) or v's (second 1). */
int smfg_adamw_values(const void *d_codes, const float *d_scales, int64_t numel, int64_t row_elems, int32_t second, void *d_out,
                      int32_t out_dtype, void *hip_stream);

/* Copies counts[0 .. 2L+2) to the host after synchronising the stream; returns SMFG_OK or, if the
 * status word is non-zero, its (positive) SMFG_ST_* value. */
int smfg_read_counts(const smfg_output_t *out, int32_t L, int64_t *h_counts, void *hip_stream);

/*
 * Stage timing for measurement.  One profile at a time per process; begin and end must not run
 * while another thread is inside any other call of this library (the record list is process-wide
 * state that the sampling calls append to).
 * Between begin and end, launches are bracketed by HIP events on the call's own stream:
 * level 1 = only the feature gather launch, level 2 = every launch.  At most max_records
 * launches are timed, later ones run untimed.  smfg_profile_end synchronises the device,
 * adds up the event-to-event milliseconds and the launch count per stage, and frees the events.
 * A launch that does the work of several stages is counted in each; its time goes to the first: one that
 * draws and partitions a hop's samples (SAMPLE, PARTITION), one that starts the counts and counts the samples
 * of wide fanouts (SEEDS, SCAN_TILES), one that assembles a hop and, in small hops, drew or deduplicated its
 * samples, draws for the next or copies the feature rows (ASSEMBLE, and SAMPLE, DEDUP or GATHER).  So the gather of a call that has
 * no launch of its own is counted, on either level, with no time.
 */
#define SMFG_STAGE_CLEAR 0
#define SMFG_STAGE_SEEDS 1
#define SMFG_STAGE_SAMPLE 2
#define SMFG_STAGE_FLAG 3
#define SMFG_STAGE_SCAN_TILES 4
#define SMFG_STAGE_ASSEMBLE 5
#define SMFG_STAGE_GATHER 6
#define SMFG_STAGE_AGGREGATE 7
#define SMFG_STAGE_LAYER 8
#define SMFG_STAGE_PARTITION 9
#define SMFG_STAGE_DEDUP 10
#define SMFG_NUM_STAGES 11
int smfg_profile_begin(int32_t level, int32_t max_records);
int smfg_profile_end(double *stage_ms /* host [SMFG_NUM_STAGES] */,
                     int64_t *stage_launches /* host [SMFG_NUM_STAGES] */);

const char *smfg_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SMFG_H_ */
