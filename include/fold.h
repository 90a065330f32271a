/*
 * fold.h -- C ABI of the MI355X dynamic-batching library.
 *
 * Dynamic batching (Looks et al., "Deep Learning with Dynamic Computation
 * Graphs", Section 2) evaluates a batch of computation graphs of different
 * shapes and sizes by
 *   1. giving every node a depth (constants have depth 0; a node whose inputs
 *      have maximum depth d has depth d + 1),
 *   2. batching together all nodes that run the same operation at the same
 *      depth,
 *   3. gathering each batch's inputs by index from the concatenated outputs of
 *      earlier depths, running the operation once per (depth, operation), and
 *      concatenating the outputs back,
 * and back-propagates through the same gathers and concatenations.  This
 * library exposes that hot path as three calls:
 *
 *   fold_schedule   CSR graphs -> per-level, per-operation gather indices
 *   fold_forward    schedule + parameters + leaf rows -> every node's state
 *                   and the roots' outputs
 *   fold_backward   reverse-level pass: gradients scatter-added into child
 *                   states, weight gradients accumulated
 *
 * Conventions shared by every entry point
 *   - Every call returns FOLD_OK (0) or a negative FOLD_E_* code; the
 *     matching text is available from fold_last_error() on the calling
 *     thread.  No C++ exception crosses this boundary.
 *   - "device" pointers are HIP device allocations on the current device;
 *     "host" pointers are ordinary host memory.  The caller owns every
 *     buffer it passes in; the library owns the fold_sched / fold_packed
 *     handles it returns and everything they point to.
 *   - All work is enqueued on the given stream.  fold_schedule and
 *     fold_pack_params synchronise that stream (they read back sizes);
 *     fold_forward and fold_backward never synchronise and never allocate.
 *   - Node states live in one pool in SCHEDULE order: row p of a pool holds
 *     node pos_node[p].  Every row-major float/bf16 matrix the library reads
 *     or writes has a row stride of fold_row_ld(width) elements (width
 *     rounded up to 64); columns beyond the width are written as zero
 *     (pools) and must hold zeros in inputs (the leaf table): the kernels
 *     load whole 128-byte row segments and meet those columns with zero
 *     weights, so any finite value there is harmless and NaN / Inf is not.
 *   - Handles are immutable after creation (fold_pack_update aside, which
 *     rewrites a packed handle's weights in place) and may be shared by
 *     concurrent calls on different streams that use different output buffers.
 */
#ifndef FOLD_H_
#define FOLD_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------ */
#define FOLD_OK 0
#define FOLD_E_INVALID -1  /* null pointer, negative count, bad dims/dtype, bad op table, broken graph_ptr/child_ptr */
#define FOLD_E_OP -2       /* node_op out of [0, num_ops) */
#define FOLD_E_ARITY -3    /* a node's child count differs from its operation's arity */
#define FOLD_E_CHILD -4    /* child id out of range or in another graph (-1, the zero state, is allowed) */
#define FOLD_E_INPUT -5    /* input row out of [0, num_inputs), or present/absent against has_input */
#define FOLD_E_CYCLE -6    /* the graph is not acyclic */
#define FOLD_E_NOMEM -7    /* device allocation failed */
#define FOLD_E_DEVICE -8   /* a HIP call failed */
#define FOLD_E_MISMATCH -9 /* schedule / parameters / workspace inconsistent with each other */

/* ---- operation kinds (the operations of the paper's experiments) ------- */
enum {
  FOLD_EMBED = 0,    /* h = table[input]                        (embedding lookup, arity 0, has_input) */
  FOLD_TREERNN = 1,  /* h = tanh([h_l; h_r] W + b)              (binary TreeRNN cell, arity 2) */
  FOLD_TREELSTM = 2, /* binary N-ary Tree-LSTM, gates (i|f_l|f_r|o|u); arity 0 with input = leaf
                        TreeLSTM(x, 0, 0), arity 2 = internal TreeLSTM(x?, h_l, h_r) */
  FOLD_LSTM = 3,     /* one LSTM step, gates (i|f|o|u), arity 1 (child -1 = zero start state) */
  FOLD_PROJ = 4,     /* h = tanh(h_c P + b), c = c_c            (unary projection, arity 1) */
  /* Feed-forward attention (Section 3.4, Appendix A): e_t = a(h_t), alpha = softmax(e),
   * c = sum_t alpha_t h_t, with the scorer a(h) = w . h + b.  The two sums over t are carried as one
   * aggregate of a set of scored items, (m, s, acc) = (max e, sum exp(e - m), sum exp(e - m) h), held in
   * a node's state as h = acc and c = [m, s, 0, ...] (needs hidden >= 2), so that a Reduce over the items
   * batches like any other operation.  Gradients hold m fixed (the value acc / s does not depend on it). */
  FOLD_ATTN_SCORE = 5, /* one item from the child's h: e = w . h_c + b, h = h_c, c = [e, 1, 0..]
                          (arity 1; parameters: W_rec = w as [H, 1], bias = [b]) */
  FOLD_ATTN_SUM = 6,   /* union of the two children's sets: m = max(m_1, m_2), x_k = exp(m_k - m),
                          s = x_1 s_1 + x_2 s_2, acc = x_1 acc_1 + x_2 acc_2; a child with s = 0 (the
                          zero state, an empty set) takes no part; two empty sets give the zero state
                          (arity 2, no parameters: W_rec and bias may be NULL) */
  FOLD_ATTN_OUT = 7    /* the attention output: h = acc / s (the zero vector for an empty set), c = 0
                          (arity 1, no parameters) */
};

/* ---- element types of weights, leaf table and h pool ------------------- */
enum { FOLD_F32 = 0, FOLD_BF16 = 1 };

/* One operation of the op table.  The paper requires every operation to be
 * specified and enumerated in advance (Section 2); the op id is the index in
 * the table, and groups of one depth are ordered by it. */
typedef struct {
  int32_t kind;      /* FOLD_EMBED .. FOLD_ATTN_OUT */
  int32_t arity;     /* number of node children (CSR entries) */
  int32_t has_input; /* 1: reads leaf-table row node_input[v] */
  int32_t param_set; /* index into fold_params.sets */
} fold_op;

/* A batch of graphs as one disconnected DAG (Section 2), CSR form.
 * Node ids are global; node order inside a graph is arbitrary.  Children
 * must belong to the node's own graph; -1 names a zero state. */
typedef struct {
  int32_t num_graphs;        /* G >= 0 */
  int32_t num_nodes;         /* N >= 0 */
  int32_t num_edges;         /* E >= 0, = child_ptr[N] */
  int32_t num_ops;           /* 1 .. 256 (more: FOLD_E_INVALID) */
  int32_t num_inputs;        /* rows of the leaf table that node_input may name */
  const int32_t* graph_ptr;  /* device [G+1], graph_ptr[0] = 0, graph_ptr[G] = N, nondecreasing */
  const int32_t* node_op;    /* device [N] */
  const int32_t* child_ptr;  /* device [N+1], child_ptr[0] = 0, nondecreasing */
  const int32_t* child_idx;  /* device [E] global node ids or -1 */
  const int32_t* node_input; /* device [N] leaf-table row, or -1 */
  const fold_op* ops;        /* host [num_ops] */
} fold_batch;

typedef struct fold_sched fold_sched;
typedef struct fold_packed fold_packed;

/* Read-only view of a schedule.  Device arrays are owned by the schedule. */
typedef struct {
  int32_t num_nodes, num_edges, num_graphs, num_ops;
  int32_t num_levels; /* D = maximum depth = number of batched steps */
  int32_t num_groups; /* non-empty (depth, op) groups */
  int32_t num_roots;  /* nodes that are nobody's child */
  int32_t max_parents;
  /* device, int32 */
  const int32_t* depth;           /* [N]   depth of node v (leaf operations: 1) */
  const int32_t* node_pos;        /* [N]   pool row of node v */
  const int32_t* pos_node;        /* [N]   node at pool row p */
  const int32_t* level_ptr;       /* [D+1] rows of depth <= l end at level_ptr[l] */
  const int32_t* group_level;     /* [num_groups] */
  const int32_t* group_op;        /* [num_groups] */
  const int32_t* group_row_begin; /* [num_groups] first pool row of the group */
  const int32_t* group_rows;      /* [num_groups] */
  const int32_t* group_idx_off;   /* [num_groups] offset of the group's edges in child_pos */
  const int32_t* child_pos;       /* [E]   pool row of child k of the group's row r at
                                     group_idx_off + r * arity + k, or -1 (zero state) */
  const int32_t* input_idx;       /* [N]   leaf-table row read by pool row p, or -1 */
  const int32_t* root_pos;        /* [num_roots] pool rows of the roots, ascending node id */
  /* host copies */
  const int32_t* h_level_ptr;
  const int32_t* h_group_level;
  const int32_t* h_group_op;
  const int32_t* h_group_row_begin;
  const int32_t* h_group_rows;
  const int32_t* h_group_idx_off;
  /* Static-graph layout, per group and child slot k = 0, 1: the pool row of the
   * slot's first child when the slot's children are the consecutive rows
   * base .. base + rows - 1 and each has exactly one parent edge (a batch of
   * identically shaped graphs with one operation per node position, i.e.
   * manual batching, has it on every slot); -1 otherwise.  The forward
   * kernels address such children as base + row, with no child_pos load.
   * Device [num_groups] each, and host copies. */
  const int32_t* group_child_base0;
  const int32_t* group_child_base1;
  const int32_t* h_group_child_base0;
  const int32_t* h_group_child_base1;
} fold_sched_info;

/* Schedule a batch (Section 2, the greedy scheduling algorithm):
 * validates the CSR (codes above), computes every node's depth on the GPU
 * (cycles -> FOLD_E_CYCLE), sorts the nodes by the key (depth - 1) * num_ops
 * + op with ties kept in node-id order (a stable counting sort), and emits
 * the per-group gather indices.  The edge label of the paper (index i into
 * the concatenated outputs of depth d) is the pool row minus
 * level_ptr[d - 1]; pass-throughs are unnecessary because the pool keeps
 * every level.  Synchronises `stream` once (error word, level and group
 * tables), and once more for a schedule of more than 4,096 levels or groups.
 * On success *out is a new handle to free with
 * fold_sched_free; on error *out is NULL. */
int32_t fold_schedule(const fold_batch* batch, hipStream_t stream, fold_sched** out);
int32_t fold_sched_get_info(const fold_sched* sched, fold_sched_info* out);
/* Waits until the device has finished everything queued on it (as hipFree
 * does), on every stream.  The schedule's device memory then stays with the
 * library for the next schedule: at most 1 GiB per device while any schedule
 * lives there (temporaries included), 256 MiB otherwise.  The library gives
 * it up by itself only when an allocation of its own fails; fold_trim gives
 * it to other allocators of the process. */
int32_t fold_sched_free(fold_sched* sched);
/* Gives back to the system all memory that the library keeps idle between
 * schedules, on every device, and its idle pinned buffers; schedules that
 * live are not touched.  Waits for the devices concerned.  *bytes (may be
 * NULL): the device memory given back. */
int32_t fold_trim(size_t* bytes);

/* ---- the paper's own form of the schedule ---------------------------------
 * Section 2 schedules a typed DAG: source nodes are constants of a tensor
 * type, other nodes invoke operations whose inputs and outputs have fixed
 * tensor types, and an edge connects output k of node u to input j of node
 * v.  Its five steps: (1) depth (constants 0, an operation node 1 + the
 * largest depth it reads); (2) pass-through (identity) operations, so that a
 * node at depth d + 1 reads only results of depth d; (3) one batch per
 * (depth, operation); (4) at each depth the outputs of one type concatenated
 * in the operations' enumeration order; (5) every edge labelled (d, t, i),
 * the depth and type of the value it reads and its index into that
 * concatenation; the schedule is the indices i grouped by depth and
 * operation.  fold_schedule above is the special case of one state type
 * (node and child states travel together) with pass-throughs elided; this
 * call produces the general form, including an int-typed state such as the
 * word ids of Figure 1.
 *
 * Readings (the paper is silent): pass-throughs are operations too, one per
 * type t, numbered num_ops + t (after the caller's operations), with one
 * input and one output of type t; one pass-through per value and depth,
 * shared by all readers of that value; a batch lists its operation nodes in
 * ascending node id and its pass-through instances in ascending value order
 * (node id, then output slot); an operation's outputs of one type enter
 * that type's concatenation in slot order, each with the whole batch in
 * batch order; the depth-0 state of type t holds the constants of type t in
 * ascending node id. */
typedef struct {
  int32_t num_inputs, num_outputs; /* 1..8 each */
  const int32_t* in_type;          /* host [num_inputs], 0..num_types-1 */
  const int32_t* out_type;         /* host [num_outputs] */
} fold_typed_op;

typedef struct {
  int32_t num_graphs, num_nodes, num_edges;
  int32_t num_ops;    /* 1..64 */
  int32_t num_types;  /* 1..16 */
  const int32_t* graph_ptr; /* device [G+1]: graph g is nodes graph_ptr[g] .. graph_ptr[g+1]-1 */
  const int32_t* node_op;   /* device [N]: operation id, or -1 - t for a constant of type t */
  const int32_t* in_ptr;    /* device [N+1]: node v's inputs are edges in_ptr[v] .. in_ptr[v+1]-1 */
  const int32_t* in_node;   /* device [E]: source node of the edge (same graph) */
  const int32_t* in_slot;   /* device [E]: source output slot */
  const fold_typed_op* ops; /* host [num_ops] */
} fold_typed_batch;

typedef struct fold_typed_sched fold_typed_sched;

typedef struct {
  int32_t num_levels;   /* D: the largest depth */
  int32_t num_batches;  /* non-empty (depth, operation) batches, pass-throughs included */
  int32_t num_passes;   /* pass-through instances */
  int32_t num_items;    /* operation nodes + pass-through instances */
  int32_t num_gather;   /* entries of gather */
  int32_t num_ops, num_types;
  /* device, int32 */
  const int32_t* depth;             /* [N] */
  const int32_t* batch_depth;       /* [num_batches] ascending (depth, operation) */
  const int32_t* batch_op;          /* [num_batches] operation, or num_ops + t: pass-through of type t */
  const int32_t* batch_rows;        /* [num_batches] */
  const int32_t* batch_gather_off;  /* [num_batches] input j of row r at gather[off + j * rows + r] */
  const int32_t* batch_item_begin;  /* [num_batches] first entry in item_node */
  const int32_t* item_node;         /* [num_items] node id, or -1 - p for pass-through instance p */
  const int32_t* gather;            /* [num_gather] indices i into the (depth - 1, input type) state */
  const int32_t* pass_node;         /* [num_passes] the value (node, output slot) carried, and the */
  const int32_t* pass_slot;         /*   depth of the instance; ascending value, then depth */
  const int32_t* pass_depth;
  const int32_t* state_size;        /* [(D + 1) * num_types]: rows of the state (d, t) at d * T + t */
  const int32_t* edge_index;        /* [E] label index i of every input edge (its d is the reader's
                                       depth - 1, its t the input's type) */
  /* host copies */
  const int32_t* h_batch_depth;
  const int32_t* h_batch_op;
  const int32_t* h_batch_rows;
  const int32_t* h_batch_gather_off;
  const int32_t* h_state_size;
} fold_typed_sched_info;

/* fold_schedule_typed: validates the batch (FOLD_E_INVALID for a malformed
 * op table, graph_ptr / in_ptr, an edge from a missing node or output or of
 * the wrong type, a constant with inputs or an operation node with the wrong
 * input count; FOLD_E_CHILD for an edge across graphs; FOLD_E_OP for an
 * operation or constant type out of range; FOLD_E_CYCLE; FOLD_E_INVALID for
 * a batch whose nodes, edges and pass-throughs reach 2^31), then schedules it
 * on the GPU.  The library allocates and owns the result.  Synchronises
 * `stream` twice: once to size the pass-through arrays, once at the end (a
 * third time where values times levels reach 2^31). */
int32_t fold_schedule_typed(const fold_typed_batch* batch, hipStream_t stream, fold_typed_sched** out);
int32_t fold_typed_sched_get_info(const fold_typed_sched* sched, fold_typed_sched_info* out);
/* Waits and keeps memory as fold_sched_free. */
int32_t fold_typed_sched_free(fold_typed_sched* sched);


/* Parameters of one operation family, canonical row-major layout, device
 * memory, element type fold_params.dtype (bias always fp32).  G gate blocks
 * (Tree-LSTM 5, LSTM 4, TreeRNN / PROJ 1, EMBED 0) of `hidden` columns each,
 * in the order given under FOLD_TREELSTM / FOLD_LSTM.  Attention sets
 * (in_dim 0): FOLD_ATTN_SCORE has arity 1, W_rec = the scorer vector w as
 * [hidden, 1] and bias = [b] (one float); FOLD_ATTN_SUM (arity 2) and
 * FOLD_ATTN_OUT (arity 1) hold no values (W_rec and bias may be NULL).  Their
 * gradients (fold_param_grads) are dW_rec [hidden] and dbias [1] for the
 * scorer, none for the other two.  hidden must be at least 2 once an
 * attention set is present. */
typedef struct {
  int32_t kind;
  int32_t in_dim;    /* width of the leaf-table rows the ops read (EMBED: = hidden) */
  int32_t arity;     /* child slots covered by W_rec */
  const void* W_in;  /* [in_dim, G*hidden] or NULL when in_dim == 0 */
  const void* W_rec; /* [arity*hidden, G*hidden]; rows k*hidden.. belong to child k */
  const float* bias; /* [G*hidden] (NULL for EMBED) */
} fold_param_set;

typedef struct {
  int32_t dtype;  /* FOLD_F32 or FOLD_BF16 */
  int32_t hidden; /* H, 1 .. 4096 */
  int32_t num_sets;
  const fold_param_set* sets; /* host [num_sets] */
} fold_params;

/* Copy the parameters into the library's MFMA-friendly layouts (gate blocks
 * interleaved per 32 hidden units, K padded per input segment, transposed
 * copies for the backward).  Reads the caller's arrays once; synchronises.
 * FOLD_E_INVALID for a set whose packed matrix, G * H' * (in_dim' + arity * H')
 * entries (primes: rounded up to 64), would reach 2^32. */
int32_t fold_pack_params(const fold_params* params, hipStream_t stream, fold_packed** out);
int32_t fold_packed_free(fold_packed* packed);

/* Re-pack new values of the same parameters into an existing handle (a
 * training loop after each optimizer step): `params` must match the handle
 * in dtype, hidden, number of sets and each set's kind, in_dim and arity
 * (FOLD_E_MISMATCH otherwise; FOLD_E_INVALID for the checks of
 * fold_pack_params).  Enqueued on `stream`; asynchronous; allocates
 * nothing; the packed buffers keep their addresses, so HIP graphs recorded
 * with the handle stay valid.  The caller orders it after every pass that
 * still reads the old weights and before every pass that needs the new. */
int32_t fold_pack_update(fold_packed* packed, const fold_params* params, hipStream_t stream);

/* Row stride, in elements, that the library uses for a row of `width`
 * elements (pools, root outputs, gradients of node states, leaf tables):
 * width rounded up to a multiple of 64. */
int32_t fold_row_ld(int32_t width);

/* Workspace needed by fold_forward (saved gate activations for the
 * backward) and by fold_backward (the same region plus per-node gradient
 * accumulators).  One buffer of bwd_bytes serves both calls. */
int32_t fold_workspace_size(const fold_sched* sched, const fold_packed* packed,
                            size_t* fwd_bytes, size_t* bwd_bytes);

/* Forward pass over every level: for each (depth, op) group in order, gather
 * the children's (h, c) rows and the leaf-table rows by index, contract
 * with the operation's weights on the matrix cores, apply the cell, and
 * write the group's rows of the pools.
 *   leaf_table  device [leaf_rows, fold_row_ld(in_dim)] of dtype (may be NULL
 *               if no op has an input)
 *   h_pool      device [N, fold_row_ld(H)] of dtype (written)
 *   c_pool      device [N, fold_row_ld(H)] fp32 (written)
 *   roots_out   device [num_roots, fold_row_ld(H)] of dtype (written; NULL skips)
 *   ws          device workspace of >= fwd_bytes; receives the activations
 *               fold_backward needs (NULL with ws_bytes 0: inference only)
 * Asynchronous; allocates nothing. */
int32_t fold_forward(const fold_sched* sched, const fold_packed* packed,
                     const void* leaf_table, int64_t leaf_rows,
                     void* h_pool, float* c_pool, void* roots_out,
                     void* ws, size_t ws_bytes, hipStream_t stream);

/* Gradients of one parameter set, canonical layout, fp32, device memory.
 * Accumulated (+=): the caller zeroes them.  NULL skips that tensor. */
typedef struct {
  float* dW_in;  /* [in_dim, G*H] */
  float* dW_rec; /* [arity*H, G*H] */
  float* dbias;  /* [G*H] */
} fold_param_grads;

typedef struct {
  int32_t num_sets;              /* must equal the packed parameters' */
  const fold_param_grads* sets;  /* host [num_sets] */
  float* d_leaf_table;           /* device [leaf_rows, fold_row_ld(in_dim)] fp32, += ; or NULL */
} fold_grads;

/* Backward pass, levels in reverse order.  The upstream gradient is
 * dh_roots on the roots (row r = root r, in ascending node id) plus, if
 * given, dh_nodes on every pool row; the roots' cell states get none.
 * For each group: dz from the saved gates, dz . W^T scatter-added into the
 * children's (h, c) gradients (every parent lies at a greater depth, so a
 * child's gradient is complete before its own level runs); then, per
 * operation, the weight gradients dW += X^T dz, db += sum dz, and the
 * leaf-table gradient: dz summed over the operation's rows of each
 * leaf-table row, times W_in^T, added into that row (the same sum as adding
 * every row's dz . W_in^T, in another order).
 *   h_pool, c_pool, ws   exactly as left by fold_forward with this schedule
 *   dh_roots             device [num_roots, ld(H)] fp32 or NULL
 *   dh_nodes             device [N, ld(H)] fp32 (pool order) or NULL
 *   dh_out, dc_out       device [N, ld(H)] fp32 (pool order) or NULL: receive every
 *                        node's total upstream gradient of h and c (every row
 *                        written whole)
 * dh_roots, dh_nodes, dh_out, dc_out and ws must be 16-byte aligned
 * (FOLD_E_INVALID otherwise).  Asynchronous; allocates nothing. */
int32_t fold_backward(const fold_sched* sched, const fold_packed* packed,
                      const void* leaf_table, int64_t leaf_rows,
                      const void* h_pool, const float* c_pool,
                      const float* dh_roots, const float* dh_nodes,
                      const fold_grads* grads, float* dh_out, float* dc_out,
                      void* ws, size_t ws_bytes, hipStream_t stream);

/* fold_forward_noalloc: fold_forward for callers that cannot allocate --
 * code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  It computes the same states as fold_forward (inference: no
 * activations are saved for a backward pass) and takes no workspace: the
 * K-split partial sums of narrow levels go to a library-owned 16 MiB device
 * array per GPU (a static __device__ array, held until the process ends).
 * A level whose K split would need more than that splits into fewer slices,
 * or none, so no batch is rejected for its size; results stay within the
 * tolerance of fold_forward's (slices may differ, so not always bit-equal).
 * Arguments, errors and asynchrony are those of fold_forward without ws;
 * FOLD_E_MISMATCH if the handles belong to another device than the current
 * one, FOLD_E_DEVICE if the array's address cannot be looked up.  It calls
 * no hipMalloc, hipFree or allocating routine.  Every call on one GPU shares
 * that GPU's array, so calls that overlap on one GPU (two streams, two host
 * threads) race: serialise them.  No contents carry over between calls that
 * matter (every slice writes its partial sums before they are read). */
int32_t fold_forward_noalloc(const fold_sched* sched, const fold_packed* packed,
                             const void* leaf_table, int64_t leaf_rows,
                             void* h_pool, float* c_pool, void* roots_out,
                             hipStream_t stream);

/* Recurrent dropout (Section 3.5 trains the Tree-LSTM with the recurrent
 * dropout of Semeniuta et al., "Recurrent dropout without memory loss"):
 * the forward and backward passes above with a mask on the candidate update
 * u where it enters the memory cell, c = i*(m*u) + sum_k f_k*c_k, so the
 * forget paths of the cell state are never dropped.  Operations of kind
 * FOLD_TREELSTM (leaf and internal) and FOLD_LSTM use the mask; the other
 * kinds ignore it.
 *   u_mask  device [N, fold_row_ld(H)] fp32, pool order (row p = node
 *           pos_node[p]); any multiplier (0 or 1/(1-p) for inverted
 *           dropout, drawn by the caller).  Caller-owned, read only; the
 *           backward must get the same mask as the forward.  NULL is
 *           FOLD_E_INVALID (use fold_forward / fold_backward instead).
 * Every other argument, error and the asynchrony are as in fold_forward /
 * fold_backward. */
int32_t fold_forward_dropout(const fold_sched* sched, const fold_packed* packed,
                             const void* leaf_table, int64_t leaf_rows,
                             void* h_pool, float* c_pool, void* roots_out,
                             const float* u_mask, void* ws, size_t ws_bytes,
                             hipStream_t stream);
int32_t fold_backward_dropout(const fold_sched* sched, const fold_packed* packed,
                              const void* leaf_table, int64_t leaf_rows,
                              const void* h_pool, const float* c_pool,
                              const float* u_mask, const float* dh_roots,
                              const float* dh_nodes, const fold_grads* grads,
                              float* dh_out, float* dc_out,
                              void* ws, size_t ws_bytes, hipStream_t stream);

/* fold_dropout_mask: draws the recurrent-dropout mask of one training step
 * (the u_mask of fold_forward_dropout / fold_backward_dropout) on the GPU
 * from the counter-based generator Philox4x32-10 (Salmon, Moraes, Dror and
 * Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).  For node
 * v and hidden unit j < hidden, with r the (j mod 4)-th output word of the
 * call on counter (v, j / 4, low and high 32 bits of step) under the key
 * (low and high 32 bits of seed):
 *     mask[pos(v)][j] = 0 if r < min(floor(p 2^32), 2^32 - 1), else (float)(1 / (1 - p))
 * (inverted dropout: kept units are scaled so the expected multiplier is 1).
 *   mask    device [N, fold_row_ld(hidden)] fp32, POOL order (row q = node
 *           pos_node[q]), 16-byte aligned; written whole, pad columns 0.
 *           Caller-owned.
 *   p       drop probability in [0, 1); p = 0 gives all ones.
 *   seed, step  any 64-bit values; a node's row depends only on (v, seed,
 *           step, p), not on the batch around it.
 * FOLD_E_INVALID for a NULL schedule, hidden outside 1..4096, p outside
 * [0, 1), or a NULL or misaligned mask (N > 0).  Asynchronous; allocates
 * nothing. */
int32_t fold_dropout_mask(const fold_sched* sched, int32_t hidden, double p, uint64_t seed, uint64_t step,
                          float* mask, hipStream_t stream);

/* ---- the training step around the path ------------------------------------
 * Section 3.5 trains the binary Tree-LSTM on trees whose every node carries a
 * class label: a linear layer and a softmax on every node's state h, the
 * cross entropy against the node's label, summed over the nodes, minimised
 * with TensorFlow's Adam optimizer (Section 3.3).  These two calls are that
 * step's loss head and update; fold_backward takes the head's dh_nodes.
 *
 * fold_loss_softmax_ce: per node v with label y_v >= 0
 *     z_v = h_v W_cls + b_cls,  loss_v = log sum_c exp(z_vc) - z_{v,y_v}
 * and the gradients of L = scale * sum_v loss_v:
 *     dz_v = scale (softmax(z_v) - onehot(y_v)),  dh_v = dz_v W_cls^T,
 *     dW_cls += h^T dz,  db_cls += sum_v dz_v;
 * a node with label -1 (or any label outside [0, num_classes)) has loss 0
 * and dh 0.  fp32 arithmetic on h of the packed parameters' dtype.
 *   h_pool     device [N, fold_row_ld(H)] pool (as left by fold_forward)
 *   labels     device [N] int32 in NODE order: class 0..num_classes-1, or -1
 *              (no label)
 *   num_classes  2..8, 10, 16 or 32, with H * num_classes <= 8000
 *   W_cls      device [H, num_classes] fp32 row-major; b_cls device [num_classes] fp32
 *   node_loss  device [N] fp32, NODE order (written)
 *   dh_nodes   device [N, fold_row_ld(H)] fp32, POOL order (written, pad
 *              columns zero): the dh_nodes argument of fold_backward
 *   dW_cls, db_cls  device, fp32, accumulated (+=; the caller zeroes them);
 *              partial sums per block of rows are added in a fixed order,
 *              but the four waves of a block meet in LDS in arrival order,
 *              so the result is reproducible up to the order of those fp32
 *              additions, not bit for bit
 *   ws         device workspace of >= fold_loss_workspace_size bytes (the
 *              per-block partial sums; contents on entry do not matter)
 * FOLD_E_INVALID for an unsupported class count, H * num_classes above
 * 8000, a non-finite scale or a NULL buffer (N > 0); FOLD_E_MISMATCH for a
 * workspace that is too small, and as fold_forward for a schedule and
 * parameters that do not belong together.  Asynchronous; allocates nothing.
 * fold_loss_workspace_size fails with FOLD_E_INVALID as above. */
int32_t fold_loss_workspace_size(const fold_packed* packed, int32_t num_classes, size_t* bytes);
int32_t fold_loss_softmax_ce(const fold_sched* sched, const fold_packed* packed, const void* h_pool,
                             const int32_t* labels, int32_t num_classes, const float* W_cls, const float* b_cls,
                             float scale, float* node_loss, float* dh_nodes, float* dW_cls, float* db_cls,
                             void* ws, size_t ws_bytes, hipStream_t stream);

/* fold_adam_step: step `step` (1, 2, ...) of Adam (Kingma and Ba) in the
 * form of TensorFlow's optimizer, elementwise over n fp32 values:
 *     m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *     p = p - lr_t m / (sqrt(v) + eps),
 *     lr_t = lr sqrt(1 - beta2^step) / (1 - beta1^step)
 * in fp32, with lr_t, 1 - beta1 and 1 - beta2 computed in double first (the
 * hyperparameters are double so that 1 - 0.999 keeps its value).
 * param, m, v are device fp32 arrays updated in place (m, v start at zero);
 * grad is read; param_bf16, if not NULL, receives param rounded to bf16
 * (round to nearest even) for models whose weights are bf16.  Any flat
 * tensor works (weights, biases, a padded leaf table whose pad columns hold
 * zero parameters and gradients, which stay zero).  FOLD_E_INVALID for n < 0,
 * step < 1, beta outside [0, 1), eps < 0, a non-finite lr or a NULL buffer
 * (n > 0).  Asynchronous; allocates nothing. */
int32_t fold_adam_step(int64_t n, float* param, uint16_t* param_bf16, const float* grad, float* m, float* v,
                       double lr, double beta1, double beta2, double eps, int32_t step, hipStream_t stream);

/* ---- the vocabulary head ---------------------------------------------------
 * Rows of node states scored against a vocabulary of tokens: the head of a
 * model whose nodes predict words (LSTM chains over text, roots that name a
 * token), where fold_loss_softmax_ce serves a few classes.  `rows` states are
 * any matrix [rows, fold_row_ld(hidden)]: a whole pool (pool order) or
 * roots_out (root order), and the gradient d_states of the same shape is
 * fold_backward's dh_nodes or dh_roots.  The weights lie as a leaf table
 * does, one row of `hidden` values a token, so the table of an embedding
 * model can be the head's W and its d_leaf_table the head's dW (tied
 * weights).  Logits are matrices [rows, fold_row_ld(vocab)] in memory: a
 * program may mask them (-inf), between the head and what reads them.
 *
 * All of these calls enqueue on `stream`, never synchronise, never allocate
 * and can be captured.  Matrices and workspaces are 16-byte aligned
 * (FOLD_E_INVALID otherwise); rows is at most 2^31 - 1, vocab at most 2^30
 * (2^21 for the products, whose launches have fewer than 2^24 tiles: rows
 * times fold_row_ld of either width up to 2^35 always fit, more may be
 * refused as FOLD_E_INVALID).  rows = 0 is allowed (buffers that would
 * be read may be NULL).  Workspaces hold nothing between calls; calls that
 * overlap need one each, and fewer rows may need a larger one (long rows that
 * are few are cut into pieces), so a size is asked for each number of rows.
 *
 * fold_vocab_logits: z = states W^T + bias.
 *   dtype         FOLD_F32 or FOLD_BF16: states and W (products of bf16 values
 *                 are summed in fp32)
 *   states        device [rows, fold_row_ld(hidden)]; hidden 1 .. 4096
 *   W             device [vocab, fold_row_ld(hidden)]; the pad columns of one
 *                 of the two hold zeros, of the other any finite values
 *   bias          device [vocab] fp32, or NULL; -inf takes a token out
 *   logits_dtype  of `logits`: FOLD_F32, or FOLD_BF16 for a bf16 head
 *   logits        device [rows, fold_row_ld(vocab)], written whole (pad
 *                 columns zero)
 * fold_vocab_backward: from dlogits, of `dtype` and finite in the pad columns
 * (fold_loss_distill writes zeros there),
 *     d_states = dlogits W                device [rows, fold_row_ld(hidden)]
 *     dW      = dlogits^T states          device [vocab, fold_row_ld(hidden)]
 *     dbias   = sum over the rows         device [vocab]
 * all fp32; any of the three may be NULL (not computed).  They are written
 * whole, pad columns zero; with FOLD_VOCAB_ACCUMULATE dW and dbias are added
 * to what is there instead (dW's pad columns are then left alone).
 *   ws  device workspace of >= fold_vocab_workspace_size bytes (may be NULL
 *       where that is 0)
 * FOLD_E_INVALID for sizes out of range, an unknown dtype or flag, NULL or
 * misaligned buffers, an output that overlaps another buffer of the call;
 * FOLD_E_MISMATCH for a workspace that is too small. */
#define FOLD_VOCAB_ACCUMULATE 1

int32_t fold_vocab_logits(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, const void* states,
                          const void* W, const float* bias, int32_t logits_dtype, void* logits, hipStream_t stream);
int32_t fold_vocab_workspace_size(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, size_t* bytes);
int32_t fold_vocab_backward(int32_t dtype, int64_t rows, int32_t hidden, int32_t vocab, const void* states,
                            const void* W, const void* dlogits, float* d_states, float* dW, float* dbias,
                            int32_t flags, void* ws, size_t ws_bytes, hipStream_t stream);

/* fold_loss_distill: the loss of a student against the largest logits of a
 * teacher, mixed with the cross entropy of a label, and its gradient.  For a
 * row with teacher entries (i_j, t_j), j < num_teacher, and label y, with
 * q = softmax(t / T) over the entries that count, p^T = softmax(z / T) and
 * p = softmax(z) over the vocabulary:
 *     loss = soft_weight T^2 sum_j q_j (log q_j - log p^T[i_j])
 *          - hard_weight log p[y]
 * and, of L = scale * (sum of the rows' losses),
 *     dz_c = scale (soft_weight T (p^T_c - sum of q_j over i_j = c)
 *                   + hard_weight (p_c - [c = y])).
 * An entry counts if its token is in [0, vocab) and its logit is not -inf; a
 * teacher with fewer than num_teacher pads with token -1.  The same token
 * twice is two entries.  Without an entry that counts the first term is 0,
 * without a label in [0, vocab) the second; a row with neither has loss 0 and
 * gradient 0, whatever its logits hold.
 *   sched       NULL: targets and losses are in row order.  Otherwise rows
 *               are the pool rows of that schedule (rows = its num_nodes) and
 *               the targets and losses are in NODE order
 *   logits      device [rows, fold_row_ld(vocab)] of dtype (the pad columns
 *               are not looked at)
 *   teacher_token, teacher_logit  device [rows, num_teacher] int32, fp32;
 *               num_teacher 0 .. 256
 *   labels      device [rows] int32, or NULL (no labels)
 *   temperature in [1e-3, 1e3]; the weights not negative
 *   row_loss    device [rows] fp32, without the scale (written)
 *   grad_dtype  of dlogits: dtype, or FOLD_BF16 for fp32 logits (a bf16 head)
 *   dlogits     device [rows, fold_row_ld(vocab)], written whole (pad columns
 *               zero); may be `logits` itself if the types are equal, must not
 *               overlap it otherwise; NULL: the losses alone
 *   ws          device workspace of >= fold_distill_workspace_size bytes (may be
 *               NULL where that is 0: rows that a workgroup holds)
 * Sums are fp32.  Logits may be any finite numbers (a mask of -1e9 or of the
 * type's lowest value is one); those of -inf (masked) have probability 0, and
 * a target there has loss +inf.  A row with a target whose logits are all
 * -inf has loss +inf and gradient 0; one with NaN or +inf has loss and gradient
 * NaN. */
int32_t fold_distill_workspace_size(int32_t dtype, int64_t rows, int32_t vocab, int32_t num_teacher, size_t* bytes);
int32_t fold_loss_distill(const fold_sched* sched, int32_t dtype, int64_t rows, int32_t vocab, const void* logits,
                          int32_t num_teacher, const int32_t* teacher_token, const float* teacher_logit,
                          const int32_t* labels, float temperature, float soft_weight, float hard_weight, float scale,
                          float* row_loss, int32_t grad_dtype, void* dlogits, void* ws, size_t ws_bytes,
                          hipStream_t stream);

/* fold_token_logprobs: what a model says about given tokens.  For every row,
 * with p = softmax(z) over the vocabulary:
 *     logp[j]  = log p[tokens[j]]; 0 for a token outside [0, vocab), so that
 *                sums over padded sequences need no mask
 *     entropy  = - sum_c p_c log p_c
 *     top_token, top_logp  the top_k largest log probabilities in order,
 *                equal ones by the lowest token; entries for which no token
 *                of probability above -inf is left hold -1 and -inf
 *   sched       as in fold_loss_distill (tokens and results in NODE order)
 *   logits      as in fold_loss_distill
 *   tokens      device [rows, num_tokens] int32; num_tokens may be 0
 *   logp        device [rows, num_tokens] fp32
 *   entropy     device [rows] fp32, or NULL
 *   top_token, top_logp  device [rows, top_k] int32, fp32; top_k 0 .. 32
 *   ws          device workspace of >= fold_token_workspace_size bytes (may be
 *               NULL where that is 0: many rows, or short ones)
 * Sums are fp32.  A row of -inf alone has log probabilities -inf and entropy
 * 0; one with NaN or +inf has NaN for all of them and top tokens -1.
 * Errors of both calls: FOLD_E_INVALID for sizes out of range, NULL or
 * misaligned buffers, overlapping logits and dlogits; FOLD_E_MISMATCH for a
 * workspace that is too small or a schedule of another size or device. */
int32_t fold_token_workspace_size(int32_t dtype, int64_t rows, int32_t vocab, int32_t top_k, size_t* bytes);
int32_t fold_token_logprobs(const fold_sched* sched, int32_t dtype, int64_t rows, int32_t vocab, const void* logits,
                            int32_t num_tokens, const int32_t* tokens, float* logp, float* entropy, int32_t top_k,
                            int32_t* top_token, float* top_logp, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- the attention block over node states -----------------------------------
 * What stands between the states of a forward pass and a head where the nodes
 * of one batch of graphs look at the states of another (a decoder's chains at
 * an encoder's trees): layer norm, linear layers with an activation and a
 * residual, and cross attention, each with its gradient.  Matrices are
 * [rows, fold_row_ld(width)], any rows (a pool in pool order, roots_out, tokens
 * of a serving step), 16-byte aligned.  All calls but fold_cross_create and
 * fold_cross_free enqueue on `stream`, never synchronise, never allocate and
 * can be captured; workspaces hold nothing between calls, calls that overlap
 * need one each, and a size is asked for each set of sizes.  Sums, statistics
 * and softmaxes are fp32; results are rounded once to their type.  Every sum's
 * order is fixed by sizes.  rows = 0 is allowed.
 *
 * fold_layer_norm: per row, over its first `width` values,
 *     mean = sum x / width,  rstd = (sum (x - mean)^2 / width + eps)^(-1/2),
 *     y = gamma (x - mean) rstd + beta.
 *   dtype  of x and y: FOLD_F32 or FOLD_BF16; width 1 .. 4096; rows to 2^31 - 1
 *   gamma, beta  device [width] fp32, or NULL (1 and 0)
 *   eps    finite, above 0
 *   y      device, written whole (pad columns zero); may be x itself
 *   mean, rstd  device [rows] fp32 (what the gradient needs), or NULL
 * The pad columns of x are not looked at.
 * fold_layer_norm_backward: with xh = (x - mean) rstd and g = gamma dy,
 *     dx = rstd (g - mean(g) - xh mean(g xh)) (+ residual)
 *     dgamma (+)= sum over the rows of dy xh,   dbeta (+)= sum of dy
 *   dy_dtype  of dy: dtype, or FOLD_F32
 *   residual  device [rows, ld] of residual_dtype (dtype, or FOLD_F32), a gradient
 *             that goes by the norm, or NULL
 *   dx_dtype  of dx: dtype, or FOLD_F32
 *   dx        device, written whole (pad columns zero), or NULL; may be dy or
 *             residual itself where the types are equal
 *   dgamma, dbeta  device [width] fp32, or NULL; written, or added to with
 *             FOLD_BLOCK_ACCUMULATE
 *   ws        device workspace of >= fold_layer_norm_workspace_size bytes (for
 *             dgamma or dbeta; may be NULL where that is 0)
 *
 * fold_linear: out = act(x W^T + bias) + residual.
 *   x         device [rows, fold_row_ld(in_dim)];  in_dim, out_dim 1 .. 16384
 *   W         device [out_dim, fold_row_ld(in_dim)], one row an output, as the
 *             vocabulary head's; the pad columns of one of x and W hold zeros,
 *             of the other any finite values
 *   bias      device [out_dim] fp32, or NULL
 *   act       FOLD_ACT_*;  gelu(z) = z Phi(z), Phi the normal distribution (fp32:
 *             within 1.9e-7, below zero also within 3.1e-6 of itself down to -8;
 *             bf16: within 2.5e-7)
 *   residual  device [rows, fold_row_ld(out_dim)], or NULL; may be out itself
 *   out       device [rows, fold_row_ld(out_dim)], written whole (pad columns
 *             zero)
 *   pre       device, as out: z = x W^T + bias, which the gradient of an
 *             activation needs, or NULL
 *   ws        device workspace of >= fwd_bytes of fold_linear_workspace_size
 *             (may be NULL where that is 0)
 * x, W, residual, out and pre are of dtype.
 * fold_linear_backward: with dz = dout act'(pre) (dout itself for FOLD_ACT_NONE;
 * relu'(0) = 0), rounded to dtype where it enters a product,
 *     dx = dz W,   dW (+)= dz^T x,   dbias (+)= sum over the rows of dz
 *   dout      device [rows, fold_row_ld(out_dim)] of dtype, finite in the pad
 *             columns (zero for FOLD_ACT_NONE)
 *   pre       as left by fold_linear (NULL for FOLD_ACT_NONE)
 *   dpre      device, as pre: receives dz, also where nothing else is asked
 *             for; may be pre or dout itself; NULL for FOLD_ACT_NONE
 *   dx_dtype, dw_dtype  of dx and dW: dtype, or FOLD_F32
 *   dx, dW, dbias  written whole (pad columns zero), or NULL; with
 *             FOLD_BLOCK_ACCUMULATE dbias and a dW of FOLD_F32 are added to
 *   ws        device workspace of >= bwd_bytes of fold_linear_workspace_size
 * A residual's gradient is dout.
 *
 * Errors of these calls: FOLD_E_INVALID for sizes out of range, unknown types,
 * activations or flags, NULL or misaligned buffers, an output that overlaps
 * another buffer where nothing above allows it, products of more than 2^24
 * tiles; FOLD_E_MISMATCH for a workspace that is too small. */
enum { FOLD_ACT_NONE = 0, FOLD_ACT_RELU = 1, FOLD_ACT_TANH = 2, FOLD_ACT_GELU = 3 };
#define FOLD_BLOCK_ACCUMULATE 1

int32_t fold_layer_norm(int32_t dtype, int64_t rows, int32_t width, const void* x, const float* gamma,
                        const float* beta, float eps, void* y, float* mean, float* rstd, hipStream_t stream);
int32_t fold_layer_norm_workspace_size(int32_t dtype, int64_t rows, int32_t width, size_t* bytes);
int32_t fold_layer_norm_backward(int32_t dtype, int64_t rows, int32_t width, const void* x, const float* gamma,
                                 const float* mean, const float* rstd, int32_t dy_dtype, const void* dy,
                                 int32_t residual_dtype, const void* residual, int32_t dx_dtype, void* dx, float* dgamma,
                                 float* dbeta, int32_t flags, void* ws, size_t ws_bytes, hipStream_t stream);
int32_t fold_linear(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, const void* x, const void* W,
                    const float* bias, int32_t act, const void* residual, void* out, void* pre, void* ws, size_t ws_bytes,
                    hipStream_t stream);
int32_t fold_linear_workspace_size(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, size_t* fwd_bytes,
                                   size_t* bwd_bytes);
int32_t fold_linear_backward(int32_t dtype, int64_t rows, int32_t in_dim, int32_t out_dim, const void* x, const void* W,
                             int32_t act, const void* pre, const void* dout, void* dpre, int32_t dx_dtype, void* dx,
                             int32_t dw_dtype, void* dW, float* dbias, int32_t flags, void* ws, size_t ws_bytes,
                             hipStream_t stream);

/* Cross attention: the rows of query sequences (a decoder's nodes) against
 * those of key sequences of other lengths (an encoder's nodes).  Per query row
 * and head, over the keys j of its sequence's source that count,
 *     s_j = scale q . k_j,   p = softmax(s),   o = sum_j p_j v_j,
 *     lse = log sum_j exp(s_j);
 * without such a key o = 0 and lse = -inf, and the row takes no part in any
 * gradient.  Heads are columns: head h is columns [h head_dim, (h+1) head_dim)
 * of q and of the output, and reads key head h / (heads / kv_heads).
 *
 * fold_cross_create checks the lists, lays the work out and returns a plan,
 * which may be used by any number of calls, concurrent ones too (with a
 * workspace each).  It synchronises `stream` and must not be captured.
 *   query_ptr   device [num_seqs + 1]: sequence b is list entries query_ptr[b]
 *               .. query_ptr[b+1] - 1; starts at 0, ends at num_queries
 *   query_row   device [num_queries]: the row of a list entry in the query
 *               matrices, below num_query_rows, each at most once; NULL: row i
 *               is entry i.  With a schedule: its graph_ptr and node_pos.
 *   key_ptr, key_row   the same for num_sources key sequences
 *   source      device [num_seqs]: the key sequence that a query sequence reads
 *               (several may read one), -1: none; NULL: b reads b
 * The lists are copied.  FOLD_E_INVALID for sizes out of range (heads to 1,024,
 * head_dim to 128, heads / kv_heads to 256, queries times heads below 2^31, 2^24
 * workgroups of a head) and for malformed lists, rows out of range or listed
 * twice.
 * fold_cross_free waits as fold_sched_free does. */
typedef struct fold_cross fold_cross;
typedef struct {
  int32_t dtype; /* of all matrices: FOLD_F32 or FOLD_BF16 */
  int32_t heads, kv_heads, head_dim;
  int32_t num_seqs, num_sources;
  int32_t num_queries, num_keys;        /* list entries */
  int32_t num_query_rows, num_key_rows; /* rows of the matrices */
  const int32_t *query_ptr, *query_row, *key_ptr, *key_row, *source;
} fold_cross_batch;

int32_t fold_cross_create(const fold_cross_batch* batch, hipStream_t stream, fold_cross** out);
int32_t fold_cross_free(fold_cross* cross);
int32_t fold_cross_workspace_size(const fold_cross* cross, size_t* fwd_bytes, size_t* bwd_bytes);

/* The matrices have strides of their own (ld*, in elements, at least their
 * width), so k and v may be columns of one matrix; they need the alignment of
 * their elements alone (rows of 16-byte multiples at 16-byte addresses are
 * faster).  Rows that no list names, and columns beyond the heads, are neither
 * read nor written.
 *   q        device [num_query_rows, ldq], heads * head_dim columns
 *   k, v     device [num_key_rows, ldk], [.., ldv], kv_heads * head_dim columns
 *   key_mask device [num_keys] bytes in LIST order (a schedule's node order),
 *            0: the key does not count, whatever its row holds; NULL: all count
 *   scale    above 0, below 2^127; scores are below 1e9 in magnitude, q . k
 *            itself finite
 *   out      device [num_query_rows, ldo] of dtype
 *   lse      device [num_query_rows, heads] fp32, or NULL
 * fold_cross_backward: the gradients of q, k and v from dout; out and lse as
 * left by fold_cross_attend.  dq, dk, dv (of dtype, any of them NULL) have the
 * shapes of q, k and v; listed rows are written (a key that does not count and
 * a source that nobody reads get 0).  dk and dv are summed over the heads of a
 * group and over the sequences that read a source, without atomics.
 * For bf16 the probabilities, and in the gradient the scores' gradients, are
 * rounded to bf16 where they enter a matrix product; everything else is fp32.
 * The gradient takes its probabilities from lse, exp(s - lse), so that a row's
 * are off by |lse| 2^-22 of themselves, and sum do o from out as it was rounded;
 * where a source has up to 32 keys (fp32: one) it sums p (do . v) over them in
 * fp32 instead, so that little of it is lost beside few keys and a single key's
 * dq and dk are 0.
 * FOLD_E_INVALID for NULL buffers, strides below the width, addresses that are
 * no multiple of an element's size, a scale out of range or an output that
 * overlaps another buffer; FOLD_E_MISMATCH for a workspace (16-byte aligned)
 * that is too small or a plan of another device. */
int32_t fold_cross_attend(const fold_cross* cross, const void* q, int64_t ldq, const void* k, int64_t ldk,
                          const void* v, int64_t ldv, const uint8_t* key_mask, float scale, void* out, int64_t ldo,
                          float* lse, void* ws, size_t ws_bytes, hipStream_t stream);
int32_t fold_cross_backward(const fold_cross* cross, const void* q, int64_t ldq, const void* k, int64_t ldk,
                            const void* v, int64_t ldv, const uint8_t* key_mask, float scale, const void* out,
                            int64_t ldo, const float* lse, const void* dout, int64_t lddo, void* dq, int64_t lddq,
                            void* dk, int64_t lddk, void* dv, int64_t lddv, void* ws, size_t ws_bytes,
                            hipStream_t stream);

/* ---- a whole step as one HIP graph ----------------------------------------
 * The level loop (Section 2: one batched iteration per depth, so a batch of
 * depth D costs O(D) launches instead of one per node) still issues a few
 * launches per (depth, operation) group.  For deep batches of narrow levels
 * the host launch cost and the gaps between dependent launches dominate.
 * fold_graph_create records, once, exactly the launches that fold_forward
 * (and, with FOLD_STEP_BACKWARD, fold_backward) would enqueue with the
 * buffers below, and instantiates them as a HIP graph; fold_graph_launch
 * submits that step on any stream with one call.
 *   - The buffers are bound at creation: every launch reads and writes the
 *     same device memory (contents may change between launches, addresses
 *     may not).  Recreate the graph to use other buffers.
 *   - With FOLD_STEP_ZERO_GRADS the step first zeroes every gradient tensor
 *     in `grads` (dW_in, dW_rec, dbias of each set, d_leaf_table of
 *     leaf_rows rows), so a launch yields the gradients of this step alone;
 *     without it they accumulate across launches as with fold_backward.
 *   - The recorded step holds kernel nodes only (no memset or copy nodes),
 *     allocates nothing and never synchronises when launched.
 *   - Launches of one graph must not overlap (they share the buffers): keep
 *     them on one stream or order them with events.
 * fold_graph_create synchronises nothing but returns only after
 * instantiation; it fails with the same codes as fold_forward /
 * fold_backward for inconsistent arguments, FOLD_E_DEVICE if capture or
 * instantiation fails, and leaves *out NULL on error.  The graph must be
 * launched on the device that was current at creation (FOLD_E_MISMATCH
 * otherwise).  The schedule and parameter handles must outlive the graph. */
typedef struct fold_graph fold_graph;

typedef struct {
  const void* leaf_table; /* as fold_forward */
  int64_t leaf_rows;
  void* h_pool;
  float* c_pool;
  void* roots_out;        /* or NULL */
  const float* dh_roots;  /* as fold_backward (used with FOLD_STEP_BACKWARD) */
  const float* dh_nodes;
  const fold_grads* grads; /* read at creation; the host arrays may be freed afterwards */
  float* dh_out;
  float* dc_out;
  void* ws;               /* >= fwd_bytes (forward only) or bwd_bytes */
  size_t ws_bytes;
} fold_step_buffers;

#define FOLD_STEP_BACKWARD 1   /* record fold_backward after fold_forward */
#define FOLD_STEP_ZERO_GRADS 2 /* zero the gradients first (needs FOLD_STEP_BACKWARD) */

int32_t fold_graph_create(const fold_sched* sched, const fold_packed* packed, const fold_step_buffers* buffers,
                          int32_t flags, fold_graph** out);
int32_t fold_graph_launch(const fold_graph* graph, hipStream_t stream);
int32_t fold_graph_num_nodes(const fold_graph* graph, int32_t* nodes); /* kernel nodes recorded */
int32_t fold_graph_free(fold_graph* graph);

/* ---- level launches --------------------------------------------------------
 * The groups of one depth are independent, so by default the narrow groups of
 * a level (up to four) run as one launch per kernel stage (one for their
 * contractions, one for their K-split epilogues, one for their cell
 * backwards, one for their dz . W^T), which removes the dependent launches of
 * levels with several operations.  fold_level_launches(0) turns this off for
 * every later call in the process (each group then launches alone, as a static
 * graph of one batched operation per node would run); fold_level_launches(1)
 * turns it back on.  Returns the previous setting (1 or 0).  Levels of at most
 * 128 rows compute the same forward states bit for bit either way for hidden
 * sizes up to 1,024; beyond, a group's tiles and K slices depend on the groups
 * beside it, so its states are the same up to the order of their fp32 sums,
 * and gradients up to that and the order of the atomic additions of shared
 * children. */
int32_t fold_level_launches(int32_t on);

/* ---- per-kernel timing (profiling aid) ----------------------------------
 * While enabled, every kernel the library launches is bracketed by a pair of
 * HIP events recorded on the launch stream, under a short kernel-class name
 * (e.g. "cell_fwd.treelstm.f32").  fold_profile_read waits for the recorded
 * events, returns one entry per class (launch count, summed and largest
 * duration in milliseconds), and clears the record.  Enabling costs one
 * event pair per launch; disabled (the default) it costs nothing. */
typedef struct {
  char name[48];
  int64_t launches;
  double total_ms;
  double max_ms;
} fold_kernel_stat;

int32_t fold_profile_enable(int32_t on);
int32_t fold_profile_read(fold_kernel_stat* out, int32_t capacity, int32_t* count);

/* The same records one by one, in launch order, each with the schedule group
 * it ran for (its index in the group table; -1 for launches of no single
 * group: gradient set-up, roots, the per-operation weight gradients) and its
 * operation id (-1 if none).  This splits a step's time by level and by
 * (depth, op) group (Section 2: one batched operation per group).
 * Writes min(capacity, records) entries to `out` (caller-owned host array),
 * sets *count to the number of records taken, and clears them all, as
 * fold_profile_read does.  With capacity 0 (`out` may be NULL) it only sets
 * *count and keeps the records.  FOLD_E_INVALID for NULL arguments;
 * FOLD_E_DEVICE if an event could not be read. */
typedef struct {
  char name[48];
  int32_t group;
  int32_t op;
  double ms;
} fold_launch_time;

int32_t fold_profile_read_launches(fold_launch_time* out, int32_t capacity, int32_t* count);

/* ---- achievable peaks (diagnostics) --------------------------------------
 * fold_probe_mfma times a loop of independent 32x32 MFMA instructions
 * (fp32 32x32x2 or bf16 32x32x16) on every compute unit and returns the
 * sustained dense TFLOP/s; fold_probe_copy copies `bytes` (a multiple of 16,
 * both buffers 16-byte aligned, caller-owned device memory) five times with
 * 16-byte loads and stores and returns read+write GB/s.  Both synchronise
 * `stream`; fold_probe_mfma allocates a small output buffer.
 * fold_probe_mfma_random is the same loop with random operand bits (four
 * registers a side per lane, uniform in [-1, 1), cycled over the
 * accumulators): the matrix cores' power draw, and so the clock the GPU
 * holds, depends on the operand bits, and random data is what the
 * contractions multiply.  FOLD_E_INVALID for a dtype other than FOLD_F32 /
 * FOLD_BF16 or a NULL result pointer. */
int32_t fold_probe_mfma(int32_t dtype, hipStream_t stream, double* tflops);
int32_t fold_probe_mfma_random(int32_t dtype, hipStream_t stream, double* tflops);
int32_t fold_probe_copy(void* dst, const void* src, size_t bytes, hipStream_t stream, double* gbs);

/* Text of the last error on the calling thread ("" if none). */
const char* fold_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* FOLD_H_ */
