/*
 * fc.h -- C ABI of the fused-combinator library for AMD MI355X (gfx950).
 *
 * The library executes array-combinator programs (paper section 2, "Language")
 * as fused clusters (section 3, "Fusion"): map / zipWith / generate producers
 * are evaluated in registers, pushed through gathers, and consumed by a fold, a
 * segmented fold, a single-pass scan or a scatter, so that no intermediate
 * array reaches memory.  Which combinators share a loop is described by a
 * clustering (section 4.1: pi, x, m; section 4.2: traversal orders) that
 * fc_plan() chooses by solving the paper's integer linear program exactly.
 *
 * Everything here is plain C: POD structs, raw pointers, sizes.  No exception
 * crosses the boundary; every function returns FC_OK (0) or a negative error
 * code and leaves a message for fc_last_error().
 *
 * Pointers are HOST pointers unless a comment says DEVICE.
 */
#ifndef FC_H
#define FC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- error codes */
#define FC_OK                   0
#define FC_E_BADGRAPH          -1  /* cycle / arity / dtype / shape mismatch, unknown function  */
#define FC_E_ILLEGAL_PARTITION -2  /* breaks a rule of section 3.4 or a constraint of Fig. "Total ILP formulation" */
#define FC_E_UNSUPPORTED       -3  /* legal cluster, but no kernel is built for its combination of consumers (e.g. three
                                      folds of flattened arrays, a scan of f32 that feeds a fold in its cluster), or its element
                                      programs exceed the limits (24 nodes, 7 external arrays, gathers nested 3 deep).
                                      Element programs of maps, generates and gathers as such always run: compiled for
                                      the shapes of the paper's programs, interpreted otherwise */
#define FC_E_UNBOUND           -4  /* an input or manifest array has no device buffer, or it is too small / misaligned */
#define FC_E_SCRATCH           -5  /* scratch missing, misaligned or smaller than fc_scratch_bytes() */
#define FC_E_HIP               -6  /* a HIP runtime call failed (message holds hipGetErrorString) */
#define FC_E_ARG               -7  /* NULL / out-of-range argument, capacity too small */
#define FC_E_LIMIT             -8  /* graph too large for the exact chooser, or a size above 2^31-1 elements */
#define FC_E_DEVICE_WAIT       -9  /* fc_check: a kernel of an earlier call gave up a bounded wait (see fc_check) */

/* ---------------------------------------------------------------- vocabulary */
/* Combinators of the language (section 2; Table 1 gives their cluster signatures).
 * One node = one combinator = the array it produces. */
typedef enum fc_kind {
  FC_INPUT    = 0,  /* array handed in by the caller; every edge out of it is infusible (section 3.4) */
  FC_MAP      = 1,  /* n-ary map: zipWith after the SoA transformation (section 2, last paragraph) */
  FC_GENERATE = 2,  /* ys[i] = f(i) */
  FC_GATHER   = 3,  /* ys[j] = src[idx[j]]; arg0 = idx (read in output order), arg1 = src (read in the gather's own order) */
  FC_FOLD     = 4,  /* shape (1): fold of the flattened argument; else fold of the innermost dimension */
  FC_FOLDSEG  = 5,  /* arg0 = flat values, arg1 = offsets[R+1] (infusible); y[r] = fold of values[off[r], off[r+1]) */
  FC_SCANL    = 6,  /* exclusive prefix combine (+), identity seeded; traversal order 0; a rank-2 array is scanned row
                       by row.  i32: exact.  f32: summed in a fixed tree order (the same bits on every launch), so
                       a prefix differs from the sequentially rounded sum by rounding only; an f32 scan can be
                       stored (also together with the array it scans) but not fused with a scatter or a fold
                       (FC_E_UNSUPPORTED) */
  FC_SCANR    = 7,  /* exclusive suffix combine; traversal order 1 */
  FC_SCATTER  = 8,  /* arg0 = dest (infusible, updated in place; none of the other arguments may be the same array:
                       FC_E_BADGRAPH), arg1 = index, arg2 = value, arg3 = flag (optional);
                       fn = OVERWRITE (kept indices distinct) or ADD (colliding indices combine: exact for i32,
                       in an unspecified order for f32) */
  FC_FORCE    = 9   /* identity; every edge out of it is infusible */
} fc_kind;

/* Programs are made of the first two; the others are element types of the operators' arrays (below). */
typedef enum fc_dtype { FC_F32 = 0, FC_I32 = 1, FC_F16 = 2, FC_BF16 = 3, FC_I64 = 4 } fc_dtype;

/* Element functions (the paper allows arbitrary lambdas; the kernels here are
 * hand written, so the lambdas form a closed vocabulary). */
typedef enum fc_fn {
  FC_FN_NONE = 0,
  /* map functions; fp32 arithmetic is rounded operation by operation (never contracted) */
  FC_FN_IDENT = 1,        /* x                                           */
  FC_FN_AFFINE = 2,       /* fparam[0]*x + fparam[1]                     */
  FC_FN_SIN_X_MUL_X = 3,  /* sin(x)*x                                    */
  FC_FN_SQ_PLUS_ONE = 4,  /* x*x + 1                                     */
  FC_FN_MUL2 = 5,         /* a*b                                         */
  FC_FN_ADD2 = 6,         /* a+b                                         */
  FC_FN_ADD3 = 7,         /* (a+b)+c                                     */
  FC_FN_ADD5 = 8,         /* (((a+b)+c)+d)+e                             */
  FC_FN_EXP_NEG = 9,      /* exp(-x)                                     */
  FC_FN_MOD_EQ = 10,      /* i32 -> i32: (x mod iparam[0] == iparam[1]) ? 1 : 0 for x >= 0; iparam[0] > 0;
                             a residue outside [0, iparam[0]) matches no x */
  /* generate functions (index -> i32) */
  FC_FN_IOTA = 32,            /* i                                                       */
  FC_FN_IOTA_REV = 33,        /* n-1-i                                                   */
  FC_FN_CLAMP_SHIFT_2D = 34,  /* (i,j) -> clamp(i+iparam[0],0,H-1)*W + clamp(j+iparam[1],0,W-1) */
  FC_FN_ROW_OF_2D = 35,       /* (i,j) -> i                                              */
  FC_FN_CONST_I32 = 36,       /* iparam[0]                                               */
  /* reducers of fold / foldSeg / scan and combination functions of scatter */
  FC_OP_ADD = 64,
  FC_OP_MAX = 65,
  FC_OP_MUL = 66,
  FC_OP_OVERWRITE = 67        /* scatter only: the new value wins (section 2.1) */
} fc_fn;

#define FC_MAX_ARGS 6

/* node flags */
#define FC_NODE_OUTPUT 1u   /* a result of the program: must be manifest (m = 0) */
#define FC_NODE_SINGLE_PASS 2u /* on a fold or foldSeg node: its cluster must run as ONE pass over the arrays it reads,
                                  every gather issued at the position that asks for it (section 2: a fold inside a
                                  cluster is one stage of a parallel reduction).  Without the flag the library may, for
                                  a gathered table larger than the L2 of an XCD, run a kernel that visits the positions
                                  in another order and in more than one kernel (elements sorted by table range in a
                                  first kernel and gathered from on-chip memory; for small inputs the streams of a
                                  segmented fold read once per column range), which is faster and, the reducers
                                  being commutative, gives the same result up to rounding */

typedef struct fc_node {
  int32_t  kind;              /* fc_kind  */
  int32_t  dtype;             /* fc_dtype of the produced array */
  int32_t  fn;                /* fc_fn    */
  float    fparam[2];
  int32_t  iparam[4];
  int32_t  nargs;
  int32_t  arg[FC_MAX_ARGS];  /* indices of the producing nodes; each < own index (topological order) */
  int32_t  rank;              /* 1 or 2 */
  int64_t  shape[2];          /* row-major extents; unused extents are 1 */
  uint32_t flags;
  uint32_t infusible_args;    /* bit k set: the edge from arg[k] is infusible whatever the kinds say
                                 (the argument is indexed with `!`, wrapped in force, or passed to foreign code) */
} fc_node;

/* The data dependence graph (n, N, F, I) of section 4.1.  Edges are implied by
 * the argument lists; edge e is the e-th (consumer ascending, slot ascending)
 * argument reference.  Fusible / infusible follows from the kinds (inputs,
 * force, scatter destination and scatter result, foldSeg offsets are infusible). */
typedef struct fc_graph {
  int32_t        n;
  const fc_node *nodes;
} fc_graph;

/* A clustering in the variables of Fig. "Total ILP formulation".  All arrays are
 * caller allocated: n_nodes entries for the per-node arrays, n_edges for the
 * per-edge array. */
typedef struct fc_partition {
  int32_t  n_nodes;       /* capacity of pi / fused_away / order_out (in) */
  int32_t  n_edges;       /* capacity of edge_unfused (in)                */
  int32_t *pi;            /* cluster number; clusters run in ascending order           */
  uint8_t *fused_away;    /* m_a: 1 = the array never reaches memory, 0 = manifest      */
  int32_t *order_out;     /* d^o_a: 0, 1 or the label (2 + ordinal) of a gather         */
  uint8_t *edge_unfused;  /* x_ab: 0 = fused over, 1 = not                              */
  int32_t  n_clusters;    /* (out) clusters after the connected-component split         */
  double   cost;          /* (out) value of the requested cost function                 */
  int32_t  proven;        /* (out, fc_plan and fc_plan_weighted) 1: the clustering is optimal; 0: it is the
                             best one found when the search budget of FC_PLAN_ANYTIME ran out */
} fc_partition;

/* cost functions of section 4.1 ("Cost function"), evaluated on the ILP solution */
typedef enum fc_cost {
  FC_COST_CLUSTERS    = 0,  /* (a) largest cluster number + 1                                  */
  FC_COST_FUSED_EDGES = 1,  /* (b) sum of x over fusible edges                                 */
  FC_COST_ARRAYS      = 2,  /* (c) number of manifest non-input arrays                         */
  FC_COST_READS       = 3,  /* (d) array reads: one per (array, consuming cluster, order)      */
  FC_COST_READS_WRITES= 4,  /* (e) reads + manifest arrays                                     */
  FC_COST_BYTES       = 5   /* (e) with every read / write weighted by the array's bytes       */
} fc_cost;

/* plan flags */
#define FC_PLAN_NO_SPLIT 1u  /* keep the raw ILP solution (skip the connected-component split) */
#define FC_PLAN_EXECUTABLE 2u /* choose among the clusterings fc_run_fused has kernels for: the kernels are a fixed
                                 set of cluster shapes, and the optimum of the ILP may contain a legal cluster that
                                 is not among them (fc_run_fused would answer FC_E_UNSUPPORTED).  With this flag the
                                 result is the cheapest clustering that runs; FC_E_UNSUPPORTED if there is none,
                                 i.e. some combinator has no kernel even on its own */
#define FC_PLAN_ANYTIME 4u    /* the chooser is an exact branch and bound: its time grows exponentially with the
                                 number of combinators (seconds up to 24, half a minute at 30, much longer from 36 on).
                                 With this flag it starts from a clustering built greedily and improved by
                                 moving combinators between neighbouring clusters, searches for 1.2 seconds at
                                 most, spends what is left of two seconds on further (random) moves if the search
                                 had not finished, and returns the best clustering found, which is legal at any
                                 moment; fc_partition.proven says whether the search had finished.  Programs of
                                 more than 64 combinators get the greedy clustering improved by two seconds of moves.
                                 Without the flag a search that exceeds its (much larger) budget, or a program
                                 of more than 64 combinators, ends in FC_E_LIMIT */

typedef struct fc_buffer {
  void   *ptr;    /* DEVICE pointer, 16-byte aligned; NULL = not bound */
  int64_t bytes;
} fc_buffer;

/* ---------------------------------------------------------------- planning (host only) */

/* Number of edges of the graph (length of fc_partition.edge_unfused). */
int fc_num_edges(const fc_graph *g, int32_t *n_edges);

/* Choose the clustering that minimises `cost_fn` subject to the constraints of
 * Fig. "Total ILP formulation" (sections 4.1, 4.2), by exact branch and bound over
 * the edge variables x, then split clusters into connected components (section
 * 4.1, "Performance and correctness").  Fills every array of *out, n_clusters, cost
 * and proven.  Graphs of more than 64 non-input nodes, and searches that exceed their
 * budget, are refused (FC_E_LIMIT) unless FC_PLAN_ANYTIME is set. */
int fc_plan(const fc_graph *g, int cost_fn, uint32_t flags, fc_partition *out);

/* fc_plan for a linear combination of the cost functions: minimises
 * sum_k weights[k] * cost_k, k over the FC_COST_COUNT values of fc_cost (section 5.1,
 * "Runtime analysis", proposes such a combination with coefficients found by tuning as
 * the way to a cost function that models run time on a given machine).  weights: HOST,
 * FC_COST_COUNT entries, none negative, not all zero (else FC_E_ARG).  out->cost is the
 * weighted sum for the chosen clustering.  Same outputs and limits as fc_plan. */
#define FC_COST_COUNT 6
int fc_plan_weighted(const fc_graph *g, const double *weights, uint32_t flags, fc_partition *out);

/* The greedy comparison arms of section 5 ("Greedy"): direction 0 walks the fusible edges
 * from the top of the graph, 1 from the bottom, and fuses an edge whenever a legal
 * clustering still exists that fuses it together with the edges already taken.  The
 * result is locally maximal, not optimal.  Same outputs and limits as fc_plan; cost is the
 * value of cost_fn for the returned clustering. */
int fc_plan_greedy(const fc_graph *g, int direction, int cost_fn, uint32_t flags, fc_partition *out);

/* The clustering with every combinator in a cluster of its own (no fusion). */
int fc_partition_trivial(const fc_graph *g, fc_partition *out);

/* Check a clustering against the rules of section 3.4 and the ILP constraints;
 * only pi is read, the other arrays and n_clusters are (re)derived and written.
 * *cost receives the value of cost_fn for it (may be NULL). */
int fc_partition_check(const fc_graph *g, fc_partition *p, int cost_fn, double *cost);

/* Work duplication (named in sections 1 and 6, outside the paper's ILP): clone
 * every map / generate node that a gather reads as its source and that has other
 * consumers, once per such gather, so that each clone has a single traversal
 * order.  Writes the rewritten graph to out_nodes (capacity entries), its size to
 * *out_n, and for each new node the index of the node it came from to origin. */
int fc_duplicate(const fc_graph *g, fc_node *out_nodes, int32_t capacity, int32_t *out_n, int32_t *origin);

/* ---------------------------------------------------------------- execution (device work) */

/* Bytes of device scratch fc_run_* needs for this graph and clustering
 * (p == NULL: the unfused clustering): the control block, the manifest
 * intermediates, and the workspace of the cluster kernel that asks for the most. */
int fc_scratch_bytes(const fc_graph *g, const fc_partition *p, size_t *bytes);

/* Execute the program cluster by cluster, one kernel launch per cluster (two for a
 * fold over a gather from a table larger than the L2 of an XCD), on `hip_stream`
 * (a hipStream_t; NULL = the default stream).  The call only enqueues work and
 * returns; results are valid after the stream is synchronised.
 *
 * bufs[i] is the DEVICE buffer of node i.  Inputs and manifest arrays (m = 0) of
 * the clustering must be bound, fused-away arrays are ignored.  Arrays made
 * manifest by the clustering but not bound by the caller are placed in scratch.
 * A scatter updates its destination buffer in place (section 2, scatter), its own
 * buffer must be NULL or equal to the destination's.  Scalar results (fold of
 * shape (1)) are 4-byte device buffers.  Gather and scatter indices out of range
 * are undefined behaviour, as in the paper.
 *
 * scratch: DEVICE, 256-byte aligned, at least fc_scratch_bytes().  Its first
 * FC_SCRATCH_CONTROL_BYTES must be zero the first time a buffer is used; every
 * call leaves them ready for the next one.  Two calls that overlap in time must
 * not share a scratch buffer. */
int fc_run_fused(const fc_graph *g, const fc_partition *p, const fc_buffer *bufs,
                 void *scratch, size_t scratch_bytes, void *hip_stream);

/* fc_run_fused for callers that cannot allocate device memory or bring a scratch buffer:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, checks, kernels and results as fc_run_fused, but the scratch is a buffer
 * of FC_STATIC_SCRATCH_BYTES inside the library's code object (one copy per device, zero
 * when the library is loaded, kept until the process ends).  The call allocates nothing,
 * on the device or through any library.  The first call on a device looks the buffer's
 * address up (make that call outside a graph capture).
 *
 * Programs whose fc_scratch_bytes() exceeds FC_STATIC_SCRATCH_BYTES (manifest
 * intermediates the caller did not bind, or a kernel workspace, too large) are refused
 * with FC_E_LIMIT before anything is enqueued: bind the intermediates, or use fc_run_fused.
 * All calls on one device share the one buffer: calls that overlap in time on a device
 * (two streams, two host threads) race, as two fc_run_fused calls on one scratch buffer
 * would.  Nothing has to be cleared between calls: words left by earlier calls carry
 * older launch tags.  fc_check(NULL, stream) reports on this buffer. */
#define FC_STATIC_SCRATCH_BYTES (32u << 20)
int fc_run_fused_static(const fc_graph *g, const fc_partition *p, const fc_buffer *bufs, void *hip_stream);

/* Same program, no fusion: one kernel per combinator, every intermediate array
 * (generated index arrays included) materialised in scratch unless bound. */
int fc_run_unfused(const fc_graph *g, const fc_buffer *bufs,
                   void *scratch, size_t scratch_bytes, void *hip_stream);

/* fc_run_fused (p == NULL: fc_run_unfused) in two halves, for callers that run one program on
 * the same buffers many times.  fc_bind does everything a run does on the host -- the checks, the
 * choice of the kernels, the arguments and the sizes of their launches -- and enqueues nothing;
 * fc_run_bound enqueues the launches.  The graph, the clustering and the buffer table are not
 * needed after fc_bind; the device memory they name and the scratch buffer are, until the last run
 * has finished.  A bound program belongs to the device that was current in fc_bind.  It is not
 * changed by running: any number of threads and streams may run it, under the rule for runs that
 * share a scratch buffer.  Same errors as fc_run_fused / fc_run_unfused; fc_unbind(NULL) does nothing. */
typedef struct fc_bound fc_bound;
int fc_bind(const fc_graph *g, const fc_partition *p, const fc_buffer *bufs, void *scratch, size_t scratch_bytes,
            fc_bound **out);
int fc_run_bound(const fc_bound *b, void *hip_stream);
int fc_unbind(fc_bound *b);

/* ---------------------------------------------------------------- operators of a serving cache */
/* The pattern of this library -- index arrays decide what a reduction reads and a scatter writes, and nothing in between
 * reaches memory -- at the place where language models meet it: a cache of keys and values in pages.  FC_PAGE_MAP scans the
 * requests' lengths into block tables and slot maps, FC_HEAD_NORM_ROPE writes keys and values through the slot map,
 * FC_PAGED_ATTENTION folds over the cache gathered through the block table.  Three more leave most of a long cache unread:
 * FC_PAGE_BOUNDS folds the keys of a page into their least and largest, FC_PAGE_SELECT picks by these the pages of a request that each key
 * head reads, and FC_PREFIX_ATTENTION reads what many requests begin with once for all of them.  The language above cannot say them (rank 2,
 * 32-bit elements, a closed vocabulary), so each is an operator of its own.
 *
 * An operator is a kind and a struct of its arrays.  Lists of operators run in order on a stream under the rules of programs:
 * fc_run_operators enqueues and returns; fc_bind_operators does the host's work once, for callers that run the
 * same operators on the same arrays step after step (the bound list is an fc_bound: fc_run_bound, fc_unbind); nothing is
 * allocated, nothing synchronises, no memset or copy is enqueued, so a step can be captured into a graph.  Scratch is that of
 * fc_run_fused: 256-byte aligned, its first FC_SCRATCH_CONTROL_BYTES zero the first time, not shared by calls that overlap in time.
 *
 * Shapes, types, strides and alignment are checked before anything is enqueued (FC_E_ARG: wrong, FC_E_UNSUPPORTED: right but not
 * built, FC_E_UNBOUND: no memory or misaligned, FC_E_LIMIT: an extent beyond 2^31-1).  What lies in device memory cannot be: lengths,
 * page numbers, slots and positions out of range are defined below, and no kernel reads or writes outside its arrays for
 * them.  Outputs must not overlap inputs or each other except where it is said. */

/* A DEVICE array.  rank 0: absent.  Strides in elements; the innermost is 1, and those of an array that is written keep its
 * elements apart.  ptr is aligned to the element, and may be NULL where an extent is 0. */
typedef struct fc_tensor {
  void   *ptr;
  int32_t dtype;      /* fc_dtype */
  int32_t rank;       /* 0 to 4 */
  int64_t shape[4];
  int64_t stride[4];
} fc_tensor;

typedef enum fc_operator_kind {
  FC_PAGE_MAP            = 0,  /* args: fc_page_map            */
  FC_HEAD_NORM_ROPE      = 1,  /* args: fc_head_norm_rope      */
  FC_HEAD_NORM_ROPE_GRAD = 2,  /* args: fc_head_norm_rope_grad */
  FC_PAGED_ATTENTION     = 3,  /* args: fc_paged_attention     */
  FC_PAGE_BOUNDS         = 4,  /* args: fc_page_bounds         */
  FC_PAGE_SELECT         = 5,  /* args: fc_page_select         */
  FC_PREFIX_ATTENTION    = 6   /* args: fc_prefix_attention    */
} fc_operator_kind;

typedef struct fc_operator {
  int32_t     kind;
  const void *args;
} fc_operator;

/* Block table and slot map of one step of a server.  B requests, tables of W pages each, pages of P = page_size tokens, a ring of
 * C page numbers that holds the free pages from cursor[0] (taken from there) up to cursor[1] (given back there), both counting on
 * for ever, C at least the number of pages.  new_tokens[r] > 0: tokens request r adds in this step; < 0: tokens it drops from its
 * end (-lengths[r]: it leaves).  With pages(n) = min(ceil(n / P), W), len = max(lengths[r], 0), want = max(len + new_tokens[r], 0):
 *   the pages pages(len) .. pages(want)-1 are taken from the ring, requests in order, and entered in the table; where the ring
 *   runs out the rest stay as they are, and the request keeps the tokens that fit: lengths_after[r] = want, or the least of want
 *   and what its pages hold.  The pages pages(want) .. pages(len)-1 of a request that shrinks go to the ring, requests in order;
 *   pages given back are not taken in the same step.
 *   row_start[r] = number of new tokens of the requests before r.  Token t of the step, j-th new token of request r:
 *   request[t] = r, positions[t] = len + j, slots[t] = table[r][positions[t] / P] * P + positions[t] mod P, or -1 if it has no place
 *   (positions[t] >= lengths_after[r], or its entry is negative).  Past the last token: -1, 0, -1.
 *   cursor_after: the cursor of the next step; unplaced[0]: tokens of all requests that found no page.
 * cursor, lengths and new_tokens are not written, so a step that is run again gives the same; the ring and the table
 * are written in place.  Tokens beyond the extent of slots have no entry.  Where the new tokens are 2^31 or more together,
 * row_start stays at 2^31-1. */
typedef struct fc_page_map {
  int32_t   page_size;
  fc_tensor lengths;        /* i32 [B] */
  fc_tensor new_tokens;     /* i32 [B] */
  fc_tensor pool;           /* i32 [C], in and out */
  fc_tensor cursor;         /* i64 [2] */
  fc_tensor table;          /* i32 [B, W], in and out */
  fc_tensor lengths_after;  /* i32 [B], out */
  fc_tensor row_start;      /* i32 [B + 1], out */
  fc_tensor slots;          /* i64 [T], out */
  fc_tensor positions;      /* i32 [T], out */
  fc_tensor request;        /* i32 [T], out */
  fc_tensor cursor_after;   /* i64 [2], out */
  fc_tensor unplaced;       /* i64 [1], out */
} fc_page_map;

/* Norm of every query and key head and rotation by position, in one pass.  x, one head of one token, D elements:
 *   y = x * rsqrt(mean(x^2) + eps) * weight   (y = x where the weight is absent),
 *   the first R elements of y are turned in pairs, the i-th pair, i < R/2, by the angle whose cosine and sine are cos_sin[p][i] and
 *   cos_sin[p][R/2 + i], p = positions[axis_of[i]][t] (axis 0 where axis_of is absent; no rotation where cos_sin is); a pair is
 *   (y[i], y[i + R/2]), interleaved: (y[2i], y[2i + 1]);  (a, b) -> (a c - b s, b c + a s).
 * In 32 bits, rounded once.  Keys go to k_out, or, with values as they are, to row slots[t] of the caches (page slots[t] / P, place
 * slots[t] mod P); slots outside the cache, -1 among them, are skipped; slots of one call are distinct.  A position or an axis outside
 * its table gives NaN in the rotated elements that need it.  q_out may be q and k_out may be k (same memory, same strides: FC_E_ARG otherwise).
 * At most 255 axes, 2^31-1 places of the cache and 2^31-1 heads of a token, all of q, k and (with slots) v (FC_E_LIMIT).  With N elements the
 * largest power of two, of 16 bytes at most, that D/2, R/2 (not interleaved), the strides and the alignment of the rows are multiples
 * of, D is at most 128 N (FC_E_UNSUPPORTED); rows are read N elements at a time, or more where R/2 alone makes N one or two. */
typedef struct fc_head_norm_rope {
  fc_tensor q;            /* [T, Hq, D]: f32, f16 or bf16; D even, at most 512 */
  fc_tensor k;            /* [T, Hk, D] */
  fc_tensor q_weight;     /* [D] of the same type, or absent */
  fc_tensor k_weight;
  fc_tensor cos_sin;      /* f32 [positions there are, R], R even, R <= D; or absent.  Without rows every position is outside it */
  fc_tensor positions;    /* i32 [axes, T]; absent with cos_sin */
  fc_tensor axis_of;      /* i32 [R / 2], or absent */
  fc_tensor q_out;        /* [T, Hq, D], out */
  fc_tensor k_out;        /* [T, Hk, D], out; absent with slots */
  fc_tensor v;            /* [T, Hk, D]; with slots */
  fc_tensor k_cache;      /* [pages, P, Hk, D], out; with slots */
  fc_tensor v_cache;
  fc_tensor slots;        /* i64 [T], or absent */
  double    eps;
  int32_t   interleaved;
} fc_head_norm_rope;

/* Its gradient: dq and dk from the gradients of q_out and k_out, and (f32) those of the weights, summed over tokens and heads in a
 * fixed order.  With g = dy turned back, u = x * rsqrt(mean(x^2) + eps): dweight = sum g u, dx = rsqrt(...) * (w g - u mean(w g u)).
 * dq may be dq_out and dk may be dk_out, as above. */
typedef struct fc_head_norm_rope_grad {
  fc_tensor q, k, q_weight, k_weight, cos_sin, positions, axis_of;   /* as above */
  fc_tensor dq_out;       /* [T, Hq, D] */
  fc_tensor dk_out;       /* [T, Hk, D] */
  fc_tensor dq;           /* [T, Hq, D], out */
  fc_tensor dk;           /* [T, Hk, D], out */
  fc_tensor dq_weight;    /* f32 [D], out; absent with q_weight */
  fc_tensor dk_weight;    /* f32 [D], out; absent with k_weight */
  double    eps;
  int32_t   interleaved;
} fc_head_norm_rope_grad;

/* Attention of one new token of each request over its pages of the cache.  Request b sees the keys j of
 * [max(0, len - window), len), len = lengths[b] (window 0: all), at place j mod P of page table[b][j / P]; keys on pages that are
 * outside the cache or the table are not there.  Query head h reads key head h / (Hq / Hk).
 *   s_j = scale q.k_j, out = sum_j exp(s_j) v_j / sum_j exp(s_j), lse = log sum_j exp(s_j)
 * In 32 bits, rounded once, but for the weights exp(s_j - max) of 16-bit values: two numbers of 16 bits hold them, together 16 bits of a
 * weight (bf16) or 22, and those below 2^-39 of the largest count as none (f16).
 * A request without keys, or with no score above -inf, gets zeros and -inf.  Pieces of a call's work (at most 128 keys of a request's key
 * head, of as many keys as its table could hold, 2^31-1 at most) are counted in 31 bits, the elements of a request's heads, four at a time, too (FC_E_LIMIT).  What lies
 * in the pages past a request's length is not looked at, whatever it holds.
 * With a table of rank 3 every key head has keys of its own: h sees the lengths[b][h] keys that lie, one page after the other, on the pages
 * table[b][h]; all else is as above, positions and the window counted in what the head sees. */
typedef struct fc_paged_attention {
  fc_tensor q;            /* [B, Hq, D]: f32, f16 or bf16; D a multiple of 8, at most 256; rows 16-byte aligned */
  fc_tensor k_cache;      /* [pages, P, Hk, D], in any order of strides with D innermost; rows 16-byte aligned */
  fc_tensor v_cache;
  fc_tensor table;        /* i32 [B, W], or [B, Hk, W] */
  fc_tensor lengths;      /* i32 [B], or [B, Hk] */
  fc_tensor out;          /* [B, Hq, D], out */
  fc_tensor lse;          /* f32 [B, Hq], out, or absent */
  double    scale;
  int32_t   window;
} fc_paged_attention;

/* Bounds of the keys of a page, for the pages that got new keys.  Request b has new keys at the positions max(lengths_before[b], 0) ..
 * lengths[b]-1 (and below W P), which lie where fc_paged_attention finds them.  For each page that holds any, and each key head:
 *   bounds[page][h][0] = the least, bounds[page][h][1] = the largest of every element of its new keys, and of what was there before where
 *   the page's first position is below lengths_before[b].
 * A NaN among the keys makes a NaN of both.  Pages outside the cache are left out; a page takes new keys of one request only, at one place of its table.  Keys that a request drops from its end
 * leave bounds that are still bounds.  A step that is run again gives the same.  Pages of a request that can have new keys times heads: 2^31-1 of all
 * requests together (FC_E_LIMIT). */
typedef struct fc_page_bounds {
  fc_tensor k_cache;         /* [pages, P, Hk, D]: f32, f16 or bf16; D a multiple of 8, at most 256; rows 16-byte aligned */
  fc_tensor table;           /* i32 [B, W] */
  fc_tensor lengths_before;  /* i32 [B] */
  fc_tensor lengths;         /* i32 [B] */
  fc_tensor bounds;          /* [pages, Hk, 2, D] of the type of the cache, in and out; rows 16-byte aligned */
} fc_page_bounds;

/* The pages of a request that count most for each of its key heads.  Request b has pages(b) = min(ceil(lengths[b] / P), W) pages, P = page_size, its
 * keys end at len = min(lengths[b], W P); an entry of the table that is no page of bounds is not there.  The score of a page for key head h
 * bounds what any of its keys scores with a query head of the group:
 *   s = max over the query heads of h of  sum over d of  max(q_d, 0) bounds[page][h][1][d] + min(q_d, 0) bounds[page][h][0][d]
 * in 64 bits, a NaN counted as +inf.  Taken are the first `first` and the last `last` of the pages (1 and 1 keep what began the text and
 * what is newest), and of the others those of the largest scores, of equal ones those that come first, S in all; all that are there where they are no more.
 * selected[b][h]: their numbers in the order of the table, -1 behind them.  selected_lengths[b][h]: the keys they hold, which is P each but for
 * the last page of the request.  Both are what fc_paged_attention takes as a table of rank 3 and its lengths.
 * S P is at most 2^31-1, B Hk 2^24-1, B Hk times the pages of a request 2^36 (FC_E_LIMIT).  How rows are spread over the device goes by W: a table much
 * wider than its requests are long costs time. */
typedef struct fc_page_select {
  fc_tensor q;                 /* [B, Hq, D]: f32, f16 or bf16; D a multiple of 8, at most 256; rows 16-byte aligned */
  fc_tensor bounds;            /* [pages, Hk, 2, D] of the same type; rows 16-byte aligned */
  fc_tensor table;             /* i32 [B, W] */
  fc_tensor lengths;           /* i32 [B] */
  fc_tensor selected;          /* i32 [B, Hk, S], out */
  fc_tensor selected_lengths;  /* i32 [B, Hk], out */
  int32_t   page_size;
  int32_t   first;
  int32_t   last;              /* first + last <= S */
} fc_page_select;

/* Attention of one new token of each request whose keys are those of a prefix, which all requests of a group share, and its own behind them.
 * Group g: the requests group_start[g] .. group_start[g+1]-1, whose prefix are the prefix_lengths[g] keys on the pages prefix_table[g]; requests
 * before group_start[0] and from group_start[G] on have no prefix.  A start below an earlier one counts as that one, below 0 as 0, above B as B.  Request
 * b's own keys are the lengths[b] keys on the pages table[b].  The result is that of fc_paged_attention without a window over both, each key
 * of a prefix read once for 16 to 128 of the query heads that see it.  A request may have no keys of its own, a group no prefix.
 * scale is below 2^126 (FC_E_UNSUPPORTED).  At most 1024 groups; pieces of a prefix (32 keys of a key head for 128 query heads, at least) are counted in 31 bits, of as many keys as its
 * table could hold (FC_E_LIMIT).  How many query heads read a prefix together goes by B Hq / (Hk G): places for groups that have no requests, and many requests
 * without a group, cost time. */
typedef struct fc_prefix_attention {
  fc_tensor q;               /* as in fc_paged_attention */
  fc_tensor k_cache;
  fc_tensor v_cache;
  fc_tensor prefix_table;    /* i32 [G, Wp] */
  fc_tensor prefix_lengths;  /* i32 [G] */
  fc_tensor group_start;     /* i32 [G + 1] */
  fc_tensor table;           /* i32 [B, W] */
  fc_tensor lengths;         /* i32 [B] */
  fc_tensor out;             /* [B, Hq, D], out */
  fc_tensor lse;             /* f32 [B, Hq], out, or absent */
  double    scale;
} fc_prefix_attention;

/* Bytes of scratch a list of operators needs. */
int fc_operators_scratch_bytes(const fc_operator *ops, int32_t n, size_t *bytes);

/* Enqueue the operators in order on `hip_stream`. */
int fc_run_operators(const fc_operator *ops, int32_t n, void *scratch, size_t scratch_bytes, void *hip_stream);

/* The same in two halves, as fc_bind: *out is run by fc_run_bound and released by fc_unbind. */
int fc_bind_operators(const fc_operator *ops, int32_t n, void *scratch, size_t scratch_bytes, fc_bound **out);

/* Status of the device work enqueued so far by fc_run_* calls that used `scratch`.
 *
 * Kernels whose workgroups hand partial results to each other (the last stage of a fold,
 * the tiles of a single-pass scan, the teams of the column-blocked segmented fold; section
 * 2 asks of a fold or scan inside a cluster only that it is one pass, and names the chained
 * scan) never wait without bound: a workgroup polls for a word of another workgroup of its
 * launch at most a fixed number of times (about a second), then takes the operator's
 * identity in place of the missing value, sets word 1 of the control block at the start of
 * scratch (word 0 counts the launches that used the block) and goes on, so that no launch
 * can hang the device.  The results of such a launch are wrong.  It cannot happen while the
 * assumptions the kernels rest on hold (workgroups of a launch start in index order; the
 * device is not shared with work that holds compute units for seconds), and fc_run_* does
 * not look: it only enqueues.  A caller that wants the guarantee calls fc_check after the
 * calls whose results it is about to use.
 *
 * fc_check waits until the work enqueued on `hip_stream` has finished (it synchronises the
 * stream), reads the word, and returns FC_OK if it is zero.  Otherwise it clears the word
 * and returns FC_E_DEVICE_WAIT: every result produced with this scratch buffer since the
 * last check is to be discarded.  scratch: DEVICE, the buffer given to fc_run_*; NULL: the
 * buffer fc_run_fused_static uses on the current device.  Allocates nothing.
 * Errors: FC_E_SCRATCH (misaligned), FC_E_HIP. */
int fc_check(void *scratch, void *hip_stream);

/* Name of the kernel instance chosen for cluster `cluster` of the clustering
 * (p == NULL: the unfused clustering), for reports and profiles. */
int fc_cluster_kernel(const fc_graph *g, const fc_partition *p, int32_t cluster,
                      char *name, size_t capacity);

#define FC_SCRATCH_CONTROL_BYTES (1u << 23)

/* Message of the last error on the calling thread; valid until the next call. */
const char *fc_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FC_H */
