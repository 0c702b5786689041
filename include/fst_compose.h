/*
 * fst_compose.h -- C ABI of the MI355X (gfx950) eager transducer composition
 * library, libfstcompose.so.
 *
 * Operation (paper "Parallel Composition of Weighted Finite-State
 * Transducers", Section 3.1, Eq. (1) and Algorithm 1): given weighted
 * transducers A and B in the log semiring, build the trim composed transducer
 * C = A o B, which maps an input string x to an output string z with score
 * log-sum over y of exp(A(x, y) + B(y, z)).  Arcs of A are matched on their
 * output label and arcs of B on their input label.  Label 0 is epsilon.
 *
 * States of C are keys (qa, qb, f): a state of A, a state of B and one filter
 * bit.  From (qa, qb, f) there are three moves:
 *   matching move : arcs ea of qa, eb of qb with olabel(ea) = ilabel(eb) != 0
 *                   -> (dst(ea), dst(eb), 0); label ilabel(ea):olabel(eb);
 *                   weight = w(ea) + w(eb), one IEEE binary32 add (RNE)
 *   A-epsilon move: only when f = 0; arc ea with olabel(ea) = 0
 *                   -> (dst(ea), qb, 0); label ilabel(ea):0; weight w(ea)
 *   B-epsilon move: arc eb with ilabel(eb) = 0
 *                   -> (qa, dst(eb), epsOutA(qa)); label 0:olabel(eb); weight w(eb)
 * where epsOutA(q) says whether q has an out-arc with output label 0.  (The
 * filter bit keeps A's epsilon moves ahead of B's between two matching moves,
 * so each pair of paths of A and B maps to exactly one path of C.)  Start
 * keys are (sa, sb, 0) over start states of A and B.  A key accepts iff both
 * of its states accept.  C keeps only keys reachable from a start key that
 * can reach an accepting key (Section 3.1: the composed graph is trim).
 * Parallel arcs are kept; no weights are summed.
 *
 * Output is canonical and deterministic: states are numbered in ascending
 * key order (qa, qb, f); the arcs of a state are ordered by (l, a, b), where
 * l is the matched label (0 for epsilon moves), a and b are the arcs of A and
 * B the arc came from, and a missing arc sorts last.
 *
 * Graph layout (Section 3.2: structure of arrays, arcs consecutive by node,
 * offsets with V+1 entries).  All pointers passed to the library are DEVICE
 * pointers (hipMalloc or torch CUDA/HIP tensors) on the context's device.
 *
 * Errors: every entry point returns an int status (FST_OK = 0).  Nothing
 * aborts or throws across this interface.
 */
#ifndef FST_COMPOSE_H
#define FST_COMPOSE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__) || defined(__clang__)
#define FST_API __attribute__((visibility("default")))
#else
#define FST_API
#endif

#define FST_EPS 0

enum fst_status {
  FST_OK = 0,
  FST_ERR_INVALID_ARG = 1,   /* null pointer, negative size, bad option      */
  FST_ERR_INVALID_GRAPH = 2, /* input failed validation (see fst_graph)      */
  FST_ERR_TOO_LARGE = 3,     /* key space > 2^32 keys, or |C| > INT32_MAX    */
  FST_ERR_NOMEM = 4,         /* device allocation failed or over the cap     */
  FST_ERR_HIP = 5,           /* a HIP runtime call failed                    */
  FST_ERR_STATE = 6,         /* fill without a successful run               */
  FST_ERR_CYCLIC = 7,        /* fst_score on a graph with a cycle            */
  FST_ERR_NOT_CONVERGED = 8  /* fst_score_cyclic: sweeps did not settle      */
};

/* Read-only transducer view (device memory, caller-owned).
 *   num_states V >= 0, num_arcs E >= 0
 *   arc_offset[V+1]  arcs of state v are [arc_offset[v], arc_offset[v+1]);
 *                    arc_offset[0] = 0, arc_offset[V] = E, non-decreasing
 *   src[E], dst[E]   source / destination state; src consistent with offsets
 *   ilabel[E], olabel[E]  labels >= 0, 0 = epsilon
 *   weight[E]        binary32 log weights (any value, not checked)
 *   start[V], accept[V]   0 or 1; any number of start states
 * Every run validates these rules (unless FST_OPT_VALIDATE is 0) and
 * returns FST_ERR_INVALID_GRAPH on a violation.  Pointers may be NULL only
 * when the array is empty. */
typedef struct {
  int32_t num_states, num_arcs;
  const int32_t *arc_offset;
  const int32_t *src, *dst;
  const int32_t *ilabel, *olabel;
  const float *weight;
  const uint8_t *start, *accept;
} fst_graph;

/* Caller-allocated output arrays (device memory), sized from the V_C and
 * E_C that fst_compose_run reported.
 *   arc_offset[V_C+1]; src, dst, ilabel, olabel, weight [E_C];
 *   start, accept [V_C];
 *   key_a, key_b, key_f [V_C]  optional (NULL skips): the key of each state;
 *   arc_a, arc_b [E_C]         optional (NULL skips): provenance, the arc of
 *                              A / of B each arc of C came from, -1 if none. */
typedef struct {
  int32_t *arc_offset;
  int32_t *src, *dst, *ilabel, *olabel;
  float *weight;
  uint8_t *start, *accept;
  int32_t *key_a, *key_b;
  uint8_t *key_f;
  int32_t *arc_a, *arc_b;
} fst_graph_out;

/* Statistics of the last successful run. */
typedef struct {
  int64_t key_space;     /* key slots: V_A x 2^(b+1), b = max(4, bits(V_B-1)) */
  int64_t accessible;    /* keys reached from the start keys                 */
  int64_t coaccessible;  /* accessible keys that reach an accepting key = V_C */
  int64_t generated;     /* moves out of accessible keys; -1 unless
                            FST_OPT_COUNT_MOVES was set                      */
  int64_t fwd_levels;    /* frontier generations of the forward search       */
  int64_t bwd_levels;    /* frontier generations of the backward search      */
  int64_t heavy_states;  /* states of C handled one workgroup per state      */
  int64_t num_states;    /* V_C                                              */
  int64_t num_arcs;      /* E_C                                              */
  int64_t generated_backward; /* predecessor moves of the co-accessible keys
                            (each probed once by the backward search); -1
                            unless FST_OPT_COUNT_MOVES was set               */
} fst_stats;

typedef struct fst_ctx fst_ctx;

/* Create a context on HIP device `device`.  The context owns a device
 * workspace that grows on demand and is reused across calls.  A context is
 * not thread-safe: use one per host thread / stream.  *ctx is set on success. */
FST_API int fst_ctx_create(int device, fst_ctx **ctx);

/* Release the context and its workspace (NULL is allowed). */
FST_API void fst_ctx_destroy(fst_ctx *ctx);

/* Options: FST_OPT_MAX_WORKSPACE caps the workspace in bytes (0 = no cap;
 * exceeding it gives FST_ERR_NOMEM); FST_OPT_TIMING = 1 records per-phase
 * HIP events (read with fst_compose_phase_times).  Tuning knobs that never
 * change the result: FST_OPT_LABEL_BUCKETS (1 = default: per-state label
 * bucket tables for a graph whose table fits in 256 MiB and in 64 times its
 * arc records (8 bytes per arc); 0 = binary search only) and
 * FST_OPT_CHAIN_DEPTH (default 64: how many newly found keys one search
 * thread may expand depth-first before handing keys to the next frontier,
 * where B is mostly chains; 0 = a search by levels, as elsewhere,
 * whose deep searches go on inside a launch for 16 levels at most).  FST_OPT_COUNT_MOVES = 1 makes
 * each run also count the moves out of all accessible keys and the
 * predecessor moves of all co-accessible keys (extra passes, reported in
 * fst_stats.generated and fst_stats.generated_backward).
 * FST_OPT_ORDER picks the order of the two searches (the result is the same):
 * FST_ORDER_FORWARD_FIRST searches forward from the start keys,
 * then backward from the accepting keys it reached, inside the accessible
 * set; FST_ORDER_COACCESSIBLE_FIRST is Algorithm 1's order: the co-accessible
 * set over all key pairs first (backward from every accepting pair), then the
 * forward search inside it (fst_stats.accessible then counts only keys that
 * are also co-accessible); FST_ORDER_CONCURRENT (default) runs the forward
 * search's first generations alone, then, unless it has ended (then it goes
 * on as forward-first), a backward search from every accepting pair beside
 * the rest of it in the same kernels, restricted to accessible keys once
 * the forward search has ended and held back while its frontier is far
 * wider than the forward one (kernel FST_KERNEL_SEARCH_FORWARD then times
 * the launches that advance either search, and FST_KERNEL_SEARCH_BACKWARD
 * has none).  The concurrent order searches small operands in one launch:
 * up to 8,192 state pairs, 65,536 bits of V_A rounded up to 64 times V_B
 * rounded up to a power of two (16 at least) times 2, and 81,920 work units
 * over all pairs (epsilon arcs, and the other arcs of the side with fewer; 24
 * a pair and 4,096), unless B is mostly chains (most of its states have one
 * out-arc).  Where B is and every arc of A leads from a state to the next one
 * with an output other than epsilon, it follows 64 keys of a state of B at a
 * time (generations then advance both directions).
 * FST_OPT_VALIDATE (default 1) checks every input graph's
 * structure as described at fst_graph; 0 is for callers that vouch for
 * their graphs: the checks are skipped (the composition still reads the
 * largest label, the label order and the accepting states; a score reads
 * nothing before it starts), and a graph that breaks the rules then gives
 * unspecified results, which may include reads outside its arrays.
 * FST_OPT_LIST_CAPACITY (entries, 0 = default 2^22) is the first size of
 * the search's work lists (frontier and heavy keys); a search
 * that overflows them runs again with four times the size (never more than
 * 2 V_A V_B), and the context keeps the size that sufficed for later calls;
 * the result is the same. */
enum fst_option {
  FST_OPT_MAX_WORKSPACE = 1,
  FST_OPT_TIMING = 2,
  FST_OPT_LABEL_BUCKETS = 3,
  FST_OPT_CHAIN_DEPTH = 4,
  FST_OPT_COUNT_MOVES = 5,
  FST_OPT_ORDER = 6,
  FST_OPT_VALIDATE = 7,
  FST_OPT_LIST_CAPACITY = 8
};
enum fst_order {
  FST_ORDER_FORWARD_FIRST = 0,
  FST_ORDER_COACCESSIBLE_FIRST = 1,
  FST_ORDER_CONCURRENT = 2
};
FST_API int fst_ctx_set_option(fst_ctx *ctx, int option, int64_t value);

/* Phase 1 (Algorithm 1 up to the size of C): validate A and B, search the
 * state pairs reachable from the start keys, prune to co-accessible ones,
 * number the kept states and count their arcs.  Work is queued on `stream`
 * (a hipStream_t; NULL = default stream); the call blocks until the sizes are
 * known and stores them in *num_states (V_C) and *num_arcs (E_C).  A and B
 * must stay valid and unchanged until fst_compose_fill's work has completed.
 * An empty C (V_C = 0) is a valid result. */
FST_API int fst_compose_run(fst_ctx *ctx, const fst_graph *A, const fst_graph *B, void *stream,
                    int64_t *num_states, int64_t *num_arcs);

/* Phase 2 (Section 3.3, second pass): write C into caller-allocated arrays.
 * Asynchronous on `stream`; the caller synchronises before reading C. */
FST_API int fst_compose_fill(fst_ctx *ctx, const fst_graph_out *C, void *stream);

/* Statistics of the last successful fst_compose_run. */
FST_API int fst_compose_stats(const fst_ctx *ctx, fst_stats *out);

/* With FST_OPT_TIMING on, the device time in ms of each phase of the last
 * run + fill: [0] validate+preprocess, [1] forward search, [2] backward
 * search, [3] numbering + arc count, [4] fill.  Writes min(n, 5) values;
 * returns FST_ERR_STATE if timing was off. */
FST_API int fst_compose_phase_times(const fst_ctx *ctx, float *ms, int n);

/* Kernels timed with FST_OPT_TIMING on: every launch of the forward search
 * kernel; every launch of the backward search kernel; the arc-count kernels
 * (C's keys listed, states with few moves, states with many: 3 launches, 2
 * where the workspace has no room for the keys, the more where the call
 * queued a count for too few states and counted again, none for an empty C
 * whose number of states was waited for); the fill kernels (every state's
 * offset and flags with the arcs of light states, then heavy states' arcs if
 * any). */
enum fst_kernel {
  FST_KERNEL_SEARCH_FORWARD = 0,
  FST_KERNEL_SEARCH_BACKWARD = 1,
  FST_KERNEL_COUNT = 2,
  FST_KERNEL_FILL = 3,
  FST_KERNEL_SCORE_GEN = 4,   /* fst_score: generation kernels (one launch
                                 advances every direction asked for)       */
  FST_KERNEL_SCORE_PREP = 5,  /* fst_score: in-arc structure of the graph   */
  FST_KERNEL_SEARCH3 = 6,     /* fst_compose3_run: the level launches of the
                                 forward and backward searches             */
  FST_KERNEL_COMPACT3 = 7     /* fst_compose3_run + fill: in-arc grouping,
                                 trim keys, sort and numbering, arc count,
                                 fill                                      */
};

/* With FST_OPT_TIMING on: *ms = summed device time of the launches of
 * `kernel` in the last run + fill (kernels 0-3), the last fst_score
 * (kernels 4-5) or the last fst_compose3_run + fst_compose3_fill (kernels
 * 6-7), each bracketed by HIP events on the caller's stream, and
 * *launches = how many there were.  Returns FST_ERR_STATE if timing was off
 * or no such call was timed, FST_ERR_INVALID_ARG for an unknown kernel. */
FST_API int fst_compose_kernel_time(const fst_ctx *ctx, int kernel, float *ms, int64_t *launches);

/* ---- Scores of C and their gradient ------------------------------------
 * The log-semiring weight of C's paths (Eq. (1)) is what a training user
 * differentiates through (the introduction motivates eager composition by
 * automatic differentiation).  For an acyclic graph G (any fst_graph, e.g.
 * a composed C):
 *   alpha[v] = log-sum over paths from a start state to v of exp(weight),
 *              0 for a start state's empty path;
 *   beta[v]  = log-sum over paths from v to an accepting state;
 *   total    = log-sum over all paths from a start state to an accepting
 *              state (-inf if there is none); the weight of a path is the
 *              sum of its arc weights, and sums are float64.
 * Every log-sum is exact up to its final rounding and independent of the
 * order of its terms, so results are bitwise reproducible. */

/* Forward and backward scores of G (device arrays of V doubles; either may
 * be NULL to skip that direction) and the total (one device double, the
 * log-sum of alpha over accepting states when alpha is computed, else of
 * beta over start states).  G's structure is validated as in
 * fst_compose_run (labels are not read: scores do not depend on them).  Queued on
 * `stream`; blocks on small readbacks as the recursion advances.  Returns
 * FST_ERR_CYCLIC (outputs undefined) if G has a cycle (fst_score_cyclic
 * below takes such graphs).  Weights must be
 * finite (an infinite or NaN weight gives unspecified values, never a
 * fault).  G must stay valid until the work has completed. */
FST_API int fst_score(fst_ctx *ctx, const fst_graph *G, double *alpha, double *beta,
                      double *total, void *stream);

/* The same scores (alpha, beta, total: the sums over all paths) of a graph
 * that may have cycles, where a state can have infinitely many paths; the
 * sums are finite when the spectral radius of the matrix of arc
 * probabilities, M[u][v] = sum of exp(w(e)) over the arcs from u to v, is
 * below 1 over the states that lie on such paths (the Neumann series
 * sum_k M^k of the probability domain).  Shortest distance is among the
 * operations the paper leaves to future work (Section 5); here it is
 * relaxed by Jacobi sweeps of both recursions from every value at -inf:
 * sweep k gives each state the exact log-add of fst_score over the
 * previous sweep's values (its pull list's terms and its empty path), so
 * after k sweeps the values are the sums over the paths of at most k - 1
 * arcs, rising monotonically.  The sweeps stop at the first sweep in which
 * no value rose by more than `tol` (log domain, >= 0; 0 waits for a sweep
 * that changes no value upwards); *sweeps (if not NULL) receives its
 * number.  On a graph without cycles the sweeps reach fst_score's values
 * bit for bit after at most (longest path + 2) sweeps.  Each sweep reads
 * every state's in-arcs and out-arcs once (64 states per wavefront; where
 * those have more than 512 arcs, one thread per state), in batches of 16 to
 * 64 sweeps between read-backs (a quarter of the sweeps so far; sweeps
 * queued past the one that settled do nothing).  Arguments, validation and
 * outputs as in fst_score;
 * returns FST_ERR_NOT_CONVERGED (outputs: the last sweep's values) if no
 * sweep settled within max_sweeps (>= 0) sweeps, as when the sums diverge;
 * FST_ERR_INVALID_ARG for a negative max_sweeps or tol. */
FST_API int fst_score_cyclic(fst_ctx *ctx, const fst_graph *G, double *alpha, double *beta,
                             double *total, int32_t max_sweeps, double tol, int32_t *sweeps,
                             void *stream);

/* Arc posteriors times `scale`: grad[e] = scale * exp(alpha[src e] + w(e) +
 * beta[dst e] - *total), the derivative of scale * total by w(e) (0 for every
 * arc when *total is -inf).  alpha, beta, total come from fst_score or
 * fst_score_cyclic on the same G (with cycles, an arc's posterior is its
 * expected number of uses and can exceed 1); grad has E floats (device).
 * G is validated.  Asynchronous after the validation readback. */
FST_API int fst_score_posterior(fst_ctx *ctx, const fst_graph *G, const double *alpha,
                                const double *beta, const double *total, float scale,
                                float *grad, void *stream);

/* Gradient scatter through provenance: out[i] = sum of grad[e] over the
 * e < n with idx[e] = i (idx[e] = -1 is skipped), for i < m.  With idx =
 * C's arc_a (arc_b) and grad = the gradient of a loss by C's arc weights,
 * out is its gradient by the weights of A's (B's) arcs, since an arc of C
 * weighs w(a) + w(b).  Sums are exact to 2^-64 of the largest |grad| per
 * term, rounded once to float, so they do not depend on the order of
 * accumulation.  grad, idx: n entries; out: m floats (device).  Blocks until
 * done; returns FST_ERR_INVALID_ARG if an index lies outside [-1, m). */
FST_API int fst_grad_scatter(fst_ctx *ctx, int64_t n, const float *grad, const int32_t *idx,
                             int32_t m, float *out, void *stream);

/* Largest m (number of targets) that fst_grad_scatter_noalloc accepts. */
#define FST_SCATTER_NOALLOC_MAX_TARGETS (1 << 20)

/* fst_grad_scatter for callers that cannot allocate device memory (code
 * under HIP graph capture, serving loops that must not call hipMalloc,
 * harnesses that forbid it): same arguments and the same result, bit for
 * bit, but the call allocates nothing.  Its accumulators live in a fixed
 * device array of the library (32 bytes per target, for at most
 * FST_SCATTER_NOALLOC_MAX_TARGETS targets: 32 MiB plus a small header),
 * which every device the library runs on holds until the process ends; its
 * address is looked up once per device by fst_ctx_create.  The call clears
 * the part it uses before summing; the array keeps the last call's sums
 * afterwards.  All calls on one device share that one array, so calls that
 * overlap on a device (different streams or host threads without ordering)
 * race and give wrong sums: order them.  Returns FST_ERR_TOO_LARGE if m
 * exceeds the maximum, FST_ERR_INVALID_ARG for an index outside [-1, m) or
 * bad arguments.  Blocks until done (it reads back the bad-index flag into
 * the context's host memory, set up by fst_ctx_create). */
FST_API int fst_grad_scatter_noalloc(fst_ctx *ctx, int64_t n, const float *grad,
                                     const int32_t *idx, int32_t m, float *out, void *stream);

/* ---- Batches and chains ------------------------------------------------
 * Batch (the realistic workload of Section 4.2: the emission graphs of many
 * utterances composed with one lexicon): C_i = A_i o B for i < n in one
 * pass.  The A_i (host array of n device graphs) are composed as their
 * disjoint union; keys of different items never meet, and in the canonical
 * order (qa first) item i's states and arcs are the contiguous ranges
 * [item_states[i], item_states[i+1]) and [item_arcs[i], item_arcs[i+1]) of
 * the one C that fst_compose_fill then writes.  Ids in that C are those of
 * the union: subtract item_states[i] from src, dst (and item_arcs[i] from
 * arc_offset) for item-local values; key_a and arc_a index the union of the
 * A_i (subtract the states / arcs of the items before i).  item_states and
 * item_arcs are host arrays of n + 1 entries, filled on success (the last
 * entries are V_C and E_C).  Items are composed in parts: consecutive
 * items whose union fits the key space of one composition (an item that
 * does not fit alone gives FST_ERR_TOO_LARGE); most batches are one part,
 * one search.  With several parts the run searches each part in turn, and
 * fst_compose_fill searches every part but the last again before writing
 * it, so that fill blocks until done; the A_i and B must stay valid and
 * unchanged until the fill has completed (a part that comes out with other
 * sizes gives FST_ERR_STATE).  fst_compose_stats then reports sums over the
 * parts (levels: the largest).  V_C and E_C are at most INT32_MAX.
 * Chains (N-way composition): C has the input layout, so A o B o D is two
 * calls (compose, then compose C with D). */
FST_API int fst_compose_batch_run(fst_ctx *ctx, const fst_graph *A, int32_t n,
                                  const fst_graph *B, void *stream, int64_t *num_states,
                                  int64_t *num_arcs, int64_t *item_states,
                                  int64_t *item_arcs);

/* Per-item totals of a batch: totals[i] = log-sum of exp(val[v]) over the
 * v in [bounds[i], bounds[i+1]) with flag[v] != 0, for i < n (exact as in
 * fst_score; -inf for an empty set).  With val = alpha of the batch's C,
 * flag = its accept array and bounds = item_states, totals are the items'
 * forward scores.  val, flag, totals: device; bounds: host, n + 1
 * non-decreasing entries within the arrays.  Blocks until done. */
FST_API int fst_segment_logsum(fst_ctx *ctx, const double *val, const uint8_t *flag, int32_t n,
                               const int64_t *bounds, double *totals, void *stream);

/* ---- Three inputs at once ----------------------------------------------
 * N-way composition (Section 5 names composing N inputs at once, instead
 * of two, as the next step): C = A o B o D in one search, without building
 * A o B.  Eq. (1) read for three inputs: C maps x to w with score log-sum,
 * over all y and z, of exp(A(x, y) + B(y, z) + D(z, w)).  States of C are
 * keys (qa, qb, f1, qd, f2): (qa, qb, f1) is a state of T = A o B whose
 * arcs are the three moves of two-input composition (header comment above,
 * filter bit f1), and the key composes T with D by the same three rules,
 * filter bit f2:
 *   match  : a T-arc t with output z != 0, an arc ed of qd with ilabel z
 *            -> (dst t, dst ed, 0); label in(t):olabel(ed);
 *            weight w(t) + w(ed) (a T-match weighs w(ea) + w(eb), so the
 *            adds are (w(ea) + w(eb)) + w(ed), binary32, in that order)
 *   T alone: only when f2 = 0; a T-arc t with output 0 -> (dst t, qd, 0);
 *            label in(t):0; weight w(t)
 *   D alone: an arc ed of qd with ilabel 0 -> ((qa, qb, f1), dst ed,
 *            epsOutT(qa, qb, f1)); label 0:olabel(ed); weight w(ed)
 * where epsOutT says whether the T-state has a T-arc with output 0.  Start
 * keys are (sa, sb, 0, sd, 0); a key accepts iff its three states accept;
 * C is trim.  Output is canonical: states in ascending key order (qa, qb,
 * f1, qd, f2); the arcs of a state by (l, a, b, d), where l is the label
 * the arcs of A and B were matched on (0 when they were not both used) and
 * a, b, d are the arcs of A, B and D the arc came from, a missing arc
 * sorting last.  Key bits: bits(V_A - 1) +
 * bits(V_B - 1) + bits(V_D - 1) + 2 <= 62 (each at least 1), else
 * FST_ERR_TOO_LARGE.  The workspace grows with the number of keys reached
 * (a hash set of 8 bytes per slot, at most half full, grown and searched
 * again when it fills). */
typedef struct {
  int32_t *arc_offset;
  int32_t *src, *dst, *ilabel, *olabel;
  float *weight;
  uint8_t *start, *accept;
  int32_t *key_a, *key_b;   /* optional [V_C] (NULL skips): the key of     */
  uint8_t *key_fab;         /* each state, (key_a, key_b, key_fab, key_d,  */
  int32_t *key_d;           /* key_f) = (qa, qb, f1, qd, f2)               */
  uint8_t *key_f;
  int32_t *arc_a, *arc_b, *arc_d; /* optional [E_C] provenance, -1 = none  */
} fst_graph3_out;

/* Phase 1 of C = A o B o D: validate the three graphs, search forward from
 * the start keys and backward over the generated arcs, number the trim
 * keys and count their arcs.  Blocks until *num_states and *num_arcs are
 * known.  A, B and D must stay valid and unchanged until
 * fst_compose3_fill's work has completed. */
FST_API int fst_compose3_run(fst_ctx *ctx, const fst_graph *A, const fst_graph *B,
                             const fst_graph *D, void *stream, int64_t *num_states,
                             int64_t *num_arcs);

/* Phase 2: write C into caller-allocated arrays sized from phase 1
 * (asynchronous on `stream`). */
FST_API int fst_compose3_fill(fst_ctx *ctx, const fst_graph3_out *C, void *stream);

/* Statistics of the last successful fst_compose3_run: key_space = 2^(key
 * bits), accessible = keys reached, coaccessible = num_states = V_C,
 * generated = moves out of the accessible keys, fwd_levels and bwd_levels
 * = levels of the two searches, num_arcs = E_C, heavy_states = states of
 * C with more work units than one thread takes (one workgroup each in the
 * count and the fill), generated_backward -1. */
FST_API int fst_compose3_stats(const fst_ctx *ctx, fst_stats *out);

/* ---- Between a network and its graphs ----------------------------------
 * What a recogniser computes on the other side of the arc weights: a gated
 * recurrence over the frames, attention to earlier frames (norms and rotation
 * of queries and keys, linear attention with decays, attention to a window),
 * the weights of emission graphs by a linear layer and log-softmax, a cross
 * entropy over a vocabulary of words, and the gradients of all of these.
 *
 * Activations and weights are row-major matrices of one of three types,
 * with any row stride; the matrices of a call share one type.  Sums,
 * statistics of the softmax and states are float32 whatever the type;
 * results are rounded to their type once.  Results do not depend on anything but the
 * arguments (no atomic sums).  Calls are asynchronous on `stream` after a
 * call of the same sizes has made the workspace; they read nothing back, so
 * they can be captured into a HIP graph.  The workspace that a captured call
 * uses stays allocated until the context is destroyed, beside a larger one
 * that other calls may need (FST_OPT_MAX_WORKSPACE counts both): a graph may
 * be replayed as long as the context lives.  A replay uses the workspace as a
 * call does, so replays and calls of one context have to follow one another. */
enum fst_type { FST_F32 = 0, FST_F16 = 1, FST_BF16 = 2 };

/* Element (r, c) is data[r * stride + c] (device memory, caller-owned);
 * stride >= cols, in elements; data aligned to an element. */
typedef struct {
  void *data;
  int64_t rows, cols, stride;
  int32_t type; /* enum fst_type */
} fst_matrix;

/* Ragged sequences through a gated linear recurrence: sequence s is rows
 * [offset[s], offset[s+1]) of x and gate, channel by channel
 *   f_t = sigmoid(gate_t),  h_t = f_t h_(t-1) + (1 - f_t) x_t,  y_t = h_t
 * from h = state[s] (0 where state is NULL), the first row first, or the last
 * row first if `reverse` is not 0.
 *   offset[num_seqs + 1]  device; 0, non-decreasing, ending with x.rows.
 *                         Other offsets give unspecified results, and rows
 *                         of no sequence are left as they are; no access
 *                         leaves the matrices.  A sequence may be empty.
 *   state[num_seqs * x.cols]  device, float32, or NULL
 * num_seqs is at most FST_RECURRENCE_MAX_SEQS; past 65,535 x 64 columns calls
 * give FST_ERR_TOO_LARGE (16-bit rows read two columns at a time: twice that). */
typedef struct {
  int32_t num_seqs;
  const int32_t *offset;
  int32_t reverse;
  fst_matrix x, gate;
  const float *state;
} fst_recurrence;

#define FST_RECURRENCE_MAX_SEQS (1 << 22)
#define FST_RECURRENCE_SAVE_ROWS 64

/* y (as x), last[num_seqs * x.cols] (float32, optional): the state after each
 * sequence (state[s], or 0, after an empty one).  No output may overlap an input
 * (`last` not `state` either: a long sequence is read by several workgroups) or
 * another output.  saved (float32, optional), for fst_recurrence_grads:
 * (x.rows / FST_RECURRENCE_SAVE_ROWS + num_seqs) * x.cols values, the states
 * entering every 64 steps of a sequence; rows of `saved` that stand for no
 * step are left as they are. */
FST_API int fst_recurrence_run(fst_ctx *ctx, const fst_recurrence *R, const fst_matrix *y,
                               float *last, float *saved, void *stream);

/* Gradients of a loss by x, gate and state, from its gradients by y (grad_y)
 * and by `last` (grad_last, float32, NULL = 0), with `saved` of the run on the
 * same R:
 *   D_t = grad_y_t + f_(t+1) D_(t+1)   (and grad_last at the last step)
 *   grad_x_t = (1 - f_t) D_t
 *   grad_gate_t = D_t (h_(t-1) - x_t) f_t (1 - f_t)
 *   grad_state = f_0 D_0 (grad_last for an empty sequence)
 * grad_state (float32, num_seqs * x.cols) is optional.  No output may overlap
 * an input or another output. */
FST_API int fst_recurrence_grads(fst_ctx *ctx, const fst_recurrence *R, const float *saved,
                                 const fst_matrix *grad_y, const float *grad_last,
                                 const fst_matrix *grad_x, const fst_matrix *grad_gate,
                                 float *grad_state, void *stream);

/* One step of many streams: row i of x, gate and y is a stream whose state
 * is row slot[i] of state_in and state_out (device, float32, num_slots *
 * x.cols; slot NULL: row i, num_slots >= x.rows).  A slot outside [0,
 * num_slots) marks an idle row: its y is 0 and no state is read or written.
 * Rows of state_out that no row of x names are left as they are.  state_out
 * may be state_in; slots of one call must differ. */
FST_API int fst_recurrence_step(fst_ctx *ctx, const fst_matrix *x, const fst_matrix *gate,
                                const float *state_in, float *state_out, const int32_t *slot,
                                int32_t num_slots, const fst_matrix *y, void *stream);

/* ---- Attention over frames ---------------------------------------------
 * Queries, keys and values are matrices whose row t holds a frame's heads side
 * by side, each of the same number of columns; matrices may be parts of wider
 * ones (one product's queries, keys and values side by side).  Sequences are
 * the rows [offset[s], offset[s+1]), offsets as in fst_recurrence.  No output
 * may overlap an input or another output, but for the caches of
 * fst_window_attention_step and state_out of fst_linear_attention_step.
 * No results, gradients or states of rows depend on rows that they do not see:
 * where those hold infinities or NaN, sums that these would make no number of are
 * taken again without them (slowly, and rounded in another order).  Infinities and
 * NaN in rows that they do see make infinities or NaN of them where the formulas do. */
#define FST_NORM_MAX_WIDTH 512      /* columns of a head of fst_head_norms     */
#define FST_ATTENTION_MAX_WIDTH 128 /* of the attentions (FST_ERR_TOO_LARGE,   */
                                    /* which more than 16,383 heads, rows more */
                                    /* than 2^22 numbers apart and steps of    */
                                    /* more than 2^23 rows may give as well)   */

/* Queries and keys normalised head by head, scaled, and rotated by position.
 * For each head x of a row, of `width` columns, with one of the two weights
 * (float32, width; queries' and keys' own):
 *   z = x / sqrt(mean of x^2 + eps) * weight
 * then the first 2 * num_freq columns are num_freq pairs, each turned by the
 * angle pos[row] * freq[i]:  (a, b) -> (a cos - b sin, b cos + a sin).  Pair i is
 * columns i and num_freq + i, or, with `pairs` not 0, columns 2 i and 2 i + 1.
 * Angles are taken in 64 bits: any position keeps float32's precision.  So do heads
 * whose squares are past float32's largest number, or (with such an eps) its smallest.
 *   q, k      q.cols and k.cols are multiples of width; k may be without columns
 *             (more than 2^31 - 65 heads together give FST_ERR_TOO_LARGE)
 *   freq      device, float32, num_freq <= width / 2; NULL if num_freq is 0
 *   pos       device, q.rows; NULL if num_freq is 0
 * eps is finite and not negative. */
typedef struct {
  fst_matrix q, k;
  int32_t width;
  const float *q_weight, *k_weight;
  const float *freq;
  int32_t num_freq;
  const int32_t *pos;
  int32_t pairs;
  float eps;
} fst_head_norms;

/* y_q, y_k: as q and k. */
FST_API int fst_head_norms_run(fst_ctx *ctx, const fst_head_norms *A, const fst_matrix *y_q,
                               const fst_matrix *y_k, void *stream);

/* Gradients of a loss by q, k (grad_q, grad_k: as q and k) and the weights
 * (float32, width, each optional) from those by y_q and y_k (grad_yq, grad_yk). */
FST_API int fst_head_norms_grads(fst_ctx *ctx, const fst_head_norms *A,
                                 const fst_matrix *grad_yq, const fst_matrix *grad_yk,
                                 const fst_matrix *grad_q, const fst_matrix *grad_k,
                                 float *grad_q_weight, float *grad_k_weight, void *stream);

/* Linear attention with a decay for each head: with K = q.cols / heads and
 * V = v.cols / heads columns of a head, head by head
 *   S_t = e^(log_decay) S_(t-1) + k_t v_t^T,   y_t = scale S_t^T q_t
 * from S = state[s] (num_seqs * heads * K * V float32 values, row-major; 0 where
 * state is NULL), the first row of a sequence first, or the last if `reverse` is
 * not 0.  log_decay (device, float32, heads) holds constants of the layer: no
 * gradient is taken by them.  They are meant to be <= 0; -inf keeps nothing.
 * With 16-bit matrices each score q_t . k_j of rows up to 63 apart, times its decay,
 * and each number of the state that meets q is rounded to the matrices' type
 * (float16: scaled by a power of two first) before it is multiplied; states
 * themselves and `last` are float32 sums. */
typedef struct {
  int32_t num_seqs;
  const int32_t *offset;
  int32_t reverse;
  int32_t heads;
  const float *log_decay;
  float scale;
  fst_matrix q, k, v;
  const float *state;
} fst_linear_attention;

/* y: as v.  last (float32, as state, optional): the state after each sequence
 * (state[s], or 0, after an empty one). */
FST_API int fst_linear_attention_run(fst_ctx *ctx, const fst_linear_attention *A,
                                     const fst_matrix *y, float *last, void *stream);

/* Gradients of a loss by q, k, v (as these) and state (float32, optional) from
 * those by y (grad_y) and `last` (grad_last, NULL = 0).  With D_t the gradient by
 * S_t, from the last row back:
 *   D_t = scale q_t dy_t^T + e^(log_decay) D_(t+1)   (and grad_last at the last row)
 *   dq_t = scale S_t dy_t,  dk_t = D_t v_t,  dv_t = D_t^T k_t,
 *   grad_state = e^(log_decay) D_0   (grad_last for an empty sequence) */
FST_API int fst_linear_attention_grads(fst_ctx *ctx, const fst_linear_attention *A,
                                       const fst_matrix *grad_y, const float *grad_last,
                                       const fst_matrix *grad_q, const fst_matrix *grad_k,
                                       const fst_matrix *grad_v, float *grad_state,
                                       void *stream);

/* One step of many streams: row i of q, k, v and y is a stream whose state is
 * slot[i] of state_in and state_out (num_slots of heads * K * V values; slot and
 * num_slots as in fst_recurrence_step).  state_out may be state_in. */
FST_API int fst_linear_attention_step(fst_ctx *ctx, const fst_matrix *q, const fst_matrix *k,
                                      const fst_matrix *v, int32_t heads, const float *log_decay,
                                      float scale, const float *state_in, float *state_out,
                                      const int32_t *slot, int32_t num_slots,
                                      const fst_matrix *y, void *stream);

/* Attention to a window and a sequence's first frames: frame t sees frame s <= t
 * of its sequence if t - s < window or s < sinks, and with z = scale q_t . k_s
 *   lse_t = log sum over s of e^z,   y_t = sum over s of e^(z - lse_t) v_s.
 * q has `heads` heads, k and v have kv_heads, each shared by heads / kv_heads
 * consecutive heads of q; all heads have the same number of columns.  window >= 1
 * (one as long as the sequences: all earlier frames), sinks >= 0, their sum at
 * most 2^31 - 1; blocks of 128 rows and sequences together more than 2^23 give
 * FST_ERR_TOO_LARGE.  With 16-bit matrices e^(z - maximum), and for the gradients
 * e^(z - lse) and the gradient of z, are rounded to the matrices' type (float16: scaled
 * by powers of two first) before they are multiplied. */
typedef struct {
  int32_t num_seqs;
  const int32_t *offset;
  int32_t heads, kv_heads;
  int32_t window, sinks;
  float scale;
  fst_matrix q, k, v;
} fst_window_attention;

/* y: as q; lse: float32, q.rows * heads. */
FST_API int fst_window_attention_run(fst_ctx *ctx, const fst_window_attention *A,
                                     const fst_matrix *y, float *lse, void *stream);

/* Gradients of a loss by q, k and v (as these) from that by y (grad_y), with y
 * and lse of the run on the same A. */
FST_API int fst_window_attention_grads(fst_ctx *ctx, const fst_window_attention *A,
                                       const fst_matrix *y, const float *lse,
                                       const fst_matrix *grad_y, const fst_matrix *grad_q,
                                       const fst_matrix *grad_k, const fst_matrix *grad_v,
                                       void *stream);

/* One step of many streams.  A stream's keys and values lie in the rows
 * [slot * L, (slot + 1) * L) of k_cache and v_cache, L = sinks + window: the frame
 * of position p in row p of these if p < sinks, else in row sinks + (p - sinks) %
 * window.  Row i of q, k and v is the frame of position pos[i] of stream slot[i]
 * (slot NULL: stream i): its k and v are written to the caches, and y is its
 * attention to what the caches then hold, the frames of positions 0 .. pos[i] that
 * it sees.  k_cache and v_cache have num_slots * L rows (L past 2^31 - 257 gives
 * FST_ERR_TOO_LARGE).  A slot outside
 * [0, num_slots) or a negative position marks an idle row: its y is 0, no cache is
 * read or written.  Slots of one call must differ. */
FST_API int fst_window_attention_step(fst_ctx *ctx, const fst_matrix *q, const fst_matrix *k,
                                      const fst_matrix *v, int32_t heads, int32_t kv_heads,
                                      int32_t window, int32_t sinks, float scale,
                                      const int32_t *pos, const int32_t *slot,
                                      int32_t num_slots, const fst_matrix *k_cache,
                                      const fst_matrix *v_cache, const fst_matrix *y,
                                      void *stream);

/* Fills the caches of fst_window_attention_step with whole sequences, that of
 * sequence s in stream slot[s] (NULL: s; outside [0, num_slots): left out; all others of
 * a call must differ), so that the next frame's position is its length.  Rows that no
 * frame belongs in are left as they are.  k and v have the caches' columns; window and
 * sinks are theirs. */
FST_API int fst_window_attention_fill(fst_ctx *ctx, int32_t num_seqs, const int32_t *offset,
                                      const fst_matrix *k, const fst_matrix *v, int32_t window,
                                      int32_t sinks, const int32_t *slot, int32_t num_slots,
                                      const fst_matrix *k_cache, const fst_matrix *v_cache,
                                      void *stream);

/* Heads take at most FST_HEAD_MAX_ROWS rows of x and of w, and
 * FST_HEAD_MAX_COLS columns and classes of an emission (FST_ERR_TOO_LARGE, which
 * 2^37 scores and more in one call may give as well: a launch's limit).
 * None of their outputs may overlap an input or another output.  Matrices
 * whose rows do not begin at multiples of 16 bytes, or whose width is not a
 * multiple of 64 (float32: 32), are copied into the workspace first. */
#define FST_HEAD_MAX_ROWS (1 << 25)
#define FST_HEAD_MAX_COLS (1 << 22)

/* Weights of emission graphs: weight[n * C + c] = z[n][c] - log-sum over c'
 * of exp(z[n][c']), z = x w^T, for the N rows of x (frames, of any number of
 * utterances) and the C rows of w (tokens), C >= 1 unless N is 0.  weight
 * (device, float32, N * C) is the weight array of the graph whose state n
 * has the C arcs [n C, (n + 1) C), or of several such graphs in a row.  A
 * row whose scores hold a NaN comes out NaN; scores of -inf weigh -inf. */
FST_API int fst_emission_weights(fst_ctx *ctx, const fst_matrix *x, const fst_matrix *w,
                                 float *weight, void *stream);

/* Gradients of a loss by x and w (each optional, not both) from its gradient
 * by the weights (float32, N * C; e.g. what fst_grad_scatter returns), with
 * the weights of fst_emission_weights on the same x and w:
 *   dz = grad - exp(weight) * (sum of grad over the row)
 *   grad_x = dz w,  grad_w = dz^T x
 * For the two products dz is rounded to the matrices' type (float16: scaled by a
 * power of two first, so that the smallest keep their digits): a gradient is off
 * by half a spacing of the type, at most, of the sizes of the terms that it sums.
 * Up to 2^28 products N C H dz is kept as two such numbers, which lose next to
 * nothing. */
FST_API int fst_emission_grads(fst_ctx *ctx, const fst_matrix *x, const fst_matrix *w,
                               const float *weight, const float *grad,
                               const fst_matrix *grad_x, const fst_matrix *grad_w,
                               void *stream);

/* Cross entropy over the V rows of w (words): with z = x w^T and
 * lse[n] = log-sum over v of exp(z[n][v]), loss[n] = lse[n] -
 * z[n][target[n]], or 0 where target[n] is -1 (no word).  Any other target
 * outside [0, V) gives a loss of NaN.  The scores z are not stored.
 * target: device, N; loss, lse: device, float32, N.  V >= 1 unless N is 0. */
FST_API int fst_cross_entropy(fst_ctx *ctx, const fst_matrix *x, const fst_matrix *w,
                              const int32_t *target, float *loss, float *lse, void *stream);

/* Gradients of the sum over n of grad[n] * loss[n] by x and w (each optional,
 * not both), with lse of fst_cross_entropy on the same x, w and target
 * (grad: device, float32, N, or NULL for 1):
 *   dz = grad[n] (exp(z - lse[n]) - [v = target[n]])  (0 for no word)
 *   grad_x = dz w,  grad_w = dz^T x
 * z is computed again, for a piece of the vocabulary at a time whose dz (rounded
 * as above) takes 512 MiB of workspace at most (more only where 256 words take
 * more).  The pieces depend on the sizes alone: a cap of the workspace that has
 * no room for one refuses the call.  A row without a word has dz = 0, whatever
 * its scores; its x still meets that 0 in grad_w, so it has to be finite there. */
FST_API int fst_cross_entropy_grads(fst_ctx *ctx, const fst_matrix *x, const fst_matrix *w,
                                    const int32_t *target, const float *lse, const float *grad,
                                    const fst_matrix *grad_x, const fst_matrix *grad_w,
                                    void *stream);

/* Static string for a status code. */
FST_API const char *fst_strerror(int code);

#ifdef __cplusplus
}
#endif

#endif /* FST_COMPOSE_H */
