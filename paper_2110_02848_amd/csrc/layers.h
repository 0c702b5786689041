// Declarations of the operators between a network and its graphs: the gated
// recurrence (recurrence.hip), the heads, emission weights and the cross
// entropy over a vocabulary (head.hip), and attention layers: norms of queries
// and keys with their rotation (norms.hip), linear attention (linear.hip) and
// attention to a window (window.hip).
#pragma once

#include "internal.h"

namespace fstc {

// A row-major view of caller memory: element (r, c) at data[r * stride + c].
struct Mat {
  void *data;
  long long rows, cols, stride;
  int type;  // enum fst_type
};

inline size_t type_bytes(int type) { return type == FST_F32 ? 4 : 2; }

// ---- recurrence ----------------------------------------------------------

struct RecArgs {
  const void *x, *u, *gy;        // [N, D] inputs, gate, gradient of y
  void *y, *gx, *gu;             // [N, D] outputs
  long long xs, us, ys, gys, gxs, gus;  // their strides
  const float *state;            // [n, D] or null
  float *last;                   // [n, D] or null
  float *saved;                  // [N / REC_SAVE + n, D]: states entering each 64 steps
  const float *glast;            // [n, D] or null
  float *gstate;                 // [n, D] or null
  const int32_t *off;            // [n + 1]
  float2 *agg;                   // split form: maps of the units, [N / unit + n, D]
  long long N, unit;             // rows; steps of a unit, 0: not split
  int n, D, reverse;
};

constexpr int REC_SAVE = 64;  // scan steps between saved states
static_assert(REC_SAVE == FST_RECURRENCE_SAVE_ROWS, "the header's constant");

// Called twice, as the heads below: first without workspace for its bytes.
hipError_t launch_recurrence(RecArgs a, int type, void *ws, size_t *need, hipStream_t s);
hipError_t launch_recurrence_grads(RecArgs a, int type, void *ws, size_t *need, hipStream_t s);

struct StepArgs {
  const void *x, *u;
  void *y;
  long long xs, us, ys;
  const float *in;
  float *out;
  const int32_t *slot;  // row of the states, or null: row i
  long long n;
  int D, slots;
};
hipError_t launch_recurrence_step(const StepArgs &a, int type, hipStream_t s);

// ---- heads ---------------------------------------------------------------

// An operand of the products, element (r, k) of `rows` by `depth`: at
// p[r * ld + k], or at p[k * ld + r] where it is read column by column.  Rows
// of memory begin at multiples of 16 bytes, whole groups of them.  From step
// `wrap` of the sum on, k starts over, `jump` bytes further on.
struct Operand {
  const void *p;
  long long ld;
  long long rows, depth;
  int wrap = INT32_MAX;
  long long jump = 0;
};

// Each is called twice: without workspace (ws null) it only says how many
// bytes it needs, with it it queues the work.
hipError_t launch_emission(const Mat &x, const Mat &w, float *weight, void *ws, size_t *need,
                           hipStream_t s);
hipError_t launch_emission_grads(const Mat &x, const Mat &w, const float *weight,
                                 const float *grad, const Mat *gx, const Mat *gw, void *ws,
                                 size_t *need, hipStream_t s);
hipError_t launch_loss(const Mat &x, const Mat &w, const int32_t *target, float *loss, float *lse,
                       void *ws, size_t *need, hipStream_t s);
hipError_t launch_loss_grads(const Mat &x, const Mat &w, const int32_t *target, const float *lse,
                             const float *grad, const Mat *gx, const Mat *gw, void *ws,
                             size_t *need, hipStream_t s);

// ---- norms of queries and keys, rotated ----------------------------------

struct NormSide {          // queries or keys
  const void *x, *g;       // [N, heads * D]: input, gradient of the result
  void *y;                 // [N, heads * D]: result, or gradient of x
  long long xs, gs, ys;
  const float *w;          // [D]
  float *gw;               // [D]: gradient of w
  int heads;
};
struct NormArgs {
  NormSide side[2];
  const float *freq;       // [P]
  const int32_t *pos;      // [N]
  float *part;             // gradients: a workgroup's sums for each side's w
  long long N;
  int D, P, pairs;
  float eps;
};
hipError_t launch_norms(const NormArgs &a, int type, hipStream_t s);
hipError_t launch_norms_grads(NormArgs a, int type, void *ws, size_t *need, hipStream_t s);

// ---- linear attention ----------------------------------------------------

struct LinCall {
  const void *q, *k, *v;         // [N, H K], [N, H K], [N, H V]
  void *y;                       // [N, H V]: result, or its gradient
  void *gq, *gk, *gv;            // gradients
  long long qs, ks, vs, ys, gqs, gks, gvs;
  const float *state, *glast;    // [n, H, K, V] or null
  float *last, *gstate;          // [n, H, K, V] or null
  const int32_t *off;            // [n + 1]
  const float *log_decay;        // [H]
  long long N;
  int n, H, K, V, reverse;
  float scale;
};
hipError_t launch_linear(const LinCall &c, int type, void *ws, size_t *need, hipStream_t s);
hipError_t launch_linear_grads(const LinCall &c, int type, void *ws, size_t *need,
                               hipStream_t s);

// One pass over rows, in their order or (reverse) from the last one back:
//   y_i = so (sum over rows j up to i of e^(g (i - j)) (q_i . k_j) v_j) + ss X_i^T q_i
// with X_0 = state and X_(i+1) = e^g X_i + sk k_i v_i^T, of which y_i takes e^g X_i;
// `back`: X_(i+1) = e^g (X_i + sk k_i v_i^T), of which y_i takes X_i itself.
struct LinJob {
  const void *q, *k, *v;
  void *o;
  long long qs, ks, vs, os;
  int A, B;                  // widths of q and k, of v and o
  const float *state;        // first state, or null: 0
  float *last;               // last state, or null
  long long sa, sb;          // element (a, b) of a head's state at a sa + b sb
  float *units;              // split form: states entering the units
  float so, ss, sk;
  int reverse, back;
};
struct LinArgs {
  LinJob job[3];
  const int32_t *off;
  const float *log_decay;
  long long N, unit;         // rows; steps of a unit, 0: not split
  int n, H, slices;          // slices of a head's columns of v
};
struct LinStepArgs {
  const void *q, *k, *v;
  void *y;
  long long qs, ks, vs, ys;
  const float *log_decay, *in;
  float *out;
  const int32_t *slot;       // row of the states, or null: row i
  long long n;
  int H, A, B, slots;
  float scale;
};
hipError_t launch_linear_step(const LinStepArgs &a, int type, hipStream_t s);

// ---- attention to a window -----------------------------------------------

struct WinArgs {
  const void *q, *k, *v, *y, *gy;   // y, gy: gradients only
  void *o;                          // result
  void *gq, *gk, *gv;
  long long qs, ks, vs, ys, gys, os, gqs, gks, gvs;
  float *lse;                       // [N, H]
  const int32_t *off;               // [n + 1]
  long long N;
  int n, H, G, D, window, sinks;
  float scale;
  long long unit;                   // queries of a unit.  (Here: beside `scale`, delta would
                                    // come to k_window_back by way of scratch memory)
  // workspace of the gradients
  float *delta;                     // [N, H]
  float *own, *part;                // sums for gk and gv of cut sequences' first frames:
                                    // their blocks' own, and units' (or null)
};
hipError_t launch_window(const WinArgs &a, int type, hipStream_t s);
hipError_t launch_window_grads(WinArgs a, int type, void *ws, size_t *need, hipStream_t s);

struct WinStepArgs {
  const void *q, *k, *v;
  void *y, *kc, *vc;                // caches: slots * (sinks + window) rows
  long long qs, ks, vs, ys, kcs, vcs;
  const int32_t *pos, *slot;        // [n]; slot may be null: row i
  long long n;
  int H, G, D, window, sinks, slots;
  float scale;
  float *part;                      // splits' results
  int splits;
};
hipError_t launch_window_step(WinStepArgs a, int type, void *ws, size_t *need, hipStream_t s);

struct WinFillArgs {
  const void *k, *v;
  void *kc, *vc;
  long long ks, vs, kcs, vcs;
  const int32_t *off, *slot;
  long long N;
  int n, first, width, window, sinks, slots;
};
hipError_t launch_window_fill(const WinFillArgs &a, int type, hipStream_t s);

}  // namespace fstc
