// Declarations of the operators between a network and its graphs: the gated
// recurrence (recurrence.hip) and the heads, emission weights and the cross
// entropy over a vocabulary (head.hip).
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

}  // namespace fstc
