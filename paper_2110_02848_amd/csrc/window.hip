// Attention to a window of frames and a sequence's first ones
// (fst_window_attention_run, its gradients, its single step and the filling of
// its caches).
//
// Frame t of a sequence sees frame s <= t if t - s < window or s < sinks:
//   z = scale q_t . k_s,  y_t = sum of e^(z - lse_t) v_s,  lse_t = log sum of e^z
// in one pass over the frames that a block of queries sees, with the running
// maximum and sum of the softmax.  Scores are products of (k rows) x (q columns),
// whose results are an operand of the product with v in the registers that they
// are in, and whose statistics are a lane's own.  Exponentials are powers of 2.
//
// Back, with P = e^(z - lse) and delta_t = y_t . dy_t:
//   dS = P (dy v^T - delta),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dy
// from scores that are computed again, once by queries (dq) and once by keys (dk, dv),
// so that every sum has one owner and one order.  First frames are seen by all
// later queries: in long sequences, units of queries sum what lies outside the
// window, and k_window_first adds the units.  All three are workgroups of one launch,
// the long ones first, so that none waits for another's last.
#include <initializer_list>

#include "sequences.h"
#include "tiles.h"

namespace fstc {

using namespace tile;

namespace {

constexpr int WNT = 256;             // threads
constexpr int WNW = WNT / WAVE;
constexpr int KEYS = 64;             // of a tile of keys
constexpr int QUERIES = 32;          // of a tile of queries
// Tiles of 16 queries (or keys) of a wavefront.  Two read half as much of LDS for a
// product; float32's products take eight times as long, and one leaves it more
// workgroups (6 x 211 x 6 heads of 43, gradients: 146 us with two).
template <typename T>
constexpr int QT_OF = sizeof(T) == 2 ? 2 : 1;
template <typename T>
constexpr int BLOCK_OF = 16 * QT_OF<T> * WNW;  // queries, or keys, of a workgroup
constexpr int FEW = 64;              // frames
// First frames whose queries are cut into units, at most.  A unit takes workspace and
// time for each of them, an uncut sequence walks all its queries for a block of them.
// Gradients, cut and uncut, 64, 256 and 512 of them: 16 x 2,000 x 16 + 4 x 128 bf16, window
// 1,000: 1,068 and 1,083, 1,366 and 1,116, 1,759 and 1,187 us; 64 x 500 x 8 x 64, window
// 100: 201 and 190, 286 and 211, 380 and 216; 1 x 20,000 x 8 + 2 x 64, window 256: 186 and
// 4,925, 280 and 4,867, 409 and 4,836.  (Past it the long sequence would still gain.)
constexpr int MAX_CUT = 256;
constexpr float LOG2 = 0.69314718055994530942f, LOG2E = 1.44269502162933349609375f;

// Wavefronts of a SIMD, at least, of the kernels below.  Two have half of its
// registers each, all of them ones that the vector units can add and multiply in;
// float32's operands take twice the room.
template <typename T>
constexpr int MIN_WAVES = sizeof(T) == 2 ? 2 : 1;

// float16: dS is multiplied times a power of two (tiles.h) of the result that it is
// summed into, a query's dq or a key's dk.
template <typename T>
constexpr bool SCALED = std::is_same<T, f16>::value;

// float16: log 2 of what exponentials are multiplied by.  They are at most 1 (P, but for
// lse's rounding) or 2^LATE (where the sums' maximum lags), and those of frames seen
// faintly, or among many, below 2^-14, where float16 loses digits.
template <typename T>
constexpr float RAISE = SCALED<T> ? 12.0f : 0.0f;
template <typename T>
constexpr float RAISED = SCALED<T> ? 0x1p12f : 1.0f;
template <typename T>
constexpr float LATE = SCALED<T> ? 3.0f : 8.0f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int N, int M>
__device__ __forceinline__ bool finite(const float4v (&x)[N][M]) {
  float z = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < M; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) z = fmaf(x[i][j][r], 0.0f, z);
  return __all(z == 0.0f);
}

// Sum of a[i] b[i], i < D.
template <typename T>
__device__ __forceinline__ float dot(const T *a, const T *b, int D) {
  float x = 0.0f;
  for (int i = 0; i < D; ++i) x = fmaf((float)a[i], (float)b[i], x);
  return x;
}

// Whether query t sees no frame but itself: then dS is 0, or no number where one of its
// factors is none, and no difference of two sums.
__device__ __forceinline__ bool sees_one(long long t, int window, int sinks) {
  return t == 0 || (window == 1 && sinks == 0);
}

// The frames that queries [lo, hi) of a sequence see: sinks [0, sinks), before
// the window of any of them, then [first, hi).
struct Seen {
  long long first;
  int sinks, sink_tiles, tiles;
};
__device__ __forceinline__ Seen seen_by(long long lo, long long hi, int window, int sinks) {
  Seen s;
  s.first = lo - window + 1 > 0 ? lo - window + 1 : 0;
  s.sinks = (int)(sinks < s.first ? sinks : s.first);
  s.sink_tiles = (s.sinks + KEYS - 1) / KEYS;
  s.tiles = s.sink_tiles + (int)((hi - s.first + KEYS - 1) / KEYS);
  return s;
}

// Of a tile of keys from s0 on, which of a lane's (s0 + 4 lg + at, at = 16 kt + r)
// query t sees: at <= last, and at >= from or at < upto.  A tile that no query has
// the near, or the far, end of its frames in needs no such choice.
struct Edge {
  int last, from, upto;
  bool near, far;
};
__device__ __forceinline__ int within_tile(long long x) {
  int y = (int)(x < -KEYS ? -KEYS : x > KEYS ? KEYS : x);
  // (as it is: comparisons with it would be made with x, in 64 bits, and the choices
  // for tiles at an edge for all of them)
  asm volatile("" : "+v"(y));
  return y;
}
__device__ __forceinline__ Edge edge_of(const WinArgs &a, const Seen &sn, bool sink, long long s0,
                                        long long t, int lg) {
  Edge e;
  const long long at0 = s0 + 4 * lg;
  e.last = sink ? KEYS : within_tile(t - at0);
  e.from = sink ? KEYS : within_tile(t - a.window + 1 - at0);
  e.upto = within_tile((sink ? sn.sinks : a.sinks) - at0);
  e.near = __any(e.last < KEYS);
  e.far = __any(e.from > 0);
  return e;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// A query row against the frames that it sees alone, term by term, for four columns
// from d0 on.  The products also take the others' v, times 0, which makes no number
// of an infinity or a NaN that the query does not see: where a result is none, it
// is taken again.  The same below for the gradients.  (Behind the results' stores:
// registers that had to hold results across these calls would be missing in the
// products.)
template <typename T>
__device__ __noinline__ float4v exact_row(const T *q, const T *k, long long ks, const T *v,
                                          long long vs, int D, long long t, int window,
                                          int sinks, float c, float m, int d0) {
  float4v x{};
  for (long long s = 0; s <= t; ++s) {
    if (t - s >= window && s >= sinks) {
      s = t - window;
      continue;
    }
    const float p = exp2_of(dot(q, k + s * ks, D) * c - m);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      x[r] = fmaf(p, d0 + r < D ? (float)v[s * vs + d0 + r] : p, x[r]);
    if (all_nan(x)) break;  // (and so they stay)
  }
  return x;
}

// Tiles of 64 keys come to two pairs of buffers in turn, the next one's loads under
// way while one is multiplied.  m is the maximum that exponents are taken from: it
// follows a row's maximum only once that is past it by LATE (powers of 2), so that
// most tiles leave the sums as they are; p stays below 2^LATE, times 2^RAISE.
//
// Bound by the vector units: a wavefront takes 2,910 of their instructions for up to 11
// tiles, and a tile's 32 exponentials last four times as long as the others (40,000 x 8 x
// 64 bf16, window 512: 87 to 90 us, 63 % of cycles on the vector units, 24 % on the matrix
// cores; 16 x 2,000 x 16 x 128, window 1,000: 225 to 242 us, 43 and 30 %).  Rows that are
// no whole groups of 16 bytes go through registers number by number, for which there is
// not room enough at widths past 64 (16 x 2,000 x 16 x 100: 1,234 us, back 6,427; of 60
// 430 and 1,246, of 64 173 and 624).
template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(WNT, MIN_WAVES<T>) void k_window(WinArgs a) {
  constexpr int QT = QT_OF<T>, DT = P / 16, DS = P / 32, TILE = KEYS * P * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) char s_dyn[];  // [2][k, v][TILE]
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const long long piece = piece_of((long long)blockIdx.y * gridDim.x + blockIdx.x,
                                   (long long)gridDim.x * gridDim.y);
  const int h = (int)(piece / gridDim.x), g = h / (a.H / a.G), D = a.D;
  Unit u;
  if (!unit_of(a.off, a.n, a.N, BLOCK_OF<T>, false, piece % gridDim.x, u) || u.lo >= u.hi) return;

  const T *q = static_cast<const T *>(a.q) + u.b * a.qs + (long long)h * D;
  const T *k = static_cast<const T *>(a.k) + u.b * a.ks + (long long)g * D;
  const T *v = static_cast<const T *>(a.v) + u.b * a.vs + (long long)g * D;
  const Seen sn = seen_by(u.lo, u.hi, a.window, a.sinks);
  Carry<T, P, KEYS, WNT, WIDE> ck, cv;
  ck.init(a.ks, D);
  cv.init(a.vs, D);
  const auto start = [&](int tile) {
    return tile < sn.sink_tiles ? (long long)tile * KEYS
                                : sn.first + (long long)(tile - sn.sink_tiles) * KEYS;
  };
  const auto fetch = [&](int tile, char *to) {
    const long long s0 = start(tile), end = tile < sn.sink_tiles ? sn.sinks : u.hi;
    const int count = (int)(end - s0 < KEYS ? end - s0 : KEYS);
    ck.fetch(k, a.ks, D, s0, count, to);
    cv.fetch(v, a.vs, D, s0, count, to + TILE);
  };
  fetch(0, s_dyn);
  const long long tw = u.lo + w * 16 * QT;  // the wavefront's first query
  // (exponents are taken of sizes: a negative scale turns q's signs)
  const uint32_t sign = a.scale < 0.0f ? sizeof(T) == 2 ? 0x80008000u : 0x80000000u : 0u;
  const float c = fmaxf(fabsf(a.scale) * LOG2E, 0x1p-120f);
  Frag<T> qf[QT][DS];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long t = tw + 16 * i + l16;
#pragma unroll
    for (int s = 0; s < DS; ++s)
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e)
        qf[i][s].v[e] =
            load_group<T, WIDE>(q + t * a.qs, 32 * s + 8 * lg + e * PER<T>, D, t < u.hi, q) ^
            (int)sign;
  }
  float m[QT], l[QT];  // (m in units of scores)
  float4v o[DT][QT] = {};
#pragma unroll
  for (int i = 0; i < QT; ++i) m[i] = -INFINITY, l[i] = 0.0f;

  for (int tile = 0; tile < sn.tiles; ++tile) {
    char *s_k = s_dyn + (tile & 1) * 2 * TILE, *s_v = s_k + TILE;
    char *s_next = s_dyn + (~tile & 1) * 2 * TILE;
    if (tile == 0 || WIDE) {
      ck.finish(s_k);
      cv.finish(s_v);
    }
    __syncthreads();
    const bool more = tile + 1 < sn.tiles;
    if (more) fetch(tile + 1, s_next);
    const bool sink = tile < sn.sink_tiles;
    const long long s0 = start(tile);
    // unless none of the wavefront's queries sees the tile
    if (sink ||
        !(s0 > tw + 16 * QT - 1 || (tw - (s0 + KEYS - 1) >= a.window && s0 >= a.sinks))) {
      // whether all see all of it
      const bool whole = sink ? s0 + KEYS <= sn.sinks
                              : s0 + KEYS - 1 <= tw && tw + 16 * QT - 1 - s0 < a.window;
      float4v x[4][QT] = {};
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int s = 0; s < DS; ++s) {
          const Frag<T> f = Packed<T, P>::rows(s_k, 16 * kt, 32 * s, lane);
#pragma unroll
          for (int i = 0; i < QT; ++i) x[kt][i] = mac(f, qf[i][s], x[kt][i]);
        }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          const Edge e = edge_of(a, sn, sink, s0, tw + 16 * i + l16, lg);
          if (e.near) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                x[kt][i][r] = 16 * kt + r <= e.last ? x[kt][i][r] : -INFINITY;
          }
          if (e.far) {
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
              for (int r = 0; r < 4; ++r)
                x[kt][i][r] = ((16 * kt + r >= e.from) | (16 * kt + r < e.upto)) ? x[kt][i][r]
                                                                              : -INFINITY;
          }
        }
      }
      float top[QT];  // a lane's own, until a row is late
      bool late = false;
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        top[i] = fmaxf(fmaxf(x[0][i][0], x[0][i][1]), x[0][i][2]);
        top[i] = fmaxf(top[i], x[0][i][3]);
#pragma unroll
        for (int kt = 1; kt < 4; ++kt) {
          top[i] = fmaxf(fmaxf(top[i], x[kt][i][0]), x[kt][i][1]);
          top[i] = fmaxf(fmaxf(top[i], x[kt][i][2]), x[kt][i][3]);
        }
        late = late || !((top[i] - m[i]) * c <= LATE<T>);
      }
      if (__any(late)) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          // (while a row has seen nothing, m is -infinity and the sums are 0)
          const float shift = fmaxf(m[i], column_max(top[i]));
          const float less = shift == -INFINITY ? 1.0f : exp2_of((m[i] - shift) * c);
          m[i] = shift;
          l[i] *= less;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[d][i] *= less;
        }
      }
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        const float mc = (m[i] == -INFINITY ? 0.0f : m[i] * c) - RAISE<T>;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[kt][i][r] = exp2_of(fmaf(x[kt][i][r], c, -mc));
            l[i] += x[kt][i][r];
          }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag<T> p[QT];
#pragma unroll
        for (int i = 0; i < QT; ++i) p[i] = pack<T>(x[2 * t][i], x[2 * t + 1][i]);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const Frag<T> f = Packed<T, P>::columns(s_v, 32 * t, 16 * d, lane);
#pragma unroll
          for (int i = 0; i < QT; ++i) o[d][i] = mac(f, p[i], o[d][i]);
        }
      }
    }
    if (!WIDE && more) {
      ck.finish(s_next);
      cv.finish(s_next + TILE);
    }
  }
  const bool fine = finite(o);
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    l[i] = column_sum(l[i]);
    const long long t = tw + 16 * i + l16;
    if (t >= u.hi) continue;
    const float f = 1.0f / l[i];
    T *y = static_cast<T *>(a.o) + (u.b + t) * a.os + (long long)h * D;
#pragma unroll
    for (int d = 0; d < DT; ++d) store_four<T, WIDE>(y, 16 * d + 4 * lg, D, o[d][i] * f);
    if (lg == 0)
      a.lse[(u.b + t) * a.H + h] = fmaf(m[i], c, log2f(l[i] * (1.0f / RAISED<T>))) * LOG2;
  }
  if (fine) return;
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long t = tw + 16 * i + l16;
    if (t >= u.hi) continue;
    T *y = static_cast<T *>(a.o) + (u.b + t) * a.os + (long long)h * D;
    for (int d = 4 * lg; d < D; d += 16)
      if (none_of_four(y, d, D))
        mend_four(y, d, D,
                  exact_row<T>(q + t * a.qs, k, a.ks, v, a.vs, D, t, a.window, a.sinks,
                               a.scale < 0.0f ? -c : c,
                               (m[i] == -INFINITY ? 0.0f : m[i] * c) - RAISE<T>, d) *
                      (1.0f / l[i]));
  }
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------

// delta = y . dy of each row and head, a lane for 16 bytes of it.  Bound by memory (200
// MB of y and dy: 31 us).
template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(WNT) void k_window_delta(WinArgs a) {
  constexpr int LANES = P / PER<T>, EACH = WNT / LANES;
  const long long all = a.N * a.H;
  const int c = threadIdx.x % LANES * PER<T>;
  struct alignas(16) Group { T v[PER<T>]; };
  const auto read = [&](const void *p, long long at) {
    const T *row = static_cast<const T *>(p) + at;
    return __builtin_bit_cast(Group, load_group<T, WIDE>(row, c, a.D, true, row));
  };
  for (long long i = (long long)blockIdx.x * EACH + threadIdx.x / LANES; i < all;
       i += (long long)gridDim.x * EACH) {
    const long long row = (uint64_t)i / (uint32_t)a.H;
    const int h = (int)(i - row * a.H);
    const Group y = read(a.y, row * a.ys + (long long)h * a.D);
    const Group gy = read(a.gy, row * a.gys + (long long)h * a.D);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < PER<T>; ++j) s = fmaf((float)y.v[j], (float)gy.v[j], s);
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) s += __shfl_xor(s, o, WAVE);
    if (c == 0) a.delta[i] = s;
  }
}

template <typename T>
__device__ __noinline__ float4v exact_dq(const T *q, const T *gy, const T *k, long long ks,
                                         const T *v, long long vs, int D, long long t,
                                         int window, int sinks, float c, float lse, float delta,
                                         int d0) {
  float4v x{};
  for (long long s = 0; s <= t; ++s) {
    if (t - s >= window && s >= sinks) {
      s = t - window;
      continue;
    }
    const float e = exp2_of(fmaf(dot(q, k + s * ks, D), c, -lse));
    const float d = e * (dot(gy, v + s * vs, D) - delta);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      x[r] = fmaf(d, d0 + r < D ? (float)k[s * ks + d0 + r] : d, x[r]);
    if (all_nan(x)) break;
  }
  return x;
}

// What queries [t0, t1) of a head that see key s add to the gradients by it; or (run
// > 0) the wave-th 32 in each run of them, those that are a window past it.
struct TwoFours {
  float4v k, v;
};
template <typename T>
__device__ __noinline__ TwoFours exact_dkv(const T *q, long long qs, const T *gy, long long gys,
                                           const float *lse, const float *delta, int H, int D,
                                           const T *k, const T *v, long long s, long long t0,
                                           long long t1, int run, int wave, int window,
                                           int sinks, float c, int d0) {
  TwoFours x{};
  for (long long t = t0; t < t1; ++t) {
    if (run && ((t - t0) % run / 32 != wave || t - s < window)) continue;
    const T *qt = q + t * qs, *gt = gy + t * gys;
    const float e = exp2_of(fmaf(dot(qt, k, D), c, -lse[t * H] * LOG2E));
    float d = e * (dot(gt, v, D) - delta[t * H]);
    if (sees_one(t, window, sinks)) d *= 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x.k[r] = fmaf(d, d0 + r < D ? (float)qt[d0 + r] : d, x.k[r]);
      x.v[r] = fmaf(e, d0 + r < D ? (float)gt[d0 + r] : e, x.v[r]);
    }
    if (all_nan(x.k) && all_nan(x.v)) break;
  }
  return x;
}

// Gradients by queries; SUMS: only their delta, from P and dy v^T.
template <typename T, int P, bool WIDE, bool SUMS>
__device__ __forceinline__ void dq_block(const WinArgs &a, const Unit &u, int h, char *s_dyn) {
  // s_dyn: [2][k, v][TILE]
  constexpr int QT = QT_OF<T>, DT = P / 16, DS = P / 32, TILE = KEYS * P * (int)sizeof(T);
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int g = h / (a.H / a.G), D = a.D;
  const T *q = static_cast<const T *>(a.q) + u.b * a.qs + (long long)h * D;
  const T *gy = static_cast<const T *>(a.gy) + u.b * a.gys + (long long)h * D;
  const T *k = static_cast<const T *>(a.k) + u.b * a.ks + (long long)g * D;
  const T *v = static_cast<const T *>(a.v) + u.b * a.vs + (long long)g * D;
  const Seen sn = seen_by(u.lo, u.hi, a.window, a.sinks);
  Carry<T, P, KEYS, WNT, WIDE> ck, cv;
  ck.init(a.ks, D);
  cv.init(a.vs, D);
  const auto start = [&](int tile) {
    return tile < sn.sink_tiles ? (long long)tile * KEYS
                                : sn.first + (long long)(tile - sn.sink_tiles) * KEYS;
  };
  const auto fetch = [&](int tile, char *to) {
    const long long s0 = start(tile), end = tile < sn.sink_tiles ? sn.sinks : u.hi;
    const int count = (int)(end - s0 < KEYS ? end - s0 : KEYS);
    ck.fetch(k, a.ks, D, s0, count, to);
    cv.fetch(v, a.vs, D, s0, count, to + TILE);
  };
  fetch(0, s_dyn);
  const long long tw = u.lo + w * 16 * QT;
  Frag<T> qf[QT][DS], gf[QT][DS];
  float lse[QT], delta[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long t = tw + 16 * i + l16;
    const bool there = t < u.hi;
#pragma unroll
    for (int s = 0; s < DS; ++s)
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e) {
        const int at = 32 * s + 8 * lg + e * PER<T>;
        qf[i][s].v[e] = load_group<T, WIDE>(q + t * a.qs, at, D, there, q);
        gf[i][s].v[e] = load_group<T, WIDE>(gy + t * a.gys, at, D, there, gy);
      }
    lse[i] = there ? a.lse[(u.b + t) * a.H + h] * LOG2E : INFINITY;
    if (sees_one(t, a.window, a.sinks)) lse[i] = fmaf(lse[i], 0.0f, INFINITY);
    delta[i] = there ? a.delta[(u.b + t) * a.H + h] : 0.0f;
  }
  const float c = a.scale * LOG2E;
  float4v o[DT][QT] = {};
  float sum[QT] = {}, up[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) up[i] = SCALED<T> ? UNMET : 1.0f;
  for (int tile = 0; tile < sn.tiles; ++tile) {
    char *s_k = s_dyn + (tile & 1) * 2 * TILE, *s_v = s_k + TILE;
    char *s_next = s_dyn + (~tile & 1) * 2 * TILE;
    if (tile == 0 || WIDE) {
      ck.finish(s_k);
      cv.finish(s_v);
    }
    __syncthreads();
    const bool more = tile + 1 < sn.tiles, sink = tile < sn.sink_tiles;
    if (more) fetch(tile + 1, s_next);
    const long long s0 = start(tile);
    const bool none = !sink && (s0 > tw + 16 * QT - 1 ||
                                (tw - (s0 + KEYS - 1) >= a.window && s0 >= a.sinks));
    const bool whole = sink ? s0 + KEYS <= sn.sinks
                            : s0 + KEYS - 1 <= tw && tw + 16 * QT - 1 - s0 < a.window;
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2) {
      if (none) continue;
      float4v x[2][QT] = {}, y[2][QT] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int s = 0; s < DS; ++s) {
          const Frag<T> f = Packed<T, P>::rows(s_k, 32 * t2 + 16 * b, 32 * s, lane);
          const Frag<T> f2 = Packed<T, P>::rows(s_v, 32 * t2 + 16 * b, 32 * s, lane);
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            x[b][i] = mac(f, qf[i][s], x[b][i]);
            y[b][i] = mac(f2, gf[i][s], y[b][i]);
          }
        }
      Frag<T> p[QT];
#pragma unroll
      for (int i = 0; i < QT; ++i) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = exp2_of(fmaf(x[b][i][r], c, -lse[i]));
            x[b][i][r] = SUMS ? e * y[b][i][r] : e * (y[b][i][r] - delta[i]);
          }
        if (!whole) {
          const Edge e = edge_of(a, sn, sink, s0 + 32 * t2, tw + 16 * i + l16, lg);
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int at = 16 * b + r;
              const bool sees = (at <= e.last) & ((at >= e.from) | (at < e.upto));
              x[b][i][r] = sees ? x[b][i][r] : 0.0f;
            }
        }
        if constexpr (SUMS) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[i] += x[b][i][r];
        }
      }
      if constexpr (SUMS) continue;
      if constexpr (SCALED<T>) {
        bool late = false;
#pragma unroll
        for (int i = 0; i < QT; ++i) late = late || largest_of(x[0][i], x[1][i]) * up[i] > PAST;
        if (__any(late)) {
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            const float less = lowered(up[i], largest_of(x[0][i], x[1][i]));
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d][i] *= less;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < QT; ++i)
        p[i] = SCALED<T> ? pack<T>(x[0][i] * up[i], x[1][i] * up[i]) : pack<T>(x[0][i], x[1][i]);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const Frag<T> f = Packed<T, P>::columns(s_k, 32 * t2, 16 * d, lane);
#pragma unroll
        for (int i = 0; i < QT; ++i) o[d][i] = mac(f, p[i], o[d][i]);
      }
    }
    if (!WIDE && more) {
      ck.finish(s_next);
      cv.finish(s_next + TILE);
    }
  }
  if constexpr (SUMS) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      sum[i] = column_sum(sum[i]);
      const long long t = tw + 16 * i + l16;
      if (lg == 0 && t < u.hi) a.delta[(u.b + t) * a.H + h] = sum[i];
    }
    return;
  }
  const bool fine = finite(o);
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long t = tw + 16 * i + l16;
    if (t >= u.hi) continue;
    const float f = a.scale / up[i];
    T *gq = static_cast<T *>(a.gq) + (u.b + t) * a.gqs + (long long)h * D;
#pragma unroll
    for (int d = 0; d < DT; ++d) store_four<T, WIDE>(gq, 16 * d + 4 * lg, D, o[d][i] * f);
  }
  if (fine) return;
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long t = tw + 16 * i + l16;
    if (t >= u.hi) continue;
    T *gq = static_cast<T *>(a.gq) + (u.b + t) * a.gqs + (long long)h * D;
    for (int d = 4 * lg; d < D; d += 16)
      if (none_of_four(gq, d, D))
        mend_four(gq, d, D,
                  exact_dq<T>(q + t * a.qs, gy + t * a.gys, k, a.ks, v, a.vs, D, t, a.window,
                              a.sinks, c, lse[i], delta[i], d) * a.scale);
  }
}

// Whether the queries outside the window of a sequence's first frames are cut into
// units: where there are more than one of them.
__device__ __forceinline__ bool in_units(const WinArgs &a, const Unit &u) {
  return a.part && u.len > a.window && u.len > a.unit;
}
// Sums [2][P] for a first frame of such a sequence: its block's own, and unit j's.
// Such sequences are longer than a unit, so floor(b / unit) differs, and floor(2 b /
// unit) by as much as they have units.
__device__ __forceinline__ float *own_part(const WinArgs &a, const Unit &u, int g, int s, int P) {
  return a.own + ((u.b / a.unit * a.G + g) * a.sinks + s) * 2 * P;
}
__device__ __forceinline__ float *unit_part(const WinArgs &a, const Unit &u, long long j, int g,
                                            int s, int P) {
  return a.part + (((2 * u.b / a.unit + j) * a.G + g) * a.sinks + s) * 2 * P;
}

// Gradients by keys and values: a workgroup has BLOCK keys of a key head and walks
// the queries that see them, head after head of its group.
template <typename T, int P, bool WIDE>
__device__ __forceinline__ void dkv_block(const WinArgs &a, const Unit &u, int g, char *s_dyn) {
  // s_dyn: [2][q, dy][TILE], v, lse and delta [2][2][QUERIES]
  constexpr int QT = QT_OF<T>, BLOCK = BLOCK_OF<T>, DT = P / 16, DS = P / 32;
  constexpr int TILE = QUERIES * P * (int)sizeof(T);
  char *s_v = s_dyn + 4 * TILE;
  float *s_row = reinterpret_cast<float *>(s_v + BLOCK * P * (int)sizeof(T));
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int E = a.H / a.G, D = a.D;
  // first frames among the keys: their queries outside the window are units', or
  // (short sequences) walked here too
  const bool split = in_units(a, u), onward = u.lo < a.sinks && !split;
  const T *k = static_cast<const T *>(a.k) + u.b * a.ks + (long long)g * D;
  const T *v = static_cast<const T *>(a.v) + u.b * a.vs + (long long)g * D;
  const long long sw = u.lo + w * 16 * QT;  // the wavefront's first key
  Carry<T, P, BLOCK, WNT, WIDE> cv;
  cv.init(a.vs, D);
  cv.fetch(v, a.vs, D, u.lo, (int)(u.hi - u.lo), s_v);
  Frag<T> kf[QT][DS];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long s = sw + 16 * i + l16;
#pragma unroll
    for (int t = 0; t < DS; ++t)
#pragma unroll
      for (int e = 0; e < (int)sizeof(T) / 2; ++e) {
        const int at = 32 * t + 8 * lg + e * PER<T>;
        kf[i][t].v[e] = load_group<T, WIDE>(k + s * a.ks, at, D, s < u.hi, k);
      }
  }
  cv.finish(s_v);
  const float c = a.scale * LOG2E;
  float4v ok[DT][QT] = {}, ov[DT][QT] = {};
  float up[QT];
#pragma unroll
  for (int i = 0; i < QT; ++i) up[i] = SCALED<T> ? UNMET : 1.0f;
  const long long end =
      u.hi - 1 + a.window < u.len && !onward ? u.hi - 1 + a.window : u.len;
  const int tiles = (int)((end - u.lo + QUERIES - 1) / QUERIES), all = tiles * E;
  Carry<T, P, QUERIES, WNT, WIDE> cq, cg;
  cq.init(a.qs, D);
  cg.init(a.gys, D);
  float r_lse = 0.0f, r_delta = 0.0f;
  const auto fetch = [&](int h, int tile, char *to) {
    const long long t0 = u.lo + (long long)tile * QUERIES;
    const int count = (int)(end - t0 < QUERIES ? end - t0 : QUERIES);
    cq.fetch(static_cast<const T *>(a.q) + u.b * a.qs + (long long)h * D, a.qs, D, t0, count, to);
    cg.fetch(static_cast<const T *>(a.gy) + u.b * a.gys + (long long)h * D, a.gys, D, t0, count,
             to + TILE);
    if (threadIdx.x < QUERIES) {
      const bool there = (int)threadIdx.x < count;
      const long long at = (u.b + t0 + threadIdx.x) * a.H + h;
      r_lse = there ? a.lse[at] * LOG2E - RAISE<T> : INFINITY;
      r_delta = there ? a.delta[at] : 0.0f;
    }
  };
  const auto finish = [&](int j) {
    cq.finish(s_dyn + (j & 1) * 2 * TILE);
    cg.finish(s_dyn + (j & 1) * 2 * TILE + TILE);
    if (threadIdx.x < QUERIES) {
      s_row[(j & 1) * 2 * QUERIES + threadIdx.x] = r_lse;
      s_row[((j & 1) * 2 + 1) * QUERIES + threadIdx.x] = r_delta;
    }
  };
  int h = g * E, tile = 0;
  fetch(h, 0, s_dyn);
  finish(0);
  for (int j = 0; j < all; ++j) {
    const char *s_q = s_dyn + (j & 1) * 2 * TILE, *s_g = s_q + TILE;
    const float *s_lse = s_row + (j & 1) * 2 * QUERIES, *s_delta = s_lse + QUERIES;
    __syncthreads();
    const long long t0 = u.lo + (long long)tile * QUERIES;
    const bool more = j + 1 < all;
    if (++tile == tiles) tile = 0, ++h;
    if (more) fetch(h, tile, s_dyn + (~j & 1) * 2 * TILE);
    const bool none = t0 + QUERIES - 1 < sw || (t0 - (sw + 16 * QT - 1) >= a.window &&
                                                !(onward && sw < a.sinks));
    const bool whole = t0 >= sw + 16 * QT - 1 && t0 + QUERIES - 1 - sw < a.window;
    if (!none) {
      float4v x[2][QT] = {}, y[2][QT] = {};
#pragma unroll
      for (int s = 0; s < DS; ++s) {
        Frag<T> vf[QT];
#pragma unroll
        for (int i = 0; i < QT; ++i)
          vf[i] = Packed<T, P>::rows(s_v, (w * QT + i) * 16, 32 * s, lane);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const Frag<T> f = Packed<T, P>::rows(s_q, 16 * b, 32 * s, lane);
          const Frag<T> f2 = Packed<T, P>::rows(s_g, 16 * b, 32 * s, lane);
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            x[b][i] = mac(f, kf[i][s], x[b][i]);
            y[b][i] = mac(f2, vf[i], y[b][i]);
          }
        }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int at = 16 * b + 4 * lg;
        const float4v lse = *reinterpret_cast<const float4v *>(s_lse + at);
        const float4v delta = *reinterpret_cast<const float4v *>(s_delta + at);
#pragma unroll
        for (int i = 0; i < QT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = exp2_of(fmaf(x[b][i][r], c, -lse[r]));
            x[b][i][r] = e;
            y[b][i][r] = e * (y[b][i][r] - delta[r]);
          }
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          // of a lane's queries t0 + 4 lg + at: those from the key on, up to `end` and
          // to the end of the window
          const long long s = sw + 16 * i + l16, at0 = t0 + 4 * lg;
          const long long past = onward && s < a.sinks ? end : s + a.window;
          const int from = within_tile(s - at0);
          const int upto = within_tile((past < end ? past : end) - at0);
          const int first = a.window == 1 && a.sinks == 0 ? KEYS : within_tile(-at0);
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int at = 16 * b + r;
              const bool sees = (at >= from) & (at < upto);
              x[b][i][r] = sees ? x[b][i][r] : 0.0f;
              y[b][i][r] = (sees & (at > first)) ? y[b][i][r] : 0.0f;
            }
        }
      }
      if constexpr (SCALED<T>) {
        bool late = false;
#pragma unroll
        for (int i = 0; i < QT; ++i) late = late || largest_of(y[0][i], y[1][i]) * up[i] > PAST;
        if (__any(late)) {
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            const float less = lowered(up[i], largest_of(y[0][i], y[1][i]));
#pragma unroll
            for (int d = 0; d < DT; ++d) ok[d][i] *= less;
          }
        }
      }
      Frag<T> p[QT], ds[QT];
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        p[i] = pack<T>(x[0][i], x[1][i]);
        ds[i] = SCALED<T> ? pack<T>(y[0][i] * up[i], y[1][i] * up[i])
                          : pack<T>(y[0][i], y[1][i]);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const Frag<T> f = Packed<T, P>::columns(s_g, 0, 16 * d, lane);
        const Frag<T> f2 = Packed<T, P>::columns(s_q, 0, 16 * d, lane);
#pragma unroll
        for (int i = 0; i < QT; ++i) {
          ov[d][i] = mac(f, p[i], ov[d][i]);
          ok[d][i] = mac(f2, ds[i], ok[d][i]);
        }
      }
    }
    if (more) finish(j + 1);
  }
  // (what the loop leaves out of queries that see only themselves: their lse and delta
  // tell whether dS is no number)
  if (sees_one(sw, a.window, a.sinks)) {
#pragma unroll
    for (int i = 0; i < QT; ++i) {
      const long long s = sw + 16 * i + l16;
      if (s >= u.hi || !sees_one(s, a.window, a.sinks)) continue;
      float z = 0.0f;
      for (int hh = g * E; hh < g * E + E; ++hh) {
        const long long at = (u.b + s) * a.H + hh;
        z = fmaf(a.lse[at] + a.delta[at], 0.0f, z);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) ok[d][i] += z;
    }
  }
  const bool fine = finite(ok) && finite(ov);
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const long long s = sw + 16 * i + l16;
    if (s >= u.hi) continue;
    T *gk = static_cast<T *>(a.gk) + (u.b + s) * a.gks + (long long)g * D;
    T *gv = static_cast<T *>(a.gv) + (u.b + s) * a.gvs + (long long)g * D;
    float *own = split && s < a.sinks ? own_part(a, u, g, (int)s, P) : nullptr;
    const float f = a.scale / (up[i] * RAISED<T>);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      ok[d][i] *= f;
      ov[d][i] *= 1.0f / RAISED<T>;
      if (own) {
        *reinterpret_cast<float4v *>(own + 16 * d + 4 * lg) = ok[d][i];
        *reinterpret_cast<float4v *>(own + P + 16 * d + 4 * lg) = ov[d][i];
      } else {
        store_four<T, WIDE>(gk, 16 * d + 4 * lg, D, ok[d][i]);
        store_four<T, WIDE>(gv, 16 * d + 4 * lg, D, ov[d][i]);
      }
    }
  }
  if (fine) return;
#pragma unroll 1
  for (int i = 0; i < QT; ++i) {
    const long long s = sw + 16 * i + l16;
    if (s >= u.hi) continue;
    T *gk = static_cast<T *>(a.gk) + (u.b + s) * a.gks + (long long)g * D;
    T *gv = static_cast<T *>(a.gv) + (u.b + s) * a.gvs + (long long)g * D;
    float *own = split && s < a.sinks ? own_part(a, u, g, (int)s, P) : nullptr;
    const long long t1 =
        s + a.window < u.len && !(onward && s < a.sinks) ? s + a.window : u.len;
    for (int d = 4 * lg; d < D; d += 16) {
      if (own ? !none_of_four(own, d, D) && !none_of_four(own + P, d, D)
              : !none_of_four(gk, d, D) && !none_of_four(gv, d, D))
        continue;
      float4v xk{}, xv{};
      for (int hh = g * E; hh < g * E + E; ++hh) {
        const T *qh = static_cast<const T *>(a.q) + u.b * a.qs + (long long)hh * D;
        const T *gh = static_cast<const T *>(a.gy) + u.b * a.gys + (long long)hh * D;
        const TwoFours x = exact_dkv<T>(
            qh, a.qs, gh, a.gys, a.lse + u.b * a.H + hh, a.delta + u.b * a.H + hh, a.H, D,
            k + s * a.ks, v + s * a.vs, s, s, t1, 0, 0, a.window, a.sinks, c, d);
        xk += x.k;
        xv += x.v;
      }
      if (own) {
        mend_four(own, d, D, xk * a.scale);
        mend_four(own + P, d, D, xv);
      } else {
        mend_four(gk, d, D, xk * a.scale);
        mend_four(gv, d, D, xv);
      }
    }
  }
}

// What a unit of queries adds to the gradients of 16 first frames that it sees
// from outside its window: 32 queries a wavefront at a time, the wavefronts'
// sums joined in LDS.  Rows of `part` of units without such a query are not
// written, nor read.
template <typename T, int P, bool WIDE>
__device__ __forceinline__ void sinks_block(const WinArgs &a, const Unit &u, int g, int first,
                                            char *s_dyn) {
  constexpr int Q = 32 * WNW, DT = P / 16, DS = P / 32;
  T *s_q = reinterpret_cast<T *>(s_dyn), *s_g = s_q + Q * LD<T, P>;
  float *s_lse = reinterpret_cast<float *>(s_g + Q * LD<T, P>), *s_delta = s_lse + Q;
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int E = a.H / a.G, D = a.D;
  const long long s = first + l16;  // the lane's key
  if (!in_units(a, u) || u.hi <= a.window) return;

  const T *k = static_cast<const T *>(a.k) + u.b * a.ks + (long long)g * D;
  const T *v = static_cast<const T *>(a.v) + u.b * a.vs + (long long)g * D;
  const bool mine = s < a.sinks && s < u.len;
  Frag<T> kf[DS], vf[DS];
#pragma unroll
  for (int t = 0; t < DS; ++t)
#pragma unroll
    for (int e = 0; e < (int)sizeof(T) / 2; ++e) {
      const int at = 32 * t + 8 * lg + e * PER<T>;
      kf[t].v[e] = load_group<T, WIDE>(k + s * a.ks, at, D, mine, k);
      vf[t].v[e] = load_group<T, WIDE>(v + s * a.vs, at, D, mine, v);
    }
  const float c = a.scale * LOG2E;
  float up = SCALED<T> ? UNMET : 1.0f;
  float4v ok[DT] = {}, ov[DT] = {};
  const long long lo = u.lo > a.window ? u.lo : a.window;
  const int tiles = (int)((u.hi - lo + Q - 1) / Q), all = tiles * E;
  Stage<T, P, Q, WNT, WIDE> rq, rg;
  float r_lse = 0.0f, r_delta = 0.0f;
  const auto fetch = [&](int j) {
    const int h = g * E + j / tiles;
    const long long t0 = lo + (long long)(j % tiles) * Q;
    const int count = (int)(u.hi - t0 < Q ? u.hi - t0 : Q);
    rq.fetch(static_cast<const T *>(a.q) + u.b * a.qs + (long long)h * D, a.qs, D, t0, 1, count);
    rg.fetch(static_cast<const T *>(a.gy) + u.b * a.gys + (long long)h * D, a.gys, D, t0, 1,
             count);
    if (threadIdx.x < Q) {
      const bool there = (int)threadIdx.x < count;
      const long long at = (u.b + t0 + threadIdx.x) * a.H + h;
      r_lse = there ? a.lse[at] * LOG2E - RAISE<T> : INFINITY;
      r_delta = there ? a.delta[at] : 0.0f;
    }
  };
  fetch(0);
  for (int j = 0; j < all; ++j) {
    __syncthreads();
    rq.store(s_q);
    rg.store(s_g);
    if (threadIdx.x < Q) s_lse[threadIdx.x] = r_lse, s_delta[threadIdx.x] = r_delta;
    __syncthreads();
    if (j + 1 < all) fetch(j + 1);
    const long long t0 = lo + (long long)(j % tiles) * Q;
    float4v x[2] = {}, y[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int at = 32 * w + 16 * b;
#pragma unroll
      for (int t = 0; t < DS; ++t) {
        x[b] = mac(rows<T, P>(s_q, at, 32 * t, lane), kf[t], x[b]);
        y[b] = mac(rows<T, P>(s_g, at, 32 * t, lane), vf[t], y[b]);
      }
      const float4v lse = *reinterpret_cast<const float4v *>(s_lse + at + 4 * lg);
      const float4v delta = *reinterpret_cast<const float4v *>(s_delta + at + 4 * lg);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const long long t = t0 + at + 4 * lg + r;
        const bool sees = mine && t - s >= a.window && t < u.hi;
        const float e = exp2_of(fmaf(x[b][r], c, -lse[r]));
        const float d = e * (y[b][r] - delta[r]);
        x[b][r] = sees ? e : 0.0f;
        y[b][r] = sees ? d : 0.0f;
      }
    }
    if constexpr (SCALED<T>) {
      const float top = largest_of(y[0], y[1]);
      if (__any(top * up > PAST)) {
        const float less = lowered(up, top);
#pragma unroll
        for (int d = 0; d < DT; ++d) ok[d] *= less;
      }
    }
    const Frag<T> p = pack<T>(x[0], x[1]);
    const Frag<T> ds = SCALED<T> ? pack<T>(y[0] * up, y[1] * up) : pack<T>(y[0], y[1]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      ov[d] = mac(columns<T, P>(s_g, 32 * w, 16 * d, lane), p, ov[d]);
      ok[d] = mac(columns<T, P>(s_q, 32 * w, 16 * d, lane), ds, ok[d]);
    }
  }
  float z = 0.0f;
  const float f = a.scale / (up * RAISED<T>);
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    ok[d] *= f;
    ov[d] *= 1.0f / RAISED<T>;
#pragma unroll
    for (int r = 0; r < 4; ++r) z = fmaf(ok[d][r], 0.0f, fmaf(ov[d][r], 0.0f, z));
  }
  if (!__all(z == 0.0f) && mine) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      if (16 * d + 4 * lg >= D) continue;
      float4v xk{}, xv{};
      for (int h = g * E; h < g * E + E; ++h) {
        const T *qh = static_cast<const T *>(a.q) + u.b * a.qs + (long long)h * D;
        const T *gh = static_cast<const T *>(a.gy) + u.b * a.gys + (long long)h * D;
        const TwoFours x = exact_dkv<T>(
            qh, a.qs, gh, a.gys, a.lse + u.b * a.H + h, a.delta + u.b * a.H + h, a.H, D,
            k + s * a.ks, v + s * a.vs, s, lo, u.hi, Q, w, a.window, a.sinks, c,
            16 * d + 4 * lg);
        xk += x.k;
        xv += x.v;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        ok[d][r] = fabsf(ok[d][r]) < INFINITY ? ok[d][r] : xk[r] * a.scale;
        ov[d][r] = fabsf(ov[d][r]) < INFINITY ? ov[d][r] : xv[r];
      }
    }
  }
  // (the sums take as much of LDS as the tiles of a 16-bit type)
  float *s_sum = reinterpret_cast<float *>(s_dyn);
  static_assert(WNW * 16 * P * 4 <= 2 * Q * LD<T, P> * (int)sizeof(T), "room for the sums");
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; ++d)
      *reinterpret_cast<float4v *>(s_sum + (w * 16 + l16) * P + 16 * d + 4 * lg) =
          o ? ov[d] : ok[d];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * P; i += WNT) {
      float v = 0.0f;
#pragma unroll
      for (int q = 0; q < WNW; ++q) v += s_sum[q * 16 * P + i];
      const int key = first + i / P;
      if (key < a.sinks)
        unit_part(a, u, u.lo / a.unit, g, key, P)[o * P + i % P] = v;
    }
  }
}

// Workgroups of all three: blocks of keys, blocks of queries, units for the first
// frames.  Seven products where five are needed: scores and dy v^T are computed for dq
// and again for dk and dv.  Bound by what a wavefront waits for between them with
// two a SIMD (16 x 2,000 x 16 heads of 128 bf16, window 1,000: 764 to 809 us, 28 % of
// cycles on the matrix cores, 28 % on the vector units).
template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(WNT, MIN_WAVES<T>) void k_window_back(WinArgs a) {
  extern __shared__ __attribute__((aligned(16))) char s_dyn[];
  constexpr int BLOCK = BLOCK_OF<T>;
  const long long blocks = a.N / BLOCK + a.n;
  long long id = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  Unit u;
  if (id < blocks * a.G) {
    id = piece_of(id, blocks * a.G);
    if (unit_of(a.off, a.n, a.N, BLOCK, false, id % blocks, u) && u.lo < u.hi)
      dkv_block<T, P, WIDE>(a, u, (int)(id / blocks), s_dyn);
    return;
  }
  id -= blocks * a.G;
  if (id < blocks * a.H) {
    id = piece_of(id, blocks * a.H);
    if (unit_of(a.off, a.n, a.N, BLOCK, false, id % blocks, u) && u.lo < u.hi)
      dq_block<T, P, WIDE, false>(a, u, (int)(id / blocks), s_dyn);
    return;
  }
  id -= blocks * a.H;
  const long long units = a.N / a.unit + a.n, part = id / units;
  if (part < (long long)a.G * ((a.sinks + 15) / 16) &&
      unit_of(a.off, a.n, a.N, a.unit, false, id % units, u) && u.lo < u.hi)
    sinks_block<T, P, WIDE>(a, u, (int)(part % a.G), (int)(part / a.G) * 16, s_dyn);
}

// delta from y as it was rounded is off by half a spacing of y, which is next to
// nothing beside dS of many frames but as much as the rounding of dS beside few:
// queries of a sequence's first block, and of windows up to FEW frames, have it
// summed again from P and dy v^T (the same case: 11 us).  (Where one of many frames takes
// nearly all the weight, dS keeps of it what y's rounding leaves: to sum it again for
// all queries would be two of seven products more.)
template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(WNT, MIN_WAVES<T>) void k_window_sums(WinArgs a, int every) {
  constexpr int BLOCK = BLOCK_OF<T>;
  extern __shared__ __attribute__((aligned(16))) char s_dyn[];
  Unit u;
  if (!unit_of(a.off, a.n, a.N, every ? BLOCK : 0, false, blockIdx.x, u)) return;
  if (u.hi > u.lo + BLOCK) u.hi = u.lo + BLOCK;
  if (u.lo < u.hi) dq_block<T, P, WIDE, true>(a, u, blockIdx.y, s_dyn);
}

// Gradients of first frames whose sums lie in parts: their own, then the units' (the
// same case: 5 us, a launch and a trip to memory).
template <typename T, int P>
__global__ __launch_bounds__(P) void k_window_first(WinArgs a) {
  Unit u;
  if (!unit_of(a.off, a.n, a.N, 0, false, blockIdx.x, u) || !in_units(a, u)) return;
  const int d = threadIdx.x, g = blockIdx.y;
  if (d >= a.D) return;
  const long long n = (u.len + a.unit - 1) / a.unit;
  for (int s = blockIdx.z; s < a.sinks && s < u.len; s += gridDim.z) {
    const float *own = own_part(a, u, g, s, P);
    float k = own[d], v = own[P + d];
    for (long long j = a.window / a.unit; j < n; ++j) {
      const float *p = unit_part(a, u, j, g, s, P);
      k += p[d];
      v += p[P + d];
    }
    static_cast<T *>(a.gk)[(u.b + s) * a.gks + (long long)g * a.D + d] = (T)k;
    static_cast<T *>(a.gv)[(u.b + s) * a.gvs + (long long)g * a.D + d] = (T)v;
  }
}

// ---------------------------------------------------------------------------
// one step
// ---------------------------------------------------------------------------

// Row of a cache where the frame of position p lies.
__device__ __forceinline__ int ring(int p, int window, int sinks) {
  return p < sinks ? p : sinks + (p - sinks) % window;
}

// 16 query heads of a key head (its group, or a part of it) of a row against a
// part of its cache, 32 frames a wavefront at a time: k straight from memory as
// an operand, v through LDS of the wavefront's own.  The row's own frame comes
// from k and v, and the first part writes it to the cache, where no one reads it.
// Bound by memory (256 rows of 16 + 4 heads of 128 f16, window 1,000: 81 to 86 us for 441
// MB, 5.1 to 5.4 TB/s); few rows by a load's way and the parts' join.
template <typename T, int P, bool WIDE>
__global__ __launch_bounds__(WNT) void k_window_step(WinStepArgs a) {
  constexpr int DT = P / 16, DS = P / 32, GROUPS = P / PER<T>, LOADS = 32 * GROUPS / WAVE;
  __shared__ __attribute__((aligned(16))) T s_v[WNW][32 * LD<T, P>];
  __shared__ float s_m[WNW][16], s_l[WNW][16];
  static_assert(WNW * BYTES<T, P, 32> >= WNW / 2 * 16 * P * 4, "room for half of the results");
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int E = a.H / a.G, parts = (E + 15) / 16, D = a.D;
  const int g = blockIdx.y / parts, e0 = blockIdx.y % parts * 16;
  const int heads = E - e0 < 16 ? E - e0 : 16;  // of this workgroup
  const long long i = blockIdx.x;
  const int h0 = g * E + e0;
  const long long slot = a.slot ? (long long)a.slot[i] : i;
  const int pos = a.pos[i];
  const bool idle = slot < 0 || slot >= a.slots || pos < 0;
  T *y = static_cast<T *>(a.y) + i * a.ys + (long long)h0 * D;
  if (idle) {
    if (blockIdx.z == 0)
      for (int d = threadIdx.x; d < heads * D; d += WNT) y[d] = (T)0.0f;
    return;
  }
  const int L = a.sinks + a.window, own = ring(pos, a.window, a.sinks);
  const int count = pos < L ? pos + 1 : L;
  T *kc = static_cast<T *>(a.kc) + slot * L * a.kcs + (long long)g * D;
  T *vc = static_cast<T *>(a.vc) + slot * L * a.vcs + (long long)g * D;
  const T *kn = static_cast<const T *>(a.k) + i * a.ks + (long long)g * D;
  const T *vn = static_cast<const T *>(a.v) + i * a.vs + (long long)g * D;
  if (blockIdx.z == 0 && e0 == 0)
    for (int d = threadIdx.x; d < D; d += WNT) {
      kc[own * a.kcs + d] = kn[d];
      vc[own * a.vcs + d] = vn[d];
    }
  // the part's frames, whole tiles of all wavefronts
  const int tiles = (count + 31) / 32, share = (tiles + a.splits - 1) / a.splits;
  const int first = blockIdx.z * share, last = first + share < tiles ? first + share : tiles;

  Frag<T> qf[DS];
  const T *q = static_cast<const T *>(a.q) + i * a.qs + (long long)(h0 + l16) * D;
#pragma unroll
  for (int s = 0; s < DS; ++s)
#pragma unroll
    for (int e = 0; e < (int)sizeof(T) / 2; ++e)
      qf[s].v[e] = load_group<T, WIDE>(q, 32 * s + 8 * lg + e * PER<T>, D, l16 < heads, kn);
  const float c = a.scale * LOG2E;
  float m = -INFINITY, l = 0.0f;
  float4v o[DT] = {};
  // a tile's keys, as operands, and values: the next one's are read as soon as this
  // one's are used
  Frag<T> kr[2][DS];
  int4v vr[LOADS];
  const auto read_keys = [&](int c0) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int r = c0 + 16 * b + l16;
      const T *p = r == own ? kn : kc + (long long)r * a.kcs;
#pragma unroll
      for (int s = 0; s < DS; ++s)
#pragma unroll
        for (int e = 0; e < (int)sizeof(T) / 2; ++e)
          kr[b][s].v[e] =
              load_group<T, WIDE>(p, 32 * s + 8 * lg + e * PER<T>, D, r < count, kn);
    }
  };
  const auto read_values = [&](int c0) {
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      const int at = e * WAVE + lane, r = c0 + at / GROUPS;
      vr[e] = load_group<T, WIDE>(r == own ? vn : vc + (long long)r * a.vcs,
                                  at % GROUPS * PER<T>, D, r < count, vn);
    }
  };
  if (first + w < last) {
    read_keys((first + w) * 32);
    read_values((first + w) * 32);
  }
  for (int tile = first + w; tile < last; tile += WNW) {
    const int c0 = tile * 32, next0 = c0 + 32 * WNW;
    const bool more = tile + WNW < last;
    float4v x[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int s = 0; s < DS; ++s) x[b] = mac(kr[b][s], qf[s], x[b]);
    if (more) read_keys(next0);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < LOADS; ++e) {
      const int at = e * WAVE + lane;
      *reinterpret_cast<int4v *>(&s_v[w][at / GROUPS * LD<T, P> + at % GROUPS * PER<T>]) = vr[e];
    }
    __builtin_amdgcn_wave_barrier();
    if (more) read_values(next0);
    float top = -INFINITY;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[b][r] = c0 + 16 * b + 4 * lg + r < count ? x[b][r] * c : -INFINITY;
        top = fmaxf(top, x[b][r]);
      }
    top = column_max(top);
    const float next = fmaxf(m, top), shift = next == -INFINITY ? 0.0f : next;
    const float less = exp2_of(m - shift);
    m = next;
    l *= less;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[b][r] = exp2_of(x[b][r] - (shift - RAISE<T>));
        l += x[b][r];
      }
    const Frag<T> p = pack<T>(x[0], x[1]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      o[d] = mac(columns<T, P>(s_v[w], 0, 16 * d, lane), p, o[d] * less);
  }
  l = column_sum(l);
  if (lg == 0) s_m[w][l16] = m, s_l[w][l16] = l;
  __syncthreads();
  // the wavefronts' results joined: each scaled to the largest maximum, then summed
  float most = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int v = 0; v < WNW; ++v) most = fmaxf(most, s_m[v][l16]);
  const float shift = most == -INFINITY ? 0.0f : most;
#pragma unroll
  for (int v = 0; v < WNW; ++v) sum += s_l[v][l16] * exp2_of(s_m[v][l16] - shift);
  const float less = exp2_of(m - shift);
  float *s_o = reinterpret_cast<float *>(&s_v[0][0]);  // [half of the waves][16][P]
#pragma unroll
  for (int half = WNW / 2; half; half /= 2) {
    __syncthreads();
    if (w >= half && w < 2 * half)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<float4v *>(s_o + ((w - half) * 16 + l16) * P + 16 * d + 4 * lg) =
            half == WNW / 2 ? o[d] * less : o[d];
    __syncthreads();
    if (w < half)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = (half == WNW / 2 ? o[d] * less : o[d]) +
               *reinterpret_cast<float4v *>(s_o + (w * 16 + l16) * P + 16 * d + 4 * lg);
  }
  if (w || l16 >= heads) return;
  if (a.splits == 1) {
    const float f = 1.0f / sum;
#pragma unroll
    for (int d = 0; d < DT; ++d)
      store_four<T, WIDE>(y + (long long)l16 * D, 16 * d + 4 * lg, D, o[d] * f);
    return;
  }
  float *part = a.part + ((i * a.H + h0 + l16) * a.splits + blockIdx.z) * (P + 4);
#pragma unroll
  for (int d = 0; d < DT; ++d)
    *reinterpret_cast<float4v *>(part + 4 + 16 * d + 4 * lg) = o[d];
  if (lg == 0) part[0] = most, part[1] = sum;
}

// Joins the parts of a row's head.
template <typename T, int P>
__global__ __launch_bounds__(P) void k_window_join(WinStepArgs a) {
  const long long i = blockIdx.x;
  const int h = blockIdx.y, d = threadIdx.x;
  const long long slot = a.slot ? (long long)a.slot[i] : i;
  if (slot < 0 || slot >= a.slots || a.pos[i] < 0 || d >= a.D) return;
  const float *part = a.part + (i * a.H + h) * (long long)a.splits * (P + 4);
  float m = -INFINITY;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, part[s * (P + 4)]);
  const float shift = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, x = 0.0f;
  for (int s = 0; s < a.splits; ++s) {
    const float *p = part + s * (P + 4);
    const float f = exp2_of(p[0] - shift);
    l = fmaf(f, p[1], l);
    x = fmaf(f, p[4 + d], x);
  }
  static_cast<T *>(a.y)[i * a.ys + (long long)h * a.D + d] = (T)(x / l);
}

// Rows of the caches from the frames of whole sequences: entry c holds the last
// frame that the ring puts there.  (256 streams of 1,004 frames of 4 heads of 128 f16: 419 us
// for 1.05 GB, 2.5 TB/s: two bytes a lane.)
template <typename T>
__global__ __launch_bounds__(WNT) void k_window_fill(WinFillArgs a) {
  const int s = a.first + blockIdx.y, L = a.sinks + a.window;
  const long long slot = a.slot ? (long long)a.slot[s] : s;
  if (slot < 0 || slot >= a.slots) return;
  const long long b = clamped(a.off[s], 0, a.N), len = clamped(a.off[s + 1], b, a.N) - b;
  for (long long e = blockIdx.x; e < L && e < len; e += gridDim.x) {
    const long long t = e < a.sinks ? e : e + (len - 1 - e) / a.window * a.window;
    const T *k = static_cast<const T *>(a.k) + (b + t) * a.ks;
    const T *v = static_cast<const T *>(a.v) + (b + t) * a.vs;
    T *kc = static_cast<T *>(a.kc) + (slot * L + e) * a.kcs;
    T *vc = static_cast<T *>(a.vc) + (slot * L + e) * a.vcs;
    for (int d = threadIdx.x; d < a.width; d += WNT) kc[d] = k[d], vc[d] = v[d];
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

// Whether every head's row of each tensor begins at a multiple of 16 bytes and is
// whole groups of them.  (Rows without columns are: the other form reads a first
// number in the place of those that are not there, and here there is none.)
bool wide_rows(size_t e, int D, std::initializer_list<long long> strides,
               std::initializer_list<const void *> data) {
  if (D == 0) return true;
  if (D * e % 16) return false;
  for (long long t : strides)
    if (t * e % 16) return false;
  for (const void *p : data)
    if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  return true;
}

// LDS of a walk over keys: two pairs of tiles; over queries: two pairs of smaller
// ones, a block of v, their rows' numbers; of a unit's queries.
template <typename T, int P>
constexpr int WALK = 4 * KEYS * P * (int)sizeof(T);
template <typename T, int P>
constexpr int WALK_BACK = (4 * QUERIES + BLOCK_OF<T>) * P * (int)sizeof(T) + 4 * QUERIES * 4;
template <typename T, int P>
constexpr int WALK_UNIT = 2 * BYTES<T, P, 32 * WNW> + 2 * 32 * WNW * 4;
static_assert(WALK<float, 128> <= 160 * 1024 && WALK_BACK<float, 128> <= 160 * 1024 &&
                  WALK_UNIT<float, 128> <= 160 * 1024,
              "LDS of a CU");

hipError_t allow_lds(const void *kernel, int lds) {
  if (lds <= 64 * 1024) return hipSuccess;
  return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
}

constexpr int MAX_ACROSS = 65535;           // of a grid's second and third dimension
constexpr long long MAX_BLOCKS = 1 << 23;   // and of its first

template <typename T, int P, bool WIDE>
hipError_t forward_as(const WinArgs &a, hipStream_t s) {
  constexpr int lds = WALK<T, P>;
  constexpr int BLOCK = BLOCK_OF<T>;
  if (a.N / BLOCK + a.n > MAX_BLOCKS) return hipErrorInvalidValue;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(k_window<T, P, WIDE>), lds);
  if (e != hipSuccess) return e;
  k_window<T, P, WIDE><<<dim3((unsigned)(a.N / BLOCK + a.n), a.H), WNT, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T, int P, bool WIDE>
hipError_t backward_as(const WinArgs &a, hipStream_t s) {
  const long long blocks = a.N / BLOCK_OF<T> + a.n;
  constexpr int each = WNT / (P / PER<T>);
  const long long rows = (a.N * a.H + each - 1) / each;
  k_window_delta<T, P, WIDE><<<(unsigned)(rows < 8192 ? rows : 8192), WNT, 0, s>>>(a);
  if constexpr (sizeof(T) == 2) {
    constexpr int lds = WALK<T, P>;
    const hipError_t e =
        allow_lds(reinterpret_cast<const void *>(k_window_sums<T, P, WIDE>), lds);
    if (e != hipSuccess) return e;
    const int every = a.window + a.sinks <= FEW;
    k_window_sums<T, P, WIDE>
        <<<dim3((unsigned)(every ? blocks : a.n), a.H), WNT, lds, s>>>(a, every);
  }
  const long long pieces = a.part ? (a.N / a.unit + a.n) * a.G * ((a.sinks + 15) / 16) : 0;
  const long long all = blocks * (a.G + a.H) + pieces;
  const long long across = all < MAX_BLOCKS ? all : MAX_BLOCKS;
  if (blocks > MAX_BLOCKS || all > across * MAX_ACROSS) return hipErrorInvalidValue;
  constexpr int keys = WALK<T, P> > WALK_BACK<T, P> ? WALK<T, P> : WALK_BACK<T, P>;
  const int lds = pieces && WALK_UNIT<T, P> > keys ? WALK_UNIT<T, P> : keys;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(k_window_back<T, P, WIDE>), lds);
  if (e != hipSuccess) return e;
  k_window_back<T, P, WIDE>
      <<<dim3((unsigned)across, (unsigned)((all + across - 1) / across)), WNT, lds, s>>>(a);
  if (a.part)
    k_window_first<T, P>
        <<<dim3(a.n, a.G, a.sinks < 1024 ? a.sinks : 1024), P, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int P, bool WIDE>
hipError_t step_as(const WinStepArgs &a, hipStream_t s) {
  const int E = a.H / a.G;
  k_window_step<T, P, WIDE>
      <<<dim3((unsigned)a.n, a.G * ((E + 15) / 16), a.splits), WNT, 0, s>>>(a);
  if (a.splits > 1) k_window_join<T, P><<<dim3((unsigned)a.n, a.H), P, 0, s>>>(a);
  return hipGetLastError();
}

// f<T, P, WIDE>() of a type, a width and an alignment.
#define FOR_FORM(f, ...)                                                                     \
  (type == FST_F32   ? D <= 64 ? wide ? f<float, 64, true>(__VA_ARGS__)                      \
                                      : f<float, 64, false>(__VA_ARGS__)                     \
                               : wide ? f<float, 128, true>(__VA_ARGS__)                     \
                                      : f<float, 128, false>(__VA_ARGS__)                    \
   : type == FST_F16 ? D <= 64 ? wide ? f<f16, 64, true>(__VA_ARGS__)                        \
                                      : f<f16, 64, false>(__VA_ARGS__)                       \
                               : wide ? f<f16, 128, true>(__VA_ARGS__)                       \
                                      : f<f16, 128, false>(__VA_ARGS__)                      \
                     : D <= 64 ? wide ? f<bf16, 64, true>(__VA_ARGS__)                       \
                                      : f<bf16, 64, false>(__VA_ARGS__)                      \
                               : wide ? f<bf16, 128, true>(__VA_ARGS__)                      \
                                      : f<bf16, 128, false>(__VA_ARGS__))

int padded(int D) { return D <= 64 ? 64 : 128; }

}  // namespace

hipError_t launch_window(const WinArgs &a, int type, hipStream_t s) {
  if (a.H > MAX_ACROSS || a.ks > MAX_STRIDE || a.vs > MAX_STRIDE) return hipErrorInvalidValue;
  const int D = a.D;
  const bool wide = wide_rows(type_bytes(type), D, {a.qs, a.ks, a.vs, a.os}, {a.q, a.k, a.v, a.o});
  return FOR_FORM(forward_as, a, s);
}

// (also without workspace: then `need` is all that is set)
hipError_t launch_window_grads(WinArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  if (a.H > MAX_ACROSS) return hipErrorInvalidValue;
  for (long long t : {a.qs, a.ks, a.vs, a.gys})
    if (t > MAX_STRIDE) return hipErrorInvalidValue;
  const int D = a.D;
  const size_t delta = ((size_t)a.N * a.H + 3) / 4 * 4;
  // (a sequence has to be longer than the window, and than a unit, for the queries of
  // its first frames to be cut; units give small calls 256 workgroups; many first
  // frames are workgroups enough)
  const long long unit = a.N * a.G / 256 / 128 * 128;
  a.unit = unit < 128 ? 128 : unit > 512 ? 512 : unit;
  const bool cut =
      a.sinks > 0 && a.sinks <= MAX_CUT && a.N > a.window && a.N > a.unit;
  const size_t first = cut ? (size_t)a.G * a.sinks * 2 * padded(D) : 0;
  const size_t own = (a.N / a.unit + 1) * first, part = (2 * a.N / a.unit + 1) * first;
  *need = (delta + own + part) * sizeof(float);
  if (!ws) return hipSuccess;
  a.delta = static_cast<float *>(ws);
  a.own = a.delta + delta;
  a.part = cut ? a.own + own : nullptr;
  const bool wide = wide_rows(type_bytes(type), D,
                              {a.qs, a.ks, a.vs, a.ys, a.gys, a.gqs, a.gks, a.gvs},
                              {a.q, a.k, a.v, a.y, a.gy, a.gq, a.gk, a.gv});
  return FOR_FORM(backward_as, a, s);
}

hipError_t launch_window_step(WinStepArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  const int D = a.D, E = a.H / a.G;
  const long long groups = (long long)a.G * ((E + 15) / 16);
  if (groups > MAX_ACROSS || a.H > MAX_ACROSS || a.n > MAX_BLOCKS) return hipErrorInvalidValue;
  // enough workgroups for the card, none with less than three tiles a wavefront: the
  // parts' join is a launch of its own (8 query and 2 key heads of 64, bf16, replayed:
  // one stream of 256 frames 7.6 us with parts of one tile, 6.3 in one piece; of 2,000
  // 14.5 with 16 parts, 11 with 4)
  const long long most = ((long long)a.sinks + a.window) / (96 * WNW);
  long long splits = (512 + a.n * groups - 1) / (a.n * groups);
  splits = splits < most ? splits : most > 1 ? most : 1;
  a.splits = (int)(splits < 64 ? splits : 64);
  *need = a.splits > 1
              ? (size_t)a.n * a.H * a.splits * (padded(D) + 4) * sizeof(float)
              : 0;
  if (!ws) return hipSuccess;
  a.part = static_cast<float *>(ws);
  const bool wide = wide_rows(type_bytes(type), D, {a.qs, a.ks, a.vs, a.ys, a.kcs, a.vcs},
                              {a.q, a.k, a.v, a.y, a.kc, a.vc});
  return FOR_FORM(step_as, a, s);
}

hipError_t launch_window_fill(const WinFillArgs &a, int type, hipStream_t s) {
  const long long L = (long long)a.sinks + a.window;
  for (int s0 = 0; s0 < a.n; s0 += MAX_ACROSS) {
    WinFillArgs b = a;
    b.first = s0;
    const int n = a.n - s0 < MAX_ACROSS ? a.n - s0 : MAX_ACROSS;
    const dim3 grid((unsigned)(L < 1024 ? L : 1024), n);
    if (type == FST_F32)
      k_window_fill<float><<<grid, WNT, 0, s>>>(b);
    else if (type == FST_F16)
      k_window_fill<f16><<<grid, WNT, 0, s>>>(b);
    else
      k_window_fill<bf16><<<grid, WNT, 0, s>>>(b);
  }
  return hipGetLastError();
}

}  // namespace fstc
