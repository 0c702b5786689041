// Gated linear recurrence over ragged sequences (fst_recurrence_run, its
// gradients and its single step).
//
//   f = sigmoid(u),  h_t = f_t h_(t-1) + (1 - f_t) x_t,  y_t = h_t
//
// Steps of a channel compose as affine maps h -> F h + H, and maps compose
// associatively: (F2, H2) after (F1, H1) is (F1 F2, F2 H1 + H2).  A wavefront
// takes CHUNK consecutive steps of 64 lanes' channels in registers, the
// wavefronts of a workgroup take consecutive chunks (a tile), their maps meet
// in LDS, and every input is read once.  The gradient runs the same maps the
// other way (D_t = gy_t + f_(t+1) D_(t+1): the carry f_t D_t into the step
// before is R + F carry with the same F) next to the states, which it
// recomputes from float32 states saved every 64 steps: five streams of
// the activations' type instead of six, and no state rounded to it.
#include <initializer_list>

#include "layers.h"

namespace fstc {

namespace {

constexpr int CHUNK = 8;  // steps of a wavefront

typedef _Float16 f16;
typedef __bf16 bf16;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(f16 v) { return (float)v; }
__device__ __forceinline__ float to_float(bf16 v) { return (float)v; }

// V consecutive channels of a lane.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
  T v[V];
};

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load(const void *p, long long i) {
  return *reinterpret_cast<const Pack<T, V> *>(static_cast<const T *>(p) + i);
}
template <typename T, int V>
__device__ __forceinline__ void store(void *p, long long i, const float (&v)[V]) {
  Pack<T, V> o;
#pragma unroll
  for (int c = 0; c < V; ++c) o.v[c] = (T)v[c];
  *reinterpret_cast<Pack<T, V> *>(static_cast<T *>(p) + i) = o;
}

// keep = sigmoid(u) and add = 1 - sigmoid(u), neither a difference of near
// numbers: keep = 1 / (1 + e), add = e keep with e = exp(-u).
//
// float32: from exp(-|u|) = 2^t (1 + r ln 2), with t = fl(-|u| log2 e) and r
// what t lost, so that large |u| keep 32 bits' precision.
__device__ __forceinline__ void gate(float u, float &keep, float &add) {
  const float a = -fabsf(u);
  const float L = 1.44269502162933349609375f, l = 1.925963033500e-8f;
  const float t = a * L;
  const float r = fmaf(a, l, fmaf(a, L, -t));
  float e = __builtin_amdgcn_exp2f(t);
  // (r is no number where u is infinite: there e = 0)
  e = fmaf(e, a > -200.0f ? r * 0.693147182464599609375f : 0.0f, e);
  const float big = __builtin_amdgcn_rcpf(1.0f + e);
  const float small = e * big;
  keep = u >= 0.0f ? big : small;
  add = u >= 0.0f ? small : big;
}
// 16-bit gates: e to within |u| 2^-24 of itself, far inside a 16-bit number,
// and half the instructions (the vector units, not memory, bounded these
// kernels: 0.37 ms for the gradients of 64 x 1500 x 1024, 0.29 so).  e is at
// most 2^126, so that add stays a number where keep vanishes, and a NaN stays
// one: this minimum, unlike fminf, passes it on (a comparison and a choice
// instead take 1 to 3 % longer in the scans).
__device__ __forceinline__ void gate16(float u, float &keep, float &add) {
  const float all = __builtin_amdgcn_exp2f(u * -1.44269502162933349609375f);
  const float e = __builtin_elementwise_minimum(all, 0x1p126f);
  keep = __builtin_amdgcn_rcpf(1.0f + e);
  add = e * keep;
}
__device__ __forceinline__ void gate(f16 u, float &keep, float &add) {
  gate16((float)u, keep, add);
}
__device__ __forceinline__ void gate(bf16 u, float &keep, float &add) {
  gate16((float)u, keep, add);
}

// What a workgroup works on: steps [lo, hi) of a sequence of `len` rows from
// row b, the first step's row `first` and each next one `step` rows on.
struct Unit {
  int s;
  long long b, len, lo, hi;
  long long first, step;
};

__device__ __forceinline__ long long clamped(long long v, long long lo, long long hi) {
  return v < lo ? lo : v > hi ? hi : v;
}

// First of the rows that sequence s, from row b, has in an array with a row
// for every `per` steps of a sequence: ceil(len / per) rows fit before the
// next sequence's, as floor(b / per) + s grows by at least that.
__device__ __forceinline__ long long rows_before(long long b, int s, long long per) {
  return b / per + s;
}

// The unit of workgroup k: a whole sequence, or (a.unit steps each) the
// sequence that owns row k of an array with a row for every unit.  All of it
// lies inside [0, N) whatever the offsets hold.  False: there is none.
__device__ __forceinline__ bool unit_of(const RecArgs &a, long long k, Unit &u) {
  int s = (int)k;
  if (a.unit) {
    int lo = 0, hi = a.n - 1;  // the last s with rows_before <= k
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (rows_before(clamped(a.off[mid], 0, a.N), mid, a.unit) <= k)
        lo = mid;
      else
        hi = mid - 1;
    }
    s = lo;
  }
  u.s = s;
  u.b = clamped(a.off[s], 0, a.N);
  u.len = clamped(a.off[s + 1], u.b, a.N) - u.b;
  u.lo = 0;
  u.hi = u.len;
  if (a.unit) {
    const long long j = k - rows_before(u.b, s, a.unit);
    u.lo = j * a.unit;
    if (j < 0 || (j > 0 && u.lo >= u.len)) return false;
    u.hi = u.lo + a.unit < u.len ? u.lo + a.unit : u.len;
  }
  u.step = a.reverse ? -1 : 1;
  u.first = a.reverse ? u.b + u.len - 1 : u.b;
  return true;
}

// Rows of a chunk's steps: i counts from the sequence's start, and steps past
// its end read its last row (what they read is not used).
template <typename T, int V>
__device__ __forceinline__ void fetch(Pack<T, V> (&r)[CHUNK], const void *p, long long stride,
                                      const Unit &u, long long i, int d) {
#pragma unroll
  for (int k = 0; k < CHUNK; ++k) {
    const long long j = i + k < u.len ? i + k : u.len - 1;
    r[k] = load<T, V>(static_cast<const T *>(p) + (u.first + j * u.step) * stride, d);
  }
}

// The maps (F, H) of a sequence's units before this one, in order, or (back)
// after it, last first, applied to v.  The wavefronts share them out.
template <int V, int NW>
__device__ __forceinline__ void carry_in(const RecArgs &a, const Unit &u, bool back, int lane,
                                         int w, int d, float2 (&s_map)[NW][V][WAVE],
                                         float (&v)[V]) {
  const long long base = rows_before(u.b, u.s, a.unit), j = u.lo / a.unit;
  const long long n = back ? (u.len - 1) / a.unit - j : j;
  const long long share = (n + NW - 1) / NW;
  const long long k0 = w * share, k1 = k0 + share < n ? k0 + share : n;
  float F[V], H[V];
#pragma unroll
  for (int c = 0; c < V; ++c) F[c] = 1.0f, H[c] = 0.0f;
#pragma unroll 4
  for (long long k = k0; k < k1; ++k) {
    const long long q = back ? j + n - k : k;
    const float2 *m = a.agg + (base + q) * a.D + d;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      F[c] *= m[c].x;
      H[c] = fmaf(m[c].x, H[c], m[c].y);
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) s_map[w][c][lane] = make_float2(F[c], H[c]);
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NW; ++q)
#pragma unroll
    for (int c = 0; c < V; ++c) v[c] = fmaf(s_map[q][c][lane].x, v[c], s_map[q][c][lane].y);
  __syncthreads();
}

// ---------------------------------------------------------------------------
// maps of units (the split form's first pass)
// ---------------------------------------------------------------------------

// Forward: (F, H) of the states; back: (F, R) of the gradient's carry.  Bound by
// memory: reads two streams and writes next to nothing (40,000 x 512 bf16, 157
// units by 4: 18 us, 4.6 TB/s).
template <typename T, int V, int NW, bool BACK>
__global__ __launch_bounds__(NW *WAVE) void k_rec_units(RecArgs a) {
  __shared__ float2 s_map[NW][V][WAVE];
  const int lane = threadIdx.x & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int dt = (blockIdx.y * WAVE + lane) * V;
  const bool there = dt < a.D;
  const int d = there ? dt : 0;
  Unit u;
  if (!unit_of(a, blockIdx.x, u) || u.len == 0) return;
  // a contiguous share of the unit's chunks for each wavefront
  const long long share = a.unit / CHUNK / NW * CHUNK;
  const long long i0 = u.lo + w * share;
  const long long i1 = i0 + share < u.hi ? i0 + share : u.hi;
  const void *p = BACK ? a.gy : a.x;
  const long long ps = BACK ? a.gys : a.xs;
  float F[V], H[V];
#pragma unroll
  for (int c = 0; c < V; ++c) F[c] = 1.0f, H[c] = 0.0f;
  if (i0 < i1) {
    const long long n = (i1 - i0 + CHUNK - 1) / CHUNK;
    Pack<T, V> pr[CHUNK], ur[CHUNK];
    fetch<T, V>(pr, p, ps, u, BACK ? i0 + (n - 1) * CHUNK : i0, d);
    fetch<T, V>(ur, a.u, a.us, u, BACK ? i0 + (n - 1) * CHUNK : i0, d);
    for (long long q = 0; q < n; ++q) {
      const long long i = i0 + (BACK ? n - 1 - q : q) * CHUNK;
      float f[CHUNK][V], v[CHUNK][V];
#pragma unroll
      for (int k = 0; k < CHUNK; ++k) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          float g;
          gate(ur[k].v[c], f[k][c], g);
          v[k][c] = to_float(pr[k].v[c]);
          if (!BACK) v[k][c] *= g;
        }
      }
      if (i + CHUNK > i1) {  // past the end: steps that change nothing
#pragma unroll
        for (int k = 0; k < CHUNK; ++k)
          if (i + k >= i1)
#pragma unroll
            for (int c = 0; c < V; ++c) f[k][c] = 1.0f, v[k][c] = 0.0f;
      }
      if (q + 1 < n) {
        fetch<T, V>(pr, p, ps, u, BACK ? i - CHUNK : i + CHUNK, d);
        fetch<T, V>(ur, a.u, a.us, u, BACK ? i - CHUNK : i + CHUNK, d);
      }
#pragma unroll
      for (int kk = 0; kk < CHUNK; ++kk) {
        const int k = BACK ? CHUNK - 1 - kk : kk;
#pragma unroll
        for (int c = 0; c < V; ++c) {
          H[c] = BACK ? f[k][c] * (H[c] + v[k][c]) : fmaf(f[k][c], H[c], v[k][c]);
          F[c] *= f[k][c];
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) s_map[w][c][lane] = make_float2(F[c], H[c]);
  __syncthreads();
  if (w || !there) return;
#pragma unroll
  for (int q = 1; q < NW; ++q) {
    const int k = BACK ? NW - 1 - q : q;
#pragma unroll
    for (int c = 0; c < V; ++c) {
      if (q == 1) {
        F[c] = s_map[BACK ? NW - 1 : 0][c][lane].x;
        H[c] = s_map[BACK ? NW - 1 : 0][c][lane].y;
      }
      const float2 m = s_map[k][c][lane];
      F[c] *= m.x;
      H[c] = fmaf(m.x, H[c], m.y);
    }
  }
#pragma unroll
  for (int c = 0; c < V; ++c) a.agg[(long long)blockIdx.x * a.D + d + c] = make_float2(F[c], H[c]);
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// A workgroup walks its unit tile by tile: from each chunk's map and the state
// before the tile every wavefront knows its first state.  Bound by memory (64
// sequences of up to 2000 x 1024 bf16, 1500 on average: 146 us, 4.1 TB/s of three
// streams, although the shorter sequences' workgroups end first; a large copy
// reaches 5.0), by the barrier and the loads of each tile where there are few
// workgroups (6 sequences of up to 211 x 333 float32: 11 us, 36 workgroups).
template <typename T, int V, int NW>
__global__ __launch_bounds__(NW *WAVE) void k_rec_forward(RecArgs a) {
  __shared__ float2 s_map[2][NW][V][WAVE];
  const int lane = threadIdx.x & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int dt = (blockIdx.y * WAVE + lane) * V;
  const bool there = dt < a.D;
  const int d = there ? dt : 0;  // (idle lanes read where others do, and write nothing)
  Unit u;
  if (!unit_of(a, blockIdx.x, u)) return;
  float h[V];
#pragma unroll
  for (int c = 0; c < V; ++c) h[c] = a.state ? a.state[(long long)u.s * a.D + d + c] : 0.0f;
  if (u.lo > 0) carry_in<V, NW>(a, u, false, lane, w, d, s_map[0], h);
  if (u.len > 0) {
    constexpr int TILE = NW * CHUNK;
    float *saved =
        a.saved ? a.saved + rows_before(u.b, u.s, REC_SAVE) * a.D + d : nullptr;
    Pack<T, V> xr[CHUNK], ur[CHUNK];
    fetch<T, V>(xr, a.x, a.xs, u, u.lo + w * CHUNK, d);
    fetch<T, V>(ur, a.u, a.us, u, u.lo + w * CHUNK, d);
    int par = 0;
    for (long long i0 = u.lo; i0 < u.hi; i0 += TILE, par ^= 1) {
      const long long i = i0 + w * CHUNK;
      // the chunk's states from a zero state, and the products of its gates
      float hl[CHUNK][V], fl[CHUNK][V];
#pragma unroll
      for (int k = 0; k < CHUNK; ++k) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          float g;
          gate(ur[k].v[c], fl[k][c], g);
          hl[k][c] = g * to_float(xr[k].v[c]);
        }
      }
      if (i + CHUNK > u.hi) {  // past the end: steps that change nothing
#pragma unroll
        for (int k = 0; k < CHUNK; ++k)
          if (i + k >= u.hi)
#pragma unroll
            for (int c = 0; c < V; ++c) fl[k][c] = 1.0f, hl[k][c] = 0.0f;
      }
#pragma unroll
      for (int k = 1; k < CHUNK; ++k)
#pragma unroll
        for (int c = 0; c < V; ++c) {
          hl[k][c] = fmaf(fl[k][c], hl[k - 1][c], hl[k][c]);
          fl[k][c] *= fl[k - 1][c];
        }
      if (i0 + TILE < u.hi) {
        fetch<T, V>(xr, a.x, a.xs, u, i + TILE, d);
        fetch<T, V>(ur, a.u, a.us, u, i + TILE, d);
      }
#pragma unroll
      for (int c = 0; c < V; ++c)
        s_map[par][w][c][lane] = make_float2(fl[CHUNK - 1][c], hl[CHUNK - 1][c]);
      // one barrier a tile: who writes this half again has passed the next
      // tile's, which all reach after reading it
      __syncthreads();
      float in[V];
#pragma unroll
      for (int j = 0; j < NW; ++j) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          if (j == w) in[c] = h[c];
          const float2 m = s_map[par][j][c][lane];
          h[c] = fmaf(m.x, h[c], m.y);
        }
      }
      if (there) {
        if (saved && i % REC_SAVE == 0 && i < u.hi) {
#pragma unroll
          for (int c = 0; c < V; ++c) saved[i / REC_SAVE * a.D + c] = in[c];
        }
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
          if (i + k < u.hi) {
            float y[V];
#pragma unroll
            for (int c = 0; c < V; ++c) y[c] = fmaf(fl[k][c], in[c], hl[k][c]);
            store<T, V>(static_cast<T *>(a.y) + (u.first + (i + k) * u.step) * a.ys, d, y);
          }
        }
      }
    }
  }
  if (there && w == 0 && a.last && u.hi == u.len) {
#pragma unroll
    for (int c = 0; c < V; ++c) a.last[(long long)u.s * a.D + d + c] = h[c];
  }
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------

// The same from the last tile to the first, with two maps a chunk: its states
// again (from the saved one before its 64 steps), and the carry.  Bound as the
// forward pass is (64 sequences of up to 2000 x 1024 bf16: 254 us, 3.9 TB/s of
// five streams; 6 of up to 211 x 333 float32: 14 us).
template <typename T, int V, int NW>
__global__ __launch_bounds__(NW *WAVE) void k_rec_backward(RecArgs a) {
  __shared__ float2 s_map[2][NW][V][WAVE];  // (F, H) of each chunk
  __shared__ float s_back[2][NW][V][WAVE];  // R of each chunk
  const int lane = threadIdx.x & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int dt = (blockIdx.y * WAVE + lane) * V;
  const bool there = dt < a.D;
  const int d = there ? dt : 0;
  Unit u;
  if (!unit_of(a, blockIdx.x, u)) return;
  float carry[V];
#pragma unroll
  for (int c = 0; c < V; ++c)
    carry[c] = a.glast ? a.glast[(long long)u.s * a.D + d + c] : 0.0f;
  if (u.hi < u.len) carry_in<V, NW>(a, u, true, lane, w, d, s_map[0], carry);
  if (u.len > 0) {
    constexpr int TILE = NW * CHUNK;
    constexpr int PER = REC_SAVE / CHUNK;
    const float *saved = a.saved + rows_before(u.b, u.s, REC_SAVE) * a.D + d;
    const long long top = u.lo + (u.hi - u.lo - 1) / TILE * TILE;
    Pack<T, V> xr[CHUNK], ur[CHUNK], gr[CHUNK];
    fetch<T, V>(xr, a.x, a.xs, u, top + w * CHUNK, d);
    fetch<T, V>(ur, a.u, a.us, u, top + w * CHUNK, d);
    fetch<T, V>(gr, a.gy, a.gys, u, top + w * CHUNK, d);
    int par = 0;
    for (long long i0 = top; i0 >= u.lo; i0 -= TILE, par ^= 1) {
      const long long i = i0 + w * CHUNK;
      float h[V];  // the state entering the 64 steps that hold this chunk
#pragma unroll
      for (int c = 0; c < V; ++c) h[c] = i < u.hi ? saved[i / REC_SAVE * a.D + c] : 0.0f;
      float f[CHUNK][V], g[CHUNK][V], x[CHUNK][V], D[CHUNK][V];
#pragma unroll
      for (int k = 0; k < CHUNK; ++k) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          gate(ur[k].v[c], f[k][c], g[k][c]);
          x[k][c] = to_float(xr[k].v[c]);
          D[k][c] = to_float(gr[k].v[c]);
        }
      }
      if (i + CHUNK > u.hi) {  // past the end: steps that change nothing
#pragma unroll
        for (int k = 0; k < CHUNK; ++k)
          if (i + k >= u.hi)
#pragma unroll
            for (int c = 0; c < V; ++c)
              f[k][c] = 1.0f, g[k][c] = 0.0f, x[k][c] = 0.0f, D[k][c] = 0.0f;
      }
      if (i0 > u.lo) {
        fetch<T, V>(xr, a.x, a.xs, u, i - TILE, d);
        fetch<T, V>(ur, a.u, a.us, u, i - TILE, d);
        fetch<T, V>(gr, a.gy, a.gys, u, i - TILE, d);
      }
#pragma unroll
      for (int c = 0; c < V; ++c) {
        float F = 1.0f, H = 0.0f, R = 0.0f;
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
          F *= f[k][c];
          H = fmaf(f[k][c], H, g[k][c] * x[k][c]);
          R = f[CHUNK - 1 - k][c] * (R + D[CHUNK - 1 - k][c]);
        }
        s_map[par][w][c][lane] = make_float2(F, H);
        s_back[par][w][c][lane] = R;
      }
      __syncthreads();
      float in[V];
#pragma unroll
      for (int j = NW - 1; j >= 0; --j) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          if (j == w) in[c] = carry[c];
          const float2 m = s_map[par][j][c][lane];
          carry[c] = fmaf(m.x, carry[c], s_back[par][j][c][lane]);
          // (ascending: chunk NW - 1 - j, of the 64 steps before this one)
          const int q = NW - 1 - j;
          if (q / PER == w / PER && q < w) {
            const float2 o = s_map[par][q][c][lane];
            h[c] = fmaf(o.x, h[c], o.y);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < V; ++c) {
#pragma unroll
        for (int k = CHUNK - 1; k >= 0; --k) {
          D[k][c] += in[c];
          in[c] = f[k][c] * D[k][c];
        }
      }
      if (there) {
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
          if (i + k < u.hi) {
            float gx[V], gu[V];
#pragma unroll
            for (int c = 0; c < V; ++c) {
              gx[c] = g[k][c] * D[k][c];
              gu[c] = D[k][c] * (h[c] - x[k][c]) * (f[k][c] * g[k][c]);
              h[c] = fmaf(f[k][c], h[c], g[k][c] * x[k][c]);
            }
            const long long r = u.first + (i + k) * u.step;
            store<T, V>(static_cast<T *>(a.gx) + r * a.gxs, d, gx);
            store<T, V>(static_cast<T *>(a.gu) + r * a.gus, d, gu);
          }
        }
      }
    }
  }
  if (there && w == 0 && a.gstate && u.lo == 0) {
#pragma unroll
    for (int c = 0; c < V; ++c) a.gstate[(long long)u.s * a.D + d + c] = carry[c];
  }
}

// ---------------------------------------------------------------------------
// one step of many streams
// ---------------------------------------------------------------------------

// Bound by memory (4096 x 1024 f16: 11.4 us, 5.1 TB/s), or by its launch (8 x 256:
// 2.2 us); four channels a lane, so that a wavefront's states are 1 KiB loads.
template <typename T, int V>
__global__ __launch_bounds__(NT) void k_rec_step(StepArgs a) {
  const int per = (a.D + V - 1) / V;
  for (long long i = (long long)blockIdx.x * NT + threadIdx.x; i < a.n * per;
       i += (long long)gridDim.x * NT) {
    const long long r = i / per;
    const int d = (int)(i - r * per) * V;
    float y[V];
    const long long q = a.slot ? a.slot[r] : r;
    const bool there = q >= 0 && q < a.slots;
#pragma unroll
    for (int c = 0; c < V; ++c) y[c] = 0.0f;
    if (there) {
      const Pack<T, V> x = load<T, V>(a.x, r * a.xs + d);
      const Pack<T, V> u = load<T, V>(a.u, r * a.us + d);
      const Pack<float, V> h = load<float, V>(a.in, q * a.D + d);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        float f, g;
        gate(u.v[c], f, g);
        y[c] = fmaf(f, h.v[c], g * to_float(x.v[c]));
      }
      store<float, V>(a.out, q * a.D + d, y);
    }
    store<T, V>(a.y, r * a.ys + d, y);
  }
}

// Whether lanes may take V channels at once: widths, strides and addresses
// are multiples of V elements.
template <int V>
bool packs(int D, size_t e, std::initializer_list<long long> strides,
           std::initializer_list<const void *> ptrs) {
  if (D % V) return false;
  for (long long t : strides)
    if (t % V) return false;
  for (const void *p : ptrs)
    if ((uintptr_t)p % (V * e)) return false;
  return true;
}

constexpr int NW = 8;  // wavefronts of a workgroup

// Workgroups side by side, of 64 lanes' channels each; a launch takes MAX_ACROSS.
constexpr long long MAX_ACROSS = 65535;
long long across(const RecArgs &a, int v) { return (a.D + v * WAVE - 1ll) / (v * WAVE); }

template <typename T, int V>
void forward_as(const RecArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(a.unit ? a.N / a.unit + a.n : a.n), (unsigned)across(a, V));
  if (a.unit) k_rec_units<T, V, NW, false><<<grid, NW * WAVE, 0, s>>>(a);
  k_rec_forward<T, V, NW><<<grid, NW * WAVE, 0, s>>>(a);
}
template <typename T, int V>
void backward_as(const RecArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(a.unit ? a.N / a.unit + a.n : a.n), (unsigned)across(a, V));
  if (a.unit) k_rec_units<T, V, NW, true><<<grid, NW * WAVE, 0, s>>>(a);
  k_rec_backward<T, V, NW><<<grid, NW * WAVE, 0, s>>>(a);
}

// How a call is laid out: channels a lane takes, and steps of a unit (0: a
// sequence is one workgroup's for every 64 lanes of channels).
//
// Two channels a lane halve the workgroups: better from 256 of them on (64
// sequences of 50 x 512 bf16: 5.5 us, one channel 6.8; 32 of 500: 256 with one
// 18.5 us, 128 with two 21.5).  Up to 128 workgroups of sequences longer than
// 256 steps leave the card idle: split into units over about 768 workgroups,
// whose maps are found in a pass of their own, they read their inputs twice
// (40,000 x 512: 49 us forward, unsplit 1,028; 4 of 2000 x 512: 17.6 and 56; 16
// of 1000: 31 both ways; 32 of 500: 32 and 18.5, unsplit).  The lengths lie on the
// device, so their average decides: one of 40,000 x 512 among 16 sequences is cut (53
// us), among 64 it is not and takes as long as alone in one piece (1.27 ms with 63 of
// 100 steps beside it).
struct Layout {
  int v;
  long long unit;
};
Layout layout(const RecArgs &a, bool pairs) {
  const long long one = (a.D + WAVE - 1) / WAVE, two = (a.D + 2 * WAVE - 1) / (2 * WAVE);
  if (a.n * one <= 128 && a.N / a.n > 256) {
    constexpr long long tile = NW * CHUNK;
    const long long steps = a.N * (pairs ? two : one) / 768;
    return {pairs ? 2 : 1, steps <= tile ? tile : (steps + tile - 1) / tile * tile};
  }
  return {pairs && a.n * two >= 256 ? 2 : 1, 0};
}

}  // namespace

// (also without workspace: then `need` is all that is set)
hipError_t launch_recurrence(RecArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  const Layout l = layout(a, type != FST_F32 &&
                                 packs<2>(a.D, 2, {a.xs, a.us, a.ys}, {a.x, a.u, a.y}));
  const bool two = l.v == 2;
  if (across(a, l.v) > MAX_ACROSS) return hipErrorInvalidValue;
  a.unit = l.unit;
  *need = a.unit ? (size_t)(a.N / a.unit + a.n) * a.D * sizeof(float2) : 0;
  if (!ws) return hipSuccess;
  a.agg = static_cast<float2 *>(ws);
  if (type == FST_F32) {
    forward_as<float, 1>(a, s);
  } else if (type == FST_F16) {
    two ? forward_as<f16, 2>(a, s) : forward_as<f16, 1>(a, s);
  } else {
    two ? forward_as<bf16, 2>(a, s) : forward_as<bf16, 1>(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_recurrence_grads(RecArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  const Layout l = layout(a, type != FST_F32 && packs<2>(a.D, 2, {a.xs, a.us, a.gys, a.gxs, a.gus},
                                                         {a.x, a.u, a.gy, a.gx, a.gu}));
  const bool two = l.v == 2;
  if (across(a, l.v) > MAX_ACROSS) return hipErrorInvalidValue;
  a.unit = l.unit;
  *need = a.unit ? (size_t)(a.N / a.unit + a.n) * a.D * sizeof(float2) : 0;
  if (!ws) return hipSuccess;
  a.agg = static_cast<float2 *>(ws);
  if (type == FST_F32) {
    backward_as<float, 1>(a, s);
  } else if (type == FST_F16) {
    two ? backward_as<f16, 2>(a, s) : backward_as<f16, 1>(a, s);
  } else {
    two ? backward_as<bf16, 2>(a, s) : backward_as<bf16, 1>(a, s);
  }
  return hipGetLastError();
}

template <typename T, int V>
static void step_as(const StepArgs &a, hipStream_t s) {
  const long long blocks = (a.n * ((a.D + V - 1) / V) + NT - 1) / NT;
  k_rec_step<T, V><<<(unsigned)(blocks < 65536 ? blocks : 65536), NT, 0, s>>>(a);
}

hipError_t launch_recurrence_step(const StepArgs &a, int type, hipStream_t s) {
  const size_t e = type_bytes(type);
  const bool four = packs<4>(a.D, e, {a.xs, a.us, a.ys}, {a.x, a.u, a.y}) &&
                    packs<4>(a.D, 4, {}, {a.in, a.out});
  if (type == FST_F32) {
    four ? step_as<float, 4>(a, s) : step_as<float, 1>(a, s);
  } else if (type == FST_F16) {
    four ? step_as<f16, 4>(a, s) : step_as<f16, 1>(a, s);
  } else {
    four ? step_as<bf16, 4>(a, s) : step_as<bf16, 1>(a, s);
  }
  return hipGetLastError();
}

}  // namespace fstc
