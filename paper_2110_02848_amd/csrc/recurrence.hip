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

constexpr int CHUNK = 16;  // steps of a wavefront

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

// keep = sigmoid(u) and add = 1 - sigmoid(u), each from the exponential of
// -|u| so that neither is a difference of near numbers.  exp(-|u|) = 2^t (1 +
// r ln 2) with t = fl(-|u| log2 e) and r what t lost, so that large |u| keep
// 32 bits' precision.
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

// The sequence's rows: [b, b + len), inside [0, N) whatever the offsets hold.
__device__ __forceinline__ void bounds(const RecArgs &a, int s, long long &b, long long &len) {
  long long lo = a.off[s], hi = a.off[s + 1];
  lo = lo < 0 ? 0 : lo > a.N ? a.N : lo;
  hi = hi < lo ? lo : hi > a.N ? a.N : hi;
  b = lo;
  len = hi - lo;
}

// First of the saved rows of sequence s: ceil(len / 64) rows fit before the
// next sequence's, as floor(b / 64) + s grows by at least that.
__device__ __forceinline__ long long units_before(long long b, int s, int per) {
  return b / per + s;
}

template <bool REV>
__device__ __forceinline__ long long row_of(long long b, long long len, long long i) {
  return REV ? b + len - 1 - i : b + i;
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// One tile of NW chunks from step i0 of a sequence, its state `h` before the
// tile replaced by the one after it.
template <typename T, int V, int NW, bool REV>
struct Forward {
  Pack<T, V> xr[CHUNK], ur[CHUNK];

  __device__ __forceinline__ void fetch(const RecArgs &a, long long b, long long len,
                                        long long i0, int d) {
#pragma unroll
    for (int k = 0; k < CHUNK; ++k) {
      const long long i = i0 + k;
      if (i < len) {
        const long long r = row_of<REV>(b, len, i);
        xr[k] = load<T, V>(a.x, r * a.xs + d);
        ur[k] = load<T, V>(a.u, r * a.us + d);
      }
    }
  }

  // hl: states of the chunk's steps from a zero state, fl: products so far.
  __device__ __forceinline__ void local(long long len, long long i0, float (&hl)[CHUNK][V],
                                        float (&fl)[CHUNK][V]) {
    float F[V], H[V];
#pragma unroll
    for (int c = 0; c < V; ++c) F[c] = 1.0f, H[c] = 0.0f;
#pragma unroll
    for (int k = 0; k < CHUNK; ++k) {
      const bool on = i0 + k < len;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if (on) {
          float f, g;
          gate(to_float(ur[k].v[c]), f, g);
          F[c] *= f;
          H[c] = fmaf(f, H[c], g * to_float(xr[k].v[c]));
        }
        hl[k][c] = H[c];
        fl[k][c] = F[c];
      }
    }
  }
};

template <typename T, int V, int NW, bool REV>
__global__ __launch_bounds__(NW *WAVE) void k_rec_forward(RecArgs a) {
  __shared__ float2 s_map[2][NW][V][WAVE];
  const int lane = threadIdx.x & (WAVE - 1), w = threadIdx.x / WAVE;
  const int s = blockIdx.x;
  const int d = (blockIdx.y * WAVE + lane) * V;
  const bool there = d < a.D;
  long long b, len;
  bounds(a, s, b, len);
  const long long sv = units_before(b, s, REC_SAVE);
  float h[V];
#pragma unroll
  for (int c = 0; c < V; ++c)
    h[c] = there && a.state ? a.state[(long long)s * a.D + d + c] : 0.0f;
  const long long mylen = there ? len : 0;
  Forward<T, V, NW, REV> t;
  t.fetch(a, b, mylen, (long long)w * CHUNK, d);
  int par = 0;
  for (long long i0 = 0; i0 < len; i0 += NW * CHUNK, par ^= 1) {
    const long long ic = i0 + (long long)w * CHUNK;
    float hl[CHUNK][V], fl[CHUNK][V];
    t.local(mylen, ic, hl, fl);
    t.fetch(a, b, mylen, ic + NW * CHUNK, d);
#pragma unroll
    for (int c = 0; c < V; ++c)
      s_map[par][w][c][lane] = make_float2(fl[CHUNK - 1][c], hl[CHUNK - 1][c]);
    __syncthreads();  // (the other half of s_map is free: all have passed its readers' barrier)
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
    if (there && a.saved && ic % REC_SAVE == 0 && ic < len) {
#pragma unroll
      for (int c = 0; c < V; ++c) a.saved[(sv + ic / REC_SAVE) * a.D + d + c] = in[c];
    }
#pragma unroll
    for (int k = 0; k < CHUNK; ++k) {
      if (ic + k < mylen) {
        float y[V];
#pragma unroll
        for (int c = 0; c < V; ++c) y[c] = fmaf(fl[k][c], in[c], hl[k][c]);
        store<T, V>(a.y, row_of<REV>(b, len, ic + k) * a.ys + d, y);
      }
    }
  }
  if (there && w == 0 && a.last) {
#pragma unroll
    for (int c = 0; c < V; ++c) a.last[(long long)s * a.D + d + c] = h[c];
  }
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------

template <typename T, int V, int NW, bool REV>
__global__ __launch_bounds__(NW *WAVE) void k_rec_backward(RecArgs a) {
  __shared__ float2 s_map[2][NW][V][WAVE];  // (F, H) of each chunk
  __shared__ float s_back[2][NW][V][WAVE];  // R of each chunk
  const int lane = threadIdx.x & (WAVE - 1), w = threadIdx.x / WAVE;
  const int s = blockIdx.x;
  const int d = (blockIdx.y * WAVE + lane) * V;
  const bool there = d < a.D;
  long long b, len;
  bounds(a, s, b, len);
  const long long sv = units_before(b, s, REC_SAVE);
  const long long mylen = there ? len : 0;
  float carry[V];
#pragma unroll
  for (int c = 0; c < V; ++c)
    carry[c] = there && a.glast ? a.glast[(long long)s * a.D + d + c] : 0.0f;
  constexpr int TILE = NW * CHUNK;
  int par = 0;
  for (long long i0 = (len + TILE - 1) / TILE * TILE - TILE; i0 >= 0; i0 -= TILE, par ^= 1) {
    const long long ic = i0 + (long long)w * CHUNK;
    Pack<T, V> xr[CHUNK];
    float f[CHUNK][V], g[CHUNK][V], D[CHUNK][V];
#pragma unroll
    for (int k = 0; k < CHUNK; ++k) {
#pragma unroll
      for (int c = 0; c < V; ++c) {
        xr[k].v[c] = (T)0.0f;
        f[k][c] = 1.0f;
        g[k][c] = 0.0f;
        D[k][c] = 0.0f;
      }
      if (ic + k < mylen) {
        const long long r = row_of<REV>(b, len, ic + k);
        xr[k] = load<T, V>(a.x, r * a.xs + d);
        const Pack<T, V> u = load<T, V>(a.u, r * a.us + d);
        const Pack<T, V> y = load<T, V>(a.gy, r * a.gys + d);
#pragma unroll
        for (int c = 0; c < V; ++c) {
          gate(to_float(u.v[c]), f[k][c], g[k][c]);
          D[k][c] = to_float(y.v[c]);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float F = 1.0f, H = 0.0f, R = 0.0f;
#pragma unroll
      for (int k = 0; k < CHUNK; ++k) {
        F *= f[k][c];
        H = fmaf(f[k][c], H, g[k][c] * to_float(xr[k].v[c]));
      }
#pragma unroll
      for (int k = CHUNK - 1; k >= 0; --k) R = f[k][c] * (R + D[k][c]);
      s_map[par][w][c][lane] = make_float2(F, H);
      s_back[par][w][c][lane] = R;
    }
    // the state entering the 64 steps that hold this chunk
    float h[V];
    const long long is = ic / REC_SAVE;
#pragma unroll
    for (int c = 0; c < V; ++c) h[c] = ic < mylen ? a.saved[(sv + is) * a.D + d + c] : 0.0f;
    __syncthreads();
    float in[V];
#pragma unroll
    for (int j = NW - 1; j >= 0; --j) {
#pragma unroll
      for (int c = 0; c < V; ++c) {
        if (j == w) in[c] = carry[c];
        carry[c] = fmaf(s_map[par][j][c][lane].x, carry[c], s_back[par][j][c][lane]);
      }
    }
    constexpr int PER = REC_SAVE / CHUNK;
#pragma unroll
    for (int j = 0; j < PER - 1; ++j) {
      if (j < w % PER) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float2 m = s_map[par][w / PER * PER + j][c][lane];
          h[c] = fmaf(m.x, h[c], m.y);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
      float C = in[c];
#pragma unroll
      for (int k = CHUNK - 1; k >= 0; --k) {
        D[k][c] += C;
        C = f[k][c] * D[k][c];
      }
    }
#pragma unroll
    for (int k = 0; k < CHUNK; ++k) {
      if (ic + k < mylen) {
        float gx[V], gu[V];
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float x = to_float(xr[k].v[c]);
          gx[c] = g[k][c] * D[k][c];
          gu[c] = D[k][c] * (h[c] - x) * (f[k][c] * g[k][c]);
          h[c] = fmaf(f[k][c], h[c], g[k][c] * x);
        }
        const long long r = row_of<REV>(b, len, ic + k);
        store<T, V>(a.gx, r * a.gxs + d, gx);
        store<T, V>(a.gu, r * a.gus + d, gu);
      }
    }
  }
  if (there && w == 0 && a.gstate) {
#pragma unroll
    for (int c = 0; c < V; ++c) a.gstate[(long long)s * a.D + d + c] = carry[c];
  }
}

// ---------------------------------------------------------------------------
// one step of many streams
// ---------------------------------------------------------------------------

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
        gate(to_float(u.v[c]), f, g);
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

template <typename T, int V, int NW, bool REV>
void forward(const RecArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.n, (unsigned)((a.D + V * WAVE - 1) / (V * WAVE)));
  k_rec_forward<T, V, NW, REV><<<grid, NW * WAVE, 0, s>>>(a);
}

template <typename T, int V, int NW, bool REV>
void backward(const RecArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)a.n, (unsigned)((a.D + V * WAVE - 1) / (V * WAVE)));
  k_rec_backward<T, V, NW, REV><<<grid, NW * WAVE, 0, s>>>(a);
}

template <typename T, int V>
void forward_as(const RecArgs &a, bool reverse, hipStream_t s) {
  reverse ? forward<T, V, 8, true>(a, s) : forward<T, V, 8, false>(a, s);
}
template <typename T, int V>
void backward_as(const RecArgs &a, bool reverse, hipStream_t s) {
  reverse ? backward<T, V, 8, true>(a, s) : backward<T, V, 8, false>(a, s);
}

}  // namespace

hipError_t launch_recurrence(const RecArgs &a, int type, bool reverse, hipStream_t s) {
  const bool two = packs<2>(a.D, 2, {a.xs, a.us, a.ys}, {a.x, a.u, a.y});
  if (type == FST_F32) {
    forward_as<float, 1>(a, reverse, s);
  } else if (type == FST_F16) {
    two ? forward_as<f16, 2>(a, reverse, s) : forward_as<f16, 1>(a, reverse, s);
  } else {
    two ? forward_as<bf16, 2>(a, reverse, s) : forward_as<bf16, 1>(a, reverse, s);
  }
  return hipGetLastError();
}

hipError_t launch_recurrence_grads(const RecArgs &a, int type, bool reverse, hipStream_t s) {
  const bool two = packs<2>(a.D, 2, {a.xs, a.us, a.gys, a.gxs, a.gus},
                            {a.x, a.u, a.gy, a.gx, a.gu});
  if (type == FST_F32) {
    backward_as<float, 1>(a, reverse, s);
  } else if (type == FST_F16) {
    two ? backward_as<f16, 2>(a, reverse, s) : backward_as<f16, 1>(a, reverse, s);
  } else {
    two ? backward_as<bf16, 2>(a, reverse, s) : backward_as<bf16, 1>(a, reverse, s);
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
