// Queries and keys normalised head by head, scaled and rotated by position
// (fst_head_norms_run and its gradients).
//
//   z = x r,  r = (mean of x^2 over the head + eps)^(-1/2)
//   y = R(pos) (w z): pairs of numbers, as complex ones, times e^(i pos freq)
//
// Back, with h = w (R(-pos) dy):  dx = r (h - z mean(h z)),  dw = sum of
// (R(-pos) dy) z over rows and heads.  Angles are taken in 64 bits, as turns,
// and their whole part dropped before they are rounded: positions of any size
// keep 32 bits' precision.  A row's angles are found once for all its heads.
#include <initializer_list>

#include "tiles.h"

namespace fstc {

using namespace tile;

namespace {

constexpr int MAX_WIDTH = FST_NORM_MAX_WIDTH;

// cos and sin of pos * freq.
__device__ __forceinline__ float2 turn(int32_t pos, float freq) {
  double t = (double)freq * 0.15915494309189533577 * (double)pos;  // 1 / (2 pi)
  t -= rint(t);
  float s, c;
  sincospif(2.0f * (float)t, &s, &c);
  return make_float2(c, s);
}

// Whether a head's sum of squares, or numbers below it, may have left float32 (those of
// float16 numbers do not).
template <typename T>
__device__ __forceinline__ bool leaves(float sum, float eps) {
  if constexpr (std::is_same<T, f16>::value) return false;
  return !(sum < 0x1p120f) || (sum < 0x1p-100f && eps < 0x1p-100f);
}
// Such a head again, with a power of two, which is returned, times its numbers x and the
// root of eps: `sum` is that of their squares.  The head lies in `lanes` lanes.
template <int N>
__device__ __forceinline__ float brought_back(float (&x)[N], float &sum, float eps, int lanes) {
  float most = sqrtf(eps);
#pragma unroll
  for (int j = 0; j < N; ++j) most = fmaxf(most, fabsf(x[j]));
  for (int m = lanes / 2; m; m /= 2) most = fmaxf(most, __shfl_xor(most, m, WAVE));
  const float s = power_below(most, 0);
  sum = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    x[j] *= s;
    sum = fmaf(x[j], x[j], sum);
  }
  for (int m = lanes / 2; m; m /= 2) sum += __shfl_xor(sum, m, WAVE);
  return s;
}

// Heads of whole 16-byte groups.  A lane holds V = 16 bytes' pairs of a head, a[j] and
// b[j], of angle c V + j for lane c of the head's: with `PAIRS` 32 bytes that lie
// side by side, else two groups P apart (two side by side where nothing turns).
// A workgroup takes queries or keys, `rows` rows at a time, whose angles it finds once
// for all their heads.  Bound by memory: 16,000 rows of 16 + 4 heads of 64 bf16 take 20
// us (82 MB, 4.0 TB/s) and back 31 us (123 MB, 4.0 TB/s) with 512 workgroups a side,
// 37 with 1,024, 39 with 256.
template <typename T, bool PAIRS, bool BACK>
__global__ __launch_bounds__(NT) void k_norms_wide(NormArgs a, int rows, int lanes) {
  constexpr int V = PER<T>;
  extern __shared__ __attribute__((aligned(16))) float s_dyn[];
  float *s_cos = s_dyn, *s_sin = s_dyn + rows * a.P;  // [rows][P]
  const int c = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = NT / lanes;
  const bool on = c < a.D / (2 * V), turns = c * V < a.P;
  // where the lane's two groups of a head lie
  const int at0 = PAIRS || !turns ? 2 * V * c : V * c, at1 = PAIRS || !turns ? at0 + V : a.P + at0;
  const int o = blockIdx.y;
  const NormSide &sd = a.side[o];
  float add[2 * V] = {}, w[2 * V];  // BACK: sums for the weights
#pragma unroll
  for (int j = 0; j < 2 * V; ++j)
    w[j] = on && sd.heads ? sd.w[PAIRS ? at0 + j : (j < V ? at0 : at1 - V) + j] : 0.0f;
  // a head's numbers, on their way while the one before is worked on
  struct alignas(16) Group { T v[V]; } n0{}, n1{}, m0{}, m1{};
  const auto fetch = [&](long long r0, int it) {
    if (!on) return;
    const int row = it / sd.heads;
    const long long at = (long long)(it - row * sd.heads) * a.D;
    const T *x = static_cast<const T *>(sd.x) + (r0 + row) * sd.xs + at;
    n0 = *reinterpret_cast<const Group *>(x + at0);
    n1 = *reinterpret_cast<const Group *>(x + at1);
    if constexpr (BACK) {
      const T *g = static_cast<const T *>(sd.g) + (r0 + row) * sd.gs + at;
      m0 = *reinterpret_cast<const Group *>(g + at0);
      m1 = *reinterpret_cast<const Group *>(g + at1);
    }
  };
  for (long long r0 = (long long)blockIdx.x * rows; r0 < a.N; r0 += (long long)gridDim.x * rows) {
    const int count = (int)(a.N - r0 < rows ? a.N - r0 : rows);
    if (group < count * sd.heads) fetch(r0, group);
    __syncthreads();
    for (int i = threadIdx.x; i < count * a.P; i += NT) {
      const float2 t = turn(a.pos[r0 + i / a.P], a.freq[i % a.P]);
      s_cos[i] = t.x;
      s_sin[i] = BACK ? -t.y : t.y;
    }
    __syncthreads();
    for (int it = group; it < count * sd.heads; it += groups) {
      const int row = it / sd.heads;
      const long long at = (long long)(it - row * sd.heads) * a.D;
      const Group x0 = n0, x1 = n1, g0 = m0, g1 = m1;
      if (it + groups < count * sd.heads) fetch(r0, it + groups);
      float z[2 * V], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) {
        z[j] = (float)(j < V ? x0.v[j] : x1.v[j - V]);
        sum = fmaf(z[j], z[j], sum);
      }
      for (int m = lanes / 2; m; m /= 2) sum += __shfl_xor(sum, m, WAVE);
      float s = 1.0f;
      if (leaves<T>(sum, a.eps)) s = brought_back(z, sum, a.eps, lanes);
      const float r = 1.0f / sqrtf(sum / (float)a.D + a.eps * s * s);
      float y[2 * V];
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) {
        z[j] *= r;
        y[j] = BACK ? (float)(j < V ? g0.v[j] : g1.v[j - V]) : z[j] * w[j];
      }
      if (turns) {
        const float *cs = s_cos + row * a.P + c * V, *sn = s_sin + row * a.P + c * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int p = PAIRS ? 2 * j : j, q = PAIRS ? 2 * j + 1 : V + j;
          const float u = y[p], v = y[q];
          y[p] = fmaf(v, -sn[j], u * cs[j]);
          y[q] = fmaf(u, sn[j], v * cs[j]);
        }
      }
      if constexpr (BACK) {
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) {
          add[j] = fmaf(y[j], z[j], add[j]);
          y[j] *= w[j];
          dot = fmaf(y[j], z[j], dot);
        }
        for (int m = lanes / 2; m; m /= 2) dot += __shfl_xor(dot, m, WAVE);
        dot /= (float)a.D;
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) y[j] = r * s * (y[j] - z[j] * dot);
      }
      if (on) {
        Group y0, y1;
#pragma unroll
        for (int j = 0; j < V; ++j) y0.v[j] = (T)y[j], y1.v[j] = (T)y[V + j];
        T *out = static_cast<T *>(sd.y) + (r0 + row) * sd.ys + at;
        *reinterpret_cast<Group *>(out + at0) = y0;
        *reinterpret_cast<Group *>(out + at1) = y1;
      }
    }
  }
  if constexpr (BACK) {
    // lanes of a column in one wavefront, then the wavefronts
    float *s_w = s_dyn;  // [NWAVES][D]
    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) {
      float v = add[j];
      for (int m = lanes; m < WAVE; m *= 2) v += __shfl_xor(v, m, WAVE);
      if (lane < lanes && on)
        s_w[wave * a.D + (PAIRS ? at0 + j : (j < V ? at0 : at1 - V) + j)] = v;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.D; d += NT) {
      float v = 0.0f;
      for (int q = 0; q < NWAVES; ++q) v += s_w[q * a.D + d];
      a.part[((long long)blockIdx.x * 2 + o) * a.D + d] = v;
    }
  }
}

// Any heads, up to 64 E wide.  A wavefront takes one: lane l holds numbers l, l +
// 64, ..  BACK: gradients; a workgroup's sums for w go to a row of `part`, sides side by
// side.  Bound by the way from a head's numbers to its results (1,266 rows of 5 + 5
// heads of 43 f32: 6 us, back 10; 14 where the next head's loads had to wait).
template <typename T, int E, bool BACK>
__global__ __launch_bounds__(NT) void k_norms(NormArgs a) {
  extern __shared__ float s_dyn[];
  float2 *s_turn = reinterpret_cast<float2 *>(s_dyn);              // [P]
  const int lane = threadIdx.x & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  float *s_z = s_dyn + 2 * a.P + w * a.D;                          // a wavefront's [D]
  const int heads = a.side[0].heads + a.side[1].heads;
  float gw[2][E] = {};
  // a head's numbers, on their way while the one before is worked on
  T nx[E] = {}, ng[E] = {};
  const auto fetch = [&](long long row, int hh) {
    const int o = hh >= a.side[0].heads;
    const NormSide &sd = a.side[o];
    const long long at = (long long)(hh - (o ? a.side[0].heads : 0)) * a.D;
    const T *x = static_cast<const T *>(sd.x) + row * sd.xs + at;
    const T *g = static_cast<const T *>(sd.g) + row * sd.gs + at;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = e * WAVE + lane;
      if (d < a.D) {
        nx[e] = x[d];
        if constexpr (BACK) ng[e] = g[d];
      }
    }
  };
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x) {
    if (w < heads) fetch(row, w);
    __syncthreads();
    for (int i = threadIdx.x; i < a.P; i += NT) s_turn[i] = turn(a.pos[row], a.freq[i]);
    __syncthreads();
    for (int hh = w; hh < heads; hh += NWAVES) {
      const int o = hh >= a.side[0].heads;
      const NormSide &sd = a.side[o];
      const long long at = (long long)(hh - (o ? a.side[0].heads : 0)) * a.D;
      T *y = static_cast<T *>(sd.y) + row * sd.ys + at;
      float xv[E], gv[E], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xv[e] = (float)nx[e];
        gv[e] = (float)ng[e];
        sum = fmaf(xv[e], xv[e], sum);
      }
      if (hh + NWAVES < heads) fetch(row, hh + NWAVES);
#pragma unroll
      for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m, WAVE);
      float s = 1.0f;
      if (leaves<T>(sum, a.eps)) s = brought_back(xv, sum, a.eps, WAVE);
      const float r = 1.0f / sqrtf(sum / (float)a.D + a.eps * s * s);
      // what is turned meets its pair in LDS (a wavefront's own, in order)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * WAVE + lane;
        if (d < a.D) s_z[d] = BACK ? gv[e] : xv[e] * r * sd.w[d];
      }
      __builtin_amdgcn_wave_barrier();
      float t[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * WAVE + lane;
        t[e] = 0.0f;
        if (d >= a.D) continue;
        t[e] = s_z[d];
        if (d < 2 * a.P) {
          const int p = a.pairs ? d >> 1 : d < a.P ? d : d - a.P;
          const bool second = a.pairs ? d & 1 : d >= a.P;
          const float other = s_z[a.pairs ? d ^ 1 : second ? d - a.P : d + a.P];
          const float2 cs = s_turn[p];
          const float s = second != BACK ? cs.y : -cs.y;
          t[e] = fmaf(other, s, t[e] * cs.x);
        }
      }
      __builtin_amdgcn_wave_barrier();
      if constexpr (!BACK) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int d = e * WAVE + lane;
          if (d < a.D) y[d] = (T)t[e];
        }
      } else {
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int d = e * WAVE + lane;
          const float z = xv[e] * r;
          const float add = t[e] * z;
          gw[0][e] += o ? 0.0f : add;
          gw[1][e] += o ? add : 0.0f;
          t[e] *= d < a.D ? sd.w[d] : 0.0f;
          dot = fmaf(t[e], z, dot);
        }
#pragma unroll
        for (int m = 32; m; m >>= 1) dot += __shfl_xor(dot, m, WAVE);
        dot /= (float)a.D;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int d = e * WAVE + lane;
          if (d < a.D) y[d] = (T)(r * s * (t[e] - xv[e] * r * dot));
        }
      }
    }
  }
  if constexpr (BACK) {
    float *s_w = s_dyn + 2 * a.P;  // [NWAVES][D]
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * WAVE + lane;
        if (d < a.D) s_w[w * a.D + d] = gw[o][e];
      }
      __syncthreads();
      for (int d = threadIdx.x; d < a.D; d += NT) {
        float v = 0.0f;
        for (int q = 0; q < NWAVES; ++q) v += s_w[q * a.D + d];
        a.part[((long long)blockIdx.x * 2 + o) * a.D + d] = v;
      }
    }
  }
}

// Sums over the workgroups, in 64 bits: a workgroup for four numbers of a weight (512
// workgroups' sums of 2 x 64: 4.5 us, a launch and one trip to memory).
__global__ __launch_bounds__(NT) void k_norms_sum(NormArgs a, int blocks) {
  constexpr int C = 4, R = NT / C, AHEAD = 8;
  __shared__ double s_sum[R][C];
  const int c = threadIdx.x % C, r = threadIdx.x / C, d = blockIdx.x * C + c, o = blockIdx.y;
  if (!a.side[o].gw) return;
  double v = 0.0;
  for (int b0 = r; d < a.D && b0 < blocks; b0 += R * AHEAD) {
    float x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int b = b0 + i * R;
      x[i] = b < blocks ? a.part[((long long)b * 2 + o) * a.D + d] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v += x[i];
  }
  s_sum[r][c] = v;
  for (int half = R / 2; half; half /= 2) {
    __syncthreads();
    if (r < half) s_sum[r][c] += s_sum[r + half][c];
  }
  if (r == 0 && d < a.D) a.side[o].gw[d] = (float)s_sum[0][c];
}

// Whether k_norms_wide takes the call.
bool wide(const NormArgs &a, size_t e, bool back) {
  const int V = 16 / (int)e;
  if (a.D % (2 * V) || a.P % V || (a.D - 2 * a.P) % (2 * V)) return false;
  for (const NormSide &s : a.side) {
    if (!s.heads) continue;
    if (s.xs * e % 16 || s.ys * e % 16 || (back && s.gs * e % 16)) return false;
    for (const void *p : {s.x, static_cast<const void *>(s.y), back ? s.g : nullptr})
      if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  }
  return true;
}

// Rows that a workgroup takes at a time: as many as leave 1,024 workgroups, up to 16.
int rows_at_once(const NormArgs &a) {
  int rows = 1;
  while (rows < 16 && a.N >= 2048 * (long long)rows) rows *= 2;
  return rows;
}

template <typename T, bool BACK>
void launch_of(const NormArgs &a, int blocks, hipStream_t s) {
  if (wide(a, sizeof(T), BACK)) {
    int lanes = 1;
    while (lanes < a.D / (2 * PER<T>)) lanes *= 2;
    const int rows = rows_at_once(a);
    const size_t turns = 2 * (size_t)rows * a.P, sums = BACK ? (size_t)NWAVES * a.D : 0;
    const size_t lds = (turns > sums ? turns : sums) * sizeof(float);
    if (a.pairs)
      k_norms_wide<T, true, BACK><<<dim3(blocks, 2), NT, lds, s>>>(a, rows, lanes);
    else
      k_norms_wide<T, false, BACK><<<dim3(blocks, 2), NT, lds, s>>>(a, rows, lanes);
    return;
  }
  const size_t lds = (2 * (size_t)a.P + (size_t)NWAVES * a.D) * sizeof(float);
  if (a.D <= WAVE)
    k_norms<T, 1, BACK><<<blocks, NT, lds, s>>>(a);
  else if (a.D <= 2 * WAVE)
    k_norms<T, 2, BACK><<<blocks, NT, lds, s>>>(a);
  else
    k_norms<T, MAX_WIDTH / WAVE, BACK><<<blocks, NT, lds, s>>>(a);
}
template <bool BACK>
void launch_as(const NormArgs &a, int type, int blocks, hipStream_t s) {
  if (type == FST_F32)
    launch_of<float, BACK>(a, blocks, s);
  else if (type == FST_F16)
    launch_of<f16, BACK>(a, blocks, s);
  else
    launch_of<bf16, BACK>(a, blocks, s);
}

// Workgroups: at most `most`, none without rows, no more than their rows' turns ask for.
int workgroups(const NormArgs &a, int type, bool back, int most) {
  const long long rows = wide(a, type_bytes(type), back) ? rows_at_once(a) : 1;
  const long long n = (a.N + rows - 1) / rows;
  const long long turns = n > most ? (n + most - 1) / most : 1;
  return (int)((n + turns - 1) / turns);
}

}  // namespace

hipError_t launch_norms(const NormArgs &a, int type, hipStream_t s) {
  if (a.N > 0) launch_as<false>(a, type, workgroups(a, type, false, 4096), s);
  return hipGetLastError();
}

hipError_t launch_norms_grads(NormArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  // (k_norms_wide: few, a workgroup's sums for the weights cost as much as some rows)
  const int blocks = workgroups(a, type, true, wide(a, type_bytes(type), true) ? 512 : 1024);
  *need = (size_t)blocks * 2 * a.D * sizeof(float);
  if (!ws) return hipSuccess;
  a.part = static_cast<float *>(ws);
  if (blocks) launch_as<true>(a, type, blocks, s);
  k_norms_sum<<<dim3((a.D + 3) / 4, 2), NT, 0, s>>>(a, blocks);
  return hipGetLastError();
}

}  // namespace fstc
