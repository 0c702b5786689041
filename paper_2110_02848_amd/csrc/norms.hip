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

// A wavefront takes a head: lane l holds numbers l, l + 64, ..  BACK: gradients;
// a workgroup's sums for w go to a row of `part`, sides side by side.
template <typename T, bool BACK>
__global__ __launch_bounds__(NT) void k_norms(NormArgs a) {
  extern __shared__ float s_dyn[];
  constexpr int E = MAX_WIDTH / WAVE;
  float2 *s_turn = reinterpret_cast<float2 *>(s_dyn);              // [P]
  const int lane = threadIdx.x & (WAVE - 1);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  float *s_z = s_dyn + 2 * a.P + w * a.D;                          // a wavefront's [D]
  const int heads = a.side[0].heads + a.side[1].heads;
  float gw[2][E] = {};
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x) {
    __syncthreads();
    for (int i = threadIdx.x; i < a.P; i += NT) s_turn[i] = turn(a.pos[row], a.freq[i]);
    __syncthreads();
    for (int hh = w; hh < heads; hh += NWAVES) {
      const int o = hh >= a.side[0].heads;
      const NormSide &sd = a.side[o];
      const long long at = (long long)(hh - (o ? a.side[0].heads : 0)) * a.D;
      const T *x = static_cast<const T *>(sd.x) + row * sd.xs + at;
      const T *g = static_cast<const T *>(sd.g) + row * sd.gs + at;
      T *y = static_cast<T *>(sd.y) + row * sd.ys + at;
      float xv[E], sum = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * WAVE + lane;
        xv[e] = d < a.D ? (float)x[d] : 0.0f;
        sum = fmaf(xv[e], xv[e], sum);
      }
#pragma unroll
      for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m, WAVE);
      const float r = 1.0f / sqrtf(sum / (float)a.D + a.eps);
      // what is turned meets its pair in LDS (a wavefront's own, in order)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = e * WAVE + lane;
        if (d < a.D) s_z[d] = BACK ? (float)g[d] : xv[e] * r * sd.w[d];
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
          if (d < a.D) y[d] = (T)(r * (t[e] - xv[e] * r * dot));
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

// Sums over the workgroups, in 64 bits: a workgroup for 16 numbers of a w.
__global__ __launch_bounds__(NT) void k_norms_sum(NormArgs a, int blocks) {
  __shared__ double s_sum[NT / 16][16];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, d = blockIdx.x * 16 + c, o = blockIdx.y;
  if (!a.side[o].gw) return;
  double v = 0.0;
  if (d < a.D)
    for (int b = r; b < blocks; b += NT / 16) v += a.part[((long long)b * 2 + o) * a.D + d];
  s_sum[r][c] = v;
  __syncthreads();
  if (r || d >= a.D) return;
  for (int q = 1; q < NT / 16; ++q) v += s_sum[q][c];
  a.side[o].gw[d] = (float)v;
}

template <bool BACK>
void launch_as(const NormArgs &a, int type, int blocks, hipStream_t s) {
  const size_t lds = (2 * (size_t)a.P + (size_t)NWAVES * a.D) * sizeof(float);
  if (type == FST_F32)
    k_norms<float, BACK><<<blocks, NT, lds, s>>>(a);
  else if (type == FST_F16)
    k_norms<f16, BACK><<<blocks, NT, lds, s>>>(a);
  else
    k_norms<bf16, BACK><<<blocks, NT, lds, s>>>(a);
}

}  // namespace

hipError_t launch_norms(const NormArgs &a, int type, hipStream_t s) {
  if (a.N > 0) launch_as<false>(a, type, (int)(a.N < 2048 ? a.N : 2048), s);
  return hipGetLastError();
}

hipError_t launch_norms_grads(NormArgs a, int type, void *ws, size_t *need, hipStream_t s) {
  const int blocks = (int)(a.N < 1024 ? a.N : 1024);
  *need = (size_t)blocks * 2 * a.D * sizeof(float);
  if (!ws) return hipSuccess;
  a.part = static_cast<float *>(ws);
  if (blocks) launch_as<true>(a, type, blocks, s);
  k_norms_sum<<<dim3((a.D + 15) / 16, 2), NT, 0, s>>>(a, blocks);
  return hipGetLastError();
}

}  // namespace fstc
