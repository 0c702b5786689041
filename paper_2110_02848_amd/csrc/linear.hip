// Linear attention with a decay for each head (fst_linear_attention_run, its
// gradients and its single step).
//
//   S_t = e^g S_(t-1) + k_t v_t^T,  y_t = scale S_t^T q_t
//
// CHUNK rows at a time that is three products on the matrix cores: with S
// the state before the chunk, its rows i, j counted from 0,
//   y_i = scale (sum over j <= i of e^(g (i - j)) (q_i . k_j) v_j + e^(g (i + 1)) S^T q_i)
//   S  <- e^(g CHUNK) S + sum over j of e^(g (CHUNK - 1 - j)) k_j v_j^T.
// No power of the decay is divided by another, so none overflows however fast a
// head forgets.  The gradients are the same operation (dy = the gradient of y):
//   dq: (dy, v, k) in place of (q, k, v), from the transposed state;
//   dk: (v, dy, q) and dv: (k, q, dy) from the last row to the first, from the
//       gradient of the last state, which decays after a row instead of before
//       it; what is left of it is the gradient of the first.
#include <initializer_list>

#include "sequences.h"
#include "tiles.h"

namespace fstc {

using namespace tile;

namespace {

constexpr int CHUNK = 64;   // rows that are multiplied at once, 16 of them by a wavefront
// Columns of v that four wavefronts take.  float32's products take eight times as
// long, and half the columns leave them twice the workgroups (6 x 211 x 5 heads of 41
// and 57, with gradients: 71 us with 64).
template <typename T>
constexpr int SLICE_OF = sizeof(T) == 2 ? 64 : 32;
constexpr int LNT = 256;    // threads of a step
constexpr int MANY = 12;    // units of a sequence, from which k_linear_scan has parts
static_assert(CHUNK == 16 * 4, "a wavefront has 16 rows");

// e^(g n) for 0 <= n <= CHUNK, from 64 bits: chunk after chunk multiplies them.
// (A head that keeps nothing has g = -inf, and e^(0 g) = 1 all the same.)
__device__ __forceinline__ double power_of(float g, int n) {
  const double d = g < -1e4f ? -1e4 : (double)g;
  return exp(d * n);
}

// Whether all of a wavefront's results are numbers.
template <int N>
__device__ __forceinline__ bool finite(const float4v (&x)[N]) {
  float z = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) z = fmaf(x[j][r], 0.0f, z);
  return __all(z == 0.0f);
}

// Row i against the state and the rows up to it alone, term by term, for 16 columns
// of v of which lane group lg has four at a time.  The product also takes the later
// rows of v, times 0, which makes no number of an infinity or a NaN that row i does
// not see: where a result (in memory, at o) is none, it is taken again.
template <typename T, int PA, int PB>
__device__ __noinline__ void exact_rows(T *o, int left, const T *s_q, const T *s_k, const T *s_v,
                                        const T *s_s, const float *s_pow, int i, int A, int lg,
                                        float f_past, float f_now) {
  for (int c = 4 * lg; c < SLICE_OF<T>; c += 16) {
    if (!none_of_four(o, c, left)) continue;
    float4v past{}, now{};
    for (int d = 0; d < A; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        past[r] = fmaf((float)s_q[i * LD<T, PA> + d], (float)s_s[(c + r) * LD<T, PA> + d],
                       past[r]);
    // (four NaN stay such)
    for (int row = 0; row <= i && !all_nan(past * f_past + now); ++row) {
      float p = 0.0f;
      for (int d = 0; d < A; ++d)
        p = fmaf((float)s_q[i * LD<T, PA> + d], (float)s_k[row * LD<T, PA> + d], p);
      p *= s_pow[i - row];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        now[r] = fmaf(p, (float)s_v[row * LD<T, PB> + c + r], now[r]);
    }
    mend_four(o, c, left, past * f_past + now * f_now);
  }
}

// Over the wavefronts.
template <int NW>
__device__ __forceinline__ float largest(const float (&m)[NW][3], int c) {
  float x = m[0][c];
#pragma unroll
  for (int w = 1; w < NW; ++w) x = fmaxf(x, m[w][c]);
  return x;
}

// What a workgroup of k_linear takes.  Workgroups begin in their order and go to the
// eight XCDs in turn: the jobs and slices of one unit and head go to one XCD, one
// after another, and where they walk the rows in the same order the second reads them from
// the XCD's cache; a row's heads run together, so that memory gives whole rows
// (64 x 2,000 x 8 x 128 x 128 bf16 with gradients: 1,080 us with the units of a job
// and head together, 1,027 with the jobs together, 955 with both).
struct Place {
  unsigned unit;
  int head, slice, job;
};
template <typename I>
__device__ __forceinline__ Place place_of(I X, I H, I J) {
  const I id = blockIdx.x + X * (blockIdx.y + gridDim.y * (I)blockIdx.z), pieces = X * H;
  const I turn = id / (8 * J), r = id - turn * (8 * J);
  const I wide = turn < pieces / 8 ? 8 : pieces % 8;  // pieces of the turn
  const I j = r / wide, p = turn * 8 + (r - j * wide), unit = p / H;
  return {(unsigned)unit, (int)(p - unit * H), (int)(j / gridDim.z), (int)(j % gridDim.z)};
}
__device__ __forceinline__ Place place_of(int H, int slices) {
  const unsigned X = gridDim.x, J = slices * gridDim.z;
  if ((unsigned long long)X * H <= 0xffffffffu / J) return place_of<unsigned>(X, H, J);
  return place_of<unsigned long long>(X, H, J);
}

// FULL: rows' results; otherwise a unit's own contribution to the state, written
// where the state entering the unit will be.
//
// Four wavefronts, 16 rows of the chunk each, for every 64 columns of v (CG such
// groups of wavefronts share the tiles of q and k): scores as (k rows) x (q columns),
// so that they become an operand of the product with v where they are; the state
// in registers, a quarter of its rows a wavefront, and rounded to T in LDS as
// (v rows) x (k columns) for the product with q.
//
// Roundings to 16 bits: scores and the state that meets q, once each.  The decayed k
// that go into the state are as many numbers as hold them: states are float32
// results.  float16: all three are scaled by powers of two, scores by one of the
// row's own (tiles.h), the decayed k by the largest of the chunk's, the state by a bound
// on its numbers, so that they neither overflow nor lose their digits.
//
// Bound by memory for heads of 64 (40,000 x 8 x 64 x 64 bf16: 37 us for 164 MB, 4.4 TB/s,
// the units' states 22 before it), for wider ones by a chunk's steps, each waiting for
// the one before with two wavefronts a SIMD (64 x 2,000 x 8 x 128 x 128 bf16 270 to 291
// us, its gradients 733 to 797; 40 % of cycles on the vector units, 20 % on the matrix
// cores).  Two workgroups of 64 columns a CU in place of one of 128 took as long.
//
// MIN_WAVES: wavefronts of a SIMD, at least: with one the compiler takes registers
// that the vector units cannot add in (that case by 64 columns: 1,316 us, with two 960).
// With three float16 spills 5 of them where heads are 64 wide, 18 number by number.
template <typename T, int PA, int CG>
constexpr int MIN_WAVES = CG == 2 ? 2 : sizeof(T) == 4 ? 1 : PA == 64 ? 3 : 2;
template <typename T, int PA, int CG, bool WIDE, bool FULL>
__global__ __launch_bounds__(256 * CG, (MIN_WAVES<T, PA, CG>)) void k_linear(LinArgs a) {
  static_assert(PA % 64 == 0, "whole tiles for four wavefronts");
  constexpr int NTH = 256 * CG, NW = 4 * CG, SLICE = SLICE_OF<T>, NJ = SLICE / 16, PB = SLICE * CG;
  constexpr int MT = PA / 64;  // tiles of 16 rows of the state, a wavefront
  constexpr bool SCALED = std::is_same<T, f16>::value;
  // numbers of T that hold 24 bits of a decayed k
  constexpr int TERMS = std::is_same<T, bf16>::value ? 3 : std::is_same<T, f16>::value ? 2 : 1;
  extern __shared__ __attribute__((aligned(16))) char s_dyn[];
  T *s_k = reinterpret_cast<T *>(s_dyn);       // [CHUNK][PA]
  T *s_v = s_k + CHUNK * LD<T, PA>;            // [CHUNK][PB]
  T *s_q = s_v + CHUNK * LD<T, PB>;            // FULL: [CHUNK][PA]
  T *s_s = s_q + CHUNK * LD<T, PA>;            // FULL: [PB][PA]
  __shared__ float s_pow[CHUNK + 1];
  __shared__ __attribute__((aligned(16))) float s_end[CHUNK];  // rows' powers to the end
  __shared__ float s_max[NW][3];

  const Place at = place_of(a.H, a.slices);
  const LinJob &job = a.job[at.job];
  const int lane = threadIdx.x & (WAVE - 1), l16 = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int wr = w & 3, c0 = CG == 1 ? 0 : (w >> 2) * SLICE;  // its rows and columns
  const int h = at.head, b0 = at.slice * PB;
  const int A = job.A, B = job.B, left = B - b0;
  Unit u;
  if (left <= 0 || !unit_of(a.off, a.n, a.N, a.unit, job.reverse, at.unit, u)) return;

  const float g = a.log_decay[h];
  const int end = job.back ? 0 : 1;
  if (threadIdx.x <= CHUNK) {
    const float p = (float)power_of(g, threadIdx.x);
    const int j = CHUNK - end - (int)threadIdx.x;  // the row that it takes to the end
    s_pow[threadIdx.x] = p;
    if (j >= 0 && j < CHUNK) s_end[j] = p;
  }

  // the state: rows (wr MT + m) 16 + 4 lg + r, columns c0 + 16 j + l16
  float4v S[MT][NJ];
  const long long AB = (long long)A * B;
  const int row0 = wr * MT * 16 + 4 * lg;
  float *unit_state =
      a.unit ? job.units + ((long long)at.unit * a.H + h) * AB : nullptr;
  const float *from = !FULL ? nullptr
                            : a.unit ? unit_state
                                     : job.state ? job.state + ((long long)u.s * a.H + h) * AB
                                                 : nullptr;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int ra = row0 + 16 * m + r, cb = c0 + 16 * j + l16;
        S[m][j][r] = from && ra < A && cb < left
                         ? from[(long long)ra * job.sa + (long long)(b0 + cb) * job.sb]
                         : 0.0f;
      }
  float bound = 0.0f;  // SCALED: on the state's magnitudes
  if constexpr (SCALED && FULL) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = fabsf(S[m][j][r]);
          bound = x < INFINITY ? fmaxf(bound, x) : bound;
        }
    bound = wave_max(bound);
    if (lane == 0) s_max[w][2] = bound;
  }
  __syncthreads();
  if constexpr (SCALED && FULL)
    bound = largest(s_max, 2);

  // powers that every chunk uses: of row i = 16 wr + l16 against rows j = 16 t +
  // 4 lg + r (0 where j is later) and against the state
  const int i = 16 * wr + l16;
  float dec[4][4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = i - (16 * t + 4 * lg + r);
      dec[t][r] = d >= 0 ? s_pow[d] : 0.0f;
    }
  const float over = s_pow[i + end];
  // e^(g CHUNK) as two numbers
  const double all = power_of(g, CHUNK);
  float keep = (float)all, keep_lo = (float)(all - (double)keep);
  if (!(fabsf(keep) < INFINITY)) keep_lo = 0.0f;

  const T *q = static_cast<const T *>(job.q) + (long long)h * A;
  const T *k = static_cast<const T *>(job.k) + (long long)h * A;
  const T *v = static_cast<const T *>(job.v) + (long long)h * B + b0;
  Stage<T, PA, CHUNK, NTH, WIDE> rq, rk;
  Stage<T, PB, CHUNK, NTH, WIDE> rv;
  const auto fetch = [&](long long i0) {
    const long long first = u.first + i0 * u.step;
    const int count = (int)(u.hi - i0 < CHUNK ? u.hi - i0 : CHUNK);
    if constexpr (FULL) rq.fetch(q, job.qs, A, first, u.step, count);
    rk.fetch(k, job.ks, A, first, u.step, count);
    rv.fetch(v, job.vs, left, first, u.step, count);
  };
  if (u.lo < u.hi) fetch(u.lo);
  for (long long i0 = u.lo; i0 < u.hi; i0 += CHUNK) {
    const int count = (int)(u.hi - i0 < CHUNK ? u.hi - i0 : CHUNK);
    const bool more = i0 + CHUNK < u.hi;
    float s_scale = 1.0f;
    if constexpr (SCALED && FULL) s_scale = power_below(bound, 15);
    if constexpr (FULL) {
      rq.store(s_q);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          store_four<T, true>(s_s + (c0 + 16 * j + l16) * LD<T, PA>, row0 + 16 * m, PA,
                              S[m][j] * s_scale);
    }
    rk.store(s_k);
    rv.store(s_v);
    if constexpr (SCALED) {
      const float mk = wave_max(rk.largest(s_end + (CHUNK - count), count));
      const float mv = wave_max(rv.largest());
      if (lane == 0) s_max[w][0] = mk, s_max[w][1] = mv;
    }
    __syncthreads();
    if (more) fetch(i0 + CHUNK);

    float p_scale = SCALED ? UNMET : 1.0f, k_scale = 1.0f;
    if constexpr (SCALED) {
      const float mk = largest(s_max, 0), mv = largest(s_max, 1);
      bound = fmaf(keep, bound, fabsf(job.sk) * CHUNK * mk * mv);
      k_scale = fminf(power_below(fabsf(job.sk) * mk, 12), power_below(bound, 100));
    }
    if constexpr (FULL) {
      float4v past[NJ] = {}, now[NJ] = {};
      Frag<T> qf[PA / 32];
#pragma unroll
      for (int s = 0; s < PA / 32; ++s) qf[s] = rows<T, PA>(s_q, 16 * wr, 32 * s, lane);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int s = 0; s < PA / 32; ++s)
          past[j] = mac(rows<T, PA>(s_s, c0 + 16 * j, 32 * s, lane), qf[s], past[j]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (2 * t > wr) continue;
        float4v x[2] = {};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (2 * t + c > wr) continue;
#pragma unroll
          for (int s = 0; s < PA / 32; ++s)
            x[c] = mac(rows<T, PA>(s_k, 32 * t + 16 * c, 32 * s, lane), qf[s], x[c]);
          // (later rows by a choice: what they hold may be no number)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            x[c][r] = 32 * t + 16 * c + 4 * lg + r <= i
                          ? x[c][r] * dec[2 * t + c][r]
                          : 0.0f;
        }
        if constexpr (SCALED) {
          const float top = largest_of(x[0], x[1]);
          if (__any(top * p_scale > PAST)) {
            const float less = lowered(p_scale, top);
            if (t > 0) {
#pragma unroll
              for (int j = 0; j < NJ; ++j) now[j] *= less;
            }
          }
          x[0] *= p_scale, x[1] *= p_scale;
        }
        const Frag<T> p = pack<T>(x[0], x[1]);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          now[j] = mac(columns<T, PB>(s_v, 32 * t, c0 + 16 * j, lane), p, now[j]);
      }
      const bool fine = finite(now);
      if (i < count) {
        T *o = static_cast<T *>(job.o) + (u.first + (i0 + i) * u.step) * job.os +
               (long long)h * B + b0;
        const float f = job.ss * over / s_scale, f2 = job.so / p_scale;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          store_four<T, WIDE>(o, c0 + 16 * j + 4 * lg, left, past[j] * f + now[j] * f2);
        if (!fine)
          exact_rows<T, PA, PB>(o + c0, left - c0, s_q, s_k, s_v + c0, s_s + c0 * LD<T, PA>, s_pow,
                                i, A, lg, f, job.so);
      }
    }
    if (more || !FULL || (job.last && u.hi == u.len)) {
      const bool whole = count == CHUNK;
      const float kh = whole ? keep : s_pow[count], kl = whole ? keep_lo : 0.0f;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            S[m][j][r] = fmaf(kh, S[m][j][r], kl * S[m][j][r]) * k_scale;
      const float f0 = job.sk * k_scale;
      // (what a decayed k lost to two numbers matters to `last` alone)
      const int terms = !FULL || job.last ? TERMS : TERMS < 2 ? TERMS : 2;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag<T> vf[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) vf[j] = columns<T, PB>(s_v, 32 * t, c0 + 16 * j, lane);
        float f[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int j = 32 * t + 16 * e + 4 * lg;
          float4v x;
          if (whole) {
            x = *reinterpret_cast<const float4v *>(s_end + j);
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = j + r < count ? s_end[CHUNK - count + j + r] : 0.0f;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) f[4 * e + r] = x[r] * f0;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          float x[8], y[8];
          unpack(columns<T, PA>(s_k, 32 * t, (wr * MT + m) * 16, lane), x);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= f[e];
#pragma unroll
          for (int c = 0; c < TERMS; ++c) {
            if (c >= terms) continue;
            Frag<T> part = pack<T>(x);
            // (made once: what is left of x goes by the very numbers that are
            // multiplied, where the compiler might round x for each in its own way)
            if constexpr (TERMS > 1) asm("" : "+v"(part.v[0]));
#pragma unroll
            for (int j = 0; j < NJ; ++j) S[m][j] = mac(part, vf[j], S[m][j]);
            if (c + 1 < TERMS) {
              unpack(part, y);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] -= y[e];
            }
          }
        }
      }
      if constexpr (SCALED) {
        const float back = 1.0f / k_scale;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int j = 0; j < NJ; ++j) S[m][j] *= back;
      }
    }
    __syncthreads();
  }
  float *to = !FULL ? unit_state
                    : job.last && u.hi == u.len ? job.last + ((long long)u.s * a.H + h) * AB
                                                : nullptr;
  if (!to) return;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int ra = row0 + 16 * m + r, cb = c0 + 16 * j + l16;
        if (ra < A && cb < left)
          to[(long long)ra * job.sa + (long long)(b0 + cb) * job.sb] = S[m][j][r];
      }
}

// From the units' own contributions to the states entering them, in place: a lane
// takes an element of a head's state.  PARTS > 1: its workgroup's wavefronts a part of a
// sequence's units each, and what each part makes of a zero state meets in LDS.  A
// part's units stay in registers, unless there are more than AHEAD of them.  Bound by
// two trips to memory (63 units of 8 x 64 x 64: 6 us).  Few units of many sequences
// take one part, whose lanes have one exponential (4 units of 33 sequences, 5 x 128 x
// 128: 16 us; four parts, all AHEAD units passed one by one: 132).
template <int PARTS>
__global__ __launch_bounds__(NT) void k_linear_scan(LinArgs a) {
  constexpr int AHEAD = 32, STEP = 8;
  __shared__ float s_sum[PARTS][WAVE];
  const LinJob &job = a.job[blockIdx.z];
  const int AB = job.A * job.B, all = AB * a.H;
  const int lane = threadIdx.x & (WAVE - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), w = PARTS > 1 ? wave : 0;
  const int at = (PARTS > 1 ? blockIdx.x : blockIdx.x * NWAVES + wave) * WAVE + lane;
  const int e = at < all ? at : all - 1;
  const int s = blockIdx.y;
  const long long b = clamped(a.off[s], 0, a.N);
  const long long len = clamped(a.off[s + 1], b, a.N) - b;
  const long long n = len > 0 ? over_steps(len - 1, a.unit) + 1 : 1;
  const long long share = (n + PARTS - 1) / PARTS, u0 = w * share;
  const long long u1 = u0 + share < n ? u0 + share : n;
  float *p = job.units + rows_before(b, s, a.unit) * all + e;
  float S = job.state ? job.state[(long long)s * all + e] : 0.0f;
  float x[AHEAD];
#pragma unroll
  for (int c0 = 0; c0 < AHEAD; c0 += STEP)
    if (u0 + c0 < u1) {
#pragma unroll
      for (int c = c0; c < c0 + STEP; ++c) x[c] = u0 + c < u1 ? p[(u0 + c) * all] : 0.0f;
    }
  const float g = a.log_decay[e / AB];
  const double d = (g < -1e4f ? -1e4 : (double)g) * (double)a.unit, whole = exp(d);
  const float kh = (float)whole;
  const float kl = fabsf(kh) < INFINITY ? (float)(whole - (double)kh) : 0.0f;
  if constexpr (PARTS > 1) {
    float sum = 0.0f;
#pragma unroll
    for (int c0 = 0; c0 < AHEAD; c0 += STEP)
      if (u0 + c0 < u1) {
#pragma unroll
        for (int c = c0; c < c0 + STEP; ++c)
          if (u0 + c < u1) sum = fmaf(kh, sum, fmaf(kl, sum, x[c]));
      }
    for (long long u = u0 + AHEAD; u < u1; ++u) sum = fmaf(kh, sum, fmaf(kl, sum, p[u * all]));
    s_sum[w][lane] = sum;
    __syncthreads();
    const float over = w ? (float)exp(d * (double)share) : 1.0f;
    for (int q = 0; q < w; ++q) S = fmaf(over, S, s_sum[q][lane]);
  }
  if (at >= all) return;
#pragma unroll
  for (int c0 = 0; c0 < AHEAD; c0 += STEP)
    if (u0 + c0 < u1) {
#pragma unroll
      for (int c = c0; c < c0 + STEP; ++c)
        if (u0 + c < u1) {
          p[(u0 + c) * all] = S;
          S = fmaf(kh, S, fmaf(kl, S, x[c]));
        }
    }
  for (long long u = u0 + AHEAD; u < u1; ++u) {
    const float y = p[u * all];
    p[u * all] = S;
    S = fmaf(kh, S, fmaf(kl, S, y));
  }
}

// One step: a workgroup takes a row's head, each thread V columns of every
// `groups`-th row of the state.  Bound by memory: the state is read and written
// once (1,024 rows of 8 x 64 x 64: 50 us for 272 MB, 5.4 TB/s).
template <typename T, int V>
__global__ __launch_bounds__(LNT) void k_linear_step(LinStepArgs a) {
  __shared__ float s_q[FST_ATTENTION_MAX_WIDTH], s_k[FST_ATTENTION_MAX_WIDTH];
  __shared__ float s_y[LNT][V];
  const long long i = blockIdx.x;
  const int h = blockIdx.y, tid = threadIdx.x, A = a.A, B = a.B;
  T *y = static_cast<T *>(a.y) + i * a.ys + (long long)h * B;
  const long long slot = a.slot ? (long long)a.slot[i] : i;
  if (slot < 0 || slot >= a.slots) {  // an idle row
    for (int b = tid; b < B; b += LNT) y[b] = (T)0.0f;
    return;
  }
  if (tid < A) {
    s_q[tid] = (float)static_cast<const T *>(a.q)[i * a.qs + (long long)h * A + tid];
    s_k[tid] = (float)static_cast<const T *>(a.k)[i * a.ks + (long long)h * A + tid];
  }
  const int cols = (B + V - 1) / V;
  int across = 1;
  while (across < cols) across *= 2;
  const int groups = LNT / across, c = tid % across, gr = tid / across;
  const float keep = (float)power_of(a.log_decay[h], 1);
  struct alignas(4 * V) Pack { float v[V]; };
  const long long base = (slot * a.H + h) * (long long)A * B;
  const bool on = c < cols;
  float vv[V], sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    vv[e] = on ? (float)static_cast<const T *>(a.v)[i * a.vs + (long long)h * B + c * V + e] : 0.0f;
    sum[e] = 0.0f;
  }
  __syncthreads();
  if (on) {
#pragma unroll 4
    for (int ra = gr; ra < A; ra += groups) {
      Pack p = *reinterpret_cast<const Pack *>(a.in + base + (long long)ra * B + c * V);
      const float kk = s_k[ra], qq = s_q[ra];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        p.v[e] = fmaf(keep, p.v[e], kk * vv[e]);
        sum[e] = fmaf(qq, p.v[e], sum[e]);
      }
      *reinterpret_cast<Pack *>(a.out + base + (long long)ra * B + c * V) = p;
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) s_y[tid][e] = sum[e];
  for (int half = groups / 2; half; half /= 2) {
    __syncthreads();
    if (gr < half)
#pragma unroll
      for (int e = 0; e < V; ++e) s_y[tid][e] += s_y[tid + half * across][e];
  }
  if (gr == 0 && on)
#pragma unroll
    for (int e = 0; e < V; ++e) y[c * V + e] = (T)(a.scale * s_y[tid][e]);
}

unsigned units_of(const LinArgs &a) { return (unsigned)(a.unit ? a.N / a.unit + a.n : a.n); }

template <typename T, int PA, int CG, bool WIDE, bool FULL>
hipError_t launch_as(const LinArgs &a, int jobs, hipStream_t s) {
  constexpr int PB = SLICE_OF<T> * CG;
  constexpr int lds = BYTES<T, PA, CHUNK> + BYTES<T, PB, CHUNK> +
                      (FULL ? BYTES<T, PA, CHUNK> + BYTES<T, PA, PB> : 0);
  static_assert(lds <= 150 * 1024, "LDS of a CU");
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(k_linear<T, PA, CG, WIDE, FULL>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  k_linear<T, PA, CG, WIDE, FULL>
      <<<dim3(units_of(a), a.H * a.slices, jobs), 256 * CG, lds, s>>>(a);
  return hipGetLastError();
}
template <typename T, int PA, bool WIDE, bool FULL>
hipError_t launch_by_columns(const LinArgs &a, int jobs, int B, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (B > SLICE_OF<T>) return launch_as<T, PA, 2, WIDE, FULL>(a, jobs, s);
  }
  return launch_as<T, PA, 1, WIDE, FULL>(a, jobs, s);
}
template <typename T, bool FULL>
hipError_t launch_jobs(const LinArgs &a, int jobs, int A, int B, bool wide, hipStream_t s) {
  if (A <= 64)
    return wide ? launch_by_columns<T, 64, true, FULL>(a, jobs, B, s)
                : launch_by_columns<T, 64, false, FULL>(a, jobs, B, s);
  return wide ? launch_by_columns<T, 128, true, FULL>(a, jobs, B, s)
              : launch_by_columns<T, 128, false, FULL>(a, jobs, B, s);
}

// Columns of v of a workgroup.
int slice_of(int type, int B) {
  if (type == FST_F32) return SLICE_OF<float>;
  return B > SLICE_OF<bf16> ? 2 * SLICE_OF<bf16> : SLICE_OF<bf16>;
}

// Jobs [lo, hi) of `all`, which have one width of q and k (or widths up to 64).
template <bool FULL>
hipError_t launch_range(LinArgs a, const LinJob *all, int lo, int hi, int type, bool wide,
                        hipStream_t s) {
  int B = 0;
  for (int i = lo; i < hi; ++i) {
    a.job[i - lo] = all[i];
    B = all[i].B > B ? all[i].B : B;
  }
  if (B == 0) return hipSuccess;  // (no columns of results)
  a.slices = (B + slice_of(type, B) - 1) / slice_of(type, B);
  if (type == FST_F32) return launch_jobs<float, FULL>(a, hi - lo, all[lo].A, B, wide, s);
  if (type == FST_F16) return launch_jobs<f16, FULL>(a, hi - lo, all[lo].A, B, wide, s);
  return launch_jobs<bf16, FULL>(a, hi - lo, all[lo].A, B, wide, s);
}

// Whether every row of a head, of each tensor, begins at a multiple of 16 bytes
// and is whole groups of them.
bool wide_rows(const LinCall &c, size_t e, std::initializer_list<long long> strides,
               std::initializer_list<const void *> data) {
  if (c.K * e % 16 || c.V * e % 16) return false;
  for (long long t : strides)
    if (t * e % 16) return false;
  for (const void *p : data)
    if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  return true;
}

// Steps of a unit, 0: sequences are not cut.  Uncut, a call takes as long as its longest
// sequence; cut, as all rows twice and the states, which are worth it where
// workgroups are few for the sequences' length (on average).  bf16, cut and uncut: 8
// heads of 64, 8 sequences of 1,200: 35 and 50 us; of 600: 33 and 30; 24 of 1,200: 56 and
// 50; 8 heads of 128, 4 of 600: 48 and 54; 8 of 600: 69 and 55; 16 of 1,200: 114 and 92;
// 4 heads of 128, 16 of 1,200: 77 and 91.
long long unit_steps(const LinCall &c, int type, int jobs) {
  const int slice = slice_of(type, c.V);
  const long long groups = (long long)c.H * ((c.V + slice - 1) / slice);
  const long long all = c.n * groups * jobs, length = c.N / c.n;
  if (c.K == 0 || c.V == 0) return 0;  // (no states to cut by)
  if (all >= 256 || length <= 256 || 14 * all > length) return 0;
  const long long steps = c.N * groups / 512;
  return steps <= CHUNK ? CHUNK : (steps + CHUNK - 1) / CHUNK * CHUNK;
}

LinArgs linear_args(const LinCall &c, long long unit) {
  LinArgs a{};
  a.off = c.off;
  a.log_decay = c.log_decay;
  a.N = c.N;
  a.unit = unit;
  a.n = c.n;
  a.H = c.H;
  return a;
}

// Units' states of `jobs` jobs, and the scan that makes entering states of them.
hipError_t launch_states(const LinArgs &a, const LinJob *all, int jobs, int type, bool wide,
                         hipStream_t s) {
  const hipError_t e = launch_range<false>(a, all, 0, jobs, type, wide, s);
  if (e != hipSuccess) return e;
  LinArgs b = a;
  for (int i = 0; i < jobs; ++i) b.job[i] = all[i];
  const long long n = (long long)a.H * all[0].A * all[0].B;
  if (a.N / a.unit > MANY * (long long)a.n)
    k_linear_scan<NWAVES><<<dim3((unsigned)((n + WAVE - 1) / WAVE), a.n, jobs), NT, 0, s>>>(b);
  else
    k_linear_scan<1><<<dim3((unsigned)((n + NT - 1) / NT), a.n, jobs), NT, 0, s>>>(b);
  return hipGetLastError();
}

constexpr long long MAX_ACROSS = 65535;    // of a grid's second dimension
constexpr long long MAX_ROWS = 1 << 23;    // of a step

bool too_large(const LinCall &c) {
  const int most = c.K > c.V ? c.K : c.V;
  for (long long t : {c.qs, c.ks, c.vs})
    if (t > MAX_STRIDE) return true;
  return (long long)c.H * ((most + SLICE_OF<float> - 1) / SLICE_OF<float>) > MAX_ACROSS;
}

}  // namespace

// (also without workspace: then `need` is all that is set)
hipError_t launch_linear(const LinCall &c, int type, void *ws, size_t *need, hipStream_t s) {
  if (too_large(c)) return hipErrorInvalidValue;
  const size_t e = type_bytes(type);
  const long long unit = unit_steps(c, type, 1);
  *need = unit ? (size_t)(c.N / unit + c.n) * c.H * c.K * c.V * sizeof(float) : 0;
  if (!ws) return hipSuccess;
  const LinArgs a = linear_args(c, unit);
  const bool wide = wide_rows(c, e, {c.qs, c.ks, c.vs, c.ys}, {c.q, c.k, c.v, c.y});
  const LinJob job = {c.q, c.k, c.v, c.y, c.qs, c.ks, c.vs, c.ys, c.K, c.V, c.state, c.last,
                      c.V, 1, static_cast<float *>(ws), c.scale, c.scale, 1.0f, c.reverse, 0};
  if (unit) {
    const hipError_t err = launch_states(a, &job, 1, type, wide, s);
    if (err != hipSuccess) return err;
  }
  return launch_range<true>(a, &job, 0, 1, type, wide, s);
}

hipError_t launch_linear_grads(const LinCall &c, int type, void *ws, size_t *need,
                               hipStream_t s) {
  if (too_large(c) || c.ys > MAX_STRIDE) return hipErrorInvalidValue;
  const size_t e = type_bytes(type);
  const long long unit = unit_steps(c, type, 3);
  const size_t states = unit ? (size_t)(c.N / unit + c.n) * c.H * c.K * c.V : 0;
  *need = 2 * states * sizeof(float);
  if (!ws) return hipSuccess;
  const LinArgs a = linear_args(c, unit);
  const bool wide = wide_rows(c, e, {c.qs, c.ks, c.vs, c.ys, c.gqs, c.gks, c.gvs},
                              {c.q, c.k, c.v, c.y, c.gq, c.gk, c.gv});
  float *fwd = static_cast<float *>(ws), *bwd = fwd + states;
  const int back = !c.reverse;
  if (unit) {
    const LinJob sums[2] = {
        {nullptr, c.k, c.v, nullptr, 0, c.ks, c.vs, 0, c.K, c.V, c.state, nullptr, c.V, 1, fwd,
         0.0f, 0.0f, 1.0f, c.reverse, 0},
        {nullptr, c.q, c.y, nullptr, 0, c.qs, c.ys, 0, c.K, c.V, c.glast, nullptr, c.V, 1, bwd,
         0.0f, 0.0f, c.scale, back, 1}};
    const hipError_t err = launch_states(a, sums, 2, type, wide, s);
    if (err != hipSuccess) return err;
  }
  const LinJob jobs[3] = {
      {c.y, c.v, c.k, c.gq, c.ys, c.vs, c.ks, c.gqs, c.V, c.K, c.state, nullptr, 1, c.V, fwd,
       c.scale, c.scale, 1.0f, c.reverse, 0},
      {c.v, c.y, c.q, c.gk, c.vs, c.ys, c.qs, c.gks, c.V, c.K, c.glast, nullptr, 1, c.V, bwd,
       c.scale, 1.0f, c.scale, back, 1},
      {c.k, c.q, c.y, c.gv, c.ks, c.qs, c.ys, c.gvs, c.K, c.V, c.glast, c.gstate, c.V, 1, bwd,
       c.scale, 1.0f, c.scale, back, 1}};
  if ((c.K <= 64) == (c.V <= 64)) return launch_range<true>(a, jobs, 0, 3, type, wide, s);
  const hipError_t err = launch_range<true>(a, jobs, 0, 2, type, wide, s);
  return err != hipSuccess ? err : launch_range<true>(a, jobs, 2, 3, type, wide, s);
}

template <typename T>
static void linear_step_as(const LinStepArgs &a, bool four, hipStream_t s) {
  const dim3 grid((unsigned)a.n, a.H);
  if (four)
    k_linear_step<T, 4><<<grid, LNT, 0, s>>>(a);
  else
    k_linear_step<T, 1><<<grid, LNT, 0, s>>>(a);
}

hipError_t launch_linear_step(const LinStepArgs &a, int type, hipStream_t s) {
  if (a.H > MAX_ACROSS || a.n > MAX_ROWS) return hipErrorInvalidValue;
  const bool four = a.B % 4 == 0 && reinterpret_cast<uintptr_t>(a.in) % 16 == 0 &&
                    reinterpret_cast<uintptr_t>(a.out) % 16 == 0;
  if (type == FST_F32)
    linear_step_as<float>(a, four, s);
  else if (type == FST_F16)
    linear_step_as<f16>(a, four, s);
  else
    linear_step_as<bf16>(a, four, s);
  return hipGetLastError();
}

}  // namespace fstc
