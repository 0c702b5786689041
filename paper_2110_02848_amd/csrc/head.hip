// Heads of a network: log-softmax of a linear layer as weights of emission
// graphs (fst_emission_weights), cross entropy over a vocabulary
// (fst_cross_entropy), and the gradients of both.
//
// All of them are products of matrices on the matrix cores: scores z = x w^T
// (N x C over H), and from the gradient dS of the scores dx = dS w (N x H over
// C) and dw = dS^T x (C x H over N).  One kernel computes them, with an
// epilogue for each: a row's maximum and sum of exponentials, scores, dS, or a
// sum.  Scores of a vocabulary never reach memory: the forward pass leaves
// each tile's maxima and sums, and the gradient computes them again for a
// piece of the vocabulary at a time, whose dS it keeps for its two products.
#include <math.h>

#include <type_traits>

#include "layers.h"

namespace fstc {

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef __attribute__((ext_vector_type(4))) float float4v;
typedef __attribute__((ext_vector_type(4))) int int4v;
typedef __attribute__((ext_vector_type(8))) _Float16 half8;
typedef __attribute__((ext_vector_type(8))) __bf16 bhalf8;
typedef __attribute__((ext_vector_type(4))) short short4v;

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

constexpr int KBYTES = 128;  // bytes of a row of an operand's tile along the sum

template <typename T>
constexpr int k_step() { return KBYTES / (int)sizeof(T); }

// ---------------------------------------------------------------------------
// matrix core products of fragments
// ---------------------------------------------------------------------------

// A fragment: 16 rows by 64 bytes of the sum; lane l holds row l & 15, the
// 16-byte group l >> 4.
template <typename T>
struct Frag {
  int4v v;
};

__device__ __forceinline__ float4v mac(const Frag<bf16> &a, const Frag<bf16> &b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a.v),
                                                 __builtin_bit_cast(bhalf8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ float4v mac(const Frag<f16> &a, const Frag<f16> &b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a.v),
                                                __builtin_bit_cast(half8, b.v), c, 0, 0, 0);
}
// (four steps of 4: step j sums over element j of the four groups)
__device__ __forceinline__ float4v mac(const Frag<float> &a, const Frag<float> &b, float4v c) {
  const float4v x = __builtin_bit_cast(float4v, a.v), y = __builtin_bit_cast(float4v, b.v);
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
  return c;
}

// ---------------------------------------------------------------------------
// operands' tiles in LDS
// ---------------------------------------------------------------------------

// Loads of 64 lanes by 16 bytes go from memory to LDS without registers: lane
// i's bytes land at `lds` + 16 i, zeros where they lie past the end of the
// buffer.  Written as instructions, because the compiler would wait for all of
// them before the next read of LDS; whoever reads waits with wait_loads and a
// barrier.  (m0 is the compiler's own: it warns where it is named, and only
// naming it keeps its uses of m0 clear of this one.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(uint32_t lds, uint32_t offset, int4v buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(buffer)
               : "memory", "m0");
}
#pragma clang diagnostic pop
// The buffer of `bytes` bytes at p + at (as many of them as 32 bits count; all
// arguments the same in every lane).
__device__ __forceinline__ int4v buffer_at(const char *p, long long bytes, long long at) {
  const unsigned long long q = (unsigned long long)(uintptr_t)p + at;
  const long long left = bytes - at;
  const uint32_t n = left <= 0 ? 0u : left > 0xffffffffll ? 0xffffffffu : (uint32_t)left;
  return int4v{__builtin_amdgcn_readfirstlane((int)(uint32_t)q),
               __builtin_amdgcn_readfirstlane((int)(uint32_t)(q >> 32)),
               __builtin_amdgcn_readfirstlane((int)n), 0x00027000};
}
template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the last N
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const char *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

// Where the rows of a tile part lie among the rows of the whole tile: runs of
// RUN rows, one every EVERY rows from row FIRST on.
template <int RUN_, int EVERY_>
struct Rows {
  static constexpr int RUN = RUN_;
  static __device__ __forceinline__ int of(int first, int r) {
    return first + r / RUN * EVERY_ + r % RUN;
  }
};
// The rows of B so that a lane's results of a row lie side by side in groups of
// E (16 bytes), and the groups of its four lanes side by side: of a lane group a,
// the results r of its fragments j are q = 4 j + r, and column q / E 4 E + a E +
// q % E.  FN fragments of a wavefront, PER of them from the FIRST on in this part.
template <int E, int FN, int PER>
struct Spread {
  static constexpr int RUN = 4;
  static __device__ __forceinline__ int column(int group, int q) {
    return q / E * 4 * E + group * E + q % E;
  }
  static __device__ __forceinline__ int of(int first, int r) {
    const int w = r / (PER * 16), j = first + r / 16 % PER, i = r % 16;
    return w * FN * 16 + column(i / 4, 4 * j + i % 4);
  }
};

// Row-wise operand: element (r, k) at p[r * ld + k].  A part holds R rows of
// 128 bytes; 16-byte group g of row r lies at group g ^ (r & 7), so that the
// 16 lanes of a fragment's group, a row apart, read different banks.  Rows
// past the last are zeros; k has no tail (rows are padded with zeros to whole
// steps).
template <typename T, int R, int NWV, typename ROWS>
struct RowTile {
  static constexpr int BYTES = R * KBYTES;
  static constexpr int LOADS = BYTES / 1024 / NWV;  // a wavefront
  static_assert(LOADS >= 1 && LOADS * 1024 * NWV == BYTES, "whole loads");
  uint32_t off[LOADS];

  // `first`: the part's first row in the tile
  __device__ __forceinline__ void init(const Operand &o, int first, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = (wave * LOADS + i) * 8 + (lane >> 3);
      off[i] = (uint32_t)ROWS::of(first, r) * (uint32_t)(o.ld * sizeof(T)) +
               (((lane & 7) ^ (r & 7)) << 4);
    }
  }
  static __device__ __forceinline__ const char *base(const Operand &o, long long r0) {
    return static_cast<const char *>(o.p) + r0 * o.ld * (long long)sizeof(T);
  }
  // bytes from there to the end of the last row
  static __device__ __forceinline__ long long bytes(const Operand &o, long long r0) {
    return ((o.rows - 1 - r0) * o.ld + o.depth) * (long long)sizeof(T);
  }
  static __device__ __forceinline__ int4v step(const Operand &o, const char *base,
                                               long long bytes, int t) {
    const long long more = t >= o.wrap ? o.jump - (long long)o.wrap * KBYTES : 0;
    return buffer_at(base, bytes, (long long)t * KBYTES + more);
  }
  // the i-th load of the part, of the step whose buffer it is, to `lds`
  __device__ __forceinline__ void fetch(int i, uint32_t lds, int4v buffer, int wave) const {
    load_lds(lds + (wave * LOADS + i) * 1024, off[i], buffer);
  }
  // the fragment of rows `row` on, for half of the step
  static __device__ __forceinline__ Frag<T> frag(const char *lds, int row, int half, int lane) {
    const int r = row + (lane & 15), g = half * 4 + (lane >> 4);
    return Frag<T>{*reinterpret_cast<const int4v *>(lds + r * KBYTES + ((g ^ (r & 7)) << 4))};
  }
};

// Column-wise operand: element (r, k) at p[k * ld + r].  A part holds the
// step's k, each R elements of consecutive r; of 16-bit types, 32-byte block
// b of k lies at block b ^ swizzle(k), so that the reads that transpose (16
// lanes read four k of 16 rows) meet different banks.  Past the last k there
// are zeros, past the last row what lies there in memory, or zeros.
template <typename T, int R, int NWV, typename ROWS>
struct ColTile {
  static constexpr int K = k_step<T>();
  static constexpr int ROW = R * (int)sizeof(T);  // bytes of a k
  static constexpr int BYTES = ROW * K;
  static constexpr int LOADS = BYTES / 1024 / NWV;
  static constexpr int GROUPS = ROW / 16;
  static constexpr int BLOCKS = ROW / 32;
  static_assert(LOADS >= 1 && LOADS * 1024 * NWV == BYTES, "whole loads");
  static_assert(ROWS::RUN * sizeof(T) % 32 == 0, "whole blocks");
  uint32_t off[LOADS];

  static __device__ __forceinline__ int swizzle(int k) {
    return sizeof(T) == 2 ? ((k & 3) | ((k >> 1) & 4)) & (BLOCKS - 1) : 0;
  }
  // `first`: the part's first row in the tile
  __device__ __forceinline__ void init(const Operand &o, int first, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = (wave * LOADS + i) * 64 + lane, k = q / GROUPS, g = q % GROUPS;
      const int b = (((g >> 1) ^ swizzle(k)) << 5) + ((g & 1) << 4);
      off[i] = (uint32_t)k * (uint32_t)(o.ld * sizeof(T)) +
               ROWS::of(first, b / (int)sizeof(T)) * (int)sizeof(T);
    }
  }
  static __device__ __forceinline__ const char *base(const Operand &o, long long r0) {
    return static_cast<const char *>(o.p) + r0 * (long long)sizeof(T);
  }
  static __device__ __forceinline__ long long bytes(const Operand &o, long long r0) {
    return ((o.depth - 1) * o.ld + o.rows - r0) * (long long)sizeof(T);
  }
  static __device__ __forceinline__ int4v step(const Operand &o, const char *base,
                                               long long bytes, int t) {
    const long long every = K * o.ld * (long long)sizeof(T);
    return buffer_at(base, bytes, t >= o.wrap ? (t - o.wrap) * every + o.jump : t * every);
  }
  __device__ __forceinline__ void fetch(int i, uint32_t lds, int4v buffer, int wave) const {
    load_lds(lds + (wave * LOADS + i) * 1024, off[i], buffer);
  }
  // Fragment of 16 rows: lane l wants k = half * 32 + (l >> 4) * 8 .. + 8 of
  // row l & 15 (16-bit types).  A read that transposes gives lane i of 16 the
  // i-th column of four k: lanes 4j .. 4j + 3 point at the j-th k.
  static __device__ __forceinline__ Frag<T> frag(const char *lds, int row, int half, int lane) {
    if constexpr (sizeof(T) == 2) {
      const int k = half * 32 + (lane >> 4) * 8 + ((lane >> 2) & 3);
      const int block = row / 16, in = (lane & 3) * 8;
      int2 v[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int q = k + 4 * j;
        const char *at = lds + q * ROW + ((block ^ swizzle(q)) << 5) + in;
        v[j] = __builtin_bit_cast(
            int2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                      (__attribute__((address_space(3))) short4v *)(LDS_PTR(at))));
      }
      return Frag<T>{int4v{v[0].x, v[0].y, v[1].x, v[1].y}};
    } else {
      const int k = half * 16 + (lane >> 4) * 4;
      int4v v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = *reinterpret_cast<const int *>(lds + (k + j) * ROW + (row + (lane & 15)) * 4);
      return Frag<T>{v};
    }
  }
};

// ---------------------------------------------------------------------------
// the product
// ---------------------------------------------------------------------------

// out[m][n] = sum over k of A(m, k) B(n, k), m < M, n < N, k < K, by tiles of
// BM x BN.
struct Product {
  Operand A, B;
  long long M, N, K;
  int tiles_m, tiles_n;
  int splits, steps;     // parts of the sum (grid z), `steps` K-steps each
  // epilogues
  long long n0, words;   // what column 0 stands for (a piece's first word), all words
  void *out;             // scores, dS, sums or results
  long long ldo;
  float2 *part;          // [parts, M]: maximum and sum of a row's scores in a part of a tile
  const int32_t *target; // [M]
  float *hit;            // [M]: the target's score
  const float *lse;      // [M]
  const float *grad;     // [M] or null (1)
  const float *scale;    // power of two on dS (16-bit floats), or null (1)
  long long Np, lo;      // dS: columns to write, zeros past N; what rounding lost goes
                         // `lo` columns further on (0: it is dropped)
  int add;               // sums: add to what is there
  const float *sums;     // [M, N rounded up to four] or null
  int wide;              // results: `out` and its rows are aligned to four (2: to 16 bytes)
};

enum Epilogue {
  EPI_PART,    // maxima and sums of exponentials, targets' scores
  EPI_SCORE,   // the same and the scores as float32
  EPI_LOG,     // log-probabilities, of tiles as wide as a row
  EPI_DS,      // gradient of the scores
  EPI_SUM,     // float32 sums, one block of M x N a split
  EPI_RESULT   // results in T, times 1 / scale, of this sum and earlier pieces' (`sums`)
};

// Maximum that takes no infinity as a shift (exp(inf - inf) is no number).
__device__ __forceinline__ float shift_of(float m) { return fabsf(m) == INFINITY ? 0.0f : m; }

__device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
  const float mm = fmaxf(m, m2), sh = shift_of(mm);
  s = s * __expf(m - sh) + s2 * __expf(m2 - sh);
  m = mm;
}

constexpr float LOG2E = 1.44269502162933349609375f;

// exp(z - shift), of shift log2 e.
__device__ __forceinline__ float exp_less(float z, float shift2) {
  return __builtin_amdgcn_exp2f(fmaf(z, LOG2E, -shift2));
}

// Tile (tm, tn) of workgroup `id`.  Workgroups go to the eight XCDs in turn,
// and each has a second-level cache: an XCD gets a run of consecutive tiles,
// eight rows of tiles deep, so that its workgroups share rows of both operands.
__device__ __forceinline__ void tile_of(const Product &g, unsigned id, int &tm, int &tn) {
  const unsigned all = (unsigned)g.tiles_m * (unsigned)g.tiles_n;
  const unsigned x = id % 8, per = all / 8, more = all % 8;
  const unsigned q = x * per + (x < more ? x : more) + id / 8;
  constexpr unsigned DEEP = 8;
  const unsigned band = q / (DEEP * g.tiles_n), first = band * DEEP;
  const unsigned deep = g.tiles_m - first < DEEP ? g.tiles_m - first : DEEP;
  const unsigned in = q - first * g.tiles_n;
  tm = (int)(first + in % deep);
  tn = (int)(in / deep);
}

enum Layout { ROWS_ROWS, ROWS_COLS, COLS_COLS };  // of A and B

template <typename T, int LAYOUT, int R, int NWV, typename ROWS>
using TileA = std::conditional_t<LAYOUT == COLS_COLS, ColTile<T, R, NWV, ROWS>,
                                 RowTile<T, R, NWV, ROWS>>;
template <typename T, int LAYOUT, int R, int NWV, typename SPREAD, typename ROWS>
using TileB = std::conditional_t<LAYOUT == ROWS_ROWS, RowTile<T, R, NWV, SPREAD>,
                                 ColTile<T, R, NWV, ROWS>>;

template <typename T, int LAYOUT, int WN, int FM, int FN, int EPI>
__device__ __forceinline__ void epilogue(const Product &g, float4v (&acc)[FM][FN], long long m0,
                                         long long n0, int tn, int wm, int wn, int split,
                                         int lane);

template <int BM, int BN>
constexpr int STAGE_BYTES = (BM + BN) * KBYTES;

// Tiles of BM x BN where there are too few large ones: two buffers, the loads of
// the next step under way while one step's fragments are multiplied, and several
// workgroups a CU that fill each other's gaps (three or four buffers, which leave
// room for fewer, took 5 to 60 % longer: 64,000 x 120 over 512 bf16, tiles of 32 x
// 128: 42 us with four, 27 with two).  Bound by the wait for loads and by the rounds
// of tiles (1053 x 7919 over 509 f16: 18 us, 0.46 Pflop/s, matrix cores busy 15 % of
// the time; 558 tiles for 512 places).  Whole rows of 16,000 x 69 over 512 bf16: 9 us
// for 21 MB; of 1266 x 41 over 333 float32: 8.
template <typename T, int LAYOUT, int BM, int BN, int WM, int WN, int EPI>
__device__ __forceinline__ void product_tile(const Product &g, unsigned id, int split,
                                             char *s_lds) {
  constexpr int NWV = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
  using A = TileA<T, LAYOUT, BM, NWV, Rows<BM, BM>>;
  // (whole rows are put together in LDS: any order of their columns will do)
  constexpr int SIDE = EPI == EPI_LOG ? 4 : 16 / (int)sizeof(T);
  using B = TileB<T, LAYOUT, BN, NWV, Spread<SIDE, FN, FN>, Rows<BN, BN>>;
  constexpr int STAGE = A::BYTES + B::BYTES, ROOM = 2 * STAGE;
  static_assert(STAGE == STAGE_BYTES<BM, BN>, "LDS of a step");
  const int lane = threadIdx.x & (WAVE - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  tile_of(g, id, tm, tn);
  const long long m0 = (long long)tm * BM, n0 = (long long)tn * BN;

  A ta;
  B tb;
  ta.init(g.A, 0, wave, lane);
  tb.init(g.B, 0, wave, lane);
  const char *pa = A::base(g.A, m0), *pb = B::base(g.B, n0);
  const long long na = A::bytes(g.A, m0), nb = B::bytes(g.B, n0);
  const uint32_t lds = lds_address(s_lds);
  const int all = (int)((g.K + k_step<T>() - 1) / k_step<T>());
  const int first = split * g.steps;
  const int end = all - first < g.steps ? all : first + g.steps;
  // (past the end: of empty buffers, so that there are always as many loads)
  const auto fetch = [&](int stage, int t) {
    const uint32_t to = lds + stage * STAGE;
    const int4v ba = A::step(g.A, pa, t < end ? na : 0, t);
    const int4v bb = B::step(g.B, pb, t < end ? nb : 0, t);
#pragma unroll
    for (int i = 0; i < A::LOADS; ++i) ta.fetch(i, to, ba, wave);
#pragma unroll
    for (int i = 0; i < B::LOADS; ++i) tb.fetch(i, to + A::BYTES, bb, wave);
  };

  float4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0, 0, 0, 0};
  fetch(0, first);
  int cur = 0;
  for (int t = first; t < end; ++t) {
    // step t has landed, and no one reads the buffer of the step before
    wait_loads<0>();
    __syncthreads();
    fetch(cur ^ 1, t + 1);
    const char *sa = s_lds + cur * STAGE, *sb = sa + A::BYTES;
    cur ^= 1;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      Frag<T> fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = A::frag(sa, (wm * FM + i) * 16, half, lane);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = B::frag(sb, (wn * FN + j) * 16, half, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mac(fb[j], fa[i], acc[i][j]);
    }
  }
  wait_loads<0>();  // (the empty ones, too: LDS is used for other things now, or by others)
  if constexpr (EPI == EPI_LOG) {
    // rows of log-probabilities, put together in LDS: the rows of a tile lie
    // side by side in memory (ldo is N)
    static_assert(LAYOUT == ROWS_ROWS && FM == 1, "a wavefront has 16 rows");
    static_assert(BM * BN * 4 <= ROOM, "room for the tile");
    __shared__ float2 s_row[WN][BM];
    constexpr int L = 4 * FN;
    const int group = lane >> 4, cols = (int)g.N, row = wm * 16 + (lane & 15);
    const auto column = [&](int q) {
      return wn * FN * 16 + Spread<SIDE, FN, FN>::column(group, q);
    };
    float mx = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int q = 0; q < L; ++q) {
      if (column(q) >= cols) acc[0][q / 4][q % 4] = -INFINITY;
      mx = fmaxf(mx, acc[0][q / 4][q % 4]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float sh = shift_of(mx);
#pragma unroll
    for (int q = 0; q < L; ++q) sum += exp_less(acc[0][q / 4][q % 4], sh * LOG2E);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16) s_row[wn][row] = make_float2(mx, sum);
    __syncthreads();  // and no one reads operands any more
    mx = s_row[0][row].x;
    sum = s_row[0][row].y;
#pragma unroll
    for (int q = 1; q < WN; ++q) join(mx, sum, s_row[q][row].x, s_row[q][row].y);
    const float lse = shift_of(mx) + logf(sum);
    float *s = reinterpret_cast<float *>(s_lds);
#pragma unroll
    for (int q = 0; q < L; ++q) {
      const int c = column(q);
      if (c < cols) s[row * cols + c] = acc[0][q / 4][q % 4] - lse;
    }
    __syncthreads();
    const int n = (int)(g.M - m0 < BM ? g.M - m0 : BM) * cols;
    float *out = static_cast<float *>(g.out) + m0 * cols;
    for (int i = threadIdx.x; i < n; i += NWV * WAVE) out[i] = s[i];
  } else if (EPI == EPI_RESULT && g.wide == 2 && !g.sums && n0 + BN <= g.N) {
    // results by way of LDS, so that whole rows of the tile are written
    constexpr int E = 16 / (int)sizeof(T), PITCH = BN + E, CHUNKS = BN / E;
    constexpr int ROWS = ROOM / (PITCH * (int)sizeof(T)) < BM ? BM / 2 : BM;
    static_assert(ROWS * PITCH * (int)sizeof(T) <= ROOM, "room for the rows");
    const float back = g.scale ? 1.0f / *g.scale : 1.0f;
    T *s = reinterpret_cast<T *>(s_lds);
#pragma unroll
    for (int part = 0; part < BM / ROWS; ++part) {
      __syncthreads();  // no one reads operands (the part before) any more
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int r = (wm * FM + i) * 16 + (lane & 15) - part * ROWS;
        if (r >= 0 && r < ROWS) {
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            const int c = wn * FN * 16 + (LAYOUT == ROWS_ROWS
                                              ? Spread<E, FN, FN>::column(lane >> 4, 4 * j)
                                              : j * 16 + (lane >> 4) * 4);
            typedef __attribute__((ext_vector_type(4))) T T4;
            *reinterpret_cast<T4 *>(s + r * PITCH + c) =
                T4{(T)(acc[i][j][0] * back), (T)(acc[i][j][1] * back), (T)(acc[i][j][2] * back),
                   (T)(acc[i][j][3] * back)};
          }
        }
      }
      __syncthreads();
      for (int q = threadIdx.x; q < ROWS * CHUNKS; q += NWV * WAVE) {
        const long long m = m0 + part * ROWS + q / CHUNKS;
        if (m < g.M)
          *reinterpret_cast<int4v *>(static_cast<T *>(g.out) + m * g.ldo + n0 + q % CHUNKS * E) =
              *reinterpret_cast<const int4v *>(s + q / CHUNKS * PITCH + q % CHUNKS * E);
      }
    }
  } else {
    epilogue<T, LAYOUT, WN, FM, FN, EPI>(g, acc, m0, n0, tn, wm, wn, split, lane);
  }
}

template <typename T, int LAYOUT, int BM, int BN, int WM, int WN, int EPI>
__global__ __launch_bounds__(WM *WN *WAVE) void k_product(Product g) {
  __shared__ __align__(1024) char s_lds[2 * STAGE_BYTES<BM, BN>];
  product_tile<T, LAYOUT, BM, BN, WM, WN, EPI>(g, blockIdx.x, blockIdx.z, s_lds);
}

// Both products of dS in one launch, the tiles with the longer sums first: where
// neither fills the card, its workgroups find a CU at once (two of them share
// one), and none is left to work alone at the end (1053 rows, 7919 words, 509 wide
// in f16: 33 us for both, 23 and 23 one after the other; with dx always first 64,000
// x 69 over 512 in float32 takes 230 us instead of 174).
template <typename T, int BM, int BN, int WM, int WN, int EPIX, int EPIW>
__global__ __launch_bounds__(WM *WN *WAVE) void k_products(Product dx, Product dw) {
  __shared__ __align__(1024) char s_lds[2 * STAGE_BYTES<BM, BN>];
  const unsigned tx = (unsigned)dx.tiles_m * dx.tiles_n, nx = tx * dx.splits;
  const unsigned tw = (unsigned)dw.tiles_m * dw.tiles_n, nw = tw * dw.splits;
  const bool x_first = dx.steps >= dw.steps;
  const unsigned first = x_first ? nx : nw, at = blockIdx.x;
  const unsigned id = at < first ? at : at - first;
  if ((at < first) == x_first)
    product_tile<T, ROWS_COLS, BM, BN, WM, WN, EPIX>(dx, id % tx, id / tx, s_lds);
  else
    product_tile<T, COLS_COLS, BM, BN, WM, WN, EPIW>(dw, id % tw, id / tw, s_lds);
}

__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" : : : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Tiles of 256 x 256, eight wavefronts as 2 x 4 of 128 x 64 results each.  A
// step (64 of the sum, 32 in float32) has two phases, the halves A0, A1 of a
// wavefront's rows, each with all its columns B.  A phase is a time for reading
// and one for multiplying, with a barrier after each, and the wavefronts of the
// lower half are one time behind: on every SIMD one wavefront multiplies while
// the other reads, so the matrix cores always have one to feed them.  (With four
// phases of a quarter each, a barrier for every 16 products instead of 32, a step
// took 3430 cycles; it takes 3060, of which the products are 2048.)
//
// The 256 rows of A and the 256 of B of a step are 32 KiB each; LDS holds five
// of them in a ring: B(t), A(t), B(t + 1), A(t + 1), B(t + 2), ...  One that was
// read in one phase is free in the next one's time for multiplying (the lower
// half has multiplied by then, so its reads are done).  B is read in phase 0
// and A for the last time in phase 1, so phase 0 of step t sends for B(t + 2) where
// A(t - 1) was, and phase 1 for A(t + 2) where B(t) was: four loads each.
// What the next phase reads has landed for all when each wavefront has waited
// for its own loads of it and met the others: five times of 32 products for a load
// to arrive, three for A0.
//
// What bounds it: waiting for loads, barriers and the card's power.  With 16,000
// x 32,000 over 1024 (bf16): products over long sums (dx, dw) 1.25 Pflop/s, 1.37
// in the first milliseconds, scores with their statistics 1.07, dS, whose 1 GB
// is written meanwhile, 0.91; the products alone, without reads or loads, would
// run at 2.0.
template <typename T, int LAYOUT>
struct Large {
  static constexpr int NWV = 8;
  using A = TileA<T, LAYOUT, 128, NWV, Rows<64, 128>>;
  using B = TileB<T, LAYOUT, 128, NWV, Spread<16 / (int)sizeof(T), 4, 2>, Rows<32, 64>>;
  static constexpr int PART = A::BYTES;
  static_assert(A::BYTES == B::BYTES && A::LOADS == 2 && B::LOADS == 2, "equal parts");

  static constexpr int PAIR = 2 * PART;  // an operand's rows of a step
  static constexpr int RING = 5 * PAIR;

  A ta[2];
  B tb[2];
  const char *pa, *pb;
  long long na, nb;  // bytes from there
  const char *lds;
  uint32_t at;
  int lane, wave, wm, wn;
  Frag<T> fa[4][2], fb[4][2];  // [fragment][half of the step]

  // the place `n` places on in the ring
  static __device__ __forceinline__ int on(int place, int n) {
    place += n * PAIR;
    return place >= RING ? place - RING : place;
  }
  // the i-th of four loads: A0, A0, A1, A1 or B, to a place in the ring
  __device__ __forceinline__ void load_a(int i, int4v buffer, int place) {
    ta[i / 2].fetch(i % 2, at + place + i / 2 * PART, buffer, wave);
  }
  __device__ __forceinline__ void load_b(int i, int4v buffer, int place) {
    tb[i / 2].fetch(i % 2, at + place + i / 2 * PART, buffer, wave);
  }
  template <int H>
  __device__ __forceinline__ void read_a(int place) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        fa[i][k] = A::frag(lds + place + H * PART, wm * 64 + i * 16, k, lane);
  }
  __device__ __forceinline__ void read_b(int place) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        fb[j][k] = B::frag(lds + place + j / 2 * PART, wn * 32 + j % 2 * 16, k, lane);
  }
  // The 32 products of rows' half HA, with load(0) .. load(N - 1) spread among
  // them: loads go out one in 16 cycles of a CU, and a wavefront that has to
  // wait for its turn feeds no matrix core.  The last LATE products come after
  // the barrier that ends the phase, so that there is work for the matrix core
  // while the other wavefront starts.
  template <int HA, int N, typename F>
  __device__ __forceinline__ void multiply(float4v (&acc)[8][4], F &&load) {
    constexpr int LATE = 4;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      if (q == 32 - LATE) {
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // all that was read
        meet();
      }
      const int k = q / 16, i = q / 4 % 4, j = q % 4;
      acc[HA * 4 + i][j] = mac(fb[j][k], fa[i][k], acc[HA * 4 + i][j]);
      if constexpr (N > 0) {
        constexpr int EVERY = 24 / N;
        if (q % EVERY == EVERY / 2 && q / EVERY < N) {
          __builtin_amdgcn_sched_barrier(0);
          load(q / EVERY);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
  }

  // Step t with B(t) at `place`; LEFT: steps after it (2: two at least).
  template <int LEFT>
  __device__ __forceinline__ void step(const Product &g, int t, int place,
                                       float4v (&acc)[8][4]) {
    const int4v ba = A::step(g.A, pa, na, t + 2), bb = B::step(g.B, pb, nb, t + 2);
    read_b(place);
    read_a<0>(on(place, 1));
    wait_loads<(LEFT > 0) ? 8 : 0>();
    meet();
    multiply<0, (LEFT > 1) ? 4 : 0>(acc, [&](int i) { load_b(i, bb, on(place, 4)); });
    read_a<1>(on(place, 1));
    if constexpr (LEFT > 0) wait_loads<(LEFT > 1) ? 6 : 2>();
    meet();
    multiply<1, (LEFT > 1) ? 4 : 0>(acc, [&](int i) { load_a(i, ba, place); });
  }

  // Sends for the first two steps of a tile (of those there are).
  __device__ __forceinline__ void begin(const Product &g, long long m0, long long n0, int first,
                                        int end) {
    pa = A::base(g.A, m0);
    pb = B::base(g.B, n0);
    na = A::bytes(g.A, m0);
    nb = B::bytes(g.B, n0);
    for (int s = 0; s < 2 && first + s < end; ++s) {
      const int4v ba = A::step(g.A, pa, na, first + s), bb = B::step(g.B, pb, nb, first + s);
#pragma unroll
      for (int i = 0; i < 4; ++i) load_b(i, bb, 2 * s * PAIR);
#pragma unroll
      for (int i = 0; i < 4; ++i) load_a(i, ba, (2 * s + 1) * PAIR);
    }
  }

  // Steps first .. end - 1 (one at least) of the tile that begin was called for.
  __device__ __forceinline__ void run(const Product &g, int first, int end,
                                      float4v (&acc)[8][4]) {
    const bool two = first + 1 < end;
    if (two)
      wait_loads<10>();
    else
      wait_loads<2>();
    meet();
    if (wm == 1) meet();
    int place = 0, t = first;
    for (; t + 2 < end; ++t, place = on(place, 2)) step<2>(g, t, place, acc);
    if (two) {
      step<1>(g, t, place, acc);
      ++t;
      place = on(place, 2);
    }
    step<0>(g, t, place, acc);
    if (wm == 0) meet();
  }
};

template <typename T, int LAYOUT, int EPI>
__global__ __launch_bounds__(512) void k_product_large(Product g) {
  using L = Large<T, LAYOUT>;
  __shared__ __align__(1024) char s_lds[L::RING];
  L l;
  l.lane = threadIdx.x & (WAVE - 1);
  l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  l.wm = l.wave / 4;
  l.wn = l.wave % 4;
  l.lds = s_lds;
  l.at = lds_address(s_lds);
  const int split = blockIdx.z;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l.ta[h].init(g.A, h * 64, l.wave, l.lane);
    l.tb[h].init(g.B, LAYOUT == ROWS_ROWS ? h * 2 : h * 32, l.wave, l.lane);
  }
  const int all = (int)((g.K + k_step<T>() - 1) / k_step<T>());
  const int first = split * g.steps;
  const int end = all - first < g.steps ? all : first + g.steps;
  const unsigned tiles = (unsigned)g.tiles_m * (unsigned)g.tiles_n;

  int tm, tn;
  tile_of(g, blockIdx.x, tm, tn);
  if (first < end) l.begin(g, tm * 256ll, tn * 256ll, first, end);
  for (unsigned id = blockIdx.x; id < tiles; id += gridDim.x) {
    float4v acc[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = float4v{0, 0, 0, 0};
    if (first < end) l.run(g, first, end, acc);
    const long long m0 = tm * 256ll, n0 = tn * 256ll;
    const int at = tn;
    if (id + gridDim.x < tiles) {  // the next tile's first loads, while this one is written
      tile_of(g, id + gridDim.x, tm, tn);
      if (first < end) l.begin(g, tm * 256ll, tn * 256ll, first, end);
    }
    epilogue<T, LAYOUT, 4, 8, 4, EPI>(g, acc, m0, n0, at, l.wm, l.wn, split, l.lane);
  }
}

// acc[i][j][r] is row m0 + (wm FM + i) 16 + (lane & 15).  Of the wavefront's
// columns, n0 + wn 16 FN on, it is Spread's where B is row-wise, 16 j + (lane >>
// 4) 4 + r where it is not.
template <typename T, int LAYOUT, int WN, int FM, int FN, int EPI>
__device__ __forceinline__ void epilogue(const Product &g, float4v (&acc)[FM][FN], long long m0,
                                         long long n0, int tn, int wm, int wn, int split,
                                         int lane) {
  constexpr int L = 4 * FN;  // results of a lane in a row
  const int group = lane >> 4;
  if constexpr (EPI == EPI_PART || EPI == EPI_SCORE || EPI == EPI_DS) {
    static_assert(LAYOUT == ROWS_ROWS, "a lane's results side by side");
    constexpr int E = 16 / (int)sizeof(T);
    const long long nb = n0 + wn * FN * 16;
    const bool full = nb + FN * 16 <= g.N;
    const auto col = [&](int q) { return Spread<E, FN, FN>::column(group, q); };
    // which of the lane's results the row's target is, -1: none
    const auto place = [&](long long word) {
      const long long c = word - nb;
      return c < 0 || c >= FN * 16 || c / E % 4 != group ? -1 : (int)(c / (4 * E) * E + c % E);
    };
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const long long m = m0 + (wm * FM + i) * 16 + (lane & 15);
      const bool in = m < g.M;
      if constexpr (EPI == EPI_DS) {
        const int32_t tgt = in ? g.target[m] : -1;
        float c = in && tgt != -1 ? (g.grad ? g.grad[m] : 1.0f) : 0.0f;
        if (tgt < -1 || tgt >= g.words) c = NAN;  // no such word
        if (g.scale) c *= *g.scale;
        const float lse2 = (in ? g.lse[m] : 0.0f) * LOG2E;
        float v[L];
#pragma unroll
        for (int q = 0; q < L; ++q) v[q] = c * exp_less(acc[i][q / 4][q % 4], lse2);
        const int at = place(tgt - g.n0);
        if (at >= 0) {  // (one lane in many)
#pragma unroll
          for (int q = 0; q < L; ++q)
            if (q == at) v[q] -= c;
        }
        if (__any(c == 0.0f)) {  // rows without a word: zeros, whatever their scores
#pragma unroll
          for (int q = 0; q < L; ++q)
            if (c == 0.0f) v[q] = 0.0f;
        }
        if (!full) {
#pragma unroll
          for (int q = 0; q < L; ++q)
            if (nb + col(q) >= g.N) v[q] = 0.0f;
        }
        if (in && nb < g.Np) {
          alignas(16) T o[L];
#pragma unroll
          for (int q = 0; q < L; ++q) o[q] = (T)v[q];
          T *to = static_cast<T *>(g.out) + m * g.ldo + nb;
#pragma unroll
          for (int q = 0; q < L; q += E)
            if (nb + col(q) < g.Np)
              *reinterpret_cast<int4v *>(to + col(q)) = *reinterpret_cast<const int4v *>(o + q);
          if (g.lo) {
            to += g.lo;
#pragma unroll
            for (int q = 0; q < L; ++q) o[q] = (T)(v[q] - (float)o[q]);
#pragma unroll
            for (int q = 0; q < L; q += E)
              if (nb + col(q) < g.Np)
                *reinterpret_cast<int4v *>(to + col(q)) = *reinterpret_cast<const int4v *>(o + q);
          }
        }
      } else {
        if constexpr (EPI == EPI_PART) {
          const int32_t tgt = in ? g.target[m] : -1;
          const int at = tgt < g.N ? place(tgt) : -1;
          if (at >= 0) {
#pragma unroll
            for (int q = 0; q < L; ++q)
              if (q == at) g.hit[m] = acc[i][q / 4][q % 4];
          }
        } else if (in) {
          float *to = static_cast<float *>(g.out) + m * g.ldo + nb;
#pragma unroll
          for (int q = 0; q < L; ++q)
            if (full || nb + col(q) < g.N) to[col(q)] = acc[i][q / 4][q % 4];
        }
        if (!full) {  // what is not there weighs nothing
#pragma unroll
          for (int q = 0; q < L; ++q)
            if (nb + col(q) >= g.N) acc[i][q / 4][q % 4] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int q = 0; q < L; ++q) mx = fmaxf(mx, acc[i][q / 4][q % 4]);
        // the four lanes of a row
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float s2 = shift_of(mx) * LOG2E;
        float sum = 0.0f;
#pragma unroll
        for (int q = 0; q < L; ++q) sum += exp_less(acc[i][q / 4][q % 4], s2);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (in && lane < 16) g.part[(long long)(tn * WN + wn) * g.M + m] = make_float2(mx, sum);
      }
    }
  } else {
    const float back = EPI == EPI_RESULT && g.scale ? 1.0f / *g.scale : 1.0f;
    typedef std::conditional_t<EPI == EPI_SUM, float, T> O;
    typedef __attribute__((ext_vector_type(4))) O O4;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const long long m = m0 + (wm * FM + i) * 16 + (lane & 15);
      if (m >= g.M) continue;
      O *row = static_cast<O *>(g.out) + (EPI == EPI_SUM ? split * g.M + m : m) * g.ldo;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const long long n = n0 + wn * FN * 16 +
                            (LAYOUT == ROWS_ROWS
                                 ? Spread<16 / (int)sizeof(T), FN, FN>::column(group, 4 * j)
                                 : j * 16 + group * 4);
        if (n >= g.N) continue;
        float4v v = acc[i][j];
        if (EPI == EPI_RESULT && g.sums) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r < g.N) v[r] += g.sums[m * ((g.N + 3) / 4 * 4) + n + r];
        }
        v *= back;
        if (g.wide && n + 4 <= g.N) {
          if (EPI == EPI_SUM && g.add) v += *reinterpret_cast<const float4v *>(row + n);
          *reinterpret_cast<O4 *>(row + n) = O4{(O)v[0], (O)v[1], (O)v[2], (O)v[3]};
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r < g.N)
              row[n + r] = (O)(EPI == EPI_SUM && g.add ? v[r] + (float)row[n + r] : v[r]);
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// rows and elements
// ---------------------------------------------------------------------------

// Copies of two matrices with rows padded with zeros to `cols` elements (whole
// groups of 16 bytes, one a thread; 7919 and 1053 rows of 509 f16: 5 to 7 us).
template <typename T>
struct Pad {
  const T *p;
  long long ld, rows, n, cols;
  T *out;
};
template <typename T>
struct Pads {
  Pad<T> x, w;
  long long groups() const { return (x.rows * x.cols + w.rows * w.cols) / (16 / (int)sizeof(T)); }
};
// (workgroup `block` of `blocks`)
template <typename T>
__device__ __forceinline__ void pad(const Pads<T> &pads, unsigned block, unsigned blocks) {
  constexpr int E = 16 / (int)sizeof(T);
  const Pad<T> &x = pads.x, &w = pads.w;
  const long long nx = x.rows * (x.cols / E), nw = w.rows * (w.cols / E);
  for (long long i = (long long)block * blockDim.x + threadIdx.x; i < nx + nw;
       i += (long long)blocks * blockDim.x) {
    const Pad<T> &m = i < nx ? x : w;
    const long long q = i < nx ? i : i - nx, groups = m.cols / E;
    const long long r = q / groups, c = (q - r * groups) * E;
    alignas(16) T v[E];
    const T *p = m.p + r * m.ld + c;
    if (c + E <= m.n) {
      __builtin_memcpy(v, p, 16);  // (one load, wherever it lies)
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = c + e < m.n ? p[e] : (T)0.0f;
    }
    *reinterpret_cast<int4v *>(m.out + r * m.cols + c) = *reinterpret_cast<const int4v *>(v);
  }
}
template <typename T>
__global__ __launch_bounds__(NT) void k_pad(Pads<T> pads) {
  pad(pads, blockIdx.x, gridDim.x);
}

__device__ __forceinline__ float wave_sum_f(float v) {
#pragma unroll
  for (int x = 1; x < WAVE; x <<= 1) v += __shfl_xor(v, x);
  return v;
}

// The log of the sum of exponentials of rows r0 .. r0 + ROWS - 1 from their
// parts' maxima and sums, by a workgroup, to s_lse.
template <int ROWS>
__device__ __forceinline__ void rows_lse(const float2 *__restrict__ part, int parts,
                                         long long rows, long long r0, float *s_lse) {
  constexpr int SLICES = NT / ROWS;
  __shared__ float2 s_part[NT];
  const int row = threadIdx.x % ROWS, slice = threadIdx.x / ROWS;
  float m = -INFINITY, s = 0.0f;
  if (r0 + row < rows) {
#pragma unroll 4
    for (int i = slice; i < parts; i += SLICES) {
      const float2 v = part[(long long)i * rows + r0 + row];
      join(m, s, v.x, v.y);
    }
  }
  // a wavefront's slices of a row, then the wavefronts'
#pragma unroll
  for (int x = ROWS; x < WAVE; x <<= 1) {
    const float m2 = __shfl_xor(m, x), s2 = __shfl_xor(s, x);
    join(m, s, m2, s2);
  }
  s_part[threadIdx.x] = make_float2(m, s);
  __syncthreads();
  if (slice == 0) {
    for (int i = 1; i < NWAVES; ++i) join(m, s, s_part[i * WAVE + row].x, s_part[i * WAVE + row].y);
    // (a row of infinities: the sum, or none of it, is what is left)
    s_lse[row] = shift_of(m) + logf(s);
  }
  __syncthreads();
}

template <int ROWS>
__global__ __launch_bounds__(NT) void k_loss(const float2 *__restrict__ part, int parts,
                                             long long rows, const int32_t *__restrict__ target,
                                             long long words, const float *__restrict__ hit,
                                             float *__restrict__ loss, float *__restrict__ lse) {
  __shared__ float s_lse[ROWS];
  const long long r0 = (long long)blockIdx.x * ROWS, r = r0 + threadIdx.x;
  rows_lse<ROWS>(part, parts, rows, r0, s_lse);
  if (threadIdx.x >= ROWS || r >= rows) return;
  const float l = s_lse[threadIdx.x];
  lse[r] = l;
  const int32_t t = target[r];
  loss[r] = t == -1 ? 0.0f : t < -1 || t >= words ? NAN : l - hit[r];
}

// Scores to log-probabilities, in place (bound by memory: 4 bytes read and written
// a score, after the product wrote them; with the product 13,000 x 257 over 512 bf16
// take 34 us and 13,000 x 1000 86, 256 classes as whole rows 16).
template <int ROWS>
__global__ __launch_bounds__(NT) void k_normalise(const float2 *__restrict__ part, int parts,
                                                  long long rows, long long cols,
                                                  float *__restrict__ z) {
  __shared__ float s_lse[ROWS];
  const long long r0 = (long long)blockIdx.x * ROWS;
  rows_lse<ROWS>(part, parts, rows, r0, s_lse);
  const int n = rows - r0 < ROWS ? (int)(rows - r0) : ROWS;
  for (int r = 0; r < n; ++r)
    for (long long c = threadIdx.x; c < cols; c += NT) z[(r0 + r) * cols + c] -= s_lse[r];
}

// The power of two that brings the largest |gradient| to [2^13, 2^14): 16-bit
// floats then hold dS down to 2^-38 of it, and no |dS| (at most twice the
// largest) overflows.  1 where the largest is 0, infinite or no number.
__device__ __forceinline__ float scale_of(uint32_t bits) {
  const int e = (int)(bits >> 23);
  if (e == 0 || e >= 255) return 1.0f;
  const int k = 127 + 13 - (e - 127);
  return __uint_as_float((uint32_t)(k < 1 ? 1 : k > 254 ? 254 : k) << 23);
}

__device__ __forceinline__ float block_max(float m) {
  __shared__ float s_max[16];
#pragma unroll
  for (int x = 1; x < WAVE; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
  if (__lane_id() == 0) s_max[threadIdx.x / WAVE] = m;
  __syncthreads();
  m = 0.0f;
  for (int i = 0; i < (int)(blockDim.x / WAVE); ++i) m = fmaxf(m, s_max[i]);
  return m;
}

// The largest |p[i]| of rows with a word (p null: 1): one workgroup, the power
// of two for it; several, each its own (then once more over theirs).
__global__ __launch_bounds__(1024) void k_scale(const float *__restrict__ p,
                                                const int32_t *__restrict__ target, long long n,
                                                float *__restrict__ out) {
  float m = p ? 0.0f : 1.0f;
  if (p)
    for (long long i = (long long)blockIdx.x * 1024 + threadIdx.x; i < n;
         i += (long long)gridDim.x * 1024)
      if (!target || target[i] >= 0) m = fmaxf(m, fabsf(p[i]));
  m = block_max(m);
  if (threadIdx.x == 0) out[blockIdx.x] = gridDim.x > 1 ? m : scale_of(__float_as_uint(m));
}

// Emissions: for each workgroup the largest of its rows' gradients and of their
// sums.
__global__ __launch_bounds__(NT) void k_emission_max(const float *__restrict__ grad,
                                                     long long rows, long long cols,
                                                     float *__restrict__ out) {
  const int lane = threadIdx.x & (WAVE - 1);
  float m = 0.0f;
  for (long long r = (long long)blockIdx.x * NWAVES + threadIdx.x / WAVE; r < rows;
       r += (long long)gridDim.x * NWAVES) {
    float s = 0.0f;
    for (long long c = lane; c < cols; c += WAVE) {
      const float g = grad[r * cols + c];
      s += g;
      m = fmaxf(m, fabsf(g));
    }
    m = fmaxf(m, fabsf(wave_sum_f(s)));
  }
  m = block_max(m);
  if (threadIdx.x == 0) out[blockIdx.x] = m;
}

// 16 bytes of dS, and what rounding lost `lo` columns further on (0: dropped).
template <typename T, int E>
__device__ __forceinline__ void put_ds(T *to, const float (&d)[E], long long lo) {
  alignas(16) T v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = (T)d[e];
  *reinterpret_cast<int4v *>(to) = *reinterpret_cast<const int4v *>(v);
  if (lo) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (T)(d[e] - (float)v[e]);
    *reinterpret_cast<int4v *>(to + lo) = *reinterpret_cast<const int4v *>(v);
  }
}

// dS = grad - exp(weight) sum(grad), zeros up to Cp columns; a wavefront a row.
// Workgroups past the first `blocks` make the copies (one launch less).
template <typename T>
__global__ __launch_bounds__(NT) void k_emission_ds(Pads<T> pads, unsigned blocks,
                                                    const float *__restrict__ weight,
                                                    const float *__restrict__ grad,
                                                    long long rows, long long cols,
                                                    const float *__restrict__ scale,
                                                    T *__restrict__ out, long long Cp,
                                                    long long ld) {
  if (blockIdx.x >= blocks) return pad(pads, blockIdx.x - blocks, gridDim.x - blocks);
  constexpr int E = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & (WAVE - 1);
  const long long r = (long long)blockIdx.x * NWAVES + threadIdx.x / WAVE;
  if (r >= rows) return;  // (a row's lanes together)
  const float k = scale ? *scale : 1.0f;
  const float *g = grad + r * cols, *w = weight + r * cols;
  float s = 0.0f;
#pragma unroll 4
  for (long long c = lane; c < cols; c += WAVE) s += g[c];
  s = wave_sum_f(s);
  for (long long c = (long long)lane * E; c < Cp; c += WAVE * E) {
    float d[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      d[e] = c + e < cols ? k * (g[c + e] - exp_less(w[c + e], 0.0f) * s) : 0.0f;
    put_ds(out + r * ld + c, d, ld > Cp ? Cp : 0);
  }
}

// The same where rows are short (cols <= SHORT): 16 rows a workgroup, which lie
// side by side, by way of LDS (16,000 x 69: 6 us, of which a launch is 2; 13 MB).
constexpr int SHORT = 256;
template <typename T>
__global__ __launch_bounds__(NT) void k_emission_ds_short(Pads<T> pads, unsigned blocks,
                                                          const float *__restrict__ weight,
                                                          const float *__restrict__ grad,
                                                          long long rows, int cols,
                                                          const float *__restrict__ scale,
                                                          T *__restrict__ out, int Cp, int ld) {
  if (blockIdx.x >= blocks) return pad(pads, blockIdx.x - blocks, gridDim.x - blocks);
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ float s_w[16 * SHORT], s_g[16 * SHORT];
  __shared__ float s_sum[16];
  const long long r0 = (long long)blockIdx.x * 16;
  const int n = (int)(rows - r0 < 16 ? rows - r0 : 16);
  const float k = scale ? *scale : 1.0f;
#pragma unroll 4
  for (int i = threadIdx.x; i < n * cols; i += NT) {
    s_w[i] = weight[r0 * cols + i];
    s_g[i] = grad[r0 * cols + i];
  }
  __syncthreads();
  const int row = threadIdx.x / 16;
  float s = 0.0f;
  if (row < n)
    for (int c = threadIdx.x % 16; c < cols; c += 16) s += s_g[row * cols + c];
#pragma unroll
  for (int x = 1; x < 16; x <<= 1) s += __shfl_xor(s, x);
  if (threadIdx.x % 16 == 0) s_sum[row] = s;
  __syncthreads();
  const int groups = Cp / E;
  for (int i = threadIdx.x; i < n * groups; i += NT) {
    const int r = i / groups, c = (i - r * groups) * E;
    float d[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
      d[e] = c + e < cols ? k * (s_g[r * cols + c + e] -
                                 exp_less(s_w[r * cols + c + e], 0.0f) * s_sum[r])
                          : 0.0f;
    put_ds(out + (r0 + r) * ld + c, d, ld > Cp ? Cp : 0);
  }
}

// Sums of the splits to results: 64 groups of four columns a workgroup, each
// split by its four wavefronts in turn, added in a fixed order.  (Rows of
// `sums` are padded to whole groups.  37 splits of 69 x 512: 3.9 us, nearly all
// of it launch and loads; 6 of 1053 x 509: 5.3.)
template <typename T>
struct Finish {
  const float *sums;
  int splits;
  long long rows, cols;
  T *out;
  long long ldo;
  __host__ __device__ long long groups() const { return rows * ((cols + 3) / 4); }
};
// (of two products, or of one: b has no rows)
template <typename T>
__global__ __launch_bounds__(NT) void k_finish(Finish<T> a, Finish<T> b,
                                               const float *__restrict__ scale) {
  __shared__ float4v s_sum[NWAVES][WAVE];
  const int lane = threadIdx.x & (WAVE - 1), w = threadIdx.x / WAVE;
  const float back = scale ? 1.0f / *scale : 1.0f;
  const long long na = (a.groups() + WAVE - 1) / WAVE, nb = (b.groups() + WAVE - 1) / WAVE;
  for (long long k = blockIdx.x; k < na + nb; k += gridDim.x) {
    const Finish<T> &f = k < na ? a : b;
    const long long i = (k < na ? k : k - na) * WAVE + lane, all = f.groups();
    const long long groups = (f.cols + 3) / 4;
    float4v v = {0, 0, 0, 0};
    if (i < all) {
#pragma unroll 8
      for (int s = w; s < f.splits; s += NWAVES)
        v += reinterpret_cast<const float4v *>(f.sums)[s * all + i];
    }
    s_sum[w][lane] = v;
    __syncthreads();
    if (w == 0 && i < all) {
#pragma unroll
      for (int q = 1; q < NWAVES; ++q) v += s_sum[q][lane];
      const long long r = i / groups, c = (i - r * groups) * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < f.cols) f.out[r * f.ldo + c + e] = (T)(v[e] * back);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// plans
// ---------------------------------------------------------------------------

constexpr int CUS = 256;

long long up(long long x, long long m) { return (x + m - 1) / m * m; }
unsigned blocks_for(long long items, long long per, long long most = 1 << 16) {
  const long long b = (items + per - 1) / per;
  return (unsigned)(b < 1 ? 1 : b < most ? b : most);
}

// Workspace, laid out by running a plan once without memory.
struct Bump {
  char *base;
  size_t at = 0;
  template <typename U>
  U *take(long long n) {
    U *p = reinterpret_cast<U *>(base + at);
    at += ((size_t)n * sizeof(U) + 255) & ~(size_t)255;
    return base ? p : nullptr;
  }
};

struct Tile {
  int bm, bn, wn;
};
constexpr Tile TILES[3] = {{256, 256, 4}, {128, 128, 2}, {64, 64, 2}};

// How a product is cut: the tile, and the parts of its sum.
struct Cut {
  int tile, splits, steps;
  double us;
};

// The cut that takes least, by a model in microseconds fitted to products of
// 0.5 to 35 Gflop (2000 x 4000 over 512, tiles of 256, 128 and 64: measured 19, 12
// and 19; 1600 x 26,000 over 256: 42, 43, 55; 64 x 10,000 over 512: 17, 10 and 7;
// 4096 x 4096 over 1024: 32, 38, 59).  A step of the largest tile takes a CU 1.54
// (256 of the products at once); 512 of the next take 1, 0.7 where a CU has
// one alone (eight wavefronts of 32 x 64: four of 64 x 64 take 1.2); of the
// smallest 256 take 0.22, one alone 0.5.  In float32 the matrix cores take
// longer than that.  Splitting costs a launch and the sums' way to memory and
// back.
template <typename T>
Cut cut_for(long long M, long long N, long long K, bool may_split, int only = -1) {
  const long long all = (K + k_step<T>() - 1) / k_step<T>();
  const bool wide = sizeof(T) == 4;
  Cut best{0, 1, (int)(all < 1 ? 1 : all), 0};
  double least = 1e30;
  for (int tile = 0; tile < 3; ++tile) {
    if (only >= 0 && tile != only) continue;
    const double tiles = (double)((M + TILES[tile].bm - 1) / TILES[tile].bm) *
                         (double)((N + TILES[tile].bn - 1) / TILES[tile].bn);
    for (long long p = 1; p == 1 || (may_split && p <= 256 && p <= all / 2); p += 1 + p / 4) {
      if (p > 1 && tiles * p > 8 * CUS) break;  // enough for every CU
      const double per = (double)((all + p - 1) / p), q = ceil(tiles * p / CUS);
      double us;
      if (tile == 0) {
        us = 1.5 + q * (per * (wide ? 7.0 : 1.54) + 5.5);
      } else if (tile == 1) {
        const double pairs = floor(tiles * p / (2 * CUS)), rest = tiles * p - pairs * 2 * CUS;
        us = 4 + per * (wide ? 3.5 : 1.0) *
                     (pairs + (rest <= 0 ? 0 : rest > CUS ? 1 : wide ? 0.5 : 0.7));
      } else {
        us = 3.5 + per * (wide ? 0.5 * q : fmax(0.5, 0.218 * q));
      }
      if (p > 1) us += 3.5 + (double)p * M * N * 8 / 4e6;
      if (us < least) {
        least = us;
        best = {tile, 1, (int)((all + p - 1) / p), us};
        best.splits = all ? (int)((all + best.steps - 1) / best.steps) : 1;
        if (best.steps < 1) best.steps = 1;
      }
    }
  }
  return best;
}

template <typename T, int LAYOUT, int EPI>
hipError_t product(Product g, int tile, hipStream_t s) {
  const Tile c = TILES[tile];
  const long long tm = (g.M + c.bm - 1) / c.bm, tn = (g.N + c.bn - 1) / c.bn;
  if (tm * tn * 512 >= (1ll << 32) || tm > INT32_MAX || tn > INT32_MAX) return hipErrorInvalidValue;
  g.tiles_m = (int)tm;
  g.tiles_n = (int)tn;
  const dim3 grid((unsigned)(tm * tn), 1, (unsigned)g.splits);
  if (tile == 0)
    k_product_large<T, LAYOUT, EPI>
        <<<dim3((unsigned)(tm * tn < CUS ? tm * tn : CUS), 1, (unsigned)g.splits), 512, 0, s>>>(g);
  else if (tile == 1)
    k_product<T, LAYOUT, 128, 128, 4, 2, EPI><<<grid, 512, 0, s>>>(g);
  else
    k_product<T, LAYOUT, 64, 64, 2, 2, EPI><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

#define TRY(e)                           \
  do {                                   \
    const hipError_t e_ = (e);           \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

// Bytes between rows of an operand, at most: 255 of them fit 32 bits.  (Copies
// and dS keep to it by FST_HEAD_MAX_COLS, dS with twice as many columns of 16
// bits and DS_GAP.)
constexpr long long ROW_BYTES = 1 << 24;
static_assert(255 * (ROW_BYTES + 1024) < (1ll << 32) && FST_HEAD_MAX_COLS * 4ll <= ROW_BYTES,
              "offsets in a tile");

// An operand whose rows are whole K-steps from aligned addresses, as it is or
// copied so.
template <typename T>
struct Laid {
  Operand o;
  T *copy;
  long long cols;
  Operand columns() const { return {o.p, o.ld, cols, o.rows}; }  // read column by column
};

template <typename T>
Laid<T> lay(const Mat &m, Bump &b) {
  const long long cols = up(m.cols, k_step<T>());
  if ((uintptr_t)m.data % 16 == 0 && m.stride * sizeof(T) % 16 == 0 && cols == m.cols &&
      m.stride * (long long)sizeof(T) <= ROW_BYTES)
    return {{m.data, m.stride, m.rows, cols}, nullptr, cols};
  T *p = b.take<T>(m.rows * cols);
  return {{p, cols, m.rows, cols}, p, cols};
}
// The copies there are to make.
template <typename T>
Pads<T> copies(const Laid<T> *lx, const Mat &x, const Laid<T> *lw, const Mat &w) {
  Pads<T> p{};
  if (lx && lx->copy)
    p.x = {static_cast<const T *>(x.data), x.stride, x.rows, x.cols, lx->cols, lx->copy};
  if (lw && lw->copy)
    p.w = {static_cast<const T *>(w.data), w.stride, w.rows, w.cols, lw->cols, lw->copy};
  return p;
}
template <typename T>
unsigned pad_blocks(const Pads<T> &p) {
  return p.groups() ? blocks_for(p.groups(), NT) : 0;
}
template <typename T>
hipError_t fill(const Pads<T> &p, hipStream_t s) {
  if (const unsigned n = pad_blocks(p)) k_pad<T><<<n, NT, 0, s>>>(p);
  return hipGetLastError();
}

// Whether four results side by side may be written at once, or (2) 16 bytes.
template <typename T>
int wide(const Mat &m) {
  if ((uintptr_t)m.data % 16 == 0 && m.stride * sizeof(T) % 16 == 0) return 2;
  return (uintptr_t)m.data % (4 * sizeof(T)) == 0 && m.stride % 4 == 0;
}

template <typename T>
hipError_t finish(const Finish<T> &a, const Finish<T> &b, const float *scale, hipStream_t s) {
  const long long n = (a.groups() + WAVE - 1) / WAVE + (b.groups() + WAVE - 1) / WAVE;
  if (n) k_finish<T><<<blocks_for(n, 1), NT, 0, s>>>(a, b, scale);
  return hipGetLastError();
}
// Zeros: the sum of nothing.
template <typename T>
hipError_t clear(const Mat &out, hipStream_t s) {
  return finish<T>({nullptr, 0, out.rows, out.cols, static_cast<T *>(out.data), out.stride}, {},
                   nullptr, s);
}

// out = A B^T, its sum in parts where that takes less.
template <typename T, int LAYOUT>
struct SplitProduct {
  Cut cut;
  float *sums;

  void plan(long long M, long long N, long long K, Bump &b) {
    cut = {0, 1, 1, 0};
    if (M == 0 || N == 0) return;
    cut = cut_for<T>(M, N, K, true);
    room(M, N, b);
  }
  void room(long long M, long long N, Bump &b) {
    sums = cut.splits > 1 ? b.take<float>(cut.splits * M * up(N, 4)) : nullptr;
  }
  Product of(Operand A, Operand B, long long M, long long N, long long K, const float *scale,
             const Mat &out) const {
    Product g{};
    g.A = A;
    g.B = B;
    g.M = M;
    g.N = N;
    g.K = K;
    g.splits = cut.splits;
    g.steps = cut.steps;
    if (cut.splits == 1) {
      g.out = out.data;
      g.ldo = out.stride;
      g.wide = wide<T>(out);
      g.scale = scale;
      return g;
    }
    g.out = sums;
    g.ldo = up(N, 4);
    g.wide = 1;
    return g;
  }
  Finish<T> rest(const Mat &out) const {  // what is left to do: nothing where nothing was cut
    return {sums, cut.splits, cut.splits > 1 ? out.rows : 0, out.cols, static_cast<T *>(out.data),
            out.stride};
  }
  hipError_t run(Operand A, Operand B, long long M, long long N, long long K, const float *scale,
                 const Mat &out, hipStream_t s) const {
    if (M == 0 || N == 0) return hipSuccess;
    const Product g = of(A, B, M, N, K, scale, out);
    if (cut.splits == 1) return product<T, LAYOUT, EPI_RESULT>(g, cut.tile, s);
    TRY((product<T, LAYOUT, EPI_SUM>(g, cut.tile, s)));
    return finish(rest(out), {}, scale, s);
  }
};

// dS has the matrices' type, so that the matrix cores multiply it: in 16 bits
// each element is rounded, by half a spacing of itself at most, and a gradient is
// off by that much of the sizes of the terms that it sums, whatever N and C are.
// As two numbers, the rounded one and the rest, dS loses next to nothing, for twice
// the products of dx and dw.  One and two, against 64 bits, with the forward call:
// 16,000 x 69 over 512 bf16 0.0023 and 0.0017 of the gradients' size (the latter
// is their own rounding) in 28 and 35 us; 1053 x 7919 over 509 f16 0.00033 and
// 0.00025 in 96 and 129; 16,000 x 32,000 over 1024 bf16 0.0024 and 0.0017 in 3.58
// and 5.38 ms.  What the second number takes decides: there is one up to 2^28
// products, where that is 5 us at most.
template <typename T>
bool in_two(long long N, long long C, long long H) {
  return sizeof(T) == 2 && (double)N * C * H <= (double)(1 << 28);
}

// The two products of dS, N x C with rows of `ld` (Cp columns, and again Cp of
// rests if `two`): their operands.
template <typename T>
struct Gradients {
  Operand dx_a, dx_b, dw_a, dw_b;
  long long dx_k, dw_k;

  Gradients(const T *ds, long long ld, long long N, long long Cp, bool two, Operand w, Operand x) {
    const long long Ns = up(N, k_step<T>());
    dx_a = {ds, ld, N, two ? 2 * Cp : Cp};
    dx_b = w;
    dw_a = {ds, ld, two ? 2 * Cp : Cp, N};
    dw_b = x;
    dx_k = Cp;
    dw_k = N;
    if (two) {
      dx_b.wrap = (int)(Cp / k_step<T>());
      dw_a.wrap = dw_b.wrap = (int)(Ns / k_step<T>());
      dw_a.jump = Cp * (long long)sizeof(T);
      dx_k = 2 * Cp;
      dw_k = 2 * Ns;
    }
  }
};

template <typename T, int BM, int BN, int WM, int WN>
void products(const Product &x, const Product &w, unsigned grid, hipStream_t s) {
  if (x.splits > 1 && w.splits > 1)
    k_products<T, BM, BN, WM, WN, EPI_SUM, EPI_SUM><<<grid, WM * WN * WAVE, 0, s>>>(x, w);
  else if (x.splits > 1)
    k_products<T, BM, BN, WM, WN, EPI_SUM, EPI_RESULT><<<grid, WM * WN * WAVE, 0, s>>>(x, w);
  else if (w.splits > 1)
    k_products<T, BM, BN, WM, WN, EPI_RESULT, EPI_SUM><<<grid, WM * WN * WAVE, 0, s>>>(x, w);
  else
    k_products<T, BM, BN, WM, WN, EPI_RESULT, EPI_RESULT><<<grid, WM * WN * WAVE, 0, s>>>(x, w);
}

// dx (N x H) and dw (C x H) from dS, those that are wanted: cut the same way
// whether or not the other one is.  In one launch unless one of them has the
// largest tiles (2000 rows, 1000 columns, width 512: 34 us as two, 27 as one;
// 16,000, 69, 512: 29 and 22); tiles of 128 if they would differ in 16 bits (64:
// 27 us of the last), in float32 what the model says of both.
template <typename T>
struct Both {
  SplitProduct<T, ROWS_COLS> x;
  SplitProduct<T, COLS_COLS> w;
  bool one;  // launch

  void plan(const Gradients<T> &p, bool gx, bool gw, long long N, long long C, long long H,
            Bump &b) {
    x.cut = cut_for<T>(N, H, p.dx_k, true);
    w.cut = cut_for<T>(C, H, p.dw_k, true);
    one = x.cut.tile && w.cut.tile;
    if (one && x.cut.tile != w.cut.tile) {
      double least = 1e30;
      for (int tile = 1; tile <= (sizeof(T) == 2 ? 1 : 2); ++tile) {
        const Cut cx = cut_for<T>(N, H, p.dx_k, true, tile);
        const Cut cw = cut_for<T>(C, H, p.dw_k, true, tile);
        if (cx.us + cw.us >= least) continue;
        least = cx.us + cw.us;
        x.cut = cx;
        w.cut = cw;
      }
    }
    one = one && gx && gw;
    if (gx) x.room(N, H, b);
    if (gw) w.room(C, H, b);
  }
  hipError_t run(const Gradients<T> &p, const Mat *gx, const Mat *gw, long long N, long long C,
                 long long H, const float *scale, hipStream_t s) const {
    if (!one) {
      if (gx) TRY(x.run(p.dx_a, p.dx_b, N, H, p.dx_k, scale, *gx, s));
      if (gw) TRY(w.run(p.dw_a, p.dw_b, C, H, p.dw_k, scale, *gw, s));
      return hipSuccess;
    }
    const Tile c = TILES[x.cut.tile];
    Product dx = x.of(p.dx_a, p.dx_b, N, H, p.dx_k, scale, *gx);
    Product dw = w.of(p.dw_a, p.dw_b, C, H, p.dw_k, scale, *gw);
    long long grid = 0;
    for (Product *g : {&dx, &dw}) {
      g->tiles_m = (int)((g->M + c.bm - 1) / c.bm);
      g->tiles_n = (int)((g->N + c.bn - 1) / c.bn);
      grid += (long long)g->tiles_m * g->tiles_n * g->splits;
    }
    if (grid * 512 >= (1ll << 32)) return hipErrorInvalidValue;
    if (x.cut.tile == 1)
      products<T, 128, 128, 4, 2>(dx, dw, (unsigned)grid, s);
    else
      products<T, 64, 64, 2, 2>(dx, dw, (unsigned)grid, s);
    TRY(hipGetLastError());
    return finish(x.rest(*gx), w.rest(*gw), scale, s);
  }
};

// Rows that a workgroup of the kernels over rows takes: 16 where that leaves
// enough workgroups (a row each otherwise: 165 rows of 869 columns 19 us by 16).
bool many_rows(long long N) { return N >= 4096; }

// Tiles of 32 rows, whole: four wavefronts of 16 rows and half the columns.
template <typename T>
void log_rows(const Product &g, hipStream_t s) {
  const unsigned grid = (unsigned)g.tiles_m;
  if (g.N <= 32)
    k_product<T, ROWS_ROWS, 32, 32, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
  else if (g.N <= 64)
    k_product<T, ROWS_ROWS, 32, 64, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
  else if (g.N <= 96)
    k_product<T, ROWS_ROWS, 32, 96, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
  else if (g.N <= 128)
    k_product<T, ROWS_ROWS, 32, 128, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
  else if (g.N <= 192)
    k_product<T, ROWS_ROWS, 32, 192, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
  else
    k_product<T, ROWS_ROWS, 32, 256, 2, 2, EPI_LOG><<<grid, 4 * WAVE, 0, s>>>(g);
}

template <typename T>
hipError_t emission_as(const Mat &x, const Mat &w, float *weight, Bump &b, hipStream_t s) {
  const long long N = x.rows, C = w.rows;
  const Laid<T> lx = lay<T>(x, b), lw = lay<T>(w, b);
  // a tile takes whole rows; past 128 classes in float32 only where there is one
  // for every CU (500 x 200 over 1024: 45 us whole, 28 by 64 and normalised after;
  // 13,637 x 250 over 286: 39 and 47, in bf16 21 and 39)
  const bool whole = C <= 128 || (C <= 256 && (sizeof(T) == 2 || N >= 32 * CUS));
  const Cut cut = cut_for<T>(N, C, lx.cols, false);
  const int parts = (int)((C + TILES[cut.tile].bn - 1) / TILES[cut.tile].bn) * TILES[cut.tile].wn;
  float2 *part = b.take<float2>(whole ? 1 : N * parts);
  if (!b.base) return hipSuccess;
  TRY(fill(copies(&lx, x, &lw, w), s));
  Product g{};
  g.A = lx.o;
  g.B = lw.o;
  g.M = N;
  g.N = C;
  g.K = lx.cols;
  g.splits = 1;
  g.steps = INT32_MAX;
  g.out = weight;
  g.ldo = C;
  if (whole) {
    g.tiles_m = (int)((N + 31) / 32);
    g.tiles_n = 1;
    log_rows<T>(g, s);
    return hipGetLastError();
  }
  g.part = part;
  TRY((product<T, ROWS_ROWS, EPI_SCORE>(g, cut.tile, s)));
  if (many_rows(N))
    k_normalise<16><<<(unsigned)((N + 15) / 16), NT, 0, s>>>(part, parts, N, C, weight);
  else
    k_normalise<1><<<(unsigned)N, NT, 0, s>>>(part, parts, N, C, weight);
  return hipGetLastError();
}

template <typename T>
hipError_t emission_grads_as(const Mat &x, const Mat &w, const float *weight, const float *grad,
                             const Mat *gx, const Mat *gw, Bump &b, hipStream_t s) {
  const long long N = x.rows, C = w.rows, H = x.cols;
  const long long Cp = up(C, 64);
  if (N == 0 || H == 0) {  // nothing to sum over, or nothing to write
    if (b.base && gw) TRY(clear<T>(*gw, s));
    b.take<char>(1);
    return hipSuccess;
  }
  const Laid<T> lx = lay<T>(x, b), lw = lay<T>(w, b);
  const bool two = in_two<T>(N, C, H);
  const long long ld = two ? 2 * Cp : Cp;
  T *ds = b.take<T>(N * ld);
  constexpr int GROUPS = 256;
  float *most = b.take<float>(GROUPS), *scale = b.take<float>(1);
  const Gradients<T> p(ds, ld, N, Cp, two, lw.columns(), lx.columns());
  Both<T> both{};
  both.plan(p, gx, gw, N, C, H, b);
  if (!b.base) return hipSuccess;
  if (std::is_same<T, f16>::value) {
    const unsigned n = blocks_for(N, NWAVES, GROUPS);
    k_emission_max<<<n, NT, 0, s>>>(grad, N, C, most);
    k_scale<<<1, 1024, 0, s>>>(most, nullptr, n, scale);
  } else {
    scale = nullptr;
  }
  const Pads<T> pads = copies(gw ? &lx : nullptr, x, gx ? &lw : nullptr, w);
  const unsigned n = (unsigned)(C <= SHORT ? (N + 15) / 16 : (N + 3) / 4);
  if (C <= SHORT)
    k_emission_ds_short<T><<<n + pad_blocks(pads), NT, 0, s>>>(pads, n, weight, grad, N, (int)C,
                                                               scale, ds, (int)Cp, (int)ld);
  else
    k_emission_ds<T><<<n + pad_blocks(pads), NT, 0, s>>>(pads, n, weight, grad, N, C, scale, ds,
                                                         Cp, ld);
  TRY(hipGetLastError());
  return both.run(p, gx, gw, N, C, H, scale, s);
}

template <typename T>
hipError_t loss_as(const Mat &x, const Mat &w, const int32_t *target, float *loss, float *lse,
                   Bump &b, hipStream_t s) {
  const long long N = x.rows, V = w.rows;
  const Laid<T> lx = lay<T>(x, b), lw = lay<T>(w, b);
  const int tile = cut_for<T>(N, V, lx.cols, false).tile;
  const int parts = (int)((V + TILES[tile].bn - 1) / TILES[tile].bn) * TILES[tile].wn;
  float2 *part = b.take<float2>(N * parts);
  float *hit = b.take<float>(N);
  if (!b.base) return hipSuccess;
  TRY(fill(copies(&lx, x, &lw, w), s));
  Product g{};
  g.A = lx.o;
  g.B = lw.o;
  g.M = N;
  g.N = V;
  g.K = lx.cols;
  g.splits = 1;
  g.steps = INT32_MAX;
  g.part = part;
  g.target = target;
  g.hit = hit;
  TRY((product<T, ROWS_ROWS, EPI_PART>(g, tile, s)));
  if (many_rows(N))
    k_loss<16><<<(unsigned)((N + 15) / 16), NT, 0, s>>>(part, parts, N, target, V, hit, loss, lse);
  else
    k_loss<1><<<(unsigned)N, NT, 0, s>>>(part, parts, N, target, V, hit, loss, lse);
  return hipGetLastError();
}

// Bytes of dS that a piece of the vocabulary may take.
constexpr long long PIECE_BYTES = 512ll << 20;

// Elements between rows of dS: with rows of a power of two bytes the product dx
// takes 3 % longer, all of a wavefront's rows in the same channels.
constexpr long long DS_GAP = 64;

// Words of a piece of the vocabulary, `most` at most (or 256): all of them, or
// rows of dw's tiles that fill the CUs a whole number of times (16,000 rows, 32,000
// words, width 1024: pieces of 16,640 words leave dw 260 tiles, 0.90 ms; 16,384
// leave 256, 0.50 ms).
long long piece_of(long long V, long long H, long long most) {
  if (most >= V) return V;
  const long long across = (H + 255) / 256;
  const long long fill = across < CUS ? CUS / across * 256 : 256;
  const long long unit = most >= fill ? fill : 256;
  return most < unit ? unit : most / unit * unit;
}

template <typename T>
hipError_t loss_grads_as(const Mat &x, const Mat &w, const int32_t *target, const float *lse,
                         const float *grad, const Mat *gx, const Mat *gw, Bump &b,
                         hipStream_t s) {
  const long long N = x.rows, V = w.rows, H = x.cols;
  if (N == 0 || H == 0) {  // nothing to sum over, or nothing to write
    if (b.base && gw) TRY(clear<T>(*gw, s));
    b.take<char>(1);
    return hipSuccess;
  }
  const Laid<T> lx = lay<T>(x, b), lw = lay<T>(w, b);
  long long most_words = PIECE_BYTES / (N * (long long)sizeof(T));
  if (most_words > FST_HEAD_MAX_COLS) most_words = FST_HEAD_MAX_COLS;
  const long long piece = piece_of(V, H, most_words);
  const bool whole = piece == V, two = whole && in_two<T>(N, V, H);
  const long long Pp = up(piece, 64);
  // a piece of `n` words from v0 on
  const auto products = [&](const T *ds, long long v0, long long n) {
    const long long np = up(n, 64);
    const Operand wc{static_cast<const T *>(lw.o.p) + v0 * lw.o.ld, lw.o.ld, lw.cols, n};
    return Gradients<T>(ds, (two ? 2 : 1) * np + DS_GAP, N, np, two, wc, lx.columns());
  };
  T *ds = b.take<T>(N * ((two ? 2 : 1) * Pp + DS_GAP));
  constexpr int GROUPS = 256;
  float *most_g = b.take<float>(GROUPS), *scale = b.take<float>(1);
  Both<T> both{};
  SplitProduct<T, COLS_COLS> &pw = both.w;
  float *sums = nullptr;
  if (whole) both.plan(products(ds, 0, V), gx, gw, N, V, H, b);
  if (gx && !whole) sums = b.take<float>(N * up(H, 4));
  const size_t mark = b.at;
  size_t most = mark;
  if (gw && !whole) {
    for (long long v0 = 0; v0 < V; v0 += piece) {
      const long long n = V - v0 < piece ? V - v0 : piece;
      b.at = mark;
      pw.plan(n, H, products(ds, v0, n).dw_k, b);
      most = b.at > most ? b.at : most;
    }
  }
  b.at = most;
  if (!b.base) return hipSuccess;
  TRY(fill(copies(&lx, x, &lw, w), s));
  if (std::is_same<T, f16>::value) {
    const bool one = !grad || N <= 65536;
    if (!one) k_scale<<<GROUPS, 1024, 0, s>>>(grad, target, N, most_g);
    k_scale<<<1, 1024, 0, s>>>(one ? grad : most_g, one ? target : nullptr, one ? N : GROUPS,
                               scale);
    TRY(hipGetLastError());
  } else {
    scale = nullptr;
  }
  for (long long v0 = 0; v0 < V; v0 += piece) {
    const long long n = V - v0 < piece ? V - v0 : piece, np = up(n, 64);
    const Operand wp{static_cast<const T *>(lw.o.p) + v0 * lw.o.ld, lw.o.ld, n, lw.cols};
    const Gradients<T> p = products(ds, v0, n);
    Product g{};
    g.A = lx.o;
    g.B = wp;
    g.M = N;
    g.N = n;
    g.K = lx.cols;
    g.splits = 1;
    g.steps = INT32_MAX;
    g.n0 = v0;
    g.words = V;
    g.out = ds;
    g.ldo = p.dx_a.ld;
    g.lo = two ? np : 0;
    g.target = target;
    g.lse = lse;
    g.grad = grad;
    g.scale = scale;
    g.Np = np;
    TRY((product<T, ROWS_ROWS, EPI_DS>(g, cut_for<T>(N, n, lx.cols, false).tile, s)));
    if (whole) return both.run(p, gx, gw, N, V, H, scale, s);
    if (gx) {
      Product q{};
      q.A = p.dx_a;
      q.B = p.dx_b;
      q.M = N;
      q.N = H;
      q.K = np;
      q.splits = 1;
      q.steps = INT32_MAX;
      if (v0 + n < V) {
        q.out = sums;
        q.ldo = up(H, 4);
        q.wide = 1;
        q.add = v0 > 0;
        TRY((product<T, ROWS_COLS, EPI_SUM>(q, cut_for<T>(N, H, np, false).tile, s)));
      } else {
        q.out = gx->data;
        q.ldo = gx->stride;
        q.wide = wide<T>(*gx);
        q.scale = scale;
        q.sums = sums;
        TRY((product<T, ROWS_COLS, EPI_RESULT>(q, cut_for<T>(N, H, np, false).tile, s)));
      }
    }
    if (gw) {
      Mat out = *gw;
      out.data = static_cast<T *>(out.data) + v0 * out.stride;
      out.rows = n;
      b.at = mark;
      pw.plan(n, H, p.dw_k, b);
      TRY(pw.run(p.dw_a, p.dw_b, n, H, p.dw_k, scale, out, s));
    }
  }
  return hipSuccess;
}

}  // namespace

#define BY_TYPE(type, call)                  \
  switch (type) {                            \
    case FST_F32: { typedef float T; e = call; break; }  \
    case FST_F16: { typedef f16 T; e = call; break; }    \
    default: { typedef bf16 T; e = call; break; }        \
  }

hipError_t launch_emission(const Mat &x, const Mat &w, float *weight, void *ws, size_t *need,
                           hipStream_t s) {
  Bump b{static_cast<char *>(ws)};
  hipError_t e;
  BY_TYPE(x.type, emission_as<T>(x, w, weight, b, s));
  *need = b.at;
  return e;
}

hipError_t launch_emission_grads(const Mat &x, const Mat &w, const float *weight,
                                 const float *grad, const Mat *gx, const Mat *gw, void *ws,
                                 size_t *need, hipStream_t s) {
  Bump b{static_cast<char *>(ws)};
  hipError_t e;
  BY_TYPE(x.type, emission_grads_as<T>(x, w, weight, grad, gx, gw, b, s));
  *need = b.at;
  return e;
}

hipError_t launch_loss(const Mat &x, const Mat &w, const int32_t *target, float *loss, float *lse,
                       void *ws, size_t *need, hipStream_t s) {
  Bump b{static_cast<char *>(ws)};
  hipError_t e;
  BY_TYPE(x.type, loss_as<T>(x, w, target, loss, lse, b, s));
  *need = b.at;
  return e;
}

hipError_t launch_loss_grads(const Mat &x, const Mat &w, const int32_t *target, const float *lse,
                             const float *grad, const Mat *gx, const Mat *gw, void *ws,
                             size_t *need, hipStream_t s) {
  Bump b{static_cast<char *>(ws)};
  hipError_t e;
  BY_TYPE(x.type, loss_grads_as<T>(x, w, target, lse, grad, gx, gw, b, s));
  *need = b.at;
  return e;
}

}  // namespace fstc
