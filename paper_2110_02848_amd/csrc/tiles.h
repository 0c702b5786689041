// Tiles of matrices in LDS and the fragments of them that the matrix cores
// multiply (linear.hip, window.hip).
//
// A product of 16 x 16 results takes 32 of the sum a step: of either operand
// lane l holds row l & 15 and eight numbers of the sum; of the results column
// l & 15 and rows 4 (l >> 4) + 0..3.  Which eight of the 32 a lane holds is
// free as long as both operands agree.  Here there are two orders: `rows`
// reads, along the rows of a tile, 8 (l >> 4) + 0..7; `columns` reads, down
// its columns, 4 (l >> 4) + 0..3 and 16 + 4 (l >> 4) + 0..3.  The second is
// how the results of two products above one another lie, so that these become
// an operand of the next product in the registers that they are in.
#pragma once

#include <type_traits>

#include "layers.h"

namespace fstc {
namespace tile {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef __attribute__((ext_vector_type(4))) float float4v;
typedef __attribute__((ext_vector_type(4))) int int4v;
typedef __attribute__((ext_vector_type(2))) int int2v;
typedef __attribute__((ext_vector_type(8))) _Float16 half8;
typedef __attribute__((ext_vector_type(8))) __bf16 bhalf8;
typedef __attribute__((ext_vector_type(4))) short short4v;

template <typename T>
constexpr int PER = 16 / (int)sizeof(T);  // numbers in 16 bytes

// Eight numbers of a lane.
template <typename T>
struct Frag {
  int4v v[sizeof(T) / 2];
};

__device__ __forceinline__ float4v mac(const Frag<bf16> &a, const Frag<bf16> &b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a.v[0]),
                                                 __builtin_bit_cast(bhalf8, b.v[0]), c, 0, 0, 0);
}
__device__ __forceinline__ float4v mac(const Frag<f16> &a, const Frag<f16> &b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a.v[0]),
                                                __builtin_bit_cast(half8, b.v[0]), c, 0, 0, 0);
}
// (eight steps of 4: step j sums over element j of the four lane groups)
__device__ __forceinline__ float4v mac(const Frag<float> &a, const Frag<float> &b, float4v c) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4v x = __builtin_bit_cast(float4v, a.v[i]), y = __builtin_bit_cast(float4v, b.v[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
  }
  return c;
}

// The eight numbers as they are held, and back.
template <typename T>
__device__ __forceinline__ void unpack(const Frag<T> &f, float (&x)[8]) {
  struct alignas(16) { T v[8]; } e;
  __builtin_memcpy(&e, &f, sizeof(e));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)e.v[i];
}
template <typename T>
__device__ __forceinline__ Frag<T> pack(const float (&x)[8]) {
  struct alignas(16) { T v[8]; } e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.v[i] = (T)x[i];
  Frag<T> f;
  __builtin_memcpy(&f, &e, sizeof(e));
  return f;
}
// Results of two products, rows r.. and 16 + r.., as an operand.
template <typename T>
__device__ __forceinline__ Frag<T> pack(const float4v &a, const float4v &b) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return pack<T>(x);
}

// Rows of P numbers, 16 bytes between them: reads of 16 lanes a row apart meet
// different banks but for one, reads that transpose take twice their time (no bound
// of the kernels that use them: linear attention, 64 x 2,000 x 8 x 128 x 128 bf16, took
// as long with rows as Packed below has them).
template <typename T, int P>
constexpr int LD = P + PER<T>;
template <typename T, int P, int R>
constexpr int BYTES = LD<T, P> * R * (int)sizeof(T);

// Rows `row` .. + 15, numbers `k` .. + 31 of each.
template <typename T, int P>
__device__ __forceinline__ Frag<T> rows(const T *t, int row, int k, int lane) {
  const T *p = t + (row + (lane & 15)) * LD<T, P> + k + (lane >> 4) * 8;
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i)
    f.v[i] = *reinterpret_cast<const int4v *>(p + i * PER<T>);
  return f;
}

// Columns `col` .. + 15, rows `row` .. + 31 of each.  (A read that transposes
// gives lane i of 16 the i-th column of four rows: lanes 4 j .. 4 j + 3 point
// at the j-th.)
template <typename T, int P>
__device__ __forceinline__ Frag<T> columns(const T *t, int row, int col, int lane) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    const T *p = t + (row + (lane >> 4) * 4 + ((lane >> 2) & 3)) * LD<T, P> + col + (lane & 3) * 4;
    int2v v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      v[i] = __builtin_bit_cast(
          int2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                     (__attribute__((address_space(3))) short4v *)(p + i * 16 * LD<T, P>)));
    f.v[0] = int4v{v[0].x, v[0].y, v[1].x, v[1].y};
  } else {
    const T *p = t + (row + (lane >> 4) * 4) * LD<T, P> + col + (lane & 15);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f.v[i][j] = __builtin_bit_cast(int, (float)p[(i * 16 + j) * LD<T, P>]);
  }
  return f;
}

// 16 bytes from number c on of a row of `width`, zeros past its end or where the row
// is not there; WIDE: the width is a multiple of them and the row begins at one.
// Otherwise every number is read by itself, all of them at once: one that is not
// there reads the first of `safe` instead.
template <typename T, bool WIDE>
__device__ __forceinline__ int4v load_group(const T *row, int c, int width, bool there,
                                            const T *safe) {
  int4v v{0, 0, 0, 0};
  if constexpr (WIDE) {
    if (there && c < width) v = *reinterpret_cast<const int4v *>(row + c);
  } else {
    struct alignas(16) { T v[PER<T>]; } e;
#pragma unroll
    for (int i = 0; i < PER<T>; ++i) e.v[i] = *(there && c + i < width ? row + c + i : safe);
#pragma unroll
    for (int i = 0; i < PER<T>; ++i) e.v[i] = there && c + i < width ? e.v[i] : (T)0.0f;
    __builtin_memcpy(&v, &e, 16);
  }
  return v;
}

// The number at a byte offset of a buffer, 0 past its end.
template <typename T>
__device__ __forceinline__ T load_number(__amdgpu_buffer_rsrc_t buffer, int at) {
  if constexpr (sizeof(T) == 2)
    return __builtin_bit_cast(
        T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(buffer, at, 0, 0));
  else
    return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(buffer, at, 0, 0));
}

// Row strides up to MAX_STRIDE keep 32-bit byte offsets within a tile of up to 128
// rows below PAST_END, an offset that is past any tile's end.
constexpr long long MAX_STRIDE = 1ll << 22;
constexpr int PAST_END = INT32_MIN;  // (as a number without a sign)

// A tile of R rows of P numbers on its way from memory to LDS, by NTH threads: by 16
// bytes (WIDE) or number by number, through a buffer, which gives zeros past its
// end without a branch.
template <typename T, int P, int R, int NTH, bool WIDE>
struct Stage {
  static constexpr int GROUPS = P / PER<T>;  // of a row
  static constexpr int LOADS = R * GROUPS / NTH;
  static_assert(LOADS >= 1 && LOADS * NTH == R * GROUPS, "whole loads");
  int4v v[LOADS];

  // row i of the tile is row first + i * step of the matrix (step 1 or -1), if i <
  // count (1 or more)
  __device__ __forceinline__ void fetch(const T *p, long long stride, int width, long long first,
                                        long long step, int count) {
    const long long low = step < 0 ? first - (count - 1) : first;
    const __amdgpu_buffer_rsrc_t buffer = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<T *>(p + low * stride), 0,
        (int)(((count - 1) * stride + width) * (long long)sizeof(T)), 0x00027000);
    const int row = (int)(stride * (long long)sizeof(T));
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = i * NTH + (int)threadIdx.x, r = q / GROUPS, c = q % GROUPS * PER<T>;
      // (before the first row: past the end, as a number without a sign)
      const int at = (step < 0 ? count - 1 - r : r) * row + c * (int)sizeof(T);
      if constexpr (WIDE) {
        v[i] = __builtin_bit_cast(int4v, __builtin_amdgcn_raw_buffer_load_b128(
                                             buffer, c < width ? at : PAST_END, 0, 0));
      } else {
        struct alignas(16) { T v[PER<T>]; } e;
#pragma unroll
        for (int j = 0; j < PER<T>; ++j)
          e.v[j] =
              load_number<T>(buffer, c + j < width ? at + j * (int)sizeof(T) : PAST_END);
        __builtin_memcpy(&v[i], &e, 16);
      }
    }
  }
  __device__ __forceinline__ void store(T *t) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = i * NTH + (int)threadIdx.x, r = q / GROUPS, c = q % GROUPS * PER<T>;
      *reinterpret_cast<int4v *>(t + r * LD<T, P> + c) = v[i];
    }
  }
  // the largest finite magnitude in it, or with `weight` that of a row's numbers times
  // weight[row] (of rows below `count`)
  __device__ __forceinline__ float largest(const float *weight = nullptr, int count = 0) const {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      struct alignas(16) { T v[PER<T>]; } e;
      __builtin_memcpy(&e, &v[i], 16);
      float most = 0.0f;
#pragma unroll
      for (int j = 0; j < PER<T>; ++j) {
        const float x = fabsf((float)e.v[j]);
        most = x < INFINITY ? fmaxf(most, x) : most;
      }
      const int r = (i * NTH + (int)threadIdx.x) / GROUPS;
      m = fmaxf(m, !weight ? most : r < count ? most * weight[r] : 0.0f);
    }
    return m;
  }
};

// Tiles whose rows lie side by side, without room between them: 16-byte group g of
// row r lies at group g ^ swizzle(r), so that reads meet different banks: a read of 16
// rows goes by 16 lanes, rows 0 .. 3 and 12 .. 15 of a group of numbers and the other
// eight of the next (or the other way round), one that transposes by 32 lanes, eight
// rows of 32 bytes.  They come from memory straight to LDS.
template <typename T, int P>
struct Packed {
  static constexpr int GROUPS = P / PER<T>, ROW = P * (int)sizeof(T);

  static __device__ __forceinline__ int swizzle(int r) {
    return GROUPS == 8 ? r & 6 : (r & 7) << 1;
  }
  static __device__ __forceinline__ const char *at(const char *t, int r, int g) {
    return t + r * ROW + ((g ^ swizzle(r)) << 4);
  }
  // as rows() and columns() above
  static __device__ __forceinline__ Frag<T> rows(const char *t, int row, int k, int lane) {
    const int r = row + (lane & 15), g = k / PER<T> + (lane >> 4) * (8 / PER<T>);
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      f.v[i] = *reinterpret_cast<const int4v *>(at(t, r, g + i));
    return f;
  }
  static __device__ __forceinline__ Frag<T> columns(const char *t, int row, int col, int lane) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      int2v v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row + 16 * i + (lane >> 4) * 4 + (lane >> 2 & 3);
        const char *p = at(t, r, col / 8 + (lane >> 1 & 1)) + (lane & 1) * 8;
        v[i] = __builtin_bit_cast(
            int2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) short4v *)p));
      }
      f.v[0] = int4v{v[0].x, v[0].y, v[1].x, v[1].y};
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = row + 16 * i + (lane >> 4) * 4 + j, c = col + (lane & 15);
          f.v[i][j] = *reinterpret_cast<const int *>(at(t, r, c / 4) + c % 4 * 4);
        }
    }
    return f;
  }
};

// Loads of 64 lanes by 16 bytes from memory to LDS without registers: lane i's
// bytes land at `lds` + 16 i, zeros where they lie past the end of the buffer.
// Written as instructions, because the compiler would wait for all of them before
// the next read of LDS; whoever reads waits with wait_loads and a barrier.  (m0 is
// the compiler's own: it warns where it is named, and only naming it keeps its uses
// of m0 clear of this one.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(uint32_t lds, uint32_t offset, int4v buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(buffer)
               : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

// A packed tile of R rows on its way from memory, by NTH threads; WIDE: straight to
// LDS, otherwise through registers, number by number.
template <typename T, int P, int R, int NTH, bool WIDE>
struct Carry {
  static constexpr int GROUPS = P / PER<T>;
  static constexpr int LOADS = R * GROUPS / NTH;
  static_assert(LOADS >= 1 && LOADS * NTH == R * GROUPS, "whole loads");
  int off[LOADS];
  int4v v[WIDE ? 1 : LOADS];

  // (row, group of it) of load i: lanes write 1,024 bytes in their order
  static __device__ __forceinline__ int row_of(int i) {
    return ((threadIdx.x / WAVE * LOADS + i) * WAVE + threadIdx.x % WAVE) / GROUPS;
  }
  static __device__ __forceinline__ int group_of(int i) {
    const int q = (threadIdx.x / WAVE * LOADS + i) * WAVE + threadIdx.x % WAVE;
    return q % GROUPS ^ Packed<T, P>::swizzle(row_of(i));
  }
  __device__ __forceinline__ void init(long long stride, int width) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int c = group_of(i) * PER<T>;
      off[i] = c < width ? (int)((row_of(i) * stride + c) * (long long)sizeof(T)) : PAST_END;
    }
  }
  // rows first .. first + count of a matrix (all arguments the same in every lane)
  __device__ __forceinline__ void fetch(const T *p, long long stride, int width, long long first,
                                        int count, char *to) {
    const uint32_t n =
        count > 0 ? (uint32_t)(((count - 1) * stride + width) * (long long)sizeof(T)) : 0u;
    if constexpr (WIDE) {
      const unsigned long long q = (unsigned long long)(uintptr_t)(p + first * stride);
      const int4v buffer{__builtin_amdgcn_readfirstlane((int)(uint32_t)q),
                         __builtin_amdgcn_readfirstlane((int)(uint32_t)(q >> 32)),
                         __builtin_amdgcn_readfirstlane((int)n), 0x00027000};
      const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)to +
                           threadIdx.x / WAVE * LOADS * 1024;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds(lds + i * 1024, (uint32_t)off[i], buffer);
    } else {
      const __amdgpu_buffer_rsrc_t buffer = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<T *>(p + first * stride), 0, (int)n, 0x00027000);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int c = group_of(i) * PER<T>;
        struct alignas(16) { T v[PER<T>]; } e;
#pragma unroll
        for (int j = 0; j < PER<T>; ++j)
          e.v[j] = load_number<T>(buffer, c + j < width ? off[i] + j * (int)sizeof(T) : PAST_END);
        __builtin_memcpy(&v[i], &e, 16);
      }
    }
  }
  // what fetch() began, in LDS; before the barrier behind which it is read
  __device__ __forceinline__ void finish(char *to) const {
    if constexpr (WIDE) {
      wait_loads();
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        *reinterpret_cast<int4v *>(
            to + ((threadIdx.x / WAVE * LOADS + i) * WAVE + threadIdx.x % WAVE) * 16) = v[i];
    }
  }
};

// Four results side by side, from column c on of a row of `width`.
template <typename T, bool WIDE>
__device__ __forceinline__ void store_four(T *row, int c, int width, const float4v &x) {
  if constexpr (WIDE) {
    struct alignas(4 * sizeof(T)) { T v[4]; } e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = (T)x[i];
    if (c < width) *reinterpret_cast<decltype(e) *>(row + c) = e;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < width) row[c + i] = (T)x[i];
  }
}

__device__ __forceinline__ bool all_nan(const float4v &x) {
  return x[0] != x[0] && x[1] != x[1] && x[2] != x[2] && x[3] != x[3];
}

// Of the same four, as they were written: whether one is no number, and x in the
// place of those that are none.
template <typename T>
__device__ __forceinline__ bool none_of_four(const T *row, int c, int width) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < width) bad = bad || !(fabsf((float)row[c + i]) < INFINITY);
  return bad;
}
template <typename T>
__device__ __forceinline__ void mend_four(T *row, int c, int width, const float4v &x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < width && !(fabsf((float)row[c + i]) < INFINITY)) row[c + i] = (T)x[i];
}

// Maximum, and sum, over the four lanes that hold a column of results (16 apart): a
// swap of rows of 16 lanes between two copies leaves a lane both its own and its
// partner's, then one of halves does.
__device__ __forceinline__ float2 swap16(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  return make_float2(__builtin_bit_cast(float, (uint32_t)r[0]),
                     __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float2 swap32(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return make_float2(__builtin_bit_cast(float, (uint32_t)r[0]),
                     __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float column_max(float x) {
  float2 p = swap16(x);
  x = fmaxf(p.x, p.y);
  p = swap32(x);
  return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float column_sum(float x) {
  float2 p = swap16(x);
  x = p.x + p.y;
  p = swap32(x);
  return p.x + p.y;
}

__device__ __forceinline__ float wave_max(float m) {
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, WAVE));
  return m;
}

// The power of two that takes numbers up to `most` below 2^top (1 where most is
// 0 or no number).
__device__ __forceinline__ float power_below(float most, int top) {
  if (!(most > 0.0f) || !(most < INFINITY)) return 1.0f;
  int e = top - 1 - ilogbf(most);
  e = e < -120 ? -120 : e > 120 ? 120 : e;
  return ldexpf(1.0f, e);
}

// Numbers that become 16-bit ones with few exponents (float16) before they are multiplied
// take a power of two of the column of results that they are summed into, by what that
// column sees alone.  It begins as UNMET and falls wherever a number would be past PAST
// with it, to one that leaves that number below 2^12, so that few tiles change it; the
// column's sums are multiplied by what `lowered` returns.  `top`: a lane's largest.
constexpr float UNMET = 0x1p120f, PAST = 0x1p15f;
__device__ __forceinline__ float lowered(float &up, float top) {
  top = column_max(top);
  const float was = up;
  if (top * up > PAST) up = fminf(up, power_below(top, 12));
  return up / was;
}
__device__ __forceinline__ float largest_of(const float4v &a, const float4v &b) {
  float top = 0.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) top = fmaxf(fmaxf(top, fabsf(a[r])), fabsf(b[r]));
  return top;
}

}  // namespace tile
}  // namespace fstc
