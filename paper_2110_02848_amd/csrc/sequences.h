// Ragged sequences of rows, whole or in units of steps (recurrence.hip,
// linear.hip).
#pragma once

#include "internal.h"

namespace fstc {

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

// x / per of a row x (rows fit 31 bits): a division of 64 bits takes a microsecond.
__device__ __forceinline__ long long over_steps(long long x, long long per) {
  return per > INT32_MAX ? 0 : (long long)((uint32_t)x / (uint32_t)per);
}

// First of the rows that sequence s, from row b, has in an array with a row
// for every `per` steps of a sequence: ceil(len / per) rows fit before the
// next sequence's, as floor(b / per) + s grows by at least that.
__device__ __forceinline__ long long rows_before(long long b, int s, long long per) {
  return over_steps(b, per) + s;
}

// The unit of workgroup k among n sequences of N rows: a whole sequence, or
// (`unit` steps each) the sequence that owns row k of an array with a row for
// every unit.  All of it lies inside [0, N) whatever the offsets hold.  False:
// there is none.
__device__ __forceinline__ bool unit_of(const int32_t *off, int n, long long N, long long unit,
                                        bool reverse, long long k, Unit &u) {
  int s = (int)k;
  if (unit) {
    int lo = 0, hi = n - 1;  // the last s with rows_before <= k
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (rows_before(clamped(off[mid], 0, N), mid, unit) <= k)
        lo = mid;
      else
        hi = mid - 1;
    }
    s = lo;
  }
  u.s = s;
  u.b = clamped(off[s], 0, N);
  u.len = clamped(off[s + 1], u.b, N) - u.b;
  u.lo = 0;
  u.hi = u.len;
  if (unit) {
    const long long j = k - rows_before(u.b, s, unit);
    u.lo = j * unit;
    if (j < 0 || (j > 0 && u.lo >= u.len)) return false;
    u.hi = u.lo + unit < u.len ? u.lo + unit : u.len;
  }
  u.step = reverse ? -1 : 1;
  u.first = reverse ? u.b + u.len - 1 : u.b;
  return true;
}

// Which of `all` pieces of work workgroup `id` takes.  Workgroups go to the eight XCDs
// in turn, and each has a second-level cache: an XCD gets a run of consecutive
// pieces, which read much the same rows.
__device__ __forceinline__ long long piece_of(long long id, long long all) {
  const int x = (int)(id % 8);
  const long long per = all / 8;
  const int more = (int)(all % 8);
  return x * per + (x < more ? x : more) + id / 8;
}

}  // namespace fstc
