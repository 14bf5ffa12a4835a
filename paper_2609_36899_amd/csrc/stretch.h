// Work of many units (sequences, blocks of their tokens) laid end to end and cut into
// equal stretches, one for each work group, from lengths that only the device knows.
#pragma once

#include "wave.h"

namespace pdec {

// Sum of v over the work group's T threads before this one, and of all of them.
template <int T>
__device__ __forceinline__ int group_scan(int v, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_prefix(v);
  __syncthreads();
  if (lane == 63) red[wave] = incl;
  __syncthreads();
  int before = incl - v, sum = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    before += w < wave ? red[w] : 0;
    sum += red[w];
  }
  *total = sum;
  return before;
}

struct Stretch {
  int total, per;  // work of all units, and of a group
  int unit, first;  // the unit that the group's first piece lies in, and that unit's first
};

// Stretch w of n_groups, at least min_per long; size(u) is unit u's work, u < n_units.
// Every thread of the group (T of them) calls it and gets the same; unit and first mean nothing where
// w * per >= total.  red: T / 64 ints of LDS, found: two.  One look at the
// sizes, but for more units than threads.
template <int T, typename F>
__device__ __forceinline__ Stretch stretch_of(int n_units, int n_groups, int min_per, int w,
                                              int* red, int* found, F&& size) {
  int mine = 0, total;
  for (int u = threadIdx.x; u < n_units; u += T) mine += size(u);
  int first = group_scan<T>(mine, red, &total);
  Stretch s = {total, max((total + n_groups - 1) / n_groups, min_per), 0, 0};
  const int at = w * s.per;
  if (at >= total) return s;
  if (n_units <= T) {
    if (first <= at && at < first + mine) {
      found[0] = threadIdx.x;
      found[1] = first;
    }
  } else {
    int base = 0;
    for (int u0 = 0; base <= at; u0 += T) {
      const int u = u0 + threadIdx.x, n = u < n_units ? size(u) : 0;
      first = base + group_scan<T>(n, red, &total);
      if (first <= at && at < first + n) {
        found[0] = u;
        found[1] = first;
      }
      base += total;
    }
  }
  __syncthreads();
  s.unit = found[0];
  s.first = found[1];
  return s;
}

}  // namespace pdec
