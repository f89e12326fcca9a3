// Rows of logits four columns at a time, and the scalar functions of a row's
// sums, shared by the kernels that hold a row in registers.
#pragma once

#include <cmath>

#include "internal.hpp"

namespace gnnprop {

constexpr int32_t MOST_COLS = 1 << 24;  // columns of a row

// Blocks of one launch (2^32 threads are the most that a launch can have).
constexpr int64_t LAUNCH_BLOCKS = 1 << 21;

// exp(x - top), where top = -inf only if no logit is above it: then 0 (or
// NaN for a NaN), so that the sum is 0 exactly for a row without any action.
__device__ inline float shift_of(float top) { return top == -INFINITY ? 0.f : top; }

// exp(x) to a few 2^-53 for |x| < 700: 2^k times the remainder's series
// (|r| < 0.35: the first term left out, r^14 / 14!, is below 5e-18).
__device__ inline double exp_exact(double x) {
  if (!(x > -700.0)) return x < 0.0 ? 0.0 : x;  // 0, or NaN
  if (x > 709.8) return INFINITY;
  const double k = rint(x * 1.4426950408889634);
  const double r = fma(-k, 2.3190468138462996e-17, fma(-k, 0.6931471805599453, x));
  double sum = 1.0 / 6227020800.0;
  sum = fma(sum, r, 1.0 / 479001600.0);
  sum = fma(sum, r, 1.0 / 39916800.0);
  sum = fma(sum, r, 1.0 / 3628800.0);
  sum = fma(sum, r, 1.0 / 362880.0);
  sum = fma(sum, r, 1.0 / 40320.0);
  sum = fma(sum, r, 1.0 / 5040.0);
  sum = fma(sum, r, 1.0 / 720.0);
  sum = fma(sum, r, 1.0 / 120.0);
  sum = fma(sum, r, 1.0 / 24.0);
  sum = fma(sum, r, 1.0 / 6.0);
  sum = fma(sum, r, 0.5);
  sum = fma(sum, r, 1.0);
  sum = fma(sum, r, 1.0);
  return ldexp(sum, (int)k);
}

// log(s) as k ln 2 + log(m), 0.7 < m < 1.42 (so that log(1) is 0): good to
// 4e-8.
__device__ inline double log_quick(float s) {
  int k;
  float m = frexpf(s, &k);
  if (m < 0.70710678f) {
    m *= 2.f;
    --k;
  }
  return fma((double)k, 0.6931471805599453, (double)logf(m));
}

// ---------------------------------------------------------- four at a time

// Rows start at any multiple of 4 bytes, so the vector accesses claim no more
// (global memory instructions of 16 bytes need no more).
typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4u __attribute__((aligned(4)));

// Reading columns [col, col + 4) of a row of C, in two steps.  First a load
// without a branch (what is loaded in one is waited for where the branch ends,
// and a row's loads would follow each other), of the row's last four columns
// where its end cuts the chunk or lies before it; later, when the values are
// there, those past the end made -inf.
__device__ inline f4 load_cols(const float* row, int32_t col, int32_t C) {
  if (C >= 4) return *reinterpret_cast<const f4u*>(row + min(col, C - 4));
  return {row[0], row[min(1, C - 1)], row[min(2, C - 1)], 0.f};
}
__device__ inline float pick(bool c, float x, float y) { return c ? x : y; }
__device__ inline f4 cut_cols(f4 w, int32_t col, int32_t C) {
  const float none = -INFINITY;
  const int32_t left = C - col;  // columns from col on
  if (C >= 4) {                  // w starts 4 - left columns before col
    const bool one = left == 3 || left == 1, two = left == 2 || left == 1;
    w = {pick(one, w.y, w.x), pick(one, w.z, w.y), pick(one, w.w, w.z), w.w};
    w = {pick(two, w.z, w.x), pick(two, w.w, w.y), w.z, w.w};
  }
  return {pick(left > 0, w.x, none), pick(left > 1, w.y, none), pick(left > 2, w.z, none),
          pick(left > 3, w.w, none)};
}
// Chunk k of V of a lane: those before the last are whole (V is the chunks of
// the row over the lanes, rounded up, so the row has at least 4 V - 3 columns).
template <int V>
__device__ inline f4 load_chunk(const float* row, int k, int32_t col, int32_t C) {
  if (k < V - 1) return *reinterpret_cast<const f4u*>(row + col);
  if (V > 1) return *reinterpret_cast<const f4u*>(row + min(col, C - 4));
  return load_cols(row, col, C);
}
__device__ inline void store_cols(float* row, int32_t col, int32_t C, f4 v) {
  if (col + 4 <= C) {
    *reinterpret_cast<f4u*>(row + col) = v;
    return;
  }
  if (col < C) row[col] = v.x;
  if (col + 1 < C) row[col + 1] = v.y;
  if (col + 2 < C) row[col + 2] = v.z;
}

__device__ inline float max4(f4 v) { return fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)); }
__device__ inline f4 exp4(f4 v, float shift) {
  return {expf(v.x - shift), expf(v.y - shift), expf(v.z - shift), expf(v.w - shift)};
}
__device__ inline float sum4(f4 v) { return (v.x + v.y) + (v.z + v.w); }

}  // namespace gnnprop
