// What drawing actions and finding top logits have in common: a row's range,
// its first entries, weights as whole numbers (the formulas: include/gnnprop.h).
//
// A draw must not depend on the order in which a sum is formed, and what lies
// next to a border (of the kept actions, of the random number) has to fall on
// its own side of it.  So an action's weight exp((z - top) / T) is a whole
// number: in units of 2^-51 of the largest, or more where a row's sum would
// pass 2^62.  Sums of them are exact, and equal logits have equal weights.
#pragma once

#include <cmath>

#include "abi.hpp"
#include "team.hpp"

namespace gnnprop {

// Rows past so many columns are shared by several blocks.
constexpr int32_t LONG_SAMPLE = 32768, LONG_TOP = 16384;

// 2^(i / 64), from the series of exp.
constexpr double exp2_64th(int i) {
  const double x = 0.6931471805599453094 * i / 64.0;
  double sum = 1.0;
  for (int k = 24; k > 0; --k) sum = 1.0 + sum * x / k;
  return sum;
}
struct Table {
  double at[64];
};
constexpr Table make_table() {
  Table t = {};
  for (int i = 0; i < 64; ++i) t.at[i] = exp2_64th(i);
  return t;
}
static __constant__ const Table TABLE = make_table();

// Units of a weight: 2^bits of them are the largest one.  At most 2^62 a row,
// and 51 bits leave the product below a double's first bit.  What rounding to
// them can move from one side of a border to the other is C half units of a sum
// of 2^bits or more: 2^(2 log C - 63) of it.  Past BY_SUM columns that would pass
// 2^-27 (a random number's last bit is 2^-24, and among 2^24 columns all that are
// below 2^-39 of the largest would be lost, 2^-15 of the sum), so there the units
// follow from the row's sum (long_rows.hip): at most 2^-28 of it then.
constexpr int32_t BY_SUM = 1 << 18;
inline int bits_of(int32_t C) {
  int log = 0;
  while ((int64_t)1 << log < C) ++log;
  return std::min(51, 62 - log);
}

// exp(d / T) in units of 2^-bits, d <= 0: with d / T in 64ths of an octave,
// 2^(q / 64) from the table and the remainder's series (below 4e-14 of it left
// out), added to 2^52, whose last bits the whole number then is.  The numbers
// are kept in scalar registers: as literals they took two moves a step.
struct Exponential {
  const double* table;  // TABLE's numbers times 2^bits
  double scale;
  double c1, c2, c3, c4, one52;

  __device__ __forceinline__ Exponential(const double* t, double s) : table(t), scale(s) {
    constexpr double a = 0.6931471805599453 / 64.0;
    c1 = scalar(a);
    c2 = scalar(a * a / 2.0);
    c3 = scalar(a * a * a / 6.0);
    c4 = a * a * a * a / 24.0;
    asm("" : "+v"(c4));  // (an instruction reads one of the others)
    one52 = scalar(4503599627370496.0);
  }
  static __device__ __forceinline__ double scalar(double x) {
    asm("" : "+s"(x));
    return x;
  }
  __device__ __forceinline__ uint64_t operator()(double d) const {
    const double t = fmax(d * scale, -64.0 * 56.0);
    const double k = rint(t), f = t - k;
    const int q = (int)k;
    double p = fma(f, c4, c3);
    p = fma(p, f, c2);
    p = fma(p, f, c1);
    p = fma(p, f, 1.0);
    const uint64_t unit = (uint64_t)__double_as_longlong(table[q & 63]);
    const uint32_t hi = (uint32_t)(unit >> 32) + ((uint32_t)(q >> 6) << 20);
    const double e = __longlong_as_double((long long)((uint64_t)hi << 32 | (uint32_t)unit));
    return (uint64_t)__double_as_longlong(fma(e, p, one52)) & 0xfffffffffffffull;
  }
};

// ------------------------------------------------------------------ draws

struct SampleArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  const float* u;
  double scale;  // 64 / (T ln 2); 0: the best action
  float inv_range;  // 1 / (T ln(C / (1 - top_p))): no border of top_p is as far from the top
  int32_t bits, top_k;
  double inv_t;  // 1 / T where units follow from the row's sum, or 0
  double top_p;
  double cut;   // T ln(min_p), or -inf
  double unit;  // 2^-bits where a sum of weights is that of the log-probabilities, or 0
  int32_t* action;
  float* logp;
  int32_t group;  // see row_range
  int64_t block0;
  // rows that several blocks share (long_rows.hip)
  struct LongRow* rows;
  struct LongPart* parts;
  int32_t per_row;
};

// The weights of a row's entries, 0 for those not kept.  They are formed again
// in each pass: a row's logits take half of the registers that weights would.
struct Weights {
  Exponential of;
  double top;
  Border kept;

  __device__ __forceinline__ uint64_t all(float z) const {
    return of((double)z - top);
  }
  __device__ __forceinline__ uint64_t operator()(float z, int32_t col) const {
    const uint64_t w = all(z);
    return within(kept, z, col) ? w : 0;
  }
  // Of four entries, formed side by side; lanes without a kept one pass on.
  __device__ __forceinline__ uint64_t sum4(f4 z, int32_t col) const {
    bool in[4], any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= in[j] = within(kept, z[j], col + j);
    if (!any) return 0;
    uint64_t w[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = all(z[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += in[j] ? w[j] : 0;
    return sum;
  }
};

// One for each logit from some value on (-inf never is).
struct Present {
  float from;
  __device__ __forceinline__ uint64_t operator()(float z, int32_t) const { return z >= from; }
};

// A row's largest logit, whether it is a finite number and none is a NaN; and of
// groups of `group` lanes (a power of two, at most G) how many hold a logit, and
// the least of what they hold the largest of.
template <class T, class Row>
__device__ __forceinline__ bool row_range(const T& team, const Row& row, int32_t group, float* top,
                                          float* low, int32_t* groups) {
  float most = -INFINITY;
  bool bad = false;
  row.each4([&](int32_t, f4 z) INLINE {
    most = fmaxf(most, max4(z));
    bad |= __builtin_isunordered(z.x, z.y) | __builtin_isunordered(z.z, z.w);
  });
  constexpr int32_t BAD = 1 << 16;
  if (T::G > 1 && group > 1) most = fmaxf(most, butterfly<1>(most));
  if (T::G > 2 && group > 2) most = fmaxf(most, butterfly<2>(most));
  if (T::G > 4 && group > 4) most = fmaxf(most, butterfly<4>(most));
  if (T::G > 8 && group > 8) most = fmaxf(most, butterfly<8>(most));
  *top = most;
  *low = most > -INFINITY ? most : INFINITY;
  *groups = (most > -INFINITY && team.lane % group == 0) + (bad ? BAD : 0);
  team.range(top, low, groups);
  return *groups < BAD && fabsf(*top) < INFINITY;
}
// Groups of so many lanes that there are k of them where the row is not masked:
// the first k entries are then found above the least group's largest.
inline int32_t group_of(int64_t lanes, int32_t C, int32_t k) {
  const int64_t held = std::min<int64_t>(lanes, ceil_div(C, 4));
  int32_t g = 1;
  while (g < 16 && held / (2 * g) > k) g *= 2;
  return g;
}

// The border of the first k entries; low and groups from row_range().
template <class T, class Row>
__device__ __forceinline__ Border first_entries(const T& team, Row& row, const float* from,
                                                int32_t C, int32_t k, float top, float low,
                                                int32_t groups, int32_t base_col = 0) {
  if (k > groups) {  // (else as many entries as groups are not below `low`)
    low = INFINITY;
    row.each([&](float z, int32_t) INLINE { low = fminf(low, z > -INFINITY ? z : INFINITY); });
    low = -team.max(-low);
  }
  float scale = (T::Shared::BINS - 1) / (top - low);
  if (!(scale < INFINITY)) scale = 0.f;
  team.clear();
  row.each([&](float z, int32_t) INLINE {
    team.add(T::bin_of(z, top, scale), 1, z >= low);
  });
  team.sync();
  Border b;
  int32_t bin;
  uint64_t base;
  const Present counts = {low};
  if (team.select(row, counts, top, scale, k, &b, &bin, &base)) return b;
  if constexpr (Row::CHUNKS > 0) {
    Reread<T::G, T::W> again;
    again.load(from, min(C, base_col + Row::MOST), team.t, base_col);
    b = team.search(again, counts, top, scale, bin, k, base);
    row.load(from, C, team.t, base_col);
  } else {
    b = team.search(row, counts, top, scale, bin, k, base);
  }
  return b;
}

// The least float z with (double)z - top >= cut, for a cut that is not above 0.
// The difference never falls as z grows, so the floats between -inf and the top
// are halved in their order: at most 32 times, whatever the arguments.  (Walking
// there from top + cut has no such bound.  Where the two cancel, all floats next
// to 0 have a difference that is rounded to cut: 6e8 of them for 1 and
// log(exp(-1)).)  It is nearly always next to top + cut, so that is tried first.
__host__ __device__ inline float least_near(float top, double cut) {
  uint32_t low = ordered(-INFINITY), high = ordered(top);
  const auto probe = [&](uint32_t key) INLINE {
    if (key <= low || key >= high) return;
    if ((double)float_of(key) - top >= cut) high = key;
    else low = key;
  };
  const uint32_t guess = ordered((float)((double)top + cut));
  probe(guess);
  probe(guess - 1);
  probe(guess + 1);
  while (high - low > 1) probe(low + (high - low) / 2);
  return float_of(high);
}
// The border of the entries with z - top >= cut, in doubles.
__device__ __forceinline__ Border near_entries(float top, double cut) {
  return {least_near(top, cut), 0x7fffffff};
}

__device__ __forceinline__ Border earlier(Border a, Border b) {
  const bool second = within(a, b.z, b.col);
  return {second ? b.z : a.z, second ? b.col : a.col};
}

__device__ __forceinline__ uint64_t unit_fraction(float u) {
  if (!(u > 0.f)) return 0;
  if (u >= 1.f) return ~0ull;
  return (uint64_t)((double)u * 18446744073709551616.0);
}

// The entry in whose weight `target` falls, counted from the first of the
// wavefront's.  KEPT: `sums` has the lane's sums of its chunks' weights (else
// they are formed again: one of several wavefronts does it).  The lane that holds
// the entry writes the row's action.
template <bool KEPT, class T, class Row>
__device__ __forceinline__ void pick_entry(const SampleArgs& a, const T& team, const Row& row,
                                           const Weights& weight, int32_t i, uint64_t target,
                                           double lse, const uint64_t* sums) {
  int at_chunk = 0;
  // its chunks of the wavefront, one after the other
  bool found = false;
  int32_t col = 0;
  f4 z = {};
  row.each4([&](int32_t at, f4 v) INLINE {
    const int k = at_chunk++;
    if (found) return;
    const uint64_t sum = lanes_sum<T::G>(KEPT ? sums[k] : weight.sum4(v, at));
    found = target < sum;
    if (!found) {
      target -= sum;
      return;
    }
    col = at;
    z = v;
  });
  const uint64_t w0 = weight(z.x, col), w1 = weight(z.y, col + 1), w2 = weight(z.z, col + 2),
                 mine = w0 + w1 + w2 + weight(z.w, col + 3), x = team.before(mine);
  if (target < x || target >= x + mine) return;
  target -= x;
  const int j = target < w0 ? 0 : target < w0 + w1 ? 1 : target < w0 + w1 + w2 ? 2 : 3;
  a.action[i] = col + j;
  if (a.logp) {
    const float za = j == 0 ? z.x : j == 1 ? z.y : j == 2 ? z.z : z.w;
    a.logp[i] = (float)((double)za - weight.top - lse);
  }
}

constexpr int32_t MOST_TOP = GNN_TOP_MOST;

struct TopArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  int32_t k;
  double inv_t;
  int32_t* index;
  float *logq, *rest;
  int32_t group;  // see row_range
  int64_t block0;
  // rows that several blocks share (long_rows.hip)
  struct TopPart* parts;
  uint64_t* candidates;  // k for each part
  int32_t per_row;
};

// The entries up to a border into the list (of `most` places), and the sums of
// exp((z - top) / T) over them and over the others (the lane's shares).  In any
// order, counted in team.s.count (put to 0 before); or, ORDERED, the wavefront's
// into a list of its own, by chunks and lanes, so that it is the same in every call:
// returns how many.
template <bool ORDERED, class T, class Row>
__device__ __forceinline__ int32_t collect(const T& team, const Row& row, const Border& b,
                                           float top, double inv_t, uint64_t* list, int32_t most,
                                           double* in_sum, double* out_sum) {
  static_assert(!ORDERED || T::G == 64, "whole wavefronts");
  int32_t count = 0;
  const float octaves = (float)(inv_t * 1.4426950408889634);
  double in = 0.0, out = 0.0;
  row.each4([&](int32_t col, f4 z) INLINE {
    bool kept[4], any = false;
    f4 e;
    float less = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kept[j] = within(b, z[j], col + j) & (z[j] > -INFINITY);
      any |= kept[j];
      // (exp as a power of two: what falls below the smallest normal number is 0)
      e[j] = __builtin_amdgcn_exp2f((z[j] - top) * octaves);
      less += kept[j] ? 0.f : e[j];
    }
    out += less;
    if (ORDERED ? !__ballot(any) : !any) return;
    float more = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int32_t at;
      if constexpr (ORDERED) {
        const uint64_t who = __ballot(kept[j]);
        at = count + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32),
                                               __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
        count += __popcll(who);
      }
      if (!kept[j]) continue;
      if constexpr (!ORDERED) at = atomicAdd(&team.s.count, 1);
      more += e[j];
      list[min(at, most - 1)] = place(z[j], col + j);
    }
    in += more;
  });
  *in_sum = in;
  *out_sum = out;
  return count;
}

// A row's outputs from the list of its first entries and the sums of both
// parts.
template <class T>
__device__ __forceinline__ void write_top(const TopArgs& a, const T& team, uint64_t* list,
                                          int32_t i, float top, double in, double out) {
  int32_t* index = a.index + (int64_t)i * a.k;
  float* logq = a.logq + (int64_t)i * a.k;
  const int32_t m = min(team.s.count, a.k);
  const double lse = log_quick((float)(in + out));
  // each in its place: those before it are counted, eight at a time
  for (int32_t j = m + team.t; j < (m + 7) / 8 * 8; j += T::LANES) list[j] = ~0ull;
  team.sync();
  for (int32_t j = team.t; j < a.k; j += T::LANES) {
    if (j >= m) {
      index[j] = -1;
      logq[j] = -INFINITY;
      continue;
    }
    const uint64_t own = list[j];
    int32_t rank = 0;
    for (int32_t q = 0; q < m; q += 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) rank += list[q + k] < own;
    }
    index[rank] = (int32_t)(uint32_t)own;
    logq[rank] = (float)(((double)logit_of(own) - top) * a.inv_t - lse);
  }
  if (team.t == 0 && a.rest) a.rest[i] = (float)(out / (in + out));
}

template <class T>
__device__ __forceinline__ void write_none(const TopArgs& a, const T& team, int32_t i) {
  for (int32_t j = team.t; j < a.k; j += T::LANES) {
    a.index[(int64_t)i * a.k + j] = -1;
    a.logq[(int64_t)i * a.k + j] = -INFINITY;
  }
  if (team.t == 0 && a.rest) a.rest[i] = 0.f;
}

// ---------------------------------------------------------------- launches

template <class Args>
struct Launch {
  void (*kernel)(Args);
  int32_t rows, threads;  // of a block
  int32_t lanes() const { return threads / rows; }
};

// Kernel::of<G, W, Row>() and Kernel::small<V>() (rows of up to Kernel::SMALL
// columns, a lane each), for rows of at most Kernel::MOST columns.
template <class Args, class Kernel>
struct Chosen {
  static constexpr bool SPREAD = true;
  static constexpr int32_t MOST = Kernel::MOST;
  template <int G, int W, int V>
  Launch<Args> held() const {
    return {Kernel::template of<G, W, Held<G, W, V>>(), threads_of<G, W>() / (G * W),
            threads_of<G, W>()};
  }
};
template <class Args, class Kernel>
Launch<Args> choose(int32_t n, int32_t C, int32_t places = 0) {
  const Shape s = shape_of(n, C, places, Kernel::SMALL, Chosen<Args, Kernel>::SPREAD);
  if (s.G > 1) return of_shape(s, Chosen<Args, Kernel>());
  if constexpr (Kernel::SMALL > 24)
    if (s.V == 8) return {Kernel::template small<8>(), 256, 256};
  switch (s.V) {
    case 1: return {Kernel::template small<1>(), 256, 256};
    case 2: return {Kernel::template small<2>(), 256, 256};
    case 4: return {Kernel::template small<4>(), 256, 256};
  }
  return {Kernel::template small<6>(), 256, 256};
}

template <class Args>
hipError_t run(const Launch<Args>& l, Args a, hipStream_t stream) {
  const int64_t blocks = ceil_div(a.n, l.rows);
  for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
    l.kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), l.threads, 0, stream>>>(a);
  return hipGetLastError();
}

// Rows past LONG_SAMPLE and LONG_TOP columns (long_rows.hip).
size_t sample_long_bytes(int32_t n, int32_t C);
hipError_t sample_long(SampleArgs a, void* workspace, hipStream_t stream);
size_t top_long_bytes(int32_t n, int32_t C, int32_t k);
hipError_t top_long(TopArgs a, void* workspace, hipStream_t stream);

}  // namespace gnnprop
