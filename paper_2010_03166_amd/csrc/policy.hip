// Log-probabilities of chosen actions, and the clipped policy loss with a KL
// term and its gradient (the formulas: include/gnnprop.h).
//
// Per row: top = max z, sum = sum exp(z - top), lp = z[a] - top - log sum;
// then the row's loss terms and the slope c = w dl/dlp, and the gradient
// c (1[j = a] - exp(z_j - top) / sum).
//
// Bound by memory: 4 bytes a logit read, with a gradient 4 written.  So every
// row is read once, held in registers from its sums to its gradient, by as
// many lanes as its length takes (choose() below), and all of a row's reads
// are under way before the first is waited for.  Only rows past 32,768 columns
// are read twice.  Measured, us a call (and what of it are the final sums, a
// launch of their own unless one block has all rows):
//   50,001 x 121, rows off alignment   14.8 (2.5)   3.3 TB/s
//   16,384 x 2,048                     52.8 (4)     5.1 TB/s, a large copy 5.05
//   64 x 131,071                       23.5 (2.5)   2.9 TB/s
//   2,000 x 20,011, log-probabilities  29.1         5.5 TB/s
// What the same accesses take with nothing computed: 10.6 us for the first.
// Up to 16 columns a lane has a row of its own, and its accesses are scattered:
// 200,000 x 7 9.3 us, 200,000 x 16 12.5, where the bytes take 3.2 and 6.0.
// Stores past the caches (non-temporal) take 3 to 15 % off the rows of whole
// cache lines, but the product that reads dZ next loses more than that.
#include <cmath>

#include "abi.hpp"

using namespace gnnprop;

namespace {

constexpr int THREADS = 256;
constexpr int32_t MOST_COLS = 1 << 24;  // (a long row's chunks are joined by each of its blocks)

struct Terms {  // a row's share of `out`
  double loss, kl, cut;
};
struct Chunk {  // sums of a part of a row
  double sum;   // of exp(z - top)
  float top;
  float pad;
};

struct PolicyArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  const int32_t* action;
  const float *adv, *old_lp, *ref_lp, *weight;  // adv in the place of those left out
  bool has_old, has_ref, has_weight;
  double lo, hi, beta;  // clip to [lo, hi]
  double mean;          // 1 / n
  float* out;
  float* logp;
  float* dZ;
  int64_t ld_dz;
  Terms* part;    // one per block (split rows: one per row)
  Chunk* chunks;  // split rows: per_row for each row
  double* exact;  // and, of the rows next to a border of the clip, their sums in doubles
  int32_t per_row;
  int64_t blocks, block0;  // of all launches, and in the launches before
};

// ------------------------------------------------------------- row scalars

// exp(x - top), where top = -inf only if no logit is above it: then 0 (or
// NaN for a NaN), so that the sum is 0 exactly for a row without any action.
__device__ inline float shift_of(float top) { return top == -INFINITY ? 0.f : top; }

// What a row's terms are computed from, besides its sum.
struct RowIn {
  int32_t act;
  float za, adv, old_lp, ref_lp, w;
  bool chosen;
};
// The action is read before the row's logits and the rest after them, so that
// the chosen logit's own read, which needs the action, waits for no other.
// (No branches here either: arrays that the caller left out are some other
// array of the row's, and not used.)
__device__ inline RowIn row_in(const PolicyArgs& a, int32_t i, int32_t act, bool loss) {
  RowIn r = {};
  r.act = act;
  r.chosen = act >= 0 && act < a.C;
  r.za = a.Z[(int64_t)i * a.ld_z + (r.chosen ? act : 0)];
  if (loss) {
    r.adv = a.adv[i];
    r.old_lp = a.old_lp[i];
    r.ref_lp = a.ref_lp[i];
    r.w = a.weight[i];
  }
  return r;
}

// Scalar functions.  What is fp32 in a row's logarithm, in steps u = 2^-24:
// the exponentials, 4 u each (doubles would bound the kernels by instructions)
// and ln C u, the weighted mean of their rounded arguments; the sum of at most
// 16 of a lane, five additions deep, 5 u (all beyond in doubles); a chunk's
// factor of a split row, 4 u; the sum's own rounding before its logarithm, u,
// and that, 0.7 u.  Together below (20 + ln C) u, 2.2e-6 for any C, beside
// which fp32 logarithms and ratios lose little, and library functions of
// doubles would hold a hundred registers for their coefficients.  A row whose
// ratio is as near to a border of the clip as those errors, one in 1e5 or so,
// is computed once more in doubles.
constexpr double NEAR = 4e-6;

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

// One step of third order from there (e^y is s but for 2e-7).
__device__ inline double log_exact(double s) {
  const double y = log_quick((float)s), e = exp_exact(y);
  return y + 2.0 * (s - e) / (s + e);
}

// e = exp(f) made exp(x), f being x rounded to fp32 (0 and infinity stay).
__device__ inline double refined(double e, double x, float f) {
  return e > 0.0 && e < INFINITY ? fma(e, x - (double)f, e) : e;
}
// exp(f) where fp32 would overflow too (as the eighth power of exp(f / 8)).
__device__ inline double exp_wide(float f) {
  if (!(f > 80.f)) return (double)expf(f);
  double e = (double)expf(0.125f * f);
  e *= e;
  e *= e;
  return e * e;
}
__device__ inline double exp_quick(double x) {
  const float f = (float)x;
  return refined(exp_wide(f), x, f);
}
// The factor from a chunk's top to its row's: exp(x), x <= 0.  A chunk of
// nothing but -inf has no top to come from, and x may be anything; its sum is
// 0, and a factor of at most 1 leaves it 0.
__device__ inline double exp_down(double x) {
  x = fmin(x, 0.0);
  const float f = (float)x;
  return refined((double)expf(f), x, f);
}
// e^x - 1, and e^x - 1 - x, from the series x^2 (1/2 + x/6 + ...) where the
// difference would lose digits (its first term left out is below 1e-7 of it).
__device__ inline double expm1_quick(double x, double* less_x) {
  const float f = (float)x;
  if (fabsf(f) < 0.5f) {
    float p = 1.f / 40320.f;
    p = fmaf(p, f, 1.f / 5040.f);
    p = fmaf(p, f, 1.f / 720.f);
    p = fmaf(p, f, 1.f / 120.f);
    p = fmaf(p, f, 1.f / 24.f);
    p = fmaf(p, f, 1.f / 6.f);
    p = fmaf(p, f, 0.5f);
    *less_x = (double)p * x * x;
    return x + *less_x;
  }
  const double e = refined(exp_wide(f), x, f) - 1.0;
  *less_x = x == INFINITY ? x : e - x;
  return e;
}

template <bool EXACT>
__device__ inline double log_prob(const RowIn& r, float top, double sum) {
  if (!r.chosen) return 0.0;
  if (sum == 0.0) return -INFINITY;
  return (double)r.za - top - (EXACT ? log_exact(sum) : log_quick((float)sum));
}

// The row's terms, and its slope c = w dl/dlp.  Returns whether the ratio is
// so close to a border of the clip that only doubles decide.
template <bool EXACT>
__device__ inline bool row_terms(const PolicyArgs& a, const RowIn& r, double sum, double lp,
                                 Terms* t, float* c) {
  *c = 0.f;
  *t = {0.0, 0.0, 0.0};
  const double w = a.has_weight ? (double)r.w : a.mean;
  if (!r.chosen || sum == 0.0 || w == 0.0) return false;
  const double A = r.adv, x = lp - (double)r.old_lp;
  const double rho = !a.has_old ? (lp == lp ? 1.0 : lp) : EXACT ? exp_exact(x) : exp_quick(x);
  // (a border at 0 cuts nothing, and a ratio that underflows is no nearer to it)
  const bool near = a.has_old && rho > 0.0 && rho < INFINITY &&
                    (fabs(rho - a.lo) <= NEAR * rho || fabs(rho - a.hi) <= NEAR * rho);
  const double ra = rho * A, ca = fmin(fmax(rho, a.lo), a.hi) * A;
  const bool cut = ra > ca;  // false for a NaN, which then shows in ra
  double slope = cut ? 0.0 : -ra, loss = -(cut ? ca : ra);
  if (a.has_ref) {
    double kl;
    const double e = expm1_quick((double)r.ref_lp - lp, &kl);
    t->kl = w * kl;
    if (a.beta != 0.0) {
      loss += a.beta * kl;
      slope -= a.beta * e;
    }
  }
  t->loss = w * loss;
  t->cut = cut ? w : 0.0;
  *c = (float)(w * slope);
  return near;
}

// ------------------------------------------------------------- reductions

// The block's sum of terms in thread 0, in a fixed order.
template <int T>
__device__ inline Terms block_terms(Terms t) {
  __shared__ Terms s[T / 64];
  t.loss = lanes_sum<64>(t.loss);
  t.kl = lanes_sum<64>(t.kl);
  t.cut = lanes_sum<64>(t.cut);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = t;
  __syncthreads();
  t = s[0];
  for (int k = 1; k < T / 64; ++k) {
    t.loss += s[k].loss;
    t.kl += s[k].kl;
    t.cut += s[k].cut;
  }
  return t;
}

__device__ inline void store_out(float* out, const Terms& t) {
  out[0] = (float)t.loss;
  out[1] = (float)t.kl;
  out[2] = (float)t.cut;
}

// The block's share of `out`, or `out` itself where it is the only block.
__device__ inline void store_terms(const PolicyArgs& a, const Terms& t) {
  if (threadIdx.x) return;
  if (a.blocks == 1) store_out(a.out, t);
  else a.part[a.block0 + blockIdx.x] = t;
}

// Sum of exp(z - top) over columns in doubles, by a wavefront (of a row) or by
// a block of T threads (of columns [from, to)), in all of the threads.
__device__ inline double exact_part(const float* z, int32_t at, int32_t to, int32_t step, float top) {
  const double shift = shift_of(top);
  double sum = 0.0;
#pragma unroll 1
  for (int32_t j = at; j < to; j += step) sum += exp_exact((double)z[j] - shift);
  return lanes_sum<64>(sum);
}
__device__ inline double exact_sum(const float* z, int32_t C, float top) {
  return exact_part(z, threadIdx.x & 63, C, 64, top);
}
template <int T>
__device__ inline double exact_sum_block(const float* z, int32_t from, int32_t to, float top) {
  __shared__ double s[T / 64];
  const double part = exact_part(z, from + threadIdx.x, to, T, top);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = part;
  __syncthreads();
  double sum = s[0];
#pragma unroll 1
  for (int k = 1; k < T / 64; ++k) sum += s[k];
  return sum;
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

// c (1[j = act] - e_j inv) for columns col .. col + 3; 0 where c is 0,
// whatever the logits.
__device__ inline f4 grad4(f4 e, int32_t col, int32_t act, float c, float inv) {
  f4 g = {0.f, 0.f, 0.f, 0.f};
  if (c == 0.f) return g;
  g.x = c * ((col == act ? 1.f : 0.f) - e.x * inv);
  g.y = c * ((col + 1 == act ? 1.f : 0.f) - e.y * inv);
  g.z = c * ((col + 2 == act ? 1.f : 0.f) - e.z * inv);
  g.w = c * ((col + 3 == act ? 1.f : 0.f) - e.w * inv);
  return g;
}

// ------------------------------------------------ several rows a wavefront

// G lanes to a row of at most 4 G V columns, R = 256 / G rows a block.  Every
// lane computes its row's scalars: the same instructions as for one lane, and
// no wavefront waits for another.  (One thread a row, between two barriers:
// 60,000 x 500 58.6 -> 63.5 us.)  72 registers let seven blocks share a CU:
// six and eight, with spills, are slower for some widths and faster for none.
template <int G, int V, bool LOSS>
__global__ __launch_bounds__(THREADS, 7) void rows_kernel(PolicyArgs a) {
  constexpr int R = THREADS / G;
  const int t = threadIdx.x, lane = t % G, grp = t / G;
  const int32_t first = (int32_t)(a.block0 + blockIdx.x) * R;
  const bool mine = grp < a.n - first;
  const int32_t i = first + (mine ? grp : 0);
  const float* row = a.Z + (int64_t)i * a.ld_z;
  const int32_t act = a.action[i];
  f4 z[V];
#pragma unroll
  for (int k = 0; k < V; ++k) z[k] = load_chunk<V>(row, k, (k * G + lane) * 4, a.C);
  const RowIn r = row_in(a, i, act, LOSS);
  z[V - 1] = cut_cols(z[V - 1], ((V - 1) * G + lane) * 4, a.C);
  float top = max4(z[0]);
#pragma unroll
  for (int k = 1; k < V; ++k) top = fmaxf(top, max4(z[k]));
  top = lanes_max<G>(top);
  const float shift = shift_of(top);
  float part = 0.f;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    z[k] = exp4(z[k], shift);
    part += sum4(z[k]);
  }
  double sum = lanes_sum<G>((double)part);
  const double lp = log_prob<false>(r, top, sum);
  if (lane == 0 && mine && a.logp) a.logp[i] = (float)lp;
  if (!LOSS) return;
  Terms terms;
  float c;
  const bool near = row_terms<false>(a, r, sum, lp, &terms, &c) && mine;
  if (__any(near)) {
    // each such row by the whole wavefront
    for (uint64_t rows = __ballot(near && lane == 0); rows; rows &= rows - 1) {
      const int from = __ffsll((unsigned long long)rows) - 1;
      const int32_t q = __shfl(i, from, 64);
      const double s = exact_sum(a.Z + (int64_t)q * a.ld_z, a.C, __shfl(top, from, 64));
      if ((t & 63) / G == from / G) sum = s;
    }
    if (near) row_terms<true>(a, r, sum, log_prob<true>(r, top, sum), &terms, &c);
    // read once more, so that this branch has the registers
#pragma unroll
    for (int k = 0; k < V; ++k) z[k] = load_chunk<V>(row, k, (k * G + lane) * 4, a.C);
    z[V - 1] = cut_cols(z[V - 1], ((V - 1) * G + lane) * 4, a.C);
#pragma unroll
    for (int k = 0; k < V; ++k) z[k] = exp4(z[k], shift);
  }
  if (a.dZ && mine) {
    float* to = a.dZ + (int64_t)i * a.ld_dz;
    const float inv = 1.f / (float)sum;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int32_t col = (k * G + lane) * 4;
      store_cols(to, col, a.C, grad4(z[k], col, r.act, c, inv));
    }
  }
  if (lane != 0 || !mine) terms = {0.0, 0.0, 0.0};
  store_terms(a, block_terms<THREADS>(terms));
}

// ---------------------------------------------------------- one row a block

// T threads to a row of at most 4 T V columns.  Of more than four chunks a
// thread the rest waits in LDS from the sums to the gradient (each thread
// reads what it wrote), so that 64 registers do and two blocks of 1,024
// threads share a CU: 2,000 x 20,011 79 -> 68 us, 1,000 x 32,768 67 -> 60.5
// (64 rows of 32,768, a block a CU either way: 11.5 -> 12.3).
template <int T, int V, bool LOSS>
__global__ __launch_bounds__(T, T == 1024 ? 8 : 1) void block_kernel(PolicyArgs a) {
  constexpr int KEPT = V < 4 || !LOSS ? V : 4, AWAY = V - KEPT;
  __shared__ f4 s_away[AWAY > 0 ? AWAY * T : 1];
  __shared__ float s_top[T / 64], s_c, s_inv;
  __shared__ double s_sum[T / 64];
  __shared__ int32_t s_near;
  const int t = threadIdx.x, wave = t >> 6;
  const int32_t i = (int32_t)(a.block0 + blockIdx.x);
  const float* row = a.Z + (int64_t)i * a.ld_z;
  const int32_t act = a.action[i];
  f4 z[V];
#pragma unroll
  for (int k = 0; k < V; ++k) z[k] = load_chunk<V>(row, k, (k * T + t) * 4, a.C);
  const RowIn r = row_in(a, i, act, LOSS);
  z[V - 1] = cut_cols(z[V - 1], ((V - 1) * T + t) * 4, a.C);
  float top = max4(z[0]);
#pragma unroll
  for (int k = 1; k < V; ++k) top = fmaxf(top, max4(z[k]));
  top = lanes_max<64>(top);
  if ((t & 63) == 0) s_top[wave] = top;
  __syncthreads();
  top = s_top[0];
#pragma unroll
  for (int k = 1; k < T / 64; ++k) top = fmaxf(top, s_top[k]);
  const float shift = shift_of(top);
  float some = 0.f;  // of at most four chunks
  double part = 0.0;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    z[k] = exp4(z[k], shift);
    some += sum4(z[k]);
    if (k % 4 == 3 || k == V - 1) {
      part += some;
      some = 0.f;
    }
    if (k >= KEPT) s_away[(k - KEPT) * T + t] = z[k];
  }
  part = lanes_sum<64>(part);
  if ((t & 63) == 0) s_sum[wave] = part;
  __syncthreads();
  double sum = 0.0;
  Terms terms;
  if (wave == 0) {
#pragma unroll
    for (int k = 0; k < T / 64; ++k) sum += s_sum[k];
    const double lp = log_prob<false>(r, top, sum);
    if (t == 0 && a.logp) a.logp[i] = (float)lp;
    if (LOSS) {
      float c;
      const bool near = row_terms<false>(a, r, sum, lp, &terms, &c);  // the same in all lanes
      if (t == 0) {
        s_c = c;
        s_inv = 1.f / (float)sum;
        s_near = near;
      }
    }
  }
  if (!LOSS) return;
  __syncthreads();
  if (s_near) {
    sum = exact_sum_block<T>(row, 0, a.C, top);
    if (t == 0) {
      row_terms<true>(a, r, sum, log_prob<true>(r, top, sum), &terms, &s_c);
      s_inv = 1.f / (float)sum;
    }
    __syncthreads();
    // read once more, so that this branch has the registers
#pragma unroll
    for (int k = 0; k < KEPT; ++k) z[k] = load_chunk<V>(row, k, (k * T + t) * 4, a.C);
    if (AWAY == 0) z[V - 1] = cut_cols(z[V - 1], ((V - 1) * T + t) * 4, a.C);
#pragma unroll
    for (int k = 0; k < KEPT; ++k) z[k] = exp4(z[k], shift);
  }
  store_terms(a, terms);
  if (!a.dZ) return;
  float* to = a.dZ + (int64_t)i * a.ld_dz;
  const float c = s_c, inv = s_inv;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const int32_t col = (k * T + t) * 4;
    const f4 e = k < KEPT ? z[k] : s_away[(k - KEPT) * T + t];
    store_cols(to, col, a.C, grad4(e, col, r.act, c, inv));
  }
}

// -------------------------------------------------------- several blocks a row

// Rows longer than 32,768 columns are cut into chunks, a block each: one
// launch for the chunks' sums, one that joins a row's sums, computes its
// scalars in every block of the row alike, and writes the chunk's gradient
// from a second reading (out of the caches, for the few rows that are so
// long), one that adds the rows' terms.  Where a row's ratio is next to a
// border of the clip, the second launch forms its chunks' sums in doubles
// instead of their gradients, and the third joins those and writes them: a
// row of 2^22 columns takes 44 us more than one away from the border (with
// each of its 1,024 blocks summing the whole row 6,800), 64 x 131,071 with
// every row there 68 us (443).  Blocks of 1,024
// threads with up to 16 chunks a thread in registers would take rows of up to
// 65,536 once: 600 x 40,000 56 us instead of 60, 500 x 65,536 66 instead of
// 82, but 1 x 65,536 13.3 instead of 9.9 and its log-probabilities 9.7 instead
// of 5.3.  Chunks of 2,048 / 4,096 / 8,192: 64 x 131,071 28.3 / 26.6 / 26.9
// us, 1 x 131,071 9.4 / 10.4 / 12.5.
constexpr int SPLIT_V = 4;
constexpr int SPLIT_COLS = 4 * THREADS * SPLIT_V;
__host__ __device__ inline int32_t chunks_of(int32_t C) {
  return (int32_t)ceil_div(C, SPLIT_COLS);
}

__device__ inline void split_load(const float* row, int32_t first, int32_t C, f4 (&z)[SPLIT_V]) {
#pragma unroll
  for (int k = 0; k < SPLIT_V; ++k) z[k] = load_cols(row, first + (k * THREADS + threadIdx.x) * 4, C);
}
// The gradient of the chunk at column `first` from its logits.
__device__ inline void split_store(const PolicyArgs& a, int32_t i, int32_t first, f4 (&z)[SPLIT_V],
                                   float shift, int32_t act, float c, float inv) {
  float* to = a.dZ + (int64_t)i * a.ld_dz;
#pragma unroll
  for (int k = 0; k < SPLIT_V; ++k) {
    const int32_t col = first + (k * THREADS + threadIdx.x) * 4;
    store_cols(to, col, a.C, grad4(exp4(cut_cols(z[k], col, a.C), shift), col, act, c, inv));
  }
}

__global__ __launch_bounds__(THREADS) void split_sums_kernel(PolicyArgs a) {
  __shared__ float s_top[THREADS / 64];
  __shared__ double s_sum[THREADS / 64];
  const int t = threadIdx.x, wave = t >> 6;
  const int64_t b = a.block0 + blockIdx.x;
  const int32_t i = (int32_t)(b / a.per_row), first = (int32_t)(b % a.per_row) * SPLIT_COLS;
  const float* row = a.Z + (int64_t)i * a.ld_z;
  f4 z[SPLIT_V];
  split_load(row, first, a.C, z);
#pragma unroll
  for (int k = 0; k < SPLIT_V; ++k) z[k] = cut_cols(z[k], first + (k * THREADS + t) * 4, a.C);
  float top = max4(z[0]);
#pragma unroll
  for (int k = 1; k < SPLIT_V; ++k) top = fmaxf(top, max4(z[k]));
  top = lanes_max<64>(top);
  if ((t & 63) == 0) s_top[wave] = top;
  __syncthreads();
  top = s_top[0];
#pragma unroll
  for (int k = 1; k < THREADS / 64; ++k) top = fmaxf(top, s_top[k]);
  const float shift = shift_of(top);
  float part = 0.f;
#pragma unroll
  for (int k = 0; k < SPLIT_V; ++k) part += sum4(exp4(z[k], shift));
  const double all = lanes_sum<64>((double)part);
  if ((t & 63) == 0) s_sum[wave] = all;
  __syncthreads();
  if (t == 0) {
    double sum = 0.0;
    for (int k = 0; k < THREADS / 64; ++k) sum += s_sum[k];
    a.chunks[b] = {sum, top, 0.f};
  }
}

// Terms that stand for a row that is left to the last launch, and add nothing.
// No other row's third one is a negative zero: it is 0 or a weight that is not.
constexpr Terms LEFT = {0.0, 0.0, -0.0};
__device__ inline bool is_left(const Terms& t) {
  return (uint64_t)__double_as_longlong(t.cut) == 1ull << 63;
}

// a.blocks blocks: those of a row's chunks, or one a row without a gradient.
template <bool LOSS>
__global__ __launch_bounds__(THREADS) void split_grad_kernel(PolicyArgs a) {
  const int t = threadIdx.x, lane = t & 63;
  const int32_t todo = LOSS && a.dZ ? a.per_row : 1;
  const int64_t b = a.block0 + blockIdx.x;
  const int32_t i = (int32_t)(b / todo), first = (int32_t)(b % todo) * SPLIT_COLS;
  const float* row = a.Z + (int64_t)i * a.ld_z;
  const int32_t act = a.action[i];
  f4 z[SPLIT_V];
  if (LOSS && a.dZ) split_load(row, first, a.C, z);
  const RowIn r = row_in(a, i, act, LOSS);
  // every wavefront joins the row's sums alike
  const Chunk* at = a.chunks + (int64_t)i * a.per_row;
  float top = -INFINITY;
  for (int32_t k = lane; k < a.per_row; k += 64) top = fmaxf(top, at[k].top);
  top = lanes_max<64>(top);
  const float shift = shift_of(top);
  double sum = 0.0;
  for (int32_t k = lane; k < a.per_row; k += 64) {
    const Chunk c = at[k];
    sum += c.sum * exp_down((double)shift_of(c.top) - shift);
  }
  sum = lanes_sum<64>(sum);
  const double lp = log_prob<false>(r, top, sum);
  const bool writer = t == 0 && first == 0;  // of what there is one of a row
  if (writer && a.logp) a.logp[i] = (float)lp;
  if (!LOSS) return;
  Terms terms;
  float c;
  const bool near = row_terms<false>(a, r, sum, lp, &terms, &c);  // alike in all threads of a row
  if (near) {
    const double part =
        exact_sum_block<THREADS>(row, first, a.dZ ? min(first + SPLIT_COLS, a.C) : a.C, top);
    if (a.dZ) {  // left to split_final_kernel
      if (t == 0) a.exact[b] = part;
      terms = LEFT;
    } else {
      row_terms<true>(a, r, part, log_prob<true>(r, top, part), &terms, &c);
    }
  }
  if (writer) a.part[i] = terms;
  if (a.dZ && !near) split_store(a, i, first, z, shift, r.act, c, 1.f / (float)sum);
}

constexpr int AT_ONCE = 8;  // reads under way, each from another XCD's block

// The sum of terms first, first + step, ... of `count`; left: whether one of
// them is that of a row left.
__device__ inline Terms sum_terms(const Terms* __restrict__ part, int64_t first, int64_t step,
                                  int32_t count, bool* left) {
  Terms t = {0.0, 0.0, 0.0};
  *left = false;
  for (int64_t k = first; k < count; k += AT_ONCE * step) {
    Terms x[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      x[j] = k + j * step < count ? part[k + j * step] : Terms{0.0, 0.0, 0.0};
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      t.loss += x[j].loss;
      t.kl += x[j].kl;
      t.cut += x[j].cut;
      *left |= is_left(x[j]);
    }
  }
  return t;
}

// A row that the launch before left, from its chunks' sums in doubles: by 16
// lanes, so that a block takes the terms of 16 rows at once.
struct Left {
  RowIn r;
  float top, c, inv;
  Terms terms;
};
__device__ inline Left left_row(const PolicyArgs& a, int32_t i) {
  Left x;
  x.r = row_in(a, i, a.action[i], true);
  const int64_t at = (int64_t)i * a.per_row;
  float top = -INFINITY;
  double sum = 0.0;
  for (int32_t k = threadIdx.x & 15; k < a.per_row; k += 16) {
    top = fmaxf(top, a.chunks[at + k].top);
    sum += a.exact[at + k];
  }
  x.top = lanes_max<16>(top);
  sum = lanes_sum<16>(sum);
  row_terms<true>(a, x.r, sum, log_prob<true>(x.r, x.top, sum), &x.terms, &x.c);
  x.inv = 1.f / (float)sum;
  return x;
}

// out = the sum of all rows' terms, by block 0, and the gradients of the rows
// left, a chunk of one to a block in turn.
__global__ __launch_bounds__(THREADS) void split_final_kernel(PolicyArgs a) {
  __shared__ int32_t s_left[THREADS / 64];
  const int t = threadIdx.x, lane = t & 63;
  bool left;
  Terms all = sum_terms(a.part, t, THREADS, a.n, &left);
  left = __any(left);
  if (lane == 0) s_left[t >> 6] = left;
  __syncthreads();
  left = false;
  for (int k = 0; k < THREADS / 64; ++k) left |= s_left[k] != 0;
  if (left) {
    const int32_t blocks = (int32_t)gridDim.x;
    int32_t chunk0 = (int32_t)blockIdx.x;  // of the next such row, the block's first
    for (int64_t i0 = 0; i0 < a.n; i0 += 64) {
      uint64_t rows = __ballot(i0 + lane < a.n && is_left(a.part[min(i0 + lane, (int64_t)a.n - 1)]));
      for (; rows; rows &= rows - 1) {
        int32_t chunk = chunk0;
        chunk0 -= a.per_row % blocks;
        if (chunk0 < 0) chunk0 += blocks;
        if (chunk >= a.per_row) continue;
        const int32_t i = (int32_t)i0 + __ffsll((unsigned long long)rows) - 1;
        const Left x = left_row(a, i);
        for (; chunk < a.per_row; chunk += blocks) {
          f4 z[SPLIT_V];
          split_load(a.Z + (int64_t)i * a.ld_z, chunk * SPLIT_COLS, a.C, z);
          split_store(a, i, chunk * SPLIT_COLS, z, shift_of(x.top), x.r.act, x.c, x.inv);
        }
      }
    }
    if (blockIdx.x == 0)
      for (int64_t i = t / 16; i < a.n; i += THREADS / 16) {
        if (!is_left(a.part[i])) continue;
        const Terms terms = left_row(a, (int32_t)i).terms;
        if (t % 16) continue;
        all.loss += terms.loss;
        all.kl += terms.kl;
        all.cut += terms.cut;
      }
  }
  if (blockIdx.x) return;
  all = block_terms<THREADS>(all);
  if (t == 0) store_out(a.out, all);
}

// One block: out = the sum of `count` partial terms.  More: each its share of
// them, to `shares`.  In a fixed order either way.
template <int T>
__global__ __launch_bounds__(T) void policy_final_kernel(
    int32_t count, const Terms* __restrict__ part, Terms* __restrict__ shares,
    float* __restrict__ out) {
  bool left;
  const Terms t = block_terms<T>(sum_terms(part, (int64_t)blockIdx.x * T + threadIdx.x,
                                           (int64_t)gridDim.x * T, count, &left));
  if (threadIdx.x) return;
  if (gridDim.x == 1) store_out(out, t);
  else shares[blockIdx.x] = t;
}

// ---------------------------------------------------------------- launches

struct Launch {
  void (*rows)(PolicyArgs);  // rows_kernel or block_kernel; NULL: split rows
  int32_t rows_per_block, threads;
};
template <int G, bool LOSS>
Launch rows_of(int v) {
  return {v == 3 ? rows_kernel<G, 3, LOSS> : rows_kernel<G, 4, LOSS>, THREADS / G, THREADS};
}
template <int T, bool LOSS>
Launch block_of(int v) {
  return {v == 3 ? block_kernel<T, 3, LOSS> : block_kernel<T, 4, LOSS>, 1, T};
}

// Three or four chunks of four columns a lane where the row is long enough,
// and as few lanes as that takes: few exchanges between lanes, few lanes past
// the row's end.  Measured with one chunk a lane and with this rule, us:
// 200,000 x 41 37 and 27, 200,000 x 121 82 and 58, 30,000 x 1,000 88 and 66,
// 16,384 x 2,048 87 and 66, 2,000 x 20,011 (five chunks, eight before) 104 and
// 83; two and eight chunks lie between.
template <bool LOSS>
Launch choose(int32_t C) {
  const int64_t q = ceil_div(C, 4);
  if (q == 1) return {rows_kernel<1, 1, LOSS>, THREADS, THREADS};
  if (q == 2) return {rows_kernel<1, 2, LOSS>, THREADS, THREADS};
  int64_t lanes = 1;
  while (lanes < 1024 && 4 * lanes < q) lanes *= 2;
  const int v = (int)ceil_div(q, lanes);
  switch (lanes) {
    case 1: return rows_of<1, LOSS>(v);
    case 2: return rows_of<2, LOSS>(v);
    case 4: return rows_of<4, LOSS>(v);
    case 8: return rows_of<8, LOSS>(v);
    case 16: return rows_of<16, LOSS>(v);
    case 32: return rows_of<32, LOSS>(v);
    case 64: return block_of<64, LOSS>(v);
    case 128: return block_of<128, LOSS>(v);
    case 256: return block_of<256, LOSS>(v);
    case 512: return block_of<512, LOSS>(v);
  }
  switch (v) {
    case 3:
    case 4: return block_of<1024, LOSS>(v);
    case 5: return {block_kernel<1024, 5, LOSS>, 1, 1024};
    case 6: return {block_kernel<1024, 6, LOSS>, 1, 1024};
    case 7: return {block_kernel<1024, 7, LOSS>, 1, 1024};
    case 8: return {block_kernel<1024, 8, LOSS>, 1, 1024};
  }
  return {nullptr, 0, 0};
}

// Partial terms that one block adds; more are added in SHARES blocks first (us
// a call with one launch and with two: 7,500 terms 52.1 and 52.4, 16,384 terms
// 56.2 and 54.3, 30,000 terms 58.5 and 53.3).
constexpr int32_t FINAL_MOST = 8192, SHARES = 64;
// Blocks of the last launch of split rows: for the rows next to a border of the
// clip (adding the terms takes one).
constexpr int64_t SPLIT_LAST = 256;
// Blocks of one launch (2^32 threads are the most that a launch can have).
constexpr int64_t LAUNCH_BLOCKS = 1 << 21;

int32_t parts_of(int32_t n, const Launch& l) {
  return l.rows ? (int32_t)ceil_div(n, l.rows_per_block) : n;
}

// [partial terms | shares of them | chunks' sums | those in doubles]
struct Layout {
  size_t shares, chunks, exact, total;
};
Layout layout_of(int32_t n, int32_t C, bool loss) {
  const Launch l = choose<true>(C);
  Layout o;
  const int32_t parts = loss ? parts_of(n, l) : 0;
  o.shares = round_up((size_t)parts * sizeof(Terms), 256);
  o.chunks = o.shares + (l.rows && parts > FINAL_MOST ? SHARES * sizeof(Terms) : 0);
  const size_t chunks = l.rows ? 0 : (size_t)n * chunks_of(C);
  o.exact = o.chunks + round_up(chunks * sizeof(Chunk), 256);
  o.total = o.exact + (loss ? round_up(chunks * sizeof(double), 256) : 0);
  return o;
}

template <bool LOSS>
gnn_status launch(PolicyArgs a, void* workspace, hipStream_t stream) {
  const Launch l = choose<LOSS>(a.C);
  const Layout o = layout_of(a.n, a.C, LOSS);
  char* ws = static_cast<char*>(workspace);
  a.part = reinterpret_cast<Terms*>(ws);
  a.chunks = reinterpret_cast<Chunk*>(ws + o.chunks);
  a.exact = reinterpret_cast<double*>(ws + o.exact);
  a.per_row = chunks_of(a.C);
  const auto run = [&](void (*kernel)(PolicyArgs), int32_t threads, int64_t blocks) {
    a.blocks = blocks;
    for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
      kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), threads, 0, stream>>>(a);
  };
  timer_begin(GNN_K_LOSS, stream);
  const int32_t parts = parts_of(a.n, l);
  bool done = !LOSS;
  if (l.rows) {
    run(l.rows, l.threads, parts);
    done |= parts == 1;  // (one block has written `out` itself)
  } else {
    const int64_t chunks = (int64_t)a.n * a.per_row;
    run(split_sums_kernel, THREADS, chunks);
    run(split_grad_kernel<LOSS>, THREADS, LOSS && a.dZ ? chunks : a.n);
    const unsigned last = a.dZ ? (unsigned)std::max<int64_t>(1, std::min(chunks, SPLIT_LAST)) : 1;
    if (LOSS) split_final_kernel<<<last, THREADS, 0, stream>>>(a);
    done = true;
  }
  if (!done) {
    Terms* shares = reinterpret_cast<Terms*>(ws + o.shares);
    const Terms* from = parts > FINAL_MOST ? shares : a.part;
    const int32_t count = parts > FINAL_MOST ? SHARES : parts;
    if (parts > FINAL_MOST)
      policy_final_kernel<256><<<SHARES, 256, 0, stream>>>(parts, a.part, shares, nullptr);
    if (count <= 1024)
      policy_final_kernel<256><<<1, 256, 0, stream>>>(count, from, nullptr, a.out);
    else
      policy_final_kernel<1024><<<1, 1024, 0, stream>>>(count, from, nullptr, a.out);
  }
  timer_end(GNN_K_LOSS, (a.dZ ? 8.0 : 4.0) * a.n * a.C, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // namespace

extern "C" {

size_t gnn_policy_workspace_bytes(int32_t n, int32_t C) {
  if (n < 0 || C <= 0 || C > MOST_COLS) return 0;
  return layout_of(n, C, true).total;
}

gnn_status gnn_action_logp(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, float* logp, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  if (n < 0 || C <= 0 || C > MOST_COLS || ld_z < C) return GNN_ERR_SHAPE;
  if (n == 0) return GNN_OK;
  if (!Z || !action || !logp) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = layout_of(n, C, false).total;
  if (workspace_bytes < need || (need > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  const size_t rows = (size_t)n * 4;
  const void* ins[] = {Z, action};
  const size_t inb[] = {mat_bytes(n, C, ld_z), rows};
  for (int k = 0; k < 2; ++k)
    if (ranges_overlap(logp, rows, ins[k], inb[k]) ||
        ranges_overlap(workspace, need, ins[k], inb[k]))
      return GNN_ERR_ALIAS;
  if (ranges_overlap(logp, rows, workspace, need)) return GNN_ERR_ALIAS;
  PolicyArgs a = {};
  a.n = n;
  a.C = C;
  a.Z = Z;
  a.ld_z = ld_z;
  a.action = action;
  a.logp = logp;
  return launch<false>(a, workspace, stream);
}

gnn_status gnn_policy_loss(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, const float* advantage,
                           const float* old_logp, const float* ref_logp,
                           const float* weight, double clip_lo, double clip_hi,
                           double beta, float* out, float* logp, float* dZ,
                           int64_t ld_dz, void* workspace, size_t workspace_bytes,
                           hipStream_t stream) {
  if (n < 0 || C <= 0 || C > MOST_COLS || ld_z < C || (dZ && ld_dz < C)) return GNN_ERR_SHAPE;
  // written so that a NaN is refused
  if (!(clip_lo >= 0.0 && clip_lo <= 1.0) || !(clip_hi >= 0.0) ||
      !(beta >= 0.0 && beta < INFINITY))
    return GNN_ERR_SHAPE;
  if (!out) return GNN_ERR_NULL;
  if (n > 0 && (!Z || !action || !advantage || (beta > 0.0 && !ref_logp))) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = layout_of(n, C, true).total;
  if (workspace_bytes < need || (need > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  {
    const size_t rows = (size_t)n * 4;
    const void* ins[] = {Z, action, advantage, old_logp, ref_logp, weight};
    const size_t inb[] = {mat_bytes(n, C, ld_z), rows, rows, rows, rows, rows};
    const void* outs[] = {out, logp, dZ, workspace};
    const size_t outb[] = {12, rows, mat_bytes(n, C, ld_dz), need};
    for (int i = 0; i < 4; ++i) {
      for (int k = 0; k < 6; ++k)
        if (ranges_overlap(outs[i], outb[i], ins[k], inb[k])) return GNN_ERR_ALIAS;
      for (int k = 0; k < i; ++k)
        if (ranges_overlap(outs[i], outb[i], outs[k], outb[k])) return GNN_ERR_ALIAS;
    }
  }
  PolicyArgs a = {};
  a.n = n;
  a.C = C;
  a.Z = Z;
  a.ld_z = ld_z;
  a.action = action;
  a.adv = advantage;
  a.has_old = old_logp != nullptr;
  a.has_ref = ref_logp != nullptr;
  a.has_weight = weight != nullptr;
  a.old_lp = old_logp ? old_logp : advantage;
  a.ref_lp = ref_logp ? ref_logp : advantage;
  a.weight = weight ? weight : advantage;
  a.lo = 1.0 - clip_lo;
  a.hi = 1.0 + clip_hi;
  a.beta = beta;
  a.mean = n > 0 ? 1.0 / n : 0.0;
  a.out = out;
  a.logp = logp;
  a.dZ = dZ;
  a.ld_dz = ld_dz;
  return launch<true>(a, workspace, stream);
}

}  // extern "C"
