// The loss of a student that is taught by a teacher's top logits, and its
// gradient (the formulas: include/gnnprop.h).
//
// The entries that the teacher names are taken from their list, all others
// from the row: their sums are formed apart, so that the share left over is
// never a difference of two sums that are nearly alike.  Of the others the
// gradient is one factor times exp((z - their largest) / T), so a row is read
// once and each exponential computed once.  A lane's places of the list stay in
// registers with their q and p, in doubles.
//
// Bound by memory where rows are long: 16,384 x 2,048 with 64 places 64 us (4.3
// TB/s of the bytes that it cannot do without; a large copy 5.05), 57 with 4.
// 50,001 x 121 with 16 places 21 us (11 the bytes): the list's exponentials in
// doubles, its reads after each other (index, logit) and the final sum's launch
// of 2.5.  64 x 131,071 with 256 places 30 us (13): three passes for two, three
// launches.  256 x 7 6.2 us, one launch.
#include <cmath>

#include "abi.hpp"
#include "team.hpp"

using namespace gnnprop;

namespace {

struct Part {   // of a row that several blocks share: its entries not named
  double sum;   // of exp((z - top) / T)
  float top;
  float pad;
};

struct DistillArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  int32_t k;
  const int32_t* index;
  const float *logq, *rest, *weight;
  double T, inv_t, mean;
  float* out;
  float* kl;
  float* dZ;
  int64_t ld_dz;
  double* part;   // losses, one per block (split rows: one per row)
  Part* parts;    // split rows: per_row for each row
  int32_t per_row;
  int64_t blocks, block0;  // of all launches, and in the launches before
};

// ln(x), x > 0, to a few 2^-53: k ln 2 + 2 atanh((m - 1) / (m + 1)) for
// 0.7 < m < 1.42 (the first term left out is below 1e-16).
__device__ __forceinline__ double log_of(double x) {
  if (!(x < INFINITY)) return x;
  int k;
  double m = frexp(x, &k);
  if (m < 0.7071067811865476) {
    m *= 2.0;
    --k;
  }
  const double s = (m - 1.0) / (m + 1.0), s2 = s * s;
  double sum = 1.0 / 21.0;
#pragma unroll
  for (int i = 19; i >= 1; i -= 2) sum = fma(sum, s2, 1.0 / i);
  return fma((double)k, 0.6931471805599453, 2.0 * s * sum);
}

// The teacher's list of one row.
struct Named {
  const int32_t* index;
  const float* logq;
  int32_t k, C;
  bool repeats;  // whether an index may be there twice: its first place counts

  __device__ __forceinline__ int32_t at(int32_t j) const {
    const int32_t c = index[j];
    if ((c < 0) | (c >= C)) return -1;
    if (repeats)
      for (int32_t i = 0; i < j; ++i)
        if (index[i] == c) return -1;
    return c;
  }
};

// What a row's loss and gradient are made of.
struct Scalars {
  bool live;       // whether the row takes part
  double kl;
  double scale_q, scale_p;  // q and p from exponentials relative to the largest
  float others;    // the factor of the other entries' exponentials
};

// A lane's places of the list: E of them in registers, or (E = 0) any number,
// read and computed again in each pass.
template <class T, int E>
struct Places {
  static constexpr int MOST = E > 0 ? E : 1;
  const Named& named;
  const float* row;
  int32_t t, k;
  int32_t col[MOST];
  float lq[MOST], z[MOST];
  double q[MOST], p[MOST];

  __device__ __forceinline__ Places(const Named& n, const float* r, int32_t lane)
      : named(n), row(r), t(lane), k(n.k) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int32_t j = t + e * T::LANES;
      col[e] = j < k ? named.at(j) : -1;
      lq[e] = j < k ? named.logq[j] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = col[e] >= 0 ? row[col[e]] : 0.f;
  }
  // f(column, logq, z, q, p) for the places that are used
  template <class F>
  __device__ __forceinline__ void each(F f) {
    if constexpr (E > 0) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (col[e] >= 0) f(col[e], lq[e], z[e], q[e], p[e]);
    } else {
#pragma unroll 1
      for (int32_t j = t; j < k; j += T::LANES) {
        const int32_t c = named.at(j);
        if (c < 0) continue;
        double q0 = 0.0, p0 = 0.0;
        f(c, named.logq[j], row[c], q0, p0);
      }
    }
  }
};

// From the sums over the entries not named: `high` their largest, `sum` of
// exp((z - high) / T); and the gradient's values at the named ones in columns
// [from, end) (to NULL: none; `ready` is called before the first).
template <class T, int E, class F>
__device__ __forceinline__ Scalars row_scalars(const DistillArgs& a, const T& team,
                                               const Named& named, const float* row, float rest,
                                               float high, double sum, double w, float* to,
                                               int32_t from, int32_t end, F ready) {
  Places<T, E> places(named, row, team.t);
  float most = -INFINITY, top = high;
  // (lanes with a place that is used, with a logq that is a NaN, with such a logit:
  // the largest values do not tell of them)
  constexpr int32_t BAD_Q = 1 << 10, BAD_Z = 1 << 20;
  static_assert(T::LANES < BAD_Q, "each count stays below the next");
  int32_t used = 0;
  places.each([&](int32_t, float lq, float z, double&, double&) INLINE {
    used |= 1 | (lq != lq ? BAD_Q : 0) | (z != z ? BAD_Z : 0);
    most = fmaxf(most, lq);
    top = fmaxf(top, z);
  });
  float low = -most;  // (the largest of both in one exchange)
  team.range(&top, &low, &used);
  most = -low;
  rest = rest > 0.f ? rest : rest == rest ? 0.f : rest;
  if (rest > 0.f) most = fmaxf(most, (float)log_quick(rest));
  const bool says = (used % BAD_Z >= BAD_Q) | (most > -INFINITY);
  const bool nan = (used >= BAD_Z) | (sum != sum);
  Scalars s = {};
  s.live = (used > 0) & says & (nan | (top > -INFINITY));
  if (!s.live) {
    ready(s);
    return s;
  }
  double nq = 0.0, np = 0.0, cross = 0.0;
  places.each([&](int32_t, float logq, float z, double& q, double& p) INLINE {
    const double lq = (double)logq - most, lp = ((double)z - top) * a.inv_t;
    q = exp_exact(lq);
    p = exp_exact(lp);
    nq += q;
    np += p;
    if (!(q == 0.0)) cross += q * (lq - lp);
  });
  team.sum3(&nq, &np, &cross);
  const double high_p = sum > 0.0 ? ((double)high - top) * a.inv_t : 0.0;
  const double down = sum == 0.0 ? 0.0 : exp_exact(high_p);
  const double r = rest == 0.f ? 0.0 : (double)rest * exp_exact(-(double)most);
  nq += r;
  np += sum * down;
  if (!(r == 0.0))
    cross += r * (sum == 0.0 ? INFINITY : log_of((double)rest / sum) - most - high_p);
  s.kl = a.T * a.T * (cross / nq + log_of(np / nq));
  s.scale_q = 1.0 / nq;
  s.scale_p = 1.0 / np;
  // (without entries of a share the factor is for those of -inf: 0, but for a NaN)
  s.others = sum == 0.0 ? (np == np ? 0.f : NAN)
                        : (float)(a.T * (down * s.scale_p - r * s.scale_q / sum));
  ready(s);
  if (!to) return s;
  places.each([&](int32_t c, float logq, float z, double q, double p) INLINE {
    if ((c < from) | (c >= end)) return;
    if (E == 0) {
      q = exp_exact((double)logq - most);
      p = exp_exact(((double)z - top) * a.inv_t);
    }
    to[c] = (float)(w * a.T * (p * s.scale_p - q * s.scale_q));
  });
  return s;
}

// The same with as many places in registers as the list asks for.
template <class T, class F>
__device__ __forceinline__ Scalars row_scalars(const DistillArgs& a, const T& team,
                                               const Named& named, const float* row, float rest,
                                               float high, double sum, double w, float* to,
                                               int32_t from, int32_t end, F ready) {
  if (T::LANES >= GNN_TOP_MOST || a.k <= T::LANES)
    return row_scalars<T, 1>(a, team, named, row, rest, high, sum, w, to, from, end, ready);
  if (a.k <= 4 * T::LANES)
    return row_scalars<T, 4>(a, team, named, row, rest, high, sum, w, to, from, end, ready);
  return row_scalars<T, 0>(a, team, named, row, rest, high, sum, w, to, from, end, ready);
}

// A part of a row (or the row) in registers with the entries named taken out,
// and the others' largest and sum.
template <class T, class Row>
struct Others {
  Row row;
  float high;
  double sum;
  bool repeats;

  // bits: one for each column that the team holds.
  __device__ __forceinline__ void load(const DistillArgs& a, const T& team, const float* from,
                                       int32_t col0, const int32_t* index, uint32_t* bits) {
    row.load(from, a.C, team.t, col0);
    for (int32_t k = team.t; k < (Row::MOST + 31) / 32; k += T::LANES) bits[k] = 0;
    team.sync();
    bool twice = false;
    for (int32_t j = team.t; j < a.k; j += T::LANES) {
      const int32_t c = index[j];
      if (c < col0 || c >= a.C || c - col0 >= Row::MOST) continue;
      const uint32_t bit = 1u << ((c - col0) & 31);
      twice |= (atomicOr(&bits[(c - col0) >> 5], bit) & bit) != 0;
    }
    repeats = team.any(twice);
    team.sync();
    high = -INFINITY;
#pragma unroll
    for (int k = 0; k < Row::CHUNKS; ++k) {
      const int32_t c = row.column(k) - col0;
      const uint32_t out = bits[c >> 5] >> (c & 31);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (out >> j & 1) row.z[k][j] = -INFINITY;
      high = fmaxf(high, max4(row.z[k]));
    }
    high = team.max(high);
    // (exp as a power of two: what falls below the smallest normal number is 0)
    const float shift = shift_of(high), octaves = (float)(a.inv_t * 1.4426950408889634);
    sum = 0.0;
#pragma unroll
    for (int k = 0; k < Row::CHUNKS; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        row.z[k][j] = __builtin_amdgcn_exp2f((row.z[k][j] - shift) * octaves);
      sum += sum4(row.z[k]);
    }
    sum = team.sum(sum);
  }
  __device__ __forceinline__ void store(float* to, float factor) const {
#pragma unroll
    for (int k = 0; k < Row::CHUNKS; ++k) {
      f4 g = row.z[k] * factor;
      if (factor == 0.f) g = {0.f, 0.f, 0.f, 0.f};
      store_cols(to, row.column(k), row.C, g);
    }
  }
};

__device__ __forceinline__ double weight_of(const DistillArgs& a, int32_t i) {
  return a.weight ? (double)a.weight[i] : a.mean;
}

// What all lanes of a team have written to memory is there before what they
// write next.
template <class T>
__device__ __forceinline__ void stores_done(const T& team) {
  if (T::W > 1) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
}

template <int G, int W, class Row>
__global__ __launch_bounds__((threads_of<G, W>())) void distill_kernel(DistillArgs a) {
  using T = Team<G, W, Exchange>;
  constexpr int THREADS = threads_of<G, W>(), R = THREADS / T::LANES;
  __shared__ typename T::Shared s[R];
  __shared__ uint32_t s_bits[R][(Row::MOST + 31) / 32];
  __shared__ double s_loss[THREADS / 64];
  const int own = threadIdx.x / T::LANES;
  const T team(s[own], threadIdx.x % T::LANES);
  const int64_t i = (a.block0 + blockIdx.x) * R + own;
  double loss = 0.0;
  if (i < a.n) {
    const float* from = a.Z + i * a.ld_z;
    Named named = {a.index + i * a.k, a.logq + i * a.k, a.k, a.C, false};
    Others<T, Row> others;
    others.load(a, team, from, 0, named.index, s_bits[own]);
    named.repeats = others.repeats;
    const double w = weight_of(a, (int32_t)i);
    float* to = a.dZ ? a.dZ + i * a.ld_dz : nullptr;
    const Scalars x = row_scalars(
        a, team, named, from, a.rest ? a.rest[i] : 0.f, others.high, others.sum, w,
        w != 0.0 ? to : nullptr, 0, a.C, [&](const Scalars& x) INLINE {
          if (!to) return;
          others.store(to, x.live && w != 0.0 ? (float)(w * x.others) : 0.f);
          stores_done(team);
        });
    if (x.live && w != 0.0) loss = w * x.kl;
    if (a.kl && team.t == 0) a.kl[i] = (float)x.kl;
  }
  // the block's share of the loss, in a fixed order
  if (team.t != 0) loss = 0.0;
  loss = lanes_sum<64>(loss);
  if ((threadIdx.x & 63) == 0) s_loss[threadIdx.x >> 6] = loss;
  __syncthreads();
  if (threadIdx.x) return;
  loss = 0.0;
  for (int k = 0; k < THREADS / 64; ++k) loss += s_loss[k];
  if (a.blocks == 1) a.out[0] = (float)loss;
  else a.part[a.block0 + blockIdx.x] = loss;
}

// Rows past 16,384 columns: a launch for the sums of their parts, one for the
// scalars, which every block of the row forms alike, and the gradient.
using SplitTeam = Team<64, 4, Exchange>;
using SplitRow = Held<64, 4, 4>;
constexpr int32_t SPLIT_COLS = SplitRow::MOST;

__global__ __launch_bounds__(256) void distill_sums_kernel(DistillArgs a) {
  __shared__ SplitTeam::Shared s;
  __shared__ uint32_t s_bits[SPLIT_COLS / 32];
  const SplitTeam team(s, threadIdx.x);
  const int64_t b = a.block0 + blockIdx.x, i = b / a.per_row;
  Others<SplitTeam, SplitRow> others;
  others.load(a, team, a.Z + i * a.ld_z, (int32_t)(b % a.per_row) * SPLIT_COLS, a.index + i * a.k,
              s_bits);
  if (team.t == 0) a.parts[b] = {others.sum, others.high, others.repeats ? 1.f : 0.f};
}

__global__ __launch_bounds__(256) void distill_grad_kernel(DistillArgs a) {
  __shared__ SplitTeam::Shared s;
  __shared__ uint32_t s_bits[SPLIT_COLS / 32];
  const SplitTeam team(s, threadIdx.x);
  const int32_t todo = a.dZ ? a.per_row : 1;
  const int64_t b = a.block0 + blockIdx.x, i = b / todo;
  const int32_t part = (int32_t)(b % todo);
  const float* from = a.Z + i * a.ld_z;
  Named named = {a.index + i * a.k, a.logq + i * a.k, a.k, a.C, false};
  const Part* at = a.parts + i * a.per_row;
  float high = -INFINITY;
  bool repeats = false;
  for (int32_t k = team.t; k < a.per_row; k += 256) {
    high = fmaxf(high, at[k].top);
    repeats |= at[k].pad != 0.f;
  }
  high = team.max(high);
  named.repeats = team.any(repeats);
  double sum = 0.0;
  for (int32_t k = team.t; k < a.per_row; k += 256)
    if (at[k].sum != 0.0) sum += at[k].sum * exp_exact(((double)at[k].top - high) * a.inv_t);
  sum = team.sum(sum);
  const double w = weight_of(a, (int32_t)i);
  const int32_t col0 = part * SPLIT_COLS;
  float* to = a.dZ ? a.dZ + i * a.ld_dz : nullptr;
  const Scalars x = row_scalars(
      a, team, named, from, a.rest ? a.rest[i] : 0.f, high, sum, w, w != 0.0 ? to : nullptr, col0,
      min(col0 + SPLIT_COLS, a.C), [&](const Scalars& x) INLINE {
        if (!to) return;
        Others<SplitTeam, SplitRow> others;
        others.load(a, team, from, col0, named.index, s_bits);
        const float down = others.sum == 0.0
                               ? 0.f : (float)exp_exact(((double)others.high - high) * a.inv_t);
        others.store(to, x.live && w != 0.0 ? (float)(w * x.others) * down : 0.f);
        stores_done(team);
      });
  if (part == 0 && team.t == 0) {
    a.part[i] = x.live && w != 0.0 ? w * x.kl : 0.0;
    if (a.kl) a.kl[i] = (float)x.kl;
  }
}

// out = the sum of `count` terms, in a fixed order.
__global__ __launch_bounds__(1024) void distill_final_kernel(int32_t count,
                                                             const double* __restrict__ part,
                                                             float* __restrict__ out) {
  __shared__ double s[16];
  double x = 0.0;
  for (int32_t k = threadIdx.x; k < count; k += 1024) x += part[k];
  x = lanes_sum<64>(x);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x) return;
  x = 0.0;
  for (int k = 0; k < 16; ++k) x += s[k];
  out[0] = (float)x;
}

struct Launch {
  void (*kernel)(DistillArgs);  // NULL: split rows
  int32_t rows, threads;
};
struct Chosen {
  static constexpr bool SPREAD = false;
  static constexpr int32_t MOST = 16384;
  template <int G, int W, int V>
  Launch held() const {
    constexpr int THREADS = threads_of<G, W>();
    return {distill_kernel<G, W, Held<G, W, V>>, THREADS / (G * W), THREADS};
  }
};
Launch choose(int32_t n, int32_t C, int32_t places) {
  if (C > Chosen::MOST) return {nullptr, 1, 256};
  const Shape s = shape_of(n, C, C < 4 ? 0 : places, 16, Chosen::SPREAD);
  if (s.G > 1) return of_shape(s, Chosen());
  switch (s.V) {
    case 1: return Chosen().held<1, 1, 1>();
    case 2: return Chosen().held<1, 1, 2>();
  }
  return Chosen().held<1, 1, 4>();
}

// [losses | parts' sums]; a loss a row, though most blocks have several rows: fewer
// rows are shared out over more blocks, and what is enough for the most rows has to
// be for fewer.
struct Layout {
  size_t parts, total;
};
Layout layout_of(int32_t n, int32_t C) {
  Layout o;
  o.parts = round_up((size_t)n * sizeof(double), 256);
  o.total = o.parts +
            (C > Chosen::MOST ? (size_t)n * ceil_div(C, SPLIT_COLS) * sizeof(Part) : 0);
  return o;
}

}  // namespace

extern "C" {

size_t gnn_distill_workspace_bytes(int32_t n, int32_t C, int32_t k) {
  if (n < 0 || C <= 0 || C > MOST_COLS || k <= 0 || k > GNN_TOP_MOST) return 0;
  return layout_of(n, C).total;
}

gnn_status gnn_distill_loss(int32_t n, int32_t C, const float* Z, int64_t ld_z, int32_t k,
                            const int32_t* index, const float* logq, const float* rest,
                            const float* weight, double temperature, float* out, float* kl,
                            float* dZ, int64_t ld_dz, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  if (n < 0 || C <= 0 || C > MOST_COLS || ld_z < C || k <= 0 || k > GNN_TOP_MOST ||
      (dZ && ld_dz < C) || !temperature_ok(temperature))
    return GNN_ERR_SHAPE;
  if (!out || (n > 0 && (!Z || !index || !logq))) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const Layout o = layout_of(n, C);
  if (workspace_bytes < o.total || (o.total > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  {
    const size_t rows = (size_t)n * 4, list = rows * k;
    const void* ins[] = {Z, index, logq, rest, weight};
    const size_t inb[] = {mat_bytes(n, C, ld_z), list, list, rows, rows};
    const void* outs[] = {out, kl, dZ, workspace};
    const size_t outb[] = {4, rows, mat_bytes(n, C, ld_dz), o.total};
    for (int i = 0; i < 4; ++i) {
      for (int q = 0; q < 5; ++q)
        if (ranges_overlap(outs[i], outb[i], ins[q], inb[q])) return GNN_ERR_ALIAS;
      for (int q = 0; q < i; ++q)
        if (ranges_overlap(outs[i], outb[i], outs[q], outb[q])) return GNN_ERR_ALIAS;
    }
  }
  const Launch l = choose(n, C, k);
  DistillArgs a = {};
  a.n = n;
  a.C = C;
  a.Z = Z;
  a.ld_z = ld_z;
  a.k = k;
  a.index = index;
  a.logq = logq;
  a.rest = rest;
  a.weight = weight;
  a.T = temperature;
  a.inv_t = 1.0 / temperature;
  a.mean = n > 0 ? 1.0 / n : 0.0;
  a.out = out;
  a.kl = kl;
  a.dZ = dZ;
  a.ld_dz = ld_dz;
  char* ws = static_cast<char*>(workspace);
  a.part = reinterpret_cast<double*>(ws);
  a.parts = reinterpret_cast<Part*>(ws + o.parts);
  a.per_row = (int32_t)ceil_div(C, SPLIT_COLS);
  const auto run = [&](void (*kernel)(DistillArgs), int32_t threads, int64_t blocks) {
    a.blocks = blocks;
    for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
      kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), threads, 0, stream>>>(a);
  };
  timer_begin(GNN_K_LOSS, stream);
  const int64_t parts = ceil_div(n, l.rows);
  if (l.kernel) {
    run(l.kernel, l.threads, parts);
  } else {
    const int64_t blocks = (int64_t)n * a.per_row;
    run(distill_sums_kernel, 256, blocks);
    run(distill_grad_kernel, 256, dZ ? blocks : n);
  }
  if (!l.kernel || parts != 1)
    distill_final_kernel<<<1, 1024, 0, stream>>>((int32_t)parts, a.part, out);
  timer_end(GNN_K_LOSS, (dZ ? 8.0 : 4.0) * n * C, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // extern "C"
