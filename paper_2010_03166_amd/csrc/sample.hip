// Actions drawn from rows of logits (temperature, top-k, top-p, min-p) by given
// random numbers, and the top logits of rows (the formulas: include/gnnprop.h).
//
// A draw must not depend on the order in which a sum is formed, and what lies
// next to a border (of the kept actions, of the random number) has to fall on
// its own side of it.  So an action's weight exp((z - top) / T) is a whole
// number: in units of 2^-51 of the largest, or more where a row's sum would
// pass 2^62.  Sums of them are exact, and equal logits have equal weights.
#include <cmath>

#include "abi.hpp"
#include "team.hpp"

using namespace gnnprop;

namespace {

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
__constant__ const Table TABLE = make_table();

// Units of a weight: 2^bits of them are the largest one.  At most 2^62 a row,
// and 51 bits leave the product below a double's first bit.
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
  const double* table;
  double scale;
  int bits;
  double c1, c2, c3, c4, one52;

  __device__ __forceinline__ Exponential(const double* t, double s, int b)
      : table(t), scale(s), bits(b) {
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
    const uint32_t hi = (uint32_t)(unit >> 32) + ((uint32_t)((q >> 6) + bits) << 20);
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
  double top_p;
  double cut;   // T ln(min_p), or -inf
  double unit;  // 2^-bits where a sum of weights is that of the log-probabilities, or 0
  int32_t* action;
  float* logp;
  int64_t block0;
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

// One for each logit that is there.
struct Present {
  __device__ __forceinline__ uint64_t operator()(float z, int32_t) const { return z > -INFINITY; }
};

// A row's largest logit, whether it is a finite number and none is a NaN; how
// many lanes hold a logit, and the least of what they hold the largest of.
template <class T, class Row>
__device__ __forceinline__ bool row_range(const T& team, const Row& row, float* top, float* low,
                                          int32_t* lanes) {
  float most = -INFINITY;
  bool bad = false;
  row.each4([&](int32_t, f4 z) INLINE {
    most = fmaxf(most, max4(z));
    bad |= __builtin_isunordered(z.x, z.y) | __builtin_isunordered(z.z, z.w);
  });
  constexpr int32_t BAD = 1 << 16;
  *top = most;
  *low = most > -INFINITY ? most : INFINITY;
  *lanes = (most > -INFINITY) + (bad ? BAD : 0);
  team.range(top, low, lanes);
  return *lanes < BAD && fabsf(*top) < INFINITY;
}

// The border of the first k entries; low and lanes from row_range().
template <class T, class Row>
__device__ __forceinline__ Border first_entries(const T& team, Row& row, const float* from,
                                                int32_t C, int32_t k, float top, float low,
                                                int32_t lanes) {
  if (k > lanes) {  // (else as many entries as lanes are not below `low`)
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
  if (team.select(row, Present(), top, scale, k, &b, &bin, &base)) return b;
  Reread<T::G, T::W> again;
  again.load(from, C, team.t);
  b = team.search(again, Present(), top, scale, bin, k, base);
  row.load(from, C, team.t);
  return b;
}

// The border of the entries with z - top >= cut, in doubles.
__device__ __forceinline__ Border near_entries(float top, double cut) {
  float z = (float)((double)top + cut);
  while ((double)z - top < cut) z = nextafterf(z, INFINITY);
  for (float y = nextafterf(z, -INFINITY); (double)y - top >= cut; y = nextafterf(z, -INFINITY))
    z = y;
  return {z, 0x7fffffff};
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

template <class T, class Row>
__device__ __forceinline__ void sample_row(const SampleArgs& a, const T& team, int32_t i, const double* table) {
  const float* from = a.Z + (int64_t)i * a.ld_z;
  Row row;
  row.load(from, a.C, team.t);
  float top, low;
  int32_t lanes;
  if (!row_range(team, row, &top, &low, &lanes)) {
    if (team.t == 0) {
      a.action[i] = -1;
      if (a.logp) a.logp[i] = 0.f;
    }
    return;
  }
  double lse = 0.0;  // of the logits, from the largest
  if (a.logp && a.unit == 0.0) {
    row.each4([&](int32_t, f4 z) INLINE { lse += (double)sum4(exp4(z, top)); });
    lse = log_quick((float)team.sum(lse));
  }
  if (a.scale == 0.0) {  // the first of the largest: a column's negative fits a float
    float first = -INFINITY;
    row.each([&](float z, int32_t col) INLINE {
      first = fmaxf(first, z == top ? -(float)col : -INFINITY);
    });
    first = team.max(first);
    if (team.t == 0) {
      a.action[i] = (int32_t)-first;
      if (a.logp) a.logp[i] = (float)-lse;
    }
    return;
  }
  Weights weight = {Exponential(table, a.scale, a.bits), top, NO_BORDER};
  if (a.top_k) weight.kept = first_entries(team, row, from, a.C, a.top_k, top, low, lanes);
  if (a.top_p < 1.0) {
    const float scale = (T::Shared::BINS - 1) * a.inv_range;
    uint64_t all = 0;
    team.clear();
    const auto fill = [&](f4 z, const uint64_t (&w)[4]) INLINE {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        all += w[j];
        team.add(T::bin_of(z[j], top, scale), w[j], w[j] != 0);
      }
    };
    if (a.top_k) {
      row.each4([&](int32_t col, f4 z) INLINE {
        uint64_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = weight(z[j], col + j);
        fill(z, w);
      });
    } else {
      row.each4([&](int32_t, f4 z) INLINE {
        uint64_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = weight.all(z[j]);
        fill(z, w);
      });
    }
    all = team.sum(all);
    team.sync();
    if (a.unit > 0.0) lse = log_quick((float)((double)all * a.unit));
    uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
    P = P < 1 ? 1 : P < all ? P : all;
    Border b;
    int32_t bin;
    uint64_t base;
    if (!team.select(row, weight, top, scale, P, &b, &bin, &base)) {
      Reread<T::G, T::W> again;
      again.load(from, a.C, team.t);
      b = team.search(again, weight, top, scale, bin, P, base);
      row.load(from, a.C, team.t);
    }
    weight.kept = b;
  }
  if (a.cut > -INFINITY) weight.kept = earlier(weight.kept, near_entries(top, a.cut));
  // the action that holds the random number's share of the sum
  constexpr int KEPT = Row::CHUNKS > 0 ? Row::CHUNKS : 1;
  uint64_t own = 0, sums[KEPT];
  int at_chunk = 0;
  row.each4([&](int32_t col, f4 z) INLINE {
    const uint64_t sum = weight.sum4(z, col);
    own += sum;
    if (Row::CHUNKS > 0) sums[at_chunk++] = sum;
  });
  own = lanes_sum<T::G>(own);
  uint64_t ahead = 0, all = own;
  if (T::W > 1) {
    if (team.lane == 0) team.s.sums[team.wave] = own;
    team.sync();
    all = 0;
    for (int k = 0; k < T::W; ++k) {
      all += team.s.sums[k];
      if (k < team.wave) ahead += team.s.sums[k];
    }
  }
  if (a.unit > 0.0 && a.top_p == 1.0) lse = log_quick((float)((double)all * a.unit));
  uint64_t target = __umul64hi(all, unit_fraction(a.u[i]));
  if (target < ahead || target >= ahead + own) return;
  target -= ahead;
  // its chunks of the wavefront, one after the other
  bool found = false;
  at_chunk = 0;
  int32_t col = 0;
  f4 z = {};
  row.each4([&](int32_t at, f4 v) INLINE {
    uint64_t sum = 0;
    if (Row::CHUNKS > 0) sum = sums[at_chunk++];
    if (found) return;
    if (Row::CHUNKS == 0) sum = weight.sum4(v, at);
    sum = lanes_sum<T::G>(sum);
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
    a.logp[i] = (float)((double)za - top - lse);
  }
}

// Blocks that share a CU, by the registers that a row takes.
template <int G, int W, class Row>
constexpr int blocks_of() {
  const int waves = W < 16 && Row::CHUNKS > 4 ? 12 : 16;  // of a CU
  return waves * 64 / threads_of<G, W>();
}

template <int G, int W, class Row>
__global__ __launch_bounds__((threads_of<G, W>()), (blocks_of<G, W, Row>())) void sample_kernel(SampleArgs a) {
  using T = Team<G, W>;
  constexpr int R = threads_of<G, W>() / T::LANES;
  __shared__ typename T::Shared s[R];
  __shared__ double s_table[64];
  if (threadIdx.x < 64) s_table[threadIdx.x] = TABLE.at[threadIdx.x];
  __syncthreads();
  const int own = threadIdx.x / T::LANES;
  const int64_t i = (a.block0 + blockIdx.x) * R + own;
  if (i >= a.n) return;
  const T team(s[own], threadIdx.x % T::LANES);
  sample_row<T, Row>(a, team, (int32_t)i, s_table);
}

// ------------------------------------------------------------- top logits

constexpr int32_t MOST_TOP = GNN_TOP_MOST;

struct TopArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  int32_t k;
  double inv_t;
  int32_t* index;
  float *logq, *rest;
  int64_t block0;
};

template <class T, class Row>
__device__ __forceinline__ void top_row(const TopArgs& a, const T& team, uint64_t* list, int32_t i) {
  Row row;
  row.load(a.Z + (int64_t)i * a.ld_z, a.C, team.t);
  int32_t* index = a.index + (int64_t)i * a.k;
  float* logq = a.logq + (int64_t)i * a.k;
  float top, low;
  int32_t lanes;
  if (!row_range(team, row, &top, &low, &lanes)) {
    for (int32_t j = team.t; j < a.k; j += T::LANES) {
      index[j] = -1;
      logq[j] = -INFINITY;
    }
    if (team.t == 0 && a.rest) a.rest[i] = 0.f;
    return;
  }
  const Border b = first_entries(team, row, a.Z + (int64_t)i * a.ld_z, a.C, a.k, top, low,
                                 lanes);
  // the entries kept, and the sums of both parts
  if (team.t == 0) team.s.count = 0;
  team.sync();
  const float octaves = (float)(a.inv_t * 1.4426950408889634);
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
    if (!any) return;
    float more = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!kept[j]) continue;
      more += e[j];
      list[atomicAdd(&team.s.count, 1)] = place(z[j], col + j);
    }
    in += more;
  });
  in = team.sum(in);
  out = team.sum(out);
  team.sync();
  const int32_t m = team.s.count;
  const double lse = log_quick((float)(in + out));
  // each in its place: those before it are counted, eight at a time
  if (team.t < 8 || T::LANES < 8)
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
    const uint32_t key = ~(uint32_t)(own >> 32);
    const float z = __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
    index[rank] = (int32_t)(uint32_t)own;
    logq[rank] = (float)(((double)z - top) * a.inv_t - lse);
  }
  if (team.t == 0 && a.rest) a.rest[i] = (float)(out / (in + out));
}

template <int G, int W, class Row>
__global__ __launch_bounds__((threads_of<G, W>())) void top_kernel(TopArgs a) {
  using T = Team<G, W>;
  constexpr int R = threads_of<G, W>() / T::LANES;
  constexpr int MOST = Row::MOST < MOST_TOP
                           ? (Row::MOST + 7) / 8 * 8 : MOST_TOP;
  __shared__ typename T::Shared s[R];
  __shared__ uint64_t s_list[R][MOST];
  const int own = threadIdx.x / T::LANES;
  const int64_t i = (a.block0 + blockIdx.x) * R + own;
  if (i >= a.n) return;
  const T team(s[own], threadIdx.x % T::LANES);
  top_row<T, Row>(a, team, s_list[own], (int32_t)i);
}

// ---------------------------------------------------------------- launches

template <class Args>
struct Launch {
  void (*kernel)(Args);
  int32_t rows, threads;
};
#define LAUNCH(G, W, ROW)                                                        \
  Launch<Args>{Kernel::template of<G, W, ROW>(), threads_of<G, W>() / (G * W), \
               threads_of<G, W>()}

struct SampleKernel {
  template <int G, int W, class Row>
  static constexpr auto of() { return sample_kernel<G, W, Row>; }
};
struct TopKernel {
  template <int G, int W, class Row>
  static constexpr auto of() { return top_kernel<G, W, Row>; }
};

template <class Args, class Kernel, int G, int W, int V>
Launch<Args> held() {
  using Row = Held<G, W, V>;
  return LAUNCH(G, W, Row);
}

template <class Args, class Kernel, int G>
Launch<Args> few(int32_t v) {
  return v == 3 ? held<Args, Kernel, G, 1, 3>() : held<Args, Kernel, G, 1, 4>();
}

template <class Args, class Kernel>
Launch<Args> choose(int32_t C) {
  const int32_t q = (int32_t)ceil_div(C, 4);
  if (q == 1) return held<Args, Kernel, 1, 1, 1>();
  if (q == 2) return held<Args, Kernel, 1, 1, 2>();
  if (q <= 4) return few<Args, Kernel, 1>(q);
  if (q <= 8) return few<Args, Kernel, 2>((q + 1) / 2);
  if (q <= 16) return few<Args, Kernel, 4>((q + 3) / 4);
  if (q <= 32) return few<Args, Kernel, 8>((q + 7) / 8);
  if (q <= 64) return few<Args, Kernel, 16>((q + 15) / 16);
  if (q <= 128) return few<Args, Kernel, 32>((q + 31) / 32);
  if (q <= 256) return few<Args, Kernel, 64>((q + 63) / 64);
  if (q <= 384) return held<Args, Kernel, 64, 1, 6>();
  if (q <= 512) return held<Args, Kernel, 64, 1, 8>();
  if (q <= 1024) return held<Args, Kernel, 64, 4, 4>();
  if (q <= 2048) return held<Args, Kernel, 64, 4, 8>();
  if (q <= 4096) return held<Args, Kernel, 64, 16, 4>();
  if (q <= 6144) return held<Args, Kernel, 64, 16, 6>();
  if (q <= 8192) return held<Args, Kernel, 64, 16, 8>();
  using Row = Reread<64, 16>;
  return LAUNCH(64, 16, Row);
}

template <class Args>
gnn_status run(const Launch<Args>& l, Args a, int kclass, hipStream_t stream) {
  const int64_t blocks = ceil_div(a.n, l.rows);
  timer_begin(kclass, stream);
  for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
    l.kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), l.threads, 0, stream>>>(a);
  timer_end(kclass, 4.0 * a.n * a.C, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // namespace

extern "C" {

size_t gnn_sample_workspace_bytes(int32_t n, int32_t C) {
  (void)n;
  (void)C;
  return 0;
}

gnn_status gnn_sample_actions(int32_t n, int32_t C, const float* Z, int64_t ld_z, const float* u,
                              double temperature, int32_t top_k, double top_p, double min_p,
                              int32_t* action, float* logp, void* workspace,
                              size_t workspace_bytes, hipStream_t stream) {
  if (n < 0 || C <= 0 || C > MOST_COLS || ld_z < C) return GNN_ERR_SHAPE;
  if (!(temperature == 0.0 || temperature_ok(temperature)) || top_k < 0 ||
      !(top_p > 0.0 && top_p <= 1.0) || !(min_p >= 0.0 && min_p <= 1.0))
    return GNN_ERR_SHAPE;
  if (n == 0) return GNN_OK;
  if (!Z || !action || (!u && temperature > 0.0)) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = gnn_sample_workspace_bytes(n, C);
  if (workspace_bytes < need || (need > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  {
    const size_t rows = (size_t)n * 4;
    const void* ins[] = {Z, u};
    const size_t inb[] = {mat_bytes(n, C, ld_z), rows};
    const void* outs[] = {action, logp, workspace};
    const size_t outb[] = {rows, rows, need};
    for (int i = 0; i < 3; ++i) {
      for (int k = 0; k < 2; ++k)
        if (ranges_overlap(outs[i], outb[i], ins[k], inb[k])) return GNN_ERR_ALIAS;
      for (int k = 0; k < i; ++k)
        if (ranges_overlap(outs[i], outb[i], outs[k], outb[k])) return GNN_ERR_ALIAS;
    }
  }
  SampleArgs a = {};
  a.n = n;
  a.C = C;
  a.Z = Z;
  a.ld_z = ld_z;
  a.u = u;
  a.scale = temperature > 0.0 ? 64.0 / (temperature * 0.6931471805599453) : 0.0;
  a.inv_range = top_p < 1.0 && temperature > 0.0
                    ? (float)(1.0 / (temperature * std::log(C / (1.0 - top_p)))) : 0.f;
  a.bits = bits_of(C);
  a.top_k = top_k < C ? top_k : 0;
  a.top_p = top_p;
  a.cut = min_p > 0.0 ? temperature * std::log(min_p) : -INFINITY;
  a.unit = temperature == 1.0 && logp && !a.top_k && (top_p < 1.0 || min_p == 0.0)
               ? std::ldexp(1.0, -a.bits) : 0.0;
  a.action = action;
  a.logp = logp;
  return run(choose<SampleArgs, SampleKernel>(C), a, GNN_K_SAMPLE, stream);
}

size_t gnn_top_workspace_bytes(int32_t n, int32_t C, int32_t k) {
  (void)n;
  (void)C;
  (void)k;
  return 0;
}

gnn_status gnn_top_logits(int32_t n, int32_t C, const float* Z, int64_t ld_z, int32_t k,
                          double temperature, int32_t* index, float* logq, float* rest,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (n < 0 || C <= 0 || C > MOST_COLS || ld_z < C || k <= 0 || k > MOST_TOP ||
      !temperature_ok(temperature))
    return GNN_ERR_SHAPE;
  if (n == 0) return GNN_OK;
  if (!Z || !index || !logq) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = gnn_top_workspace_bytes(n, C, k);
  if (workspace_bytes < need || (need > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  {
    const void* outs[] = {index, logq, rest, workspace};
    const size_t outb[] = {(size_t)n * k * 4, (size_t)n * k * 4, (size_t)n * 4, need};
    for (int i = 0; i < 4; ++i) {
      if (ranges_overlap(outs[i], outb[i], Z, mat_bytes(n, C, ld_z))) return GNN_ERR_ALIAS;
      for (int q = 0; q < i; ++q)
        if (ranges_overlap(outs[i], outb[i], outs[q], outb[q])) return GNN_ERR_ALIAS;
    }
  }
  TopArgs a = {};
  a.n = n;
  a.C = C;
  a.Z = Z;
  a.ld_z = ld_z;
  a.k = k;
  a.inv_t = 1.0 / temperature;
  a.index = index;
  a.logq = logq;
  a.rest = rest;
  return run(choose<TopArgs, TopKernel>(C), a, GNN_K_SAMPLE, stream);
}

}  // extern "C"
