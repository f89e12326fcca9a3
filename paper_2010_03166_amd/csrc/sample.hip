// Actions drawn from rows of logits (temperature, top-k, top-p, min-p) by given
// random numbers.
//
// A row is read once into the registers of its team (shape_of() in team.hpp), and
// every pass goes over them: its range, the border of the first top_k, weights
// into bins and top_p's border, the kept sum with the draw.  Formed once and
// kept, the weights took 64 registers beside a row's 32 and spilled (16,384 x
// 2,048 with top-p 303 us); formed again they cost 16 instructions each.  (1,024
// threads with eight chunks, past 24,576 columns, have 22 registers on the stack.)
//
// Bound by instructions where the rows are many: 16,384 x 2,048 with top-p takes
// 100 us, 3,190 vector instructions a wavefront of 2,048 entries, and the vector
// units issue in nine of ten cycles (the bytes take 27 us); without a border 52,
// the best action alone (T = 0) 31.
// 50,001 x 121 with top-k, top-p, min-p 39 us (the bytes 5): LDS where the first
// 20 are compared.  Where they are few, by one row's latency beside the launch:
// 8,000 x 41 6.7 us, 1 x 2,048 6.8.
#include "choose.hpp"

using namespace gnnprop;

namespace {

// Whether a row's first top_k entries are few enough to be compared with each
// other (each lane its share of them with all, twice) rather than weighed in the
// row (two passes over V chunks).  Measured, us so and so, top-p 0.95 after it:
//   200,000 x 121 (8 lanes, V = 4)  first 5: 68 and 120, 20: 131 and 129, 22: 139 and 129
//   16,384 x 2,048 (64 lanes, 8)    20: 72 and 115, 50: 94 and 120, 90: 183 and 129
//   4,000 x 8,192 (256 lanes, 8)    50: 91 and 114, 150: 158 and 120
template <class T, class Row>
__device__ __forceinline__ bool few_kept(int32_t top_k) {
  const int32_t compared = (top_k + T::LANES - 1) / T::LANES * top_k;
  return top_k <= T::Shared::WORDS / 2 && compared <= (T::W > 1 ? 10 : 15) * Row::CHUNKS;
}
// The draw from the entries up to a border, as a list in the place of what found
// it: what comes before an entry, in the row's order and by columns, is summed
// over the list.
template <class T, class Row>
__device__ __forceinline__ void sample_few(const SampleArgs& a, const T& team, const Row& row,
                                           const Weights& weight, int32_t i, double lse) {
  uint64_t* const list = team.s.words;
  uint64_t* const w = list + T::Shared::WORDS / 2;
  if (team.t == 0) team.s.count = 0;
  team.sync();
  row.each4([&](int32_t col, f4 z) INLINE {
    bool in[4], any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      any |= in[j] = within(weight.kept, z[j], col + j) && z[j] > -INFINITY;
    if (!any) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int32_t at = in[j] ? atomicAdd(&team.s.count, 1) : a.top_k;
      if (at < a.top_k) list[at] = place(z[j], col + j);
    }
  });
  team.sync();
  const int32_t m = min(team.s.count, a.top_k);
  uint64_t sum = 0;
  for (int32_t e = team.t; e < m; e += T::LANES) sum += w[e] = weight.all(logit_of(list[e]));
  if (a.top_p < 1.0) {
    const uint64_t all = team.sum(sum);
    team.sync();
    uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
    P = P < 1 ? 1 : P < all ? P : all;
    uint32_t out = 0, bit = 1;  // (at most 16 of a lane)
    for (int32_t e = team.t; e < m; e += T::LANES, bit *= 2) {
      const uint64_t own = list[e];
      uint64_t before = 0;
#pragma unroll 4
      for (int32_t j = 0; j < m; ++j) before += list[j] < own ? w[j] : 0;
      if (before >= P) out |= bit;
    }
    team.sync();
    for (int32_t e = team.t; e < m; e += T::LANES, out /= 2)
      if (out & 1) w[e] = 0;
  }
  sum = 0;
  for (int32_t e = team.t; e < m; e += T::LANES) {
    if ((double)logit_of(list[e]) - weight.top < a.cut) w[e] = 0;
    sum += w[e];
  }
  sum = team.sum(sum);
  team.sync();
  const uint64_t target = __umul64hi(sum, unit_fraction(a.u[i]));
  for (int32_t e = team.t; e < m; e += T::LANES) {
    const uint64_t own = w[e];
    const uint32_t col = (uint32_t)list[e];
    uint64_t with = 0;
#pragma unroll 4
    for (int32_t j = 0; j < m; ++j) with += (uint32_t)list[j] <= col ? w[j] : 0;
    if (target >= with || target < with - own) continue;
    a.action[i] = (int32_t)col;
    if (a.logp) a.logp[i] = (float)((double)logit_of(list[e]) - weight.top - lse);
  }
}

template <class T, class Row>
__device__ __forceinline__ void sample_row(const SampleArgs& a, const T& team, int32_t i,
                                           const double* table) {
  const float* from = a.Z + (int64_t)i * a.ld_z;
  Row row;
  row.load(from, a.C, team.t);
  float top, low;
  int32_t lanes;
  if (!row_range(team, row, a.group, &top, &low, &lanes)) {
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
  Weights weight = {Exponential(table, a.scale), top, NO_BORDER};
  if (a.top_k) {
    weight.kept = first_entries(team, row, from, a.C, a.top_k, top, low, lanes);
    if (few_kept<T, Row>(a.top_k)) {
      sample_few(a, team, row, weight, i, lse);
      return;
    }
  }
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
  // (the lanes' sums by chunks are kept for the draw, but of 1,024 threads, which
  // have no registers for them: 2,000 x 20,011 with top-p 302 us, 205 without)
  constexpr bool KEPT = T::W < 16;
  uint64_t own = 0, sums[KEPT ? Row::CHUNKS : 1];
  int at_chunk = 0;
  row.each4([&](int32_t col, f4 z) INLINE {
    const uint64_t sum = weight.sum4(z, col);
    own += sum;
    if (KEPT) sums[at_chunk++] = sum;
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
  pick_entry<KEPT>(a, team, row, weight, i, target, lse, sums);
}

// The wavefronts that a vector unit has to hold: four of 256 threads' kernels, three
// where a row takes more than four chunks; of 512 and 1,024 threads two and one, which
// leaves the registers to the compiler (eight chunks of 512 threads take 164, one block
// of a CU; held to 128, for two of them, 32 were spilled).
template <int G, int W, class Row>
constexpr int waves_of() {
  return W == 16 ? 1 : W == 8 ? 2 : Row::CHUNKS > 4 ? 3 : 4;
}

template <int G, int W, class Row>
__global__ __launch_bounds__((threads_of<G, W>()), (waves_of<G, W, Row>()))
void sample_kernel(SampleArgs a) {
  using T = Team<G, W>;
  constexpr int R = threads_of<G, W>() / T::LANES;
  __shared__ typename T::Shared s[R];
  __shared__ double s_table[64];
  if (threadIdx.x < 64) s_table[threadIdx.x] = ldexp(TABLE.at[threadIdx.x], a.bits);
  __syncthreads();
  const int own = threadIdx.x / T::LANES;
  const int64_t i = (a.block0 + blockIdx.x) * R + own;
  if (i >= a.n) return;
  const T team(s[own], threadIdx.x % T::LANES);
  sample_row<T, Row>(a, team, (int32_t)i, s_table);
}

// Rows of up to 24 columns, 65,536 of them or more: a lane has one to itself, and
// what comes before an entry is told by comparing it with every other one (no
// bins, nothing but the exponentials' table in LDS).  200,000 x 7 with top-p 21
// us by teams, 7 so; 200,000 x 16 40 and 19; 200,000 x 32 34 and 51.
template <int V>
__global__ __launch_bounds__(256) void sample_small_kernel(SampleArgs a) {
  constexpr int N = 4 * V;
  __shared__ double s_table[64];
  if (threadIdx.x < 64) s_table[threadIdx.x] = ldexp(TABLE.at[threadIdx.x], a.bits);
  __syncthreads();
  const int64_t i = (a.block0 + blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.n) return;
  Held<1, 1, V> row;
  row.load(a.Z + i * a.ld_z, a.C, 0);
  float z[N], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    z[j] = row.z[j / 4][j % 4];
    top = fmaxf(top, z[j]);
    bad |= z[j] != z[j];
  }
  if (bad || !(fabsf(top) < INFINITY)) {
    a.action[i] = -1;
    if (a.logp) a.logp[i] = 0.f;
    return;
  }
  double lse = 0.0;
  if (a.logp) {
#pragma unroll
    for (int k = 0; k < V; ++k) lse += (double)sum4(exp4(row.z[k], top));
    lse = log_quick((float)lse);
  }
  int32_t action = -1;
  if (a.scale == 0.0) {
#pragma unroll
    for (int j = N - 1; j >= 0; --j) action = z[j] == top ? j : action;
  } else {
    const Exponential of(s_table, a.scale);
    uint64_t w[N], all = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      w[j] = of((double)z[j] - top);
      if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (four at a time have registers)
    }
    if (a.top_k) {
      uint32_t kept = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        int32_t before = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) before += q < j ? z[q] >= z[j] : z[q] > z[j];
        kept |= (uint32_t)(before < a.top_k) << j;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = kept >> j & 1 ? w[j] : 0;
    }
    if (a.top_p < 1.0) {
#pragma unroll
      for (int j = 0; j < N; ++j) all += w[j];
      uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
      P = P < 1 ? 1 : P < all ? P : all;
      uint32_t kept = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        uint64_t before = 0;
#pragma unroll
        for (int q = 0; q < N; ++q)
          if (q != j) before += (q < j ? z[q] >= z[j] : z[q] > z[j]) ? w[q] : 0;
        kept |= (uint32_t)(before < P) << j;
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = kept >> j & 1 ? w[j] : 0;
    }
    if (a.cut > -INFINITY) {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = (double)z[j] - top >= a.cut ? w[j] : 0;
    }
    all = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) all += w[j];
    const uint64_t target = __umul64hi(all, unit_fraction(a.u[i]));
    uint64_t sum = all;
#pragma unroll
    for (int j = N - 1; j >= 0; --j) {  // (the first that the target is below of)
      action = target < sum ? j : action;
      sum -= w[j];
    }
  }
  a.action[i] = action;
  if (!a.logp) return;
  float za = z[0];
#pragma unroll
  for (int j = 1; j < N; ++j) za = action == j ? z[j] : za;
  a.logp[i] = (float)((double)za - top - lse);
}

struct SampleKernel {
  static constexpr int32_t SMALL = 24, MOST = LONG_SAMPLE;
  template <int G, int W, class Row>
  static constexpr auto of() { return sample_kernel<G, W, Row>; }
  template <int V>
  static constexpr auto small() { return sample_small_kernel<V>; }
};

}  // namespace

extern "C" {

size_t gnn_sample_workspace_bytes(int32_t n, int32_t C) {
  if (n < 0 || C <= 0 || C > MOST_COLS || C <= LONG_SAMPLE) return 0;
  return sample_long_bytes(n, C);
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
  a.inv_t = C > BY_SUM && temperature > 0.0 ? 1.0 / temperature : 0.0;
  a.top_k = top_k < C ? top_k : 0;
  a.top_p = top_p;
  a.cut = min_p > 0.0 ? temperature * std::log(min_p) : -INFINITY;
  a.unit = temperature == 1.0 && logp && !a.top_k && (top_p < 1.0 || min_p == 0.0)
               ? std::ldexp(1.0, -a.bits) : 0.0;
  a.action = action;
  a.logp = logp;
  timer_begin(GNN_K_SAMPLE, stream);
  hipError_t e;
  if (C > LONG_SAMPLE) {
    e = sample_long(a, workspace, stream);
  } else {
    const Launch<SampleArgs> l = choose<SampleArgs, SampleKernel>(n, C);
    a.group = a.top_k ? group_of(l.lanes(), C, a.top_k) : 1;
    e = run(l, a, stream);
  }
  timer_end(GNN_K_SAMPLE, 4.0 * n * C, stream);
  GNN_HIP(e);
  return GNN_OK;
}

}  // extern "C"
