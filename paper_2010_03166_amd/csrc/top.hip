// The top logits of rows, in their order, with their log-probabilities.
//
// A row stays in the registers of its team: its range, the border of the first k
// (bins in LDS above what k groups of lanes hold the largest of), then one pass
// for the exponentials of both parts and the list of the first k, in LDS in the
// place of the bins, where each entry's place is the number of those before it.
// Bound by instructions, some 1,680 a wavefront of 2,048 entries with k = 64:
// 16,384 x 2,048 51 us (the bytes take 28), k = 8 45, k = 256 135, where the
// comparisons of the list's entries with each other are most of it.  2,000 x
// 20,011, k = 128: 74 us in two launches (63 + 16; the bytes 32).
#include "choose.hpp"

using namespace gnnprop;

namespace {

template <int G, int W, class Row>
__global__ __launch_bounds__((threads_of<G, W>())) void top_kernel(TopArgs a) {
  using T = Team<G, W>;
  constexpr int R = threads_of<G, W>() / T::LANES;
  __shared__ typename T::Shared s[R];
  const int own = threadIdx.x / T::LANES;
  const int64_t i = (a.block0 + blockIdx.x) * R + own;
  if (i >= a.n) return;
  const T team(s[own], threadIdx.x % T::LANES);
  // (once the border is known, the list takes the place of what found it)
  static_assert(T::Shared::WORDS >= (Row::MOST < MOST_TOP ? (Row::MOST + 7) / 8 * 8 : MOST_TOP),
                "a row's first entries fit");
  uint64_t* list = s[own].words;
  const float* from = a.Z + i * a.ld_z;
  Row row;
  row.load(from, a.C, team.t);
  float top, low;
  int32_t lanes;
  if (!row_range(team, row, a.group, &top, &low, &lanes)) {
    write_none(a, team, (int32_t)i);
    return;
  }
  const Border b = first_entries(team, row, from, a.C, a.k, top, low, lanes);
  if (team.t == 0) team.s.count = 0;
  team.sync();
  double in, out;
  collect<false>(team, row, b, top, a.inv_t, list, a.k, &in, &out);
  in = team.sum(in);
  out = team.sum(out);
  team.sync();
  write_top(a, team, list, (int32_t)i, top, in, out);
}

// Rows of up to 32 columns, 65,536 of them or more: a lane has one to itself, and
// an entry's place is the number of those before it.  200,000 x 16, k = 8: 63 us
// by teams, 19 so; 200,000 x 32, k = 8: 74 and 28.
template <int V>
__global__ __launch_bounds__(256) void top_small_kernel(TopArgs a) {
  constexpr int N = 4 * V;
  const int64_t i = (a.block0 + blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.n) return;
  Held<1, 1, V> row;
  row.load(a.Z + i * a.ld_z, a.C, 0);
  int32_t* index = a.index + i * a.k;
  float* logq = a.logq + i * a.k;
  float z[N], top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    z[j] = row.z[j / 4][j % 4];
    top = fmaxf(top, z[j]);
    bad |= z[j] != z[j];
  }
  const bool none = bad || !(fabsf(top) < INFINITY);
  int32_t rank[N];
#pragma unroll
  for (int j = 0; j < N; ++j) rank[j] = 0;
#pragma unroll
  for (int j = 1; j < N; ++j)
#pragma unroll
    for (int q = 0; q < j; ++q) {
      const bool first = z[q] >= z[j];
      rank[j] += first;
      rank[q] += !first;
    }
  const float octaves = (float)(a.inv_t * 1.4426950408889634);
  double in = 0.0, out = 0.0;
  int32_t m = 0;  // places that are used
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float more = 0.f, less = 0.f;
#pragma unroll
    for (int j = 4 * k; j < 4 * k + 4; ++j) {
      const float e = __builtin_amdgcn_exp2f((z[j] - top) * octaves);
      const bool kept = rank[j] < a.k;
      more += kept ? e : 0.f;
      less += kept ? 0.f : e;
      m += kept & (z[j] > -INFINITY);
    }
    in += more;
    out += less;
  }
  if (none) m = 0;
  for (int32_t j = m; j < a.k; ++j) {
    index[j] = -1;
    logq[j] = -INFINITY;
  }
  if (a.rest) a.rest[i] = none ? 0.f : (float)(out / (in + out));
  if (none) return;
  const double lse = log_quick((float)(in + out));
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (rank[j] < m) {
      index[rank[j]] = j;
      logq[rank[j]] = (float)(((double)z[j] - top) * a.inv_t - lse);
    }
}

struct TopKernel {
  static constexpr int32_t SMALL = 32, MOST = LONG_TOP;
  template <int G, int W, class Row>
  static constexpr auto of() { return top_kernel<G, W, Row>; }
  template <int V>
  static constexpr auto small() { return top_small_kernel<V>; }
};

}  // namespace

extern "C" {

size_t gnn_top_workspace_bytes(int32_t n, int32_t C, int32_t k) {
  if (n < 0 || C <= 0 || C > MOST_COLS || k <= 0 || k > MOST_TOP || C <= LONG_TOP) return 0;
  return top_long_bytes(n, C, k);
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
  timer_begin(GNN_K_SAMPLE, stream);
  hipError_t e;
  if (C > LONG_TOP) {
    e = top_long(a, workspace, stream);
  } else {
    const Launch<TopArgs> l = choose<TopArgs, TopKernel>(n, C, k);
    a.group = group_of(l.lanes(), C, k);
    e = run(l, a, stream);
  }
  timer_end(GNN_K_SAMPLE, 4.0 * n * C, stream);
  GNN_HIP(e);
  return GNN_OK;
}

}  // extern "C"
