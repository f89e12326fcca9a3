// Log-probabilities of chosen actions, and the clipped policy loss with a KL
// term and its gradient (the formulas: include/gnnprop.h).
//
// Per row: top = max z, sum = sum exp(z - top), lp = z[a] - top - log sum;
// then the row's loss terms and the slope c = w dl/dlp, and the gradient
// c (1[j = a] - exp(z_j - top) / sum).
#include <cmath>

#include "abi.hpp"

using namespace gnnprop;

namespace {

constexpr int THREADS = 256;

struct Terms {  // a row's share of `out`
  double loss, kl, cut;
};

struct PolicyArgs {
  int32_t n, C;
  const float* Z;
  int64_t ld_z;
  const int32_t* action;
  const float *adv, *old_lp, *ref_lp, *weight;
  double lo, hi, beta;  // clip to [lo, hi]
  float* logp;
  float* dZ;
  int64_t ld_dz;
  Terms* part;
};

// exp(x - top) where top = -inf only if no logit is above it: then 0 (or NaN
// for a NaN), so that the sum is 0 exactly for a row without any action.
__device__ inline float exp_from(float x, float top) {
  return expf(x - (top == -INFINITY ? 0.f : top));
}

// The loss terms of row i and its slope, from its log-probability; `live`:
// the row has an action and at least one logit above -inf.
__device__ inline Terms row_terms(const PolicyArgs& a, int32_t i, bool live, double lp, float* c) {
  Terms t = {0.0, 0.0, 0.0};
  *c = 0.f;
  const double w = a.weight ? (double)a.weight[i] : 1.0 / a.n;
  if (!live || w == 0.0) return t;
  const double A = a.adv[i];
  const double rho = a.old_lp ? exp(lp - (double)a.old_lp[i]) : 1.0;
  const double ra = rho * A, ca = fmin(fmax(rho, a.lo), a.hi) * A;
  const bool cut = ra > ca;  // false for a NaN, which then shows in ra
  double slope = cut ? 0.0 : -ra;
  t.loss = -(cut ? ca : ra);
  t.cut = cut ? w : 0.0;
  if (a.ref_lp) {
    const double d = (double)a.ref_lp[i] - lp, e = exp(d);
    const double kl = d == INFINITY ? d : e - d - 1.0;
    t.kl = w * kl;
    if (a.beta != 0.0) {
      t.loss += a.beta * kl;
      slope += a.beta * (1.0 - e);
    }
  }
  t.loss *= w;
  *c = (float)(w * slope);
  return t;
}

template <typename T, typename F>
__device__ inline T block_reduce(T v, T* s, F op) {
  __syncthreads();
  s[threadIdx.x] = v;
  __syncthreads();
  for (int d = THREADS / 2; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) s[threadIdx.x] = op(s[threadIdx.x], s[threadIdx.x + d]);
    __syncthreads();
  }
  return s[0];
}

// One workgroup per row, three passes over it.
__global__ __launch_bounds__(THREADS) void policy_row_kernel(PolicyArgs a) {
  __shared__ float s_top[THREADS];
  __shared__ double s_sum[THREADS];
  const int32_t i = blockIdx.x;
  const float* z = a.Z + (int64_t)i * a.ld_z;
  const int32_t act = a.action[i];
  const bool chosen = act >= 0 && act < a.C;
  float top = -INFINITY, c = 0.f;
  double sum = 0.0;
  if (chosen) {
    for (int32_t j = threadIdx.x; j < a.C; j += THREADS) top = fmaxf(top, z[j]);
    top = block_reduce(top, s_top, [](float x, float y) { return fmaxf(x, y); });
    for (int32_t j = threadIdx.x; j < a.C; j += THREADS) sum += exp((double)z[j] - (top == -INFINITY ? 0.0 : (double)top));
    sum = block_reduce(sum, s_sum, [](double x, double y) { return x + y; });
  }
  const bool live = chosen && sum != 0.0;
  const double lp = live ? (double)z[act] - top - log(sum) : chosen ? -INFINITY : 0.0;
  if (threadIdx.x == 0 && a.logp) a.logp[i] = (float)lp;
  if (!a.part) return;
  const Terms t = row_terms(a, i, live, lp, &c);
  if (threadIdx.x == 0) a.part[i] = t;
  if (!a.dZ) return;
  float* dz = a.dZ + (int64_t)i * a.ld_dz;
  const float inv = (float)(1.0 / sum);
  for (int32_t j = threadIdx.x; j < a.C; j += THREADS)
    dz[j] = c == 0.f ? 0.f : c * ((j == act ? 1.f : 0.f) - exp_from(z[j], top) * inv);
}

// out = the sums of `count` partial terms, in a fixed order.
__global__ __launch_bounds__(THREADS) void policy_final_kernel(int32_t count,
                                                               const Terms* __restrict__ part,
                                                               float* __restrict__ out) {
  __shared__ double s[THREADS];
  Terms t = {0.0, 0.0, 0.0};
  for (int32_t k = threadIdx.x; k < count; k += THREADS) {
    t.loss += part[k].loss;
    t.kl += part[k].kl;
    t.cut += part[k].cut;
  }
  const auto add = [](double x, double y) { return x + y; };
  const double loss = block_reduce(t.loss, s, add), kl = block_reduce(t.kl, s, add),
               cut = block_reduce(t.cut, s, add);
  if (threadIdx.x == 0) {
    out[0] = (float)loss;
    out[1] = (float)kl;
    out[2] = (float)cut;
  }
}

size_t workspace_need(int32_t n, int32_t C) { return round_up((size_t)n * sizeof(Terms), 256); }

gnn_status launch(const PolicyArgs& a, float* out, hipStream_t stream) {
  timer_begin(GNN_K_LOSS, stream);
  if (a.n > 0) policy_row_kernel<<<a.n, THREADS, 0, stream>>>(a);
  if (out) policy_final_kernel<<<1, THREADS, 0, stream>>>(a.n, a.part, out);
  timer_end(GNN_K_LOSS, (a.dZ ? 8.0 : 4.0) * a.n * a.C, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // namespace

extern "C" {

size_t gnn_policy_workspace_bytes(int32_t n, int32_t C) {
  if (n < 0 || C <= 0) return 0;
  return workspace_need(n, C);
}

gnn_status gnn_action_logp(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, float* logp, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  if (n < 0 || C <= 0 || ld_z < C) return GNN_ERR_SHAPE;
  if (n == 0) return GNN_OK;
  if (!Z || !action || !logp) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = workspace_need(n, C);
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
  return launch(a, nullptr, stream);
}

gnn_status gnn_policy_loss(int32_t n, int32_t C, const float* Z, int64_t ld_z,
                           const int32_t* action, const float* advantage,
                           const float* old_logp, const float* ref_logp,
                           const float* weight, double clip_lo, double clip_hi,
                           double beta, float* out, float* logp, float* dZ,
                           int64_t ld_dz, void* workspace, size_t workspace_bytes,
                           hipStream_t stream) {
  if (n < 0 || C <= 0 || ld_z < C || (dZ && ld_dz < C)) return GNN_ERR_SHAPE;
  // written so that a NaN is refused
  if (!(clip_lo >= 0.0 && clip_lo <= 1.0) || !(clip_hi >= 0.0) ||
      !(beta >= 0.0 && beta < INFINITY))
    return GNN_ERR_SHAPE;
  if (!out) return GNN_ERR_NULL;
  if (n > 0 && (!Z || !action || !advantage || (beta > 0.0 && !ref_logp))) return GNN_ERR_NULL;
  if (!buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = workspace_need(n, C);
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
  a.old_lp = old_logp;
  a.ref_lp = ref_logp;
  a.weight = weight;
  a.lo = 1.0 - clip_lo;
  a.hi = 1.0 + clip_hi;
  a.beta = beta;
  a.logp = logp;
  a.dZ = dZ;
  a.ld_dz = ld_dz;
  a.part = static_cast<Terms*>(workspace);
  return launch(a, out, stream);
}

}  // extern "C"
