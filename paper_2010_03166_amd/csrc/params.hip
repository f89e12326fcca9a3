// The norm of all gradients and the AdamW update of a set of tensors
// (formulas and formats: include/gnnprop.h).
//
// Both are streams over the set: the norm reads 4 bytes a weight, the update
// moves 28 (32-bit moments: W, m, v read and written, G read) or 16 (8-bit
// moments, plus 16 bytes for each block of 256).  The plan in device memory
// lists the set's pieces of PIECE elements, so that one launch, one workgroup
// a piece, covers tensors of any number and size.
#include <cmath>
#include <cstdlib>

#include "abi.hpp"

using namespace gnnprop;

namespace {

constexpr int THREADS = 256;
constexpr int BLOCK = GNN_STATE_BLOCK;  // one wavefront, four elements a lane
constexpr int PIECE = 2048;
constexpr int NORM_BLOCKS = 2048;  // partial sums of the norm

struct PlanHead {
  int64_t pieces;
  int32_t n, state_bits;
};
struct Tensor {
  float* W;
  const float* G;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t count;
  int64_t first;  // blocks of BLOCK elements in the tensors before it
  double decay;
  int32_t vec;    // aligned for 16-byte accesses (8-bit moments: 4-byte)
  int32_t pad;
};
struct Piece {
  int32_t tensor, index;  // elements [index PIECE, (index + 1) PIECE)
};
constexpr size_t HEAD_BYTES = 64;

struct Plan {
  const PlanHead* head;
  const Tensor* tensors;
  const Piece* pieces;
};
__host__ __device__ inline Plan plan_at(const void* p, int32_t n) {
  const char* b = static_cast<const char*>(p);
  return {reinterpret_cast<const PlanHead*>(b), reinterpret_cast<const Tensor*>(b + HEAD_BYTES),
          reinterpret_cast<const Piece*>(b + HEAD_BYTES + n * sizeof(Tensor))};
}

// ------------------------------------------------------------------ plan

constexpr int BATCH = 32;  // tensors whose description one launch carries
struct PlanBatch {
  Tensor t[BATCH];
  int64_t piece0[BATCH];  // pieces before each tensor
  int32_t first, count;
  PlanHead head;
};

// One row of the grid per tensor of the batch.
__global__ __launch_bounds__(THREADS) void plan_kernel(PlanBatch b, void* plan) {
  const int k = blockIdx.y;
  const Plan p = plan_at(plan, b.head.n);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (k == 0) *const_cast<PlanHead*>(p.head) = b.head;
    if (k < b.count) const_cast<Tensor*>(p.tensors)[b.first + k] = b.t[k];
  }
  if (k >= b.count) return;
  Piece* to = const_cast<Piece*>(p.pieces) + b.piece0[k];
  const int64_t pieces = ceil_div(b.t[k].count, PIECE);
  for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < pieces;
       i += (int64_t)gridDim.x * THREADS)
    to[i] = {b.first + k, (int32_t)i};
}

// ------------------------------------------------------------------ norm

template <bool VEC>
__device__ inline float4 load4(const float* p, int64_t i, int64_t count) {
  if (VEC && i + 4 <= count) return *reinterpret_cast<const float4*>(p + i);
  float4 r;
  r.x = i < count ? p[i] : 0.f;
  r.y = i + 1 < count ? p[i + 1] : 0.f;
  r.z = i + 2 < count ? p[i + 2] : 0.f;
  r.w = i + 3 < count ? p[i + 3] : 0.f;
  return r;
}
template <bool VEC>
__device__ inline void store4(float* p, int64_t i, int64_t count, float4 r) {
  if (VEC && i + 4 <= count) {
    *reinterpret_cast<float4*>(p + i) = r;
    return;
  }
  if (i < count) p[i] = r.x;
  if (i + 1 < count) p[i + 1] = r.y;
  if (i + 2 < count) p[i + 2] = r.z;
  if (i + 3 < count) p[i + 3] = r.w;
}

__device__ inline double block_sum(double v) {
  __shared__ double s[THREADS];
  s[threadIdx.x] = v;
  __syncthreads();
  for (int d = THREADS / 2; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) s[threadIdx.x] += s[threadIdx.x + d];
    __syncthreads();
  }
  return s[0];
}

template <bool VEC>
__device__ inline double squares(const Tensor& t, int64_t base) {
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < PIECE / (4 * THREADS); ++k) {
    const float4 g = load4<VEC>(t.G, base + (k * THREADS + threadIdx.x) * 4, t.count);
    sum = fma((double)g.x, (double)g.x, sum);
    sum = fma((double)g.y, (double)g.y, sum);
    sum = fma((double)g.z, (double)g.z, sum);
    sum = fma((double)g.w, (double)g.w, sum);
  }
  return sum;
}

__global__ __launch_bounds__(THREADS) void norm_part_kernel(const void* plan, int32_t n,
                                                            double* __restrict__ part) {
  const Plan p = plan_at(plan, n);
  const int64_t pieces = p.head->pieces;
  double sum = 0.0;
  for (int64_t c = blockIdx.x; c < pieces; c += gridDim.x) {
    const Piece at = p.pieces[c];
    const Tensor& t = p.tensors[at.tensor];
    const int64_t base = (int64_t)at.index * PIECE;
    sum += t.vec ? squares<true>(t, base) : squares<false>(t, base);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(THREADS) void norm_final_kernel(int32_t count,
                                                             const double* __restrict__ part,
                                                             float* __restrict__ norm) {
  double sum = 0.0;
  for (int32_t k = threadIdx.x; k < count; k += THREADS) sum += part[k];
  sum = block_sum(sum);
  if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// ----------------------------------------------------------------- AdamW

struct Coef {
  double lr, b1, omb1, b2, omb2;
  float eps, c1, c2, lrf;
  const float* norm;
  double max_norm;
  uint64_t base;  // output t of the generator started at the seed
};

// The gradients' factor; false: the step is skipped.
__device__ inline bool clip_factor(const Coef& a, double* k) {
  *k = 1.0;
  if (!a.norm) return true;
  const float norm = *a.norm;
  if (!(fabsf(norm) < INFINITY)) return false;
  if ((double)norm > a.max_norm) *k = a.max_norm / (double)norm;
  return true;
}

__device__ inline float updated(float w, float m, float v, float keep, const Coef& a) {
  return keep * w - a.lrf * (m / a.c1) / (sqrtf(v / a.c2) + a.eps);
}

// 8-bit values: MAN bits of mantissa, the exponent of the smallest normal
// EMIN, the largest code TOP of value `most`.
struct FormatM {  // OCP e4m3
  static constexpr int MAN = 3, EMIN = -6, TOP = 126;
  static constexpr double most = 448.0;
};
struct FormatV {  // OCP e5m2
  static constexpr int MAN = 2, EMIN = -14, TOP = 123;
  static constexpr double most = 57344.0;
};

template <class F>
__device__ inline double decode(uint32_t code) {
  const uint32_t mag = code & 127u, ex = mag >> F::MAN;
  const int32_t man = (int32_t)(mag & ((1u << F::MAN) - 1)) + (ex ? 1 << F::MAN : 0);
  const double x = ldexp((double)man, (int)(ex ? ex : 1u) - 1 + F::EMIN - F::MAN);
  return code & 128u ? -x : x;
}

// Code of y >= 0 in units of the scale, rounded up where r / 2^16 reaches
// past the distance to the lower neighbour: with e the exponent of y (at
// least EMIN) neighbours are 2^(e - MAN) apart.
template <class F>
__device__ inline uint32_t encode(double y, uint32_t r) {
  const int e = max((int)((uint64_t)__double_as_longlong(y) >> 52) - 1023, F::EMIN);
  const double k = ldexp(y, F::MAN - e) + ((double)r + 0.5) * (1.0 / 65536.0);
  return min((uint32_t)((e - F::EMIN) << F::MAN) + (uint32_t)k, (uint32_t)F::TOP);
}

// Largest magnitude in the wavefront, ordered by bits: NaN above infinity.
__device__ inline uint64_t wave_max_bits(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = max(x, (uint64_t)__shfl_xor((unsigned long long)x, d, 64));
  return x;
}
__device__ inline uint64_t magnitude(double x) {
  return (uint64_t)__double_as_longlong(x) & 0x7FFFFFFFFFFFFFFFull;
}

// Scale of a block whose largest magnitude is `top`.
template <class F>
__device__ inline float scale_of(uint64_t top) {
  const float s = (float)(__longlong_as_double((long long)top) / F::most);
  return s < 0x1p-126f ? 0x1p-126f : s;
}

template <bool VEC>
__device__ inline uint32_t load_codes(const uint8_t* p, int64_t i, int64_t count) {
  if (VEC && i + 4 <= count) return *reinterpret_cast<const uint32_t*>(p + i);
  uint32_t r = 0;
  for (int k = 0; k < 4; ++k)
    if (i + k < count) r |= (uint32_t)p[i + k] << (8 * k);
  return r;
}
template <bool VEC>
__device__ inline void store_codes(uint8_t* p, int64_t i, int64_t count, uint32_t r) {
  if (VEC && i + 4 <= count) {
    *reinterpret_cast<uint32_t*>(p + i) = r;
    return;
  }
  for (int k = 0; k < 4; ++k)
    if (i + k < count) p[i + k] = (uint8_t)(r >> (8 * k));
}

// Four consecutive elements from i.
template <bool VEC>
__device__ inline void step32(const Tensor& t, int64_t i, float k, float keep, const Coef& a) {
  float *m = static_cast<float*>(t.m), *v = static_cast<float*>(t.v);
  float w4[4], g4[4], m4[4], v4[4];
  *reinterpret_cast<float4*>(w4) = load4<VEC>(t.W, i, t.count);
  *reinterpret_cast<float4*>(g4) = load4<VEC>(t.G, i, t.count);
  *reinterpret_cast<float4*>(m4) = load4<VEC>(m, i, t.count);
  *reinterpret_cast<float4*>(v4) = load4<VEC>(v, i, t.count);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float g = g4[j] * k;
    m4[j] = (float)a.b1 * m4[j] + (float)a.omb1 * g;
    v4[j] = (float)a.b2 * v4[j] + (float)a.omb2 * g * g;
    w4[j] = updated(w4[j], m4[j], v4[j], keep, a);
  }
  store4<VEC>(t.W, i, t.count, *reinterpret_cast<float4*>(w4));
  store4<VEC>(m, i, t.count, *reinterpret_cast<float4*>(m4));
  store4<VEC>(v, i, t.count, *reinterpret_cast<float4*>(v4));
}

// The same with 8-bit moments; the wavefront's 64 lanes hold one block.
template <bool VEC>
__device__ inline void step8(const Tensor& t, int64_t i, double k, float keep, const Coef& a) {
  uint8_t *m = static_cast<uint8_t*>(t.m), *v = static_cast<uint8_t*>(t.v);
  const int64_t block = i / BLOCK;  // the same in all lanes
  float w4[4], g4[4];
  *reinterpret_cast<float4*>(w4) = load4<VEC>(t.W, i, t.count);
  *reinterpret_cast<float4*>(g4) = load4<VEC>(t.G, i, t.count);
  const uint32_t mc = load_codes<VEC>(m, i, t.count), vc = load_codes<VEC>(v, i, t.count);
  const double ms = t.m_scale[block], vs = t.v_scale[block];
  double m4[4], v4[4];
  uint64_t mtop = 0, vtop = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const double g = (double)g4[j] * k;
    m4[j] = a.b1 * (decode<FormatM>(mc >> (8 * j) & 255u) * ms) + a.omb1 * g;
    v4[j] = a.b2 * (decode<FormatV>(vc >> (8 * j) & 255u) * vs) + a.omb2 * g * g;
    mtop = max(mtop, magnitude(m4[j]));
    vtop = max(vtop, magnitude(v4[j]));
    w4[j] = updated(w4[j], (float)m4[j], (float)v4[j], keep, a);
  }
  const float msn = scale_of<FormatM>(wave_max_bits(mtop));
  const float vsn = scale_of<FormatV>(wave_max_bits(vtop));
  uint32_t mo = 0, vo = 0;
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    const uint64_t r = splitmix(a.base, (uint64_t)(t.first * BLOCK + i + j) / 2);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t rr = (uint32_t)(r >> (32 * q));
      const double ym = fabs(m4[j + q]) / (double)msn, yv = v4[j + q] / (double)vsn;
      // a block with a NaN or an infinity: its scale says so
      uint32_t cm = msn < INFINITY ? encode<FormatM>(ym, rr & 0xFFFFu) : 0u;
      uint32_t cv = vsn < INFINITY ? encode<FormatV>(yv, rr >> 16) : 0u;
      if (m4[j + q] < 0.0) cm |= 128u;
      if (yv > 0.0 && cv == 0u) cv = 1u;
      mo |= cm << (8 * (j + q));
      vo |= cv << (8 * (j + q));
    }
  }
  store4<VEC>(t.W, i, t.count, *reinterpret_cast<float4*>(w4));
  store_codes<VEC>(m, i, t.count, mo);
  store_codes<VEC>(v, i, t.count, vo);
  if ((threadIdx.x & 63) == 0) {
    t.m_scale[block] = msn;
    t.v_scale[block] = vsn;
  }
}

template <int BITS>
__global__ __launch_bounds__(THREADS) void adamw_kernel(const void* plan, int32_t n, Coef a) {
  const Plan p = plan_at(plan, n);
  if (blockIdx.x >= p.head->pieces || p.head->state_bits != BITS) return;
  double k;
  if (!clip_factor(a, &k)) return;
  const Piece at = p.pieces[blockIdx.x];
  const Tensor& t = p.tensors[at.tensor];
  const float keep = (float)(1.0 - a.lr * t.decay);
#pragma unroll
  for (int q = 0; q < PIECE / (4 * THREADS); ++q) {
    const int64_t i = (int64_t)at.index * PIECE + (q * THREADS + threadIdx.x) * 4;
    // whole blocks past the end: nothing (uniform in a wavefront)
    if (i / BLOCK * BLOCK >= t.count) break;
    if (BITS == 32) {
      if (t.vec) step32<true>(t, i, (float)k, keep, a);
      else step32<false>(t, i, (float)k, keep, a);
    } else {
      if (t.vec) step8<true>(t, i, k, keep, a);
      else step8<false>(t, i, k, keep, a);
    }
  }
}

// ---------------------------------------------------------------- checks

gnn_status check_params(const gnn_params* s, int64_t* pieces) {
  if (!s) return GNN_ERR_NULL;
  if (s->n < 0) return GNN_ERR_SHAPE;
  if (s->state_bits != 32 && s->state_bits != 8) return GNN_ERR_UNSUPPORTED;
  if (s->n > 0 && !s->p) return GNN_ERR_NULL;
  int64_t sum = 0;
  for (int32_t k = 0; k < s->n; ++k) {
    const gnn_param& q = s->p[k];
    // (so that piece numbers and addresses stay far from overflow)
    if (q.count < 0 || q.count > ((int64_t)1 << 40)) return GNN_ERR_SHAPE;
    if (!(std::fabs(q.weight_decay) < INFINITY)) return GNN_ERR_SHAPE;
    if (q.count > 0 && !q.G) return GNN_ERR_NULL;
    sum += ceil_div(q.count, PIECE);
  }
  if (sum > INT32_MAX) return GNN_ERR_SHAPE;
  *pieces = sum;
  return GNN_OK;
}

size_t plan_need(int32_t n, int64_t pieces) {
  return round_up(HEAD_BYTES + (size_t)n * sizeof(Tensor) + (size_t)pieces * sizeof(Piece), 256);
}

inline bool aligned(const void* p, uintptr_t to) {
  return reinterpret_cast<uintptr_t>(p) % to == 0;
}

struct Range {
  uintptr_t a, b;
  bool written;
};
int by_start(const void* x, const void* y) {
  const Range *p = static_cast<const Range*>(x), *q = static_cast<const Range*>(y);
  return p->a < q->a ? -1 : p->a > q->a;
}

// Whether anything that is written overlaps anything else of the set.
gnn_status check_overlap(const gnn_params* s, const void* plan, size_t plan_bytes) {
  Range* r = static_cast<Range*>(malloc(sizeof(Range) * (6 * (size_t)s->n + 1)));
  if (!r) return GNN_ERR_HIP;
  size_t c = 0;
  const auto add = [&](const void* p, size_t bytes, bool written) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (p && bytes) r[c++] = {a, a + bytes, written};
  };
  add(plan, plan_bytes, true);
  for (int32_t k = 0; k < s->n; ++k) {
    const gnn_param& q = s->p[k];
    const size_t w = (size_t)q.count * 4, st = s->state_bits == 8 ? (size_t)q.count : w;
    add(q.W, w, true);
    add(q.G, w, false);
    add(q.m, st, true);
    add(q.v, st, true);
    if (s->state_bits == 8) {
      add(q.m_scale, (size_t)ceil_div(q.count, BLOCK) * 4, true);
      add(q.v_scale, (size_t)ceil_div(q.count, BLOCK) * 4, true);
    }
  }
  qsort(r, c, sizeof(Range), by_start);
  // ends of what was met so far, anything and written only
  uintptr_t any = 0, written = 0;
  gnn_status st = GNN_OK;
  for (size_t k = 0; k < c && st == GNN_OK; ++k) {
    if (r[k].a < (r[k].written ? any : written)) st = GNN_ERR_ALIAS;
    any = std::max(any, r[k].b);
    if (r[k].written) written = std::max(written, r[k].b);
  }
  free(r);
  return st;
}

}  // namespace

extern "C" {

size_t gnn_params_plan_bytes(const gnn_params* params) {
  int64_t pieces;
  if (check_params(params, &pieces) != GNN_OK) return 0;
  return plan_need(params->n, pieces);
}

gnn_status gnn_params_build_plan(const gnn_params* params, void* plan, size_t plan_bytes,
                                 hipStream_t stream) {
  int64_t pieces;
  gnn_status st = check_params(params, &pieces);
  if (st != GNN_OK) return st;
  if (!plan) return GNN_ERR_NULL;
  if (!buf16(plan)) return GNN_ERR_UNSUPPORTED;
  const size_t need = plan_need(params->n, pieces);
  if (plan_bytes < need) return GNN_ERR_WORKSPACE;
  const uintptr_t state_align = params->state_bits == 8 ? 1 : 4;
  for (int32_t k = 0; k < params->n; ++k) {
    const gnn_param& q = params->p[k];
    if (!aligned(q.W, 4) || !aligned(q.G, 4) || !aligned(q.m, state_align) ||
        !aligned(q.v, state_align) || !aligned(q.m_scale, 4) || !aligned(q.v_scale, 4))
      return GNN_ERR_UNSUPPORTED;
  }
  if ((st = check_overlap(params, plan, need)) != GNN_OK) return st;
  PlanBatch b = {};
  b.head = {pieces, params->n, params->state_bits};
  int64_t piece0 = 0, first = 0;
  int32_t k = 0;
  do {  // an empty set has a plan too
    b.first = k;
    b.count = std::min(params->n - k, BATCH);
    int64_t most = 0;
    for (int32_t j = 0; j < b.count; ++j) {
      const gnn_param& q = params->p[k + j];
      const uintptr_t al = params->state_bits == 8 ? 4 : 16;
      const bool vec = aligned(q.W, 16) && aligned(q.G, 16) && aligned(q.m, al) && aligned(q.v, al);
      b.t[j] = {q.W, q.G, q.m, q.v, q.m_scale, q.v_scale, q.count, first, q.weight_decay, vec, 0};
      b.piece0[j] = piece0;
      piece0 += ceil_div(q.count, PIECE);
      first += ceil_div(q.count, BLOCK);
      most = std::max(most, ceil_div(q.count, PIECE));
    }
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(most, THREADS), 64)),
                    (unsigned)std::max(b.count, 1));
    plan_kernel<<<grid, THREADS, 0, stream>>>(b, plan);
    GNN_HIP(hipGetLastError());
    k += b.count;
  } while (k < params->n);
  return GNN_OK;
}

size_t gnn_grad_norm_workspace_bytes(const gnn_params* params) {
  int64_t pieces;
  if (check_params(params, &pieces) != GNN_OK) return 0;
  return round_up((size_t)std::min<int64_t>(pieces, NORM_BLOCKS) * 8, 256);
}

gnn_status gnn_grad_norm(const gnn_params* params, float* norm, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
  int64_t pieces;
  const gnn_status st = check_params(params, &pieces);
  if (st != GNN_OK) return st;
  if (!norm || !params->plan) return GNN_ERR_NULL;
  if (!buf16(params->plan) || !buf16(workspace)) return GNN_ERR_UNSUPPORTED;
  const size_t need = gnn_grad_norm_workspace_bytes(params);
  if (workspace_bytes < need || (need > 0 && !workspace)) return GNN_ERR_WORKSPACE;
  if (ranges_overlap(norm, 4, workspace, need) ||
      ranges_overlap(norm, 4, params->plan, plan_need(params->n, pieces)) ||
      ranges_overlap(workspace, need, params->plan, plan_need(params->n, pieces)))
    return GNN_ERR_ALIAS;
  double weights = 0;
  for (int32_t k = 0; k < params->n; ++k) {
    const gnn_param& q = params->p[k];
    weights += q.count;
    if (ranges_overlap(norm, 4, q.G, (size_t)q.count * 4) ||
        ranges_overlap(workspace, need, q.G, (size_t)q.count * 4))
      return GNN_ERR_ALIAS;
  }
  double* part = static_cast<double*>(workspace);
  const int32_t blocks = (int32_t)std::min<int64_t>(pieces, NORM_BLOCKS);
  timer_begin(GNN_K_NORM, stream);
  if (blocks > 0)
    norm_part_kernel<<<blocks, THREADS, 0, stream>>>(params->plan, params->n, part);
  norm_final_kernel<<<1, THREADS, 0, stream>>>(blocks, part, norm);
  timer_end(GNN_K_NORM, 4.0 * weights, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

gnn_status gnn_adamw_step(const gnn_params* params, double lr, double beta1, double beta2,
                          double eps, int32_t t, const float* norm, double max_norm,
                          uint64_t seed, hipStream_t stream) {
  int64_t pieces;
  const gnn_status st = check_params(params, &pieces);
  if (st != GNN_OK) return st;
  // written so that a NaN is refused
  if (t < 1 || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
      !(eps >= 0.0 && eps < INFINITY) || !(std::fabs(lr) < INFINITY) || (norm && !(max_norm > 0.0)))
    return GNN_ERR_SHAPE;
  if (!params->plan) return GNN_ERR_NULL;
  if (!buf16(params->plan)) return GNN_ERR_UNSUPPORTED;
  double weights = 0;
  for (int32_t k = 0; k < params->n; ++k) {
    const gnn_param& q = params->p[k];
    if (q.count == 0) continue;
    if (!q.W || !q.m || !q.v || (params->state_bits == 8 && (!q.m_scale || !q.v_scale)))
      return GNN_ERR_NULL;
    weights += q.count;
    const size_t w = (size_t)q.count * 4, s = params->state_bits == 8 ? (size_t)q.count : w;
    if (ranges_overlap(norm, 4, q.W, w) || ranges_overlap(norm, 4, q.m, s) ||
        ranges_overlap(norm, 4, q.v, s))
      return GNN_ERR_ALIAS;
  }
  if (pieces == 0) return GNN_OK;
  const Coef a = {lr, beta1, 1.0 - beta1, beta2, 1.0 - beta2, (float)eps,
                  (float)(1.0 - std::pow(beta1, t)), (float)(1.0 - std::pow(beta2, t)), (float)lr,
                  norm, max_norm, splitmix(seed, (uint64_t)t)};
  timer_begin(GNN_K_UPDATE, stream);
  if (params->state_bits == 32)
    adamw_kernel<32><<<(unsigned)pieces, THREADS, 0, stream>>>(params->plan, params->n, a);
  else
    adamw_kernel<8><<<(unsigned)pieces, THREADS, 0, stream>>>(params->plan, params->n, a);
  timer_end(GNN_K_UPDATE, (params->state_bits == 32 ? 28.0 : 16.0) * weights, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // extern "C"
