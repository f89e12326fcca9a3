// The norm of all gradients and the AdamW update of a set of tensors
// (formulas and formats: include/gnnprop.h).
//
// Both are streams over the set: the norm reads 4 bytes a weight, the update
// moves 28 (32-bit moments: W, m, v read and written, G read) or 16 (8-bit
// moments, plus 16 bytes for each block of 256).  The plan in device memory
// lists the set's pieces of PIECE elements, so that one launch, one workgroup
// a piece, covers tensors of any number and size.  Measured on 120 million
// weights: norm 78 us (6.2 TB/s), update 613 us (5.5 TB/s; a large copy 5.05)
// and with 8-bit moments 360 us (5.4 TB/s); on 1.7 million 7.8 and 8.9 us,
// launches (the norm takes two) and their latency.  Pieces of 2,048: 86, 637
// and 399 us where 1,024 take 82, 630 and 400; blocks of 128 threads 119 us
// for the norm.
#include <cmath>
#include <cstdlib>

#include "abi.hpp"

using namespace gnnprop;

namespace {

constexpr int THREADS = 256;
constexpr int BLOCK = GNN_STATE_BLOCK;  // one wavefront, four elements a lane
constexpr int PIECE = 1024;
constexpr int NORM_BLOCKS = 2048;  // partial sums of the norm
// Pieces of one launch (2^32 threads are the most that a launch can have).
constexpr int64_t LAUNCH_PIECES = 1 << 23;

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

// Four elements at a time from any multiple of 4 bytes (codes: from any byte),
// which global memory instructions of 16 bytes allow: tensors in one flat
// buffer need no padding.  FULL: all four exist.
typedef float f4 __attribute__((ext_vector_type(4)));
typedef f4 f4u __attribute__((aligned(4)));
typedef uint32_t u32u __attribute__((aligned(1)));

// Addresses out of the plan are known to the compiler as device memory only
// where it is told.
#define GLOBAL __attribute__((address_space(1)))
template <class T>
__device__ inline GLOBAL T* global(T* p) {
  return (GLOBAL T*)p;
}

template <bool FULL>
__device__ inline f4 load4(const float* q, int64_t i, int64_t count) {
  const GLOBAL float* p = global(q);
  if (FULL || i + 4 <= count) return *(const GLOBAL f4u*)(p + i);
  f4 r = {0.f, 0.f, 0.f, 0.f};
  if (i < count) r.x = p[i];
  if (i + 1 < count) r.y = p[i + 1];
  if (i + 2 < count) r.z = p[i + 2];
  return r;
}
template <bool FULL>
__device__ inline void store4(float* q, int64_t i, int64_t count, f4 r) {
  GLOBAL float* p = global(q);
  if (FULL || i + 4 <= count) {
    *(GLOBAL f4u*)(p + i) = r;
    return;
  }
  if (i < count) p[i] = r.x;
  if (i + 1 < count) p[i + 1] = r.y;
  if (i + 2 < count) p[i + 2] = r.z;
}
template <bool FULL>
__device__ inline uint32_t load_codes(const uint8_t* q, int64_t i, int64_t count) {
  const GLOBAL uint8_t* p = global(q);
  if (FULL || i + 4 <= count) return *(const GLOBAL u32u*)(p + i);
  uint32_t r = 0;
  if (i < count) r = p[i];
  if (i + 1 < count) r |= (uint32_t)p[i + 1] << 8;
  if (i + 2 < count) r |= (uint32_t)p[i + 2] << 16;
  return r;
}
template <bool FULL>
__device__ inline void store_codes(uint8_t* q, int64_t i, int64_t count, uint32_t r) {
  GLOBAL uint8_t* p = global(q);
  if (FULL || i + 4 <= count) {
    *(GLOBAL u32u*)(p + i) = r;
    return;
  }
  if (i < count) p[i] = (uint8_t)r;
  if (i + 1 < count) p[i + 1] = (uint8_t)(r >> 8);
  if (i + 2 < count) p[i + 2] = (uint8_t)(r >> 16);
}

// The block's sum in all threads, in a fixed order.
__device__ inline double block_sum(double v) {
  __shared__ double s[THREADS / 64];
  v = lanes_sum<64>(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int k = 1; k < THREADS / 64; ++k) v += s[k];
  return v;
}

constexpr int AT_ONCE = PIECE / (4 * THREADS);  // accesses of a thread to a piece

template <bool FULL>
__device__ inline double squares(const Tensor& t, int64_t base) {
  f4 g[AT_ONCE];
#pragma unroll
  for (int k = 0; k < AT_ONCE; ++k)
    g[k] = load4<FULL>(t.G, base + (k * THREADS + threadIdx.x) * 4, t.count);
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fma((double)g[k][j], (double)g[k][j], sum);
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
    sum += base + PIECE <= t.count ? squares<true>(t, base) : squares<false>(t, base);
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
  float eps, step, root;  // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  const float* norm;
  double max_norm;
  uint64_t base;  // output t of the generator started at the seed
};

// The gradients' factor from their norm (without one: 0, and no limit to it).
__device__ inline double clip_factor(const Coef& a, float norm) {
  return (double)norm > a.max_norm ? a.max_norm / (double)norm : 1.0;
}

// The bias corrections are in the coefficients, the quotient is a product
// with a reciprocal good to 1 ulp, and the root the hardware's of doubles
// (good to 2^-25, and over the whole range of v), rounded.
__device__ inline float updated(float w, float m, double v, float keep, const Coef& a) {
  const float root = (float)__builtin_amdgcn_sqrt(v);
  return keep * w - a.step * m * __builtin_amdgcn_rcpf(root * a.root + a.eps);
}

// 8-bit values: MAN bits of mantissa, the exponent of the smallest normal
// EMIN, the largest value `most`.
struct FormatM {  // OCP e4m3
  static constexpr int MAN = 3, EMIN = -6;
  static constexpr double most = 448.0;
};
struct FormatV {  // OCP e5m2
  static constexpr int MAN = 2, EMIN = -14;
  static constexpr double most = 57344.0;
};

__device__ inline uint32_t high_word(double x) {
  return (uint32_t)((uint64_t)__double_as_longlong(x) >> 32);
}

// Code of |y|, y in units of the scale, rounded up where (r + 1/2) / 2^16
// reaches past the distance to the lower neighbour, with y's sign above it.
// y is multiplied so that the format's smallest normal comes to lie at the
// doubles' own: exponent and mantissa, read as one number, then count
// neighbours below it as above, MAN + 11 bits in, one step of the code.  The
// 16 bits of r and the half after them end above bit 32, so the upper word
// decides alone.  |y| is at most the format's largest value and 2^-24 of it,
// 2^-20 of a step: no r rounds that up.
template <class F>
__device__ inline uint32_t encode(double y, uint32_t r) {
  constexpr int SH = 20 - F::MAN;  // bits of the upper word after the code's
  const uint32_t hi = high_word(y * __builtin_ldexp(1.0, -1022 - F::EMIN));
  return ((hi & 0x7FFFFFFFu) + ((2 * r + 1) << (SH - 17))) >> SH | (hi >> 24 & 128u);
}

// A block's scale and its reciprocal (NaN, 0 where it has a NaN or an
// infinity).  `top`: the lane's largest magnitude; the wavefront's is found
// among their roundings to fp32, then read from its lane (all of those that
// round alike): six steps of 32 bits instead of 64.  `top` is no NaN.
template <class F>
__device__ inline float block_scale(double top, bool bad, double* inverse) {
  const float mine = (float)top;
  const float most = lanes_max<64>(mine);
  // doubles >= 0 are ordered as their bits; each turn finds a larger one, so
  // lanes that are all alike take one turn
  const uint64_t own = (uint64_t)__double_as_longlong(top);
  uint64_t bits = 0;
  for (uint64_t lanes = __ballot(mine == most && own > bits); lanes;
       lanes = __ballot(mine == most && own > bits)) {
    const int lane = __ffsll((unsigned long long)lanes) - 1;
    bits = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(own >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)own, lane);
  }
  const double scaled = __longlong_as_double((long long)bits) * (1.0 / F::most);
  float s = (float)scaled;
  if (s < 0x1p-126f) s = 0x1p-126f;
  if (bad || !(s < INFINITY)) {
    *inverse = 0.0;
    return NAN;
  }
  const double x = __builtin_amdgcn_rcp((double)s);
  const double x1 = fma(fma(-(double)s, x, 1.0), x, x);
  *inverse = fma(fma(-(double)s, x1, 1.0), x1, x1);
  return s;
}

struct Raw32 {
  f4 w, g, m, v;
};
struct Raw8 {
  f4 w, g;
  uint32_t m, v;
  float ms, vs;
};

// A thread's accesses to a piece are all under way before the first is used.
template <bool FULL>
__device__ inline void piece32(const Tensor& t, int64_t base, float norm, const Coef& a) {
  float *m = static_cast<float*>(t.m), *v = static_cast<float*>(t.v);
  Raw32 x[AT_ONCE];
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int64_t i = base + (q * THREADS + threadIdx.x) * 4;
    x[q] = {load4<FULL>(t.W, i, t.count), load4<FULL>(t.G, i, t.count),
            load4<FULL>(m, i, t.count), load4<FULL>(v, i, t.count)};
  }
  if (!(fabsf(norm) < INFINITY)) return;  // (asked here, when the reads are under way)
  const float keep = (float)(1.0 - a.lr * t.decay);
  const double k = clip_factor(a, norm);  // (1e-42, say, has 10 bits in fp32)
  const float b1 = (float)a.b1, omb1 = (float)a.omb1;
  const float b2 = (float)a.b2, omb2 = (float)a.omb2;
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int64_t i = base + (q * THREADS + threadIdx.x) * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float g = (float)((double)x[q].g[j] * k);
      x[q].m[j] = b1 * x[q].m[j] + omb1 * g;
      x[q].v[j] = b2 * x[q].v[j] + omb2 * g * g;
      x[q].w[j] = updated(x[q].w[j], x[q].m[j], (double)x[q].v[j], keep, a);
    }
    store4<FULL>(t.W, i, t.count, x[q].w);
    store4<FULL>(m, i, t.count, x[q].m);
    store4<FULL>(v, i, t.count, x[q].v);
  }
}

// 8-bit moments: the 64 lanes of a wavefront hold one block of 256, so that a
// scale is a reduction within the wavefront.  Instructions bound this path
// until they are few: about 90 a weight, 15 of them of doubles (as fast here
// as fp32 ones); with library roots, quotients and ldexp 210, and 666 us in
// the place of 360.  Small sets are bound by latency: a block's reads follow
// two reads of the plan, the piece's and then its tensor's (0.9 million
// weights, a single round of blocks: 6.2 us, their bytes 2.8).
template <bool FULL>
__device__ inline void piece8(const Tensor& t, int64_t base, float norm, const Coef& a) {
  uint8_t *m = static_cast<uint8_t*>(t.m), *v = static_cast<uint8_t*>(t.v);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Raw8 x[AT_ONCE];
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int64_t first = base + (q * (THREADS / 64) + wave) * BLOCK, i = first + lane * 4;
    if (!FULL && first >= t.count) break;
    x[q] = {load4<FULL>(t.W, i, t.count), load4<FULL>(t.G, i, t.count),
            load_codes<FULL>(m, i, t.count), load_codes<FULL>(v, i, t.count),
            global(t.m_scale)[first / BLOCK], global(t.v_scale)[first / BLOCK]};
  }
  if (!(fabsf(norm) < INFINITY)) return;
  const float keep = (float)(1.0 - a.lr * t.decay);
  const double k = clip_factor(a, norm);
  const double gm = a.omb1 * k, gv = a.omb2 * k * k;
  const uint64_t lane_state = (uint64_t)lane * (2 * GOLDEN);  // two draws a lane
#pragma unroll
  for (int q = 0; q < AT_ONCE; ++q) {
    const int64_t first = base + (q * (THREADS / 64) + wave) * BLOCK, i = first + lane * 4;
    if (!FULL && first >= t.count) break;
    const double ms = a.b1 * (double)x[q].ms, vs = a.b2 * (double)x[q].vs;
    const float mo[4] = {__builtin_amdgcn_cvt_f32_fp8(x[q].m, 0),
                         __builtin_amdgcn_cvt_f32_fp8(x[q].m, 1),
                         __builtin_amdgcn_cvt_f32_fp8(x[q].m, 2),
                         __builtin_amdgcn_cvt_f32_fp8(x[q].m, 3)};
    const float vo[4] = {__builtin_amdgcn_cvt_f32_bf8(x[q].v, 0),
                         __builtin_amdgcn_cvt_f32_bf8(x[q].v, 1),
                         __builtin_amdgcn_cvt_f32_bf8(x[q].v, 2),
                         __builtin_amdgcn_cvt_f32_bf8(x[q].v, 3)};
    double m4[4], v4[4], mtop = 0.0, vtop = 0.0;
    uint32_t gtop = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double g = (double)x[q].g[j];
      m4[j] = fma((double)mo[j], ms, g * gm);
      v4[j] = fma((double)vo[j], vs, g * gv * g);
      mtop = fmax(mtop, fabs(m4[j]));
      vtop = fmax(vtop, v4[j]);
      gtop = max(gtop, __float_as_uint(x[q].g[j]) & 0x7FFFFFFFu);
      x[q].w[j] = updated(x[q].w[j], (float)m4[j], v4[j], keep, a);
    }
    store4<FULL>(t.W, i, t.count, x[q].w);
    // a NaN or an infinity: the scales say so
    const bool bad = __ballot(gtop >= 0x7F800000u) != 0;
    double im, iv;
    const float msn = block_scale<FormatM>(mtop, bad || !(x[q].ms < INFINITY), &im);
    const float vsn = block_scale<FormatV>(vtop, bad || !(x[q].vs < INFINITY), &iv);
    uint32_t mc = 0, vc = 0;
    const uint64_t state = a.base + (uint64_t)(t.first * BLOCK + first + 2) / 2 * GOLDEN + lane_state;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t both = mix64(state + j / 2 * GOLDEN);
      const uint32_t r = (uint32_t)(both >> (32 * (j & 1)));
      const uint32_t cm = encode<FormatM>(m4[j] * im, r & 0xFFFFu);
      // a second moment above 0 (its upper word is, too) is not stored as 0
      const uint32_t cv = max(encode<FormatV>(v4[j] * iv, r >> 16),
                              min(high_word(v4[j]), 1u));
      mc |= cm << (8 * j);
      vc |= cv << (8 * j);
    }
    store_codes<FULL>(m, i, t.count, mc);
    store_codes<FULL>(v, i, t.count, vc);
    if (lane == 0) {
      global(t.m_scale)[first / BLOCK] = msn;
      global(t.v_scale)[first / BLOCK] = vsn;
    }
  }
}

template <int BITS>
__global__ __launch_bounds__(THREADS) void adamw_kernel(const void* plan, int32_t n,
                                                        int64_t piece0, Coef a) {
  const Plan p = plan_at(plan, n);
  const int64_t piece = piece0 + blockIdx.x;
  // three reads that do not wait for each other
  const PlanHead head = *p.head;
  const Piece at = p.pieces[piece];
  const float norm = a.norm ? *a.norm : 0.f;
  if (piece >= head.pieces || head.state_bits != BITS) return;
  const Tensor t = p.tensors[at.tensor];
  // (a plan for the norm alone has no weights)
  if (!t.W || !t.m || !t.v || (BITS == 8 && (!t.m_scale || !t.v_scale))) return;
  const int64_t base = (int64_t)at.index * PIECE;
  const bool full = base + PIECE <= t.count;
  if (BITS == 32) {
    if (full) piece32<true>(t, base, norm, a);
    else piece32<false>(t, base, norm, a);
  } else {
    if (full) piece8<true>(t, base, norm, a);
    else piece8<false>(t, base, norm, a);
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

int32_t norm_blocks(int64_t pieces) {
  return (int32_t)std::min<int64_t>(ceil_div(pieces, 2), NORM_BLOCKS);
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
      b.t[j] = {q.W, q.G, q.m, q.v, q.m_scale, q.v_scale, q.count, first, q.weight_decay};
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
  return round_up((size_t)norm_blocks(pieces) * 8, 256);
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
  const int32_t blocks = norm_blocks(pieces);
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
    const size_t sc = params->state_bits == 8 ? (size_t)ceil_div(q.count, BLOCK) * 4 : 0;
    if (ranges_overlap(norm, 4, q.W, w) || ranges_overlap(norm, 4, q.m, s) ||
        ranges_overlap(norm, 4, q.v, s) || ranges_overlap(norm, 4, q.m_scale, sc) ||
        ranges_overlap(norm, 4, q.v_scale, sc))
      return GNN_ERR_ALIAS;
  }
  if (pieces == 0) return GNN_OK;
  const Coef a = {lr, beta1, 1.0 - beta1, beta2, 1.0 - beta2, (float)eps,
                  (float)(lr / (1.0 - std::pow(beta1, t))),
                  (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, t))), norm,
                  norm ? max_norm : INFINITY, splitmix(seed, (uint64_t)t)};
  timer_begin(GNN_K_UPDATE, stream);
  for (int64_t p0 = 0; p0 < pieces; p0 += LAUNCH_PIECES) {
    const unsigned blocks = (unsigned)std::min(pieces - p0, LAUNCH_PIECES);
    if (params->state_bits == 32)
      adamw_kernel<32><<<blocks, THREADS, 0, stream>>>(params->plan, params->n, p0, a);
    else
      adamw_kernel<8><<<blocks, THREADS, 0, stream>>>(params->plan, params->n, p0, a);
  }
  timer_end(GNN_K_UPDATE, (params->state_bits == 32 ? 28.0 : 16.0) * weights, stream);
  GNN_HIP(hipGetLastError());
  return GNN_OK;
}

}  // extern "C"
