// Drawing actions from and finding the top logits of rows past LONG_COLS
// columns: parts of 4,096, a block each, and what is one of a row joined from
// them by every block alike or by a launch of a block a row.  A draw reads its
// row once for its range, twice for each border that is asked for, once for the
// kept sums and a part of it for the action, out of the caches for the few rows
// that are so long; top logits read it once, and the first k of each part go on.
// Sums over parts are of whole numbers, or in a fixed order.
#include "choose.hpp"

namespace gnnprop {

using PartTeam = Team<64, 4>;
using PartRow = Held<64, 4, 4>;
constexpr int32_t PART_COLS = PartRow::MOST;
constexpr int BINS = PartTeam::Shared::BINS, LIST = PartTeam::Shared::LIST;
constexpr int32_t BAD_LANES = 1 << 16;  // (row_range's mark, in a part's count of lanes)

// What is found of a row on its way to a border: amounts by bins, and the
// entries of the border's bin.
struct Search {
  uint64_t bins[BINS];
  uint64_t place[LIST], amount[LIST];
  int32_t count, pad;
};
struct LongRow {
  Search of[2];    // of the first top_k, of top_p's share
  Border kept[2];  // what is kept up to there
};
struct LongPart {
  float top, low, least;  // largest, least of the lanes' largest, least logit
  int32_t lanes;          // with a logit
  double sum;             // of exp(z - top)
  uint64_t kept;          // weights
};
struct TopPart {
  float top;
  int32_t lanes;
  double others;  // sum of exp((z - top) / T) over those that do not go on
};

namespace {

constexpr int THREADS = 256;

inline int32_t parts_of(int32_t C) { return (int32_t)ceil_div(C, PART_COLS); }

// A row's range, joined from its parts by the whole block.
struct Joined {
  float top, low, least;
  int32_t lanes;
  bool ok;
};
template <class P>
__device__ __forceinline__ Joined joined(const PartTeam& team, const P* parts, int32_t count) {
  Joined x = {-INFINITY, INFINITY, INFINITY, 0, true};
  bool bad = false;
  for (int32_t k = team.t; k < count; k += THREADS) {
    x.top = fmaxf(x.top, parts[k].top);
    const int32_t lanes = parts[k].lanes;
    bad |= lanes >= BAD_LANES;
    x.lanes += lanes % BAD_LANES;
    if constexpr (sizeof(P) == sizeof(LongPart)) {
      x.low = fminf(x.low, parts[k].low);
      x.least = fminf(x.least, parts[k].least);
    }
  }
  team.range(&x.top, &x.low, &x.lanes);
  x.least = -team.max(-x.least);
  x.ok = !team.any(bad) && fabsf(x.top) < INFINITY;
  return x;
}

// The block's row and part.
struct Where {
  int64_t i;
  int32_t part, col0;
};
template <class Args>
__device__ __forceinline__ Where where(const Args& a) {
  const int64_t b = a.block0 + blockIdx.x;
  const int32_t part = (int32_t)(b % a.per_row);
  return {b / a.per_row, part, part * PART_COLS};
}

// ------------------------------------------------------------------ draws

__global__ __launch_bounds__(THREADS) void long_range_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  const PartTeam team(s, threadIdx.x);
  const Where at = where(a);
  const float* from = a.Z + at.i * a.ld_z;
  PartRow row;
  row.load(from, a.C, team.t, at.col0);
  // the row's bins and counts start as zeros
  LongRow& mine = a.rows[at.i];
  for (int w = 0; w < 2; ++w) {
    for (int32_t k = at.part * THREADS + team.t; k < BINS; k += a.per_row * THREADS)
      mine.of[w].bins[k] = 0;
    if (at.part == 0 && team.t == 0) mine.of[w].count = 0;
  }
  LongPart p = {};
  row_range(team, row, &p.top, &p.low, &p.lanes);
  p.least = INFINITY;
  if (a.top_k) {
    row.each([&](float z, int32_t) INLINE { p.least = fminf(p.least, z > -INFINITY ? z : INFINITY); });
    p.least = -team.max(-p.least);
  }
  if (a.logp) {
    const float shift = shift_of(p.top);
    row.each4([&](int32_t, f4 z) INLINE { p.sum += (double)sum4(exp4(z, shift)); });
    p.sum = team.sum(p.sum);
  }
  if (team.t == 0) a.parts[at.i * a.per_row + at.part] = p;
}

// A row's search: what counts, where bins lie, and what amount is looked for.
struct Look {
  float scale, from;  // bins to a unit, the least logit that counts
};
__device__ __forceinline__ Look look_for(const SampleArgs& a, int which, const Joined& x) {
  if (which == 1) return {(BINS - 1) * a.inv_range, -INFINITY};
  const float from = a.top_k > x.lanes ? x.least : x.low;
  const float scale = (BINS - 1) / (x.top - from);
  return {scale < INFINITY ? scale : 0.f, from};
}
__device__ __forceinline__ uint64_t wanted(const SampleArgs& a, int which, const PartTeam& team) {
  if (which == 0) return (uint64_t)a.top_k;
  uint64_t all = 0;
  for (int k = team.t; k < BINS; k += THREADS) all += team.s.bins[k];
  all = team.sum(all);
  const uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
  return P < 1 ? 1 : P < all ? P : all;
}
__device__ __forceinline__ Weights weights_of(const SampleArgs& a, const double* table, int which,
                                              const Joined& x, const LongRow& mine) {
  return {Exponential(table, a.scale, a.bits), x.top,
          which == 1 && a.top_k ? mine.kept[0] : NO_BORDER};
}

// WHICH: 0 the first top_k, 1 top_p's share of those.
template <int WHICH>
__global__ __launch_bounds__(THREADS) void long_bins_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ double s_table[64];
  const PartTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  if (team.t < 64) s_table[team.t] = TABLE.at[team.t];
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  LongRow& mine = a.rows[at.i];
  const Look look = look_for(a, WHICH, x);
  team.clear();
  if (WHICH == 0) {
    row.each([&](float z, int32_t) INLINE {
      team.add(PartTeam::bin_of(z, x.top, look.scale), 1, z >= look.from);
    });
  } else {
    const Weights weight = weights_of(a, s_table, WHICH, x, mine);
    row.each4([&](int32_t col, f4 z) INLINE {
      uint64_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = weight(z[j], col + j);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        team.add(PartTeam::bin_of(z[j], x.top, look.scale), w[j], w[j] != 0);
    });
  }
  team.sync();
  for (int k = team.t; k < BINS; k += THREADS)
    if (s.bins[k])
      atomicAdd(reinterpret_cast<unsigned long long*>(&mine.of[WHICH].bins[k]),
                (unsigned long long)s.bins[k]);
}

// The row's bins in the block's, and the border's.
template <int WHICH>
__device__ __forceinline__ bool long_find(const SampleArgs& a, const PartTeam& team,
                                          const LongRow& mine, uint64_t* P, int32_t* bin,
                                          uint64_t* base) {
  for (int k = team.t; k < BINS; k += THREADS) team.s.bins[k] = mine.of[WHICH].bins[k];
  if (team.t == 0) team.s.count = 0;
  team.sync();
  *P = wanted(a, WHICH, team);
  return team.find(*P, bin, base);
}

template <int WHICH>
__global__ __launch_bounds__(THREADS) void long_list_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ double s_table[64];
  __shared__ int32_t s_at;
  const PartTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  if (team.t < 64) s_table[team.t] = TABLE.at[team.t];
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  LongRow& mine = a.rows[at.i];
  uint64_t P, base;
  int32_t bin;
  if (!long_find<WHICH>(a, team, mine, &P, &bin, &base)) return;
  const Look look = look_for(a, WHICH, x);
  const Weights weight = weights_of(a, s_table, WHICH, x, mine);
  row.each4([&](int32_t col, f4 z) INLINE {
    bool in[4], any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      any |= in[j] = PartTeam::bin_of(z[j], x.top, look.scale) == bin;
    if (!any) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t amount = !in[j] ? 0 : WHICH == 0 ? z[j] > -INFINITY : weight(z[j], col + j);
      if (amount) team.list(z[j], col + j, amount);
    }
  });
  team.sync();
  const int32_t own = s.count;
  if (own == 0) return;
  Search& to = mine.of[WHICH];
  if (team.t == 0) s_at = atomicAdd(&to.count, min(own, LIST + 1));
  team.sync();
  const int32_t first = s_at;
  for (int32_t k = team.t; k < min(own, LIST); k += THREADS)
    if (first + k < LIST) {
      to.place[first + k] = s.place[k];
      to.amount[first + k] = s.amount[k];
    }
}

// A block a row: the border.
template <int WHICH>
__global__ __launch_bounds__(THREADS) void long_border_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ double s_table[64];
  const PartTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  if (team.t < 64) s_table[team.t] = TABLE.at[team.t];
  const Joined x = joined(team, a.parts + i * a.per_row, a.per_row);
  if (!x.ok) return;
  LongRow& mine = a.rows[i];
  uint64_t P, base;
  int32_t bin;
  Border b = NO_BORDER;
  if (long_find<WHICH>(a, team, mine, &P, &bin, &base)) {
    const Search& found = mine.of[WHICH];
    const int32_t m = found.count;
    team.sync();  // (all have read the bins)
    if (m <= LIST) {
      for (int32_t k = team.t; k < m; k += THREADS) {
        s.place[k] = found.place[k];
        s.amount[k] = found.amount[k];
      }
      if (team.t == 0) s.count = m;
      team.sync();
      b = team.settle(P, base);
    } else {
      const Look look = look_for(a, WHICH, x);
      Reread<64, 4> row;
      row.load(a.Z + i * a.ld_z, a.C, team.t);
      if (WHICH == 0)
        b = team.search(row, Present(), x.top, look.scale, bin, P, base);
      else
        b = team.search(row, weights_of(a, s_table, WHICH, x, mine), x.top, look.scale, bin, P,
                        base);
    }
  }
  if (team.t == 0) mine.kept[WHICH] = b;
}

__device__ __forceinline__ Weights final_weights(const SampleArgs& a, const double* table,
                                                 const Joined& x, const LongRow& mine) {
  Weights w = {Exponential(table, a.scale, a.bits), x.top,
               a.top_p < 1.0 ? mine.kept[1] : a.top_k ? mine.kept[0] : NO_BORDER};
  if (a.cut > -INFINITY) w.kept = earlier(w.kept, near_entries(x.top, a.cut));
  return w;
}

__global__ __launch_bounds__(THREADS) void long_kept_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ double s_table[64];
  const PartTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  if (team.t < 64) s_table[team.t] = TABLE.at[team.t];
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  const Weights weight = final_weights(a, s_table, x, a.rows[at.i]);
  uint64_t sum = 0;
  row.each4([&](int32_t col, f4 z) INLINE { sum += weight.sum4(z, col); });
  sum = team.sum(sum);
  if (team.t == 0) a.parts[at.i * a.per_row + at.part].kept = sum;
}

// A block a row: its log-sum, the part that holds the random number's share of
// the kept sum (temperature 0: the first with the largest), and the action.
__global__ __launch_bounds__(THREADS) void long_draw_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ double s_table[64];
  __shared__ int32_t s_part;
  __shared__ uint64_t s_target;
  const PartTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  if (team.t < 64) s_table[team.t] = TABLE.at[team.t];
  const LongPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) {
    if (team.t == 0) {
      a.action[i] = -1;
      if (a.logp) a.logp[i] = 0.f;
    }
    return;
  }
  double lse = 0.0;
  if (a.logp) {
    for (int32_t k = team.t; k < a.per_row; k += THREADS)
      if (parts[k].sum != 0.0) lse += parts[k].sum * exp_exact((double)parts[k].top - x.top);
    lse = log_quick((float)team.sum(lse));
  }
  const float* from = a.Z + i * a.ld_z;
  PartRow row;
  if (a.scale == 0.0) {
    float first = -INFINITY;  // (a part's or a column's negative fits a float)
    for (int32_t k = team.t; k < a.per_row; k += THREADS)
      if (parts[k].top == x.top) first = fmaxf(first, -(float)k);
    row.load(from, a.C, team.t, (int32_t)-team.max(first) * PART_COLS);
    first = -INFINITY;
    row.each([&](float z, int32_t col) INLINE {
      first = fmaxf(first, z == x.top ? -(float)col : -INFINITY);
    });
    first = team.max(first);
    if (team.t == 0) {
      a.action[i] = (int32_t)-first;
      if (a.logp) a.logp[i] = (float)-lse;
    }
    return;
  }
  // each thread some parts that follow each other
  const int32_t each = (int32_t)ceil_div(a.per_row, THREADS);
  const int32_t p0 = min(team.t * each, a.per_row), p1 = min(p0 + each, a.per_row);
  uint64_t own = 0;
  for (int32_t k = p0; k < p1; ++k) own += parts[k].kept;
  const uint64_t wave = lanes_sum<64>(own);
  if (team.lane == 0) s.sums[team.wave] = wave;
  team.sync();
  uint64_t ahead = team.before(own), all = 0;
  for (int k = 0; k < 4; ++k) {
    if (k < team.wave) ahead += s.sums[k];
    all += s.sums[k];
  }
  uint64_t target = __umul64hi(all, unit_fraction(a.u[i]));
  if (target >= ahead && target < ahead + own) {
    int32_t k = p0;
    for (target -= ahead; target >= parts[k].kept; ++k) target -= parts[k].kept;
    s_part = k;
    s_target = target;
  }
  team.sync();
  target = s_target;
  row.load(from, a.C, team.t, s_part * PART_COLS);
  const Weights weight = final_weights(a, s_table, x, a.rows[i]);
  uint64_t sums[PartRow::CHUNKS];
  int at_chunk = 0;
  own = 0;
  row.each4([&](int32_t col, f4 z) INLINE {
    const uint64_t sum = weight.sum4(z, col);
    own += sum;
    sums[at_chunk++] = sum;
  });
  own = lanes_sum<64>(own);
  if (team.lane == 0) s.sums[team.wave] = own;
  team.sync();
  ahead = 0;
  for (int k = 0; k < team.wave; ++k) ahead += s.sums[k];
  if (target < ahead || target >= ahead + own) return;
  pick_entry(a, team, row, weight, (int32_t)i, target - ahead, lse, sums);
}

// ------------------------------------------------------------- top logits

__global__ __launch_bounds__(THREADS) void top_part_kernel(TopArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ uint64_t s_list[MOST_TOP];
  const PartTeam team(s, threadIdx.x);
  const Where at = where(a);
  const float* from = a.Z + at.i * a.ld_z;
  PartRow row;
  row.load(from, a.C, team.t, at.col0);
  TopPart p = {};
  float low;
  const bool ok = row_range(team, row, &p.top, &low, &p.lanes);
  const int64_t part = at.i * a.per_row + at.part;
  uint64_t* to = a.candidates + part * a.k;
  int32_t m = 0;
  if (ok) {
    const Border b = first_entries(team, row, from, a.C, a.k, p.top, low, p.lanes, at.col0);
    if (team.t == 0) s.count = 0;
    team.sync();
    double in, out;
    collect(team, row, b, p.top, a.inv_t, s_list, &in, &out);
    p.others = team.sum(out);
    team.sync();
    m = s.count;
  } else if (p.top == INFINITY) {
    p.lanes |= BAD_LANES;
  }
  for (int32_t k = team.t; k < a.k; k += THREADS)
    to[k] = k < m ? s_list[k] : place(-INFINITY, 0x7fffffff);
  if (team.t == 0) a.parts[part] = p;
}

__global__ __launch_bounds__(THREADS) void top_join_kernel(TopArgs a) {
  __shared__ PartTeam::Shared s;
  __shared__ uint64_t s_list[MOST_TOP];
  const PartTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  const TopPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) {
    write_none(a, team, (int32_t)i);
    return;
  }
  const Listed<64, 4> row = {a.candidates + i * a.per_row * a.k, (int64_t)a.per_row * a.k, team.t};
  float top = -INFINITY, low;
  row.each([&](float z, int32_t) INLINE { top = fmaxf(top, z); });
  low = top > -INFINITY ? top : INFINITY;
  int32_t lanes = top > -INFINITY;
  team.range(&top, &low, &lanes);
  const Border b = first_entries(team, row, nullptr, a.C, a.k, top, low, lanes);
  if (team.t == 0) s.count = 0;
  team.sync();
  double in = 0.0, out = 0.0;
  const float octaves = (float)(a.inv_t * 1.4426950408889634);
  row.each([&](float z, int32_t col) INLINE {
    const float e = __builtin_amdgcn_exp2f((z - top) * octaves);
    if (within(b, z, col) & (z > -INFINITY)) {
      in += e;
      s_list[atomicAdd(&s.count, 1)] = place(z, col);
    } else {
      out += e;
    }
  });
  for (int32_t k = team.t; k < a.per_row; k += THREADS)
    if (parts[k].others != 0.0)
      out += parts[k].others * exp_exact(((double)parts[k].top - top) * a.inv_t);
  in = team.sum(in);
  out = team.sum(out);
  team.sync();
  write_top(a, team, s_list, (int32_t)i, top, in, out);
}

template <class Args>
void launch(void (*kernel)(Args), Args a, int64_t blocks, hipStream_t stream) {
  for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
    kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), THREADS, 0, stream>>>(a);
}

size_t rows_bytes(int32_t n) { return round_up((size_t)n * sizeof(LongRow), 256); }

}  // namespace

size_t sample_long_bytes(int32_t n, int32_t C) {
  return rows_bytes(n) + (size_t)n * parts_of(C) * sizeof(LongPart);
}

hipError_t sample_long(SampleArgs a, void* workspace, hipStream_t stream) {
  a.rows = static_cast<LongRow*>(workspace);
  a.parts = reinterpret_cast<LongPart*>(static_cast<char*>(workspace) + rows_bytes(a.n));
  a.per_row = parts_of(a.C);
  const int64_t blocks = (int64_t)a.n * a.per_row;
  launch(long_range_kernel, a, blocks, stream);
  if (a.scale > 0.0) {
    if (a.top_k) {
      launch(long_bins_kernel<0>, a, blocks, stream);
      launch(long_list_kernel<0>, a, blocks, stream);
      launch(long_border_kernel<0>, a, a.n, stream);
    }
    if (a.top_p < 1.0) {
      launch(long_bins_kernel<1>, a, blocks, stream);
      launch(long_list_kernel<1>, a, blocks, stream);
      launch(long_border_kernel<1>, a, a.n, stream);
    }
    launch(long_kept_kernel, a, blocks, stream);
  }
  launch(long_draw_kernel, a, a.n, stream);
  return hipGetLastError();
}

size_t top_long_bytes(int32_t n, int32_t C, int32_t k) {
  const size_t parts = (size_t)n * parts_of(C);
  return round_up(parts * sizeof(TopPart), 256) + parts * k * sizeof(uint64_t);
}

hipError_t top_long(TopArgs a, void* workspace, hipStream_t stream) {
  a.per_row = parts_of(a.C);
  const int64_t blocks = (int64_t)a.n * a.per_row;
  a.parts = static_cast<TopPart*>(workspace);
  a.candidates = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) +
                                             round_up((size_t)blocks * sizeof(TopPart), 256));
  launch(top_part_kernel, a, blocks, stream);
  launch(top_join_kernel, a, a.n, stream);
  return hipGetLastError();
}

}  // namespace gnnprop
