// Drawing actions from rows past 32,768 columns and finding the top logits of
// rows past 16,384: parts of 4,096 columns, a block each, and what is one of a
// row joined from them by every block alike or by a launch of a block a row.  A
// draw reads its row once for its range, twice for each border that is asked
// for (bins, then the border's bin and the weights before it; where the first
// entries are few they are listed, and nothing after them reads the row) and a
// part of it for the action; the few rows that are so long come out of the
// caches.  Top logits read it once, and the first k of each part go on.  Sums
// over parts are of whole numbers, or in a fixed order.
//
// Bound by launches and their latency: 64 x 131,071 with top-k and top-p 52 us
// in five launches of 3 to 15 us (86 with the first 1,025, in ten), without a
// border 28 us in three; 1 x 131,071 14 us without, 46 with top-p (one block
// a row 56 and 179), 29 with top-k and top-p.  500 x 65,536 without a border 76 us,
// 64 x 131,071's first 256 37.
#include "choose.hpp"

namespace gnnprop {

// More bins and longer lists than for rows of a block: of 131,071 logits spread
// like a normal distribution some 200 lie in one.
template <int G, int W>
struct LongBins : Exchange<G, W> {
  static constexpr int BINS = 1024, LIST = 1024;
  alignas(16) uint64_t words[BINS + G + 2 * LIST];
  __device__ __forceinline__ uint64_t* bins() { return words; }
  __device__ __forceinline__ uint64_t* amount() { return words + BINS + G; }
  __device__ __forceinline__ uint64_t* place() { return words + BINS + G + LIST; }
  uint64_t lo, hi;
  Border border;
  int32_t count;
};
using PartTeam = Team<64, 4, LongBins>;   // a part's
using RowTeam = Team<64, 16, LongBins>;   // a row's, where one block has all of it
using SumTeam = Team<64, 4, Exchange>;    // a part's, of which only sums are formed
using TopTeam = Team<64, 4>;
using PartRow = Held<64, 4, 4>;
constexpr int32_t PART_COLS = PartRow::MOST;
constexpr int BINS = PartTeam::Shared::BINS, LIST = PartTeam::Shared::LIST;
constexpr int32_t BAD_LANES = 1 << 16;  // (row_range's mark, in a part's count of lanes)

// What is found of a row on its way to a border: amounts by bins, and the
// entries of the border's bin.
struct Search {
  uint64_t bins[BINS];
  uint64_t entries[2 * LIST];  // places
  uint64_t wanted, base;  // the amount looked for, and what lies in bins before
  int32_t bin;            // the border's (-1: all are kept)
  int32_t count;          // entries in it
};
struct LongRow {
  Search of[2];    // of the first top_k, of top_p's share
  Border kept[2];  // what is kept up to there
};
struct LongPart {
  float top, low, least;  // largest, least of the groups' largest, least logit
  int32_t lanes;          // groups with a logit
  double sum;             // of exp(z - top)
  double mass;            // of exp((z - top) / T), where units follow from the row's sum
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
template <class T, class P>
__device__ __forceinline__ Joined joined(const T& team, const P* parts, int32_t count) {
  Joined x = {-INFINITY, INFINITY, INFINITY, 0, true};
  bool bad = false;
  for (int32_t k = team.t; k < count; k += T::LANES) {
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

// The table of weights' exponentials, in units of all rows of a call, while the
// block's reads are under way.
__device__ __forceinline__ void start_table(const SampleArgs& a, double* table) {
  if (threadIdx.x < 64) table[threadIdx.x] = ldexp(TABLE.at[threadIdx.x], a.bits);
}
// Past BY_SUM columns in units of the row, 2^62 of which are the least power of two
// above its sum (an fp32 sum, good to 2e-5, and 1/64 for that).  Parts are added as
// whole 256ths, in any order the same: every launch has to find the same units.
template <class T>
__device__ __forceinline__ void row_table(const SampleArgs& a, const T& team,
                                          const LongPart* parts, const Joined& x,
                                          double* table) {
  if (a.inv_t == 0.0) return;
  uint64_t sum = 0;
  for (int32_t k = team.t; k < a.per_row; k += T::LANES)
    if (parts[k].mass > 0.0)
      sum += (uint64_t)ceil(256.0 * parts[k].mass *
                            exp_exact(((double)parts[k].top - x.top) * a.inv_t));
  sum = team.sum(sum);
  const int bits = min(51, 62 + 8 - (64 - __clzll((long long)(sum + sum / 64))));
  if (team.t < 64) table[team.t] = ldexp(TABLE.at[team.t], bits);
  team.sync();
}

// ------------------------------------------------------------------ draws

__global__ __launch_bounds__(THREADS) void long_range_kernel(SampleArgs a) {
  __shared__ SumTeam::Shared s;
  const SumTeam team(s, threadIdx.x);
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
  row_range(team, row, a.group, &p.top, &p.low, &p.lanes);
  p.least = INFINITY;
  if (a.top_k) {
    row.each([&](float z, int32_t) INLINE {
      p.least = fminf(p.least, z > -INFINITY ? z : INFINITY);
    });
    p.least = -team.max(-p.least);
  }
  if (a.logp) {
    const float shift = shift_of(p.top);
    row.each4([&](int32_t, f4 z) INLINE { p.sum += (double)sum4(exp4(z, shift)); });
    p.sum = team.sum(p.sum);
  }
  if (a.inv_t > 0.0) {
    const float shift = shift_of(p.top), octaves = (float)(a.inv_t * 1.4426950408889634);
    row.each4([&](int32_t, f4 z) INLINE {
      f4 e;
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f((z[j] - shift) * octaves);
      p.mass += (double)sum4(e);
    });
    p.mass = team.sum(p.mass);
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
template <class T>
__device__ __forceinline__ uint64_t wanted(const SampleArgs& a, int which, const T& team) {
  if (which == 0) return (uint64_t)a.top_k;
  uint64_t all = 0;
  for (int k = team.t; k < BINS; k += T::LANES) all += team.s.bins()[k];
  all = team.sum(all);
  const uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
  return P < 1 ? 1 : P < all ? P : all;
}
__device__ __forceinline__ Weights weights_of(const SampleArgs& a, const double* table, int which,
                                              const Joined& x, const LongRow& mine) {
  return {Exponential(table, a.scale), x.top,
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
  start_table(a, s_table);
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  if (WHICH == 1) row_table(a, team, a.parts + at.i * a.per_row, x, s_table);
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
    if (s.bins()[k])
      atomicAdd(reinterpret_cast<unsigned long long*>(&mine.of[WHICH].bins[k]),
                (unsigned long long)s.bins()[k]);
}

// A block a row: the border's bin.
template <int WHICH>
__global__ __launch_bounds__(THREADS) void long_find_kernel(SampleArgs a) {
  __shared__ PartTeam::Shared s;
  const PartTeam team(s, threadIdx.x);
  Search& mine = a.rows[a.block0 + blockIdx.x].of[WHICH];
  for (int k = team.t; k < BINS; k += THREADS) s.bins()[k] = mine.bins[k];
  team.sync();
  const uint64_t P = wanted(a, WHICH, team);
  int32_t bin = -1;
  uint64_t base = 0;
  if (!team.find(P, &bin, &base)) bin = -1;
  if (team.t) return;
  mine.wanted = P;
  mine.base = base;
  mine.bin = bin;
}

// A part's entries on their way to the row's list: one addition to its count for
// all of them (one for each made a call some 45 ns longer).
template <int MOST>
struct PartList {
  uint64_t places[MOST];
  int32_t count, base;  // (the count may pass the list's end, the row's then does)

  __device__ __forceinline__ void add(uint64_t place) {
    const int32_t k = atomicAdd(&count, 1);
    if (k < MOST) places[k] = place;
  }
  // (by the whole block; `count` has to be 0 at first)
  __device__ __forceinline__ void give(const SumTeam& team, uint64_t* to, int32_t* total) {
    team.sync();
    if (team.t == 0) base = count ? atomicAdd(total, count) : 0;
    team.sync();
    for (int32_t k = team.t; k < min(count, MOST) && k + base < MOST; k += SumTeam::LANES)
      to[base + k] = places[k];
  }
};

// The entries of the border's bin go to the row's list; LAST: it is the last
// border, and the weights of the bins before it are added up.
template <int WHICH, bool LAST>
__global__ __launch_bounds__(THREADS) void long_list_kernel(SampleArgs a) {
  __shared__ SumTeam::Shared s;
  __shared__ PartList<LIST> own;
  __shared__ double s_table[64];
  const SumTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  start_table(a, s_table);
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  if (WHICH == 1 || LAST) row_table(a, team, a.parts + at.i * a.per_row, x, s_table);
  LongRow& mine = a.rows[at.i];
  Search& to = mine.of[WHICH];
  const int32_t bin = to.bin;
  const Look look = look_for(a, WHICH, x);
  Weights weight = weights_of(a, s_table, WHICH, x, mine);
  if (team.t == 0) own.count = 0;
  team.sync();
  if (bin >= 0)
    row.each4([&](int32_t col, f4 z) INLINE {
      bool in[4], any = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) any |= in[j] = RowTeam::bin_of(z[j], x.top, look.scale) == bin;
      if (!any) return;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (in[j] && (WHICH == 0 ? z[j] >= look.from : weight(z[j], col + j) != 0))
          own.add(place(z[j], col + j));
    });
  own.give(team, to.entries, &to.count);
  if (!LAST) return;
  if (a.cut > -INFINITY) weight.kept = earlier(weight.kept, near_entries(x.top, a.cut));
  uint64_t sum = 0;
  row.each4([&](int32_t col, f4 z) INLINE {
    bool in[4], any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool ahead = bin < 0 || RowTeam::bin_of(z[j], x.top, look.scale) < bin;
      in[j] = ahead && within(weight.kept, z[j], col + j);
      any |= in[j];
    }
    if (!any) return;
    uint64_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = weight.all(z[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += in[j] ? w[j] : 0;
  });
  sum = team.sum(sum);
  if (team.t == 0) a.parts[at.i * a.per_row + at.part].kept = sum;
}

// A block a row: the border.  LAST: the weights of what is kept of its bin are
// added to their parts'.
template <int WHICH, bool LAST>
__global__ __launch_bounds__(1024) void long_border_kernel(SampleArgs a) {
  __shared__ RowTeam::Shared s;
  __shared__ double s_table[64];
  const RowTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  start_table(a, s_table);
  LongPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) return;
  if (WHICH == 1 || LAST) row_table(a, team, parts, x, s_table);
  LongRow& mine = a.rows[i];
  const Search& found = mine.of[WHICH];
  const int32_t bin = found.bin, m = found.count;
  const uint64_t P = found.wanted, base = found.base;
  const Look look = look_for(a, WHICH, x);
  Weights weight = weights_of(a, s_table, WHICH, x, mine);
  Reread<64, 16> row;
  row.load(a.Z + i * a.ld_z, a.C, team.t);
  Border b = NO_BORDER;
  if (bin >= 0) {
    if (m <= LIST) {
      for (int32_t k = team.t; k < m; k += 1024) {
        s.place()[k] = found.entries[k];
        s.amount()[k] = WHICH == 0 ? 1 : weight.all(logit_of(found.entries[k]));
      }
      if (team.t == 0) s.count = m;
      team.sync();
      b = team.settle(P, base);
    } else if (WHICH == 0) {
      b = team.search(row, Present{look.from}, x.top, look.scale, bin, P, base);
    } else {
      b = team.search(row, weight, x.top, look.scale, bin, P, base);
    }
  }
  weight.kept = b;
  if (LAST && a.cut > -INFINITY) weight.kept = earlier(b, near_entries(x.top, a.cut));
  if (team.t == 0) mine.kept[WHICH] = weight.kept;
  if (!LAST || bin < 0) return;
  const auto give = [&](int32_t part, uint64_t w) INLINE {
    if (w)
      atomicAdd(reinterpret_cast<unsigned long long*>(&parts[part].kept), (unsigned long long)w);
  };
  if (m <= LIST) {
    for (int32_t k = team.t; k < m; k += 1024) {
      const int32_t col = (int32_t)(uint32_t)found.entries[k];
      give(col / PART_COLS, weight(logit_of(found.entries[k]), col));
    }
  } else {
    int32_t part = 0;  // (a lane's columns ascend)
    uint64_t sum = 0;
    row.each([&](float z, int32_t col) INLINE {
      if (RowTeam::bin_of(z, x.top, look.scale) != bin || !within(weight.kept, z, col)) return;
      if (col / PART_COLS != part) {
        give(part, sum);
        part = col / PART_COLS;
        sum = 0;
      }
      sum += weight.all(z);
    });
    give(part, sum);
  }
}

__device__ __forceinline__ Weights final_weights(const SampleArgs& a, const double* table,
                                                 const Joined& x, const LongRow& mine) {
  Weights w = {Exponential(table, a.scale), x.top, NO_BORDER};
  if (a.top_p < 1.0) w.kept = mine.kept[1];
  else if (a.top_k) w.kept = mine.kept[0];
  else if (a.cut > -INFINITY) w.kept = near_entries(x.top, a.cut);
  return w;
}

// Where top_p's share of at most LIST first entries is looked for, the row's list
// takes all entries up to the last of the border's bin, and a block a row does the
// rest with the list in the place of the row: both borders and the draw.  Top
// 1,000 of 64 x 131,071 51 us, 85 by the two searches of the whole row, of 1,000 x
// 40,000 152 and 265; without top_p, where one search is saved, the other way is as
// fast or faster (top 129 of 1,000 x 40,000 145 us, 160 so).
__global__ __launch_bounds__(THREADS) void long_gather_kernel(SampleArgs a) {
  __shared__ SumTeam::Shared s;
  __shared__ PartList<2 * LIST> mine;
  const SumTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  Search& to = a.rows[at.i].of[0];
  const Look look = look_for(a, 0, x);
  const int32_t bin = to.bin < 0 ? BINS : to.bin;
  if (team.t == 0) mine.count = 0;
  team.sync();
  row.each4([&](int32_t col, f4 z) INLINE {
    if (!(max4(z) >= look.from)) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (z[j] >= look.from && RowTeam::bin_of(z[j], x.top, look.scale) <= bin)
        mine.add(place(z[j], col + j));
  });
  mine.give(team, to.entries, &to.count);
}

// The border of P among the list's amounts, by bins from `top` down.
// (few wavefronts wait for each other a shorter time, a crowded row's search from
// memory wants many: 1,000 x 40,000 with 4, 8 and 16 164, 168 and 206 us, 64 x
// 131,071 equal logits 611, 408 and 317)
constexpr int FEW_WAVES = 8;
using FewTeam = Team<64, FEW_WAVES, LongBins>;
using FewRow = Listed<64, FEW_WAVES>;
template <class Amount>
__device__ __forceinline__ Border border_of(const FewTeam& team, const FewRow& row, Amount amount,
                                            float top, float scale, uint64_t P) {
  Border b;
  int32_t bin;
  uint64_t base;
  if (!team.select(row, amount, top, scale, P, &b, &bin, &base))
    b = team.search(row, amount, top, scale, bin, P, base);
  team.sync();
  return b;
}

// The action among the list's entries up to a border: its column's range shrinks
// BINS times in each turn.
__device__ __forceinline__ int32_t draw_few(const SampleArgs& a, const FewTeam& team,
                                            const FewRow& row, Weights weight, float u) {
  const float top = (float)weight.top;
  uint64_t all = 0;
  if (a.top_p < 1.0) {
    const float scale = (BINS - 1) * a.inv_range;
    team.clear();
    row.each([&](float z, int32_t col) INLINE {
      const uint64_t w = weight(z, col);
      all += w;
      team.add(FewTeam::bin_of(z, top, scale), w, w != 0);
    });
    all = team.sum(all);
    const uint64_t P = (uint64_t)ceil(a.top_p * (double)all);
    weight.kept = border_of(team, row, weight, top, scale, P < 1 ? 1 : P < all ? P : all);
  }
  if (a.cut > -INFINITY) weight.kept = earlier(weight.kept, near_entries(top, a.cut));
  all = 0;
  row.each([&](float z, int32_t col) INLINE { all += weight(z, col); });
  all = team.sum(all);
  uint64_t target = __umul64hi(all, unit_fraction(u));
  int32_t from = 0, width = a.C;
  while (width > 1) {
    const int32_t end = from + width, step = (int32_t)ceil_div(width, BINS);
    team.clear();
    row.each([&](float z, int32_t col) INLINE {
      if (col < from || col >= end) return;
      const uint64_t w = weight(z, col);
      if (w) team.add((col - from) / step, w);
    });
    team.sync();
    int32_t bin = 0;
    uint64_t base = 0;
    team.find(target + 1, &bin, &base);
    team.sync();
    target -= base;
    from += bin * step;
    width = min(step, end - from);
  }
  return from;
}

__global__ __launch_bounds__(FewTeam::LANES) void long_few_kernel(SampleArgs a) {
  __shared__ FewTeam::Shared s;
  __shared__ double s_table[64];
  __shared__ uint64_t s_list[2 * LIST];
  const FewTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  const Search& found = a.rows[i].of[0];
  int32_t m = found.count;
  for (int32_t k = team.t; k < min(m, 2 * LIST); k += FewTeam::LANES) s_list[k] = found.entries[k];
  start_table(a, s_table);
  const LongPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) {
    if (team.t == 0) {
      a.action[i] = -1;
      if (a.logp) a.logp[i] = 0.f;
    }
    return;
  }
  row_table(a, team, parts, x, s_table);
  double lse = 0.0;
  if (a.logp) {
    for (int32_t k = team.t; k < a.per_row; k += FewTeam::LANES)
      if (parts[k].sum != 0.0) lse += parts[k].sum * exp_exact((double)parts[k].top - x.top);
    lse = log_quick((float)team.sum(lse));
  }
  const float* from = a.Z + i * a.ld_z;
  const Look look = look_for(a, 0, x);
  const Present counts = {look.from};
  const uint64_t P = (uint64_t)a.top_k;
  Border b;
  if (m <= 2 * LIST) {
    const FewRow all = {s_list, m, team.t};
    team.clear();
    all.each([&](float z, int32_t) INLINE {
      team.add(FewTeam::bin_of(z, x.top, look.scale), 1, z >= look.from);
    });
    team.sync();
    b = border_of(team, all, counts, x.top, look.scale, P);
  } else {  // a crowded bin: its border from memory, then what is kept to the list
    Reread<64, FEW_WAVES> row;
    row.load(from, a.C, team.t);
    b = team.search(row, counts, x.top, look.scale, found.bin, P, found.base);
    team.sync();
    if (team.t == 0) s.count = 0;
    team.sync();
    row.each([&](float z, int32_t col) INLINE {
      if (!(z >= look.from) || !within(b, z, col)) return;
      const int32_t k = atomicAdd(&s.count, 1);
      if (k < 2 * LIST) s_list[k] = place(z, col);
    });
    team.sync();
    m = min(s.count, 2 * LIST);
    team.sync();
  }
  const int32_t col = draw_few(a, team, FewRow{s_list, m, team.t},
                               {Exponential(s_table, a.scale), x.top, b}, a.u[i]);
  if (team.t) return;
  a.action[i] = col;
  if (a.logp) a.logp[i] = (float)((double)from[col] - x.top - lse);
}

// The parts' weights, where no border was searched.
__global__ __launch_bounds__(THREADS) void long_kept_kernel(SampleArgs a) {
  __shared__ SumTeam::Shared s;
  __shared__ double s_table[64];
  const SumTeam team(s, threadIdx.x);
  const Where at = where(a);
  PartRow row;
  row.load(a.Z + at.i * a.ld_z, a.C, team.t, at.col0);
  start_table(a, s_table);
  const Joined x = joined(team, a.parts + at.i * a.per_row, a.per_row);
  if (!x.ok) return;
  row_table(a, team, a.parts + at.i * a.per_row, x, s_table);
  const Weights weight = final_weights(a, s_table, x, a.rows[at.i]);
  uint64_t sum = 0;
  row.each4([&](int32_t col, f4 z) INLINE { sum += weight.sum4(z, col); });
  sum = team.sum(sum);
  if (team.t == 0) a.parts[at.i * a.per_row + at.part].kept = sum;
}

// A block a row: its log-sum, the part that holds the random number's share of
// the kept sum (temperature 0: the first with the largest), and the action.
__global__ __launch_bounds__(THREADS) void long_draw_kernel(SampleArgs a) {
  __shared__ SumTeam::Shared s;
  __shared__ double s_table[64];
  __shared__ int32_t s_part;
  __shared__ uint64_t s_target;
  const SumTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  start_table(a, s_table);
  const LongPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) {
    if (team.t == 0) {
      a.action[i] = -1;
      if (a.logp) a.logp[i] = 0.f;
    }
    return;
  }
  row_table(a, team, parts, x, s_table);
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
  if (team.t == 0) {
    s_part = 0;
    s_target = 0;
  }
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
  own = 0;
  row.each4([&](int32_t col, f4 z) INLINE { own += weight.sum4(z, col); });
  own = lanes_sum<64>(own);
  if (team.lane == 0) s.sums[team.wave] = own;
  team.sync();
  ahead = 0;
  for (int k = 0; k < team.wave; ++k) ahead += s.sums[k];
  if (target < ahead || target >= ahead + own) return;
  pick_entry<false>(a, team, row, weight, (int32_t)i, target - ahead, lse, nullptr);
}

// ------------------------------------------------------------- top logits

__global__ __launch_bounds__(THREADS) void top_part_kernel(TopArgs a) {
  __shared__ TopTeam::Shared s;
  const TopTeam team(s, threadIdx.x);
  const Where at = where(a);
  const float* from = a.Z + at.i * a.ld_z;
  PartRow row;
  row.load(from, a.C, team.t, at.col0);
  TopPart p = {};
  float low;
  const bool ok = row_range(team, row, a.group, &p.top, &low, &p.lanes);
  const int64_t part = at.i * a.per_row + at.part;
  uint64_t* to = a.candidates + part * a.k;
  int32_t m = 0;
  if (ok) {
    const Border b = first_entries(team, row, from, a.C, a.k, p.top, low, p.lanes, at.col0);
    // (in one order, since the join's sums go over them; a list for each wavefront in
    // the place of what found the border)
    static_assert(TopTeam::Shared::WORDS >= TopTeam::W * MOST_TOP, "the lists fit");
    uint64_t* list = s.words + team.wave * MOST_TOP;
    double in, out;
    const int32_t own = min(collect<true>(team, row, b, p.top, a.inv_t, list, a.k, &in, &out), a.k);
    if (team.lane == 0) s.flags[team.wave] = own;
    p.others = team.sum(out);  // (and every wavefront's count is there)
    int32_t before = 0;
    for (int k = 0; k < TopTeam::W; ++k) {
      if (k < team.wave) before += s.flags[k];
      m += s.flags[k];
    }
    for (int32_t k = team.lane; k < own && before + k < a.k; k += 64) to[before + k] = list[k];
  } else if (p.top == INFINITY) {
    p.lanes |= BAD_LANES;
  }
  for (int32_t k = m + team.t; k < a.k; k += THREADS) to[k] = place(-INFINITY, 0x7fffffff);
  if (team.t == 0) a.parts[part] = p;
}

template <int W>
__global__ __launch_bounds__(64 * W) void top_join_kernel(TopArgs a) {
  using JoinTeam = Team<64, W>;
  __shared__ typename JoinTeam::Shared s;
  __shared__ uint64_t s_list[MOST_TOP];
  const JoinTeam team(s, threadIdx.x);
  const int64_t i = a.block0 + blockIdx.x;
  const TopPart* parts = a.parts + i * a.per_row;
  const Joined x = joined(team, parts, a.per_row);
  if (!x.ok) {
    write_none(a, team, (int32_t)i);
    return;
  }
  const Listed<64, W> row = {a.candidates + i * a.per_row * a.k, (int64_t)a.per_row * a.k, team.t};
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
      const int32_t at = atomicAdd(&s.count, 1);
      if (at < a.k) s_list[at] = place(z, col);
    } else {
      out += e;
    }
  });
  for (int32_t k = team.t; k < a.per_row; k += JoinTeam::LANES)
    if (parts[k].others != 0.0)
      out += parts[k].others * exp_exact(((double)parts[k].top - top) * a.inv_t);
  in = team.sum(in);
  out = team.sum(out);
  team.sync();
  write_top(a, team, s_list, (int32_t)i, top, in, out);
}

template <class Args>
void launch(void (*kernel)(Args), Args a, int64_t blocks, hipStream_t stream,
            int32_t threads = THREADS) {
  for (a.block0 = 0; a.block0 < blocks; a.block0 += LAUNCH_BLOCKS)
    kernel<<<(unsigned)std::min(blocks - a.block0, LAUNCH_BLOCKS), threads, 0, stream>>>(a);
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
  a.group = a.top_k ? group_of((int64_t)a.per_row * THREADS, a.C, a.top_k) : 1;
  const int64_t blocks = (int64_t)a.n * a.per_row;
  launch(long_range_kernel, a, blocks, stream);
  if (a.scale > 0.0 && a.top_k && a.top_k <= LIST && a.top_p < 1.0) {
    launch(long_bins_kernel<0>, a, blocks, stream);
    launch(long_find_kernel<0>, a, a.n, stream);
    launch(long_gather_kernel, a, blocks, stream);
    launch(long_few_kernel, a, a.n, stream, FewTeam::LANES);
    return hipGetLastError();
  }
  if (a.scale > 0.0) {
    const auto search = [&](auto bins, auto find, auto list, auto border) {
      launch(bins, a, blocks, stream);
      launch(find, a, a.n, stream);
      launch(list, a, blocks, stream);
      launch(border, a, a.n, stream, RowTeam::LANES);
    };
    if (a.top_k && a.top_p < 1.0)
      search(long_bins_kernel<0>, long_find_kernel<0>, long_list_kernel<0, false>,
             long_border_kernel<0, false>);
    else if (a.top_k)
      search(long_bins_kernel<0>, long_find_kernel<0>, long_list_kernel<0, true>,
             long_border_kernel<0, true>);
    if (a.top_p < 1.0)
      search(long_bins_kernel<1>, long_find_kernel<1>, long_list_kernel<1, true>,
             long_border_kernel<1, true>);
    else if (!a.top_k)
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
  a.group = group_of(THREADS, a.C, a.k);
  launch(top_part_kernel, a, blocks, stream);
  // (2,000 rows of 640 candidates: 18 us by 256 threads, 68 by 1,024; 64 x 131,071
  // with its 8,192 candidates a row 56 us by 256 threads, both launches, 41 by 1,024)
  if ((int64_t)a.per_row * a.k <= 2048) launch(top_join_kernel<4>, a, a.n, stream);
  else launch(top_join_kernel<16>, a, a.n, stream, 1024);
  return hipGetLastError();
}

}  // namespace gnnprop
