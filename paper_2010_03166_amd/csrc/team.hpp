// The first entries of a row in its order: larger logits before smaller ones,
// and equal ones by their columns.  A row is held by a team of lanes, and what
// is kept of it is told by the last entry that is kept (the border).
//
// Amounts (1 an entry, or its weight) are whole numbers, so that their sums
// are exact, the same in any order, and every sum over a part of the row fits
// every other.  The border of an amount P is the entry with
//   sum before it < P <= sum with it.
// It is found without sorting the row: amounts are added up in bins of the
// logits' distance from the largest, and only the entries of the bin that
// holds the border are put in order.  Bins are so many that a few entries lie in
// one where logits are spread; where they are not (equal logits, logits at the
// type's lowest value beside others) the bin's entries are searched from memory:
// 16,384 x 2,048 equal logits with top-p 309 us instead of 100.
#pragma once

#include <type_traits>

#include "rows.hpp"

// (a lambda; left to itself the compiler calls some, and a row goes to the stack)
#define INLINE __attribute__((always_inline))

namespace gnnprop {

struct Border {
  float z;
  int32_t col;
};
constexpr Border NO_BORDER = {-INFINITY, 0x7fffffff};  // all are kept

__device__ __forceinline__ bool within(const Border& b, float z, int32_t col) {
  return (z > b.z) | ((z == b.z) & (col <= b.col));
}

// Bits whose unsigned order is the floats' (0 and -0 alike), and back.
__host__ __device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t x = __builtin_bit_cast(uint32_t, z + 0.f);
  return x >> 31 ? ~x : x | 0x80000000u;
}
__host__ __device__ __forceinline__ float float_of(uint32_t key) {
  return __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key);
}
// An entry's place in the order, as a number: smaller ones come first.
__device__ __forceinline__ uint64_t place(float z, int32_t col) {
  return (uint64_t)~ordered(z) << 32 | (uint32_t)col;
}

// Makes v a value that nothing computed from it before is kept for: what a later
// pass over a row in registers needs of it is formed again, since the row leaves
// few registers.
template <typename T>
__device__ __forceinline__ void refresh(T& v) {
  asm volatile("" : "+v"(v));
}

// What the wavefronts of a team give each other.
template <int G, int W>
struct Exchange {
  uint64_t sums[W];
  float tops[W], lows[W];
  int32_t flags[W];
};
// And what a border is found with: bins, and entries that are put in order at
// once.
template <int G, int W>
struct Bins : Exchange<G, W> {
  static constexpr int BINS = W > 1 ? 512 : G == 64 ? 256 : G >= 16 ? 128 : G == 8 ? 64 : 8 * G;
  static constexpr int LIST = W > 1 ? 256 : G == 64 ? 128 : G >= 16 ? 64 : G == 8 ? 32 : 16;
  static constexpr int WORDS = BINS + G + 2 * LIST;
  alignas(16) uint64_t words[WORDS];
  // the last G, one a lane, are for entries that are in no bin
  __device__ __forceinline__ uint64_t* bins() { return words; }
  __device__ __forceinline__ uint64_t* amount() { return words + BINS + G; }
  __device__ __forceinline__ uint64_t* place() { return words + BINS + G + LIST; }
  uint64_t lo, hi;
  Border border;
  int32_t count;
};

// The logit of an entry's place.
__device__ __forceinline__ float logit_of(uint64_t place) {
  return float_of(~(uint32_t)(place >> 32));
}

// G lanes of a wavefront, or W whole wavefronts, that hold a row together.
template <int G_, int W_, template <int, int> class S = Bins>
struct Team {
  static constexpr int G = G_, W = W_, LANES = G * W;
  static_assert(W == 1 || G == 64, "several wavefronts are whole ones");
  using Shared = S<G, W>;

  Shared& s;
  const int t;     // own number in the team
  const int lane;  // in its wavefront's part of it
  const int wave;

  __device__ __forceinline__ Team(Shared& shared, int number)
      : s(shared), t(number), lane(number % G), wave(number / G) {}

  // What the team wrote to LDS before is there after.  (A wavefront's LDS
  // accesses are done in their order.)
  __device__ __forceinline__ void sync() const {
    if (W > 1) {
      __syncthreads();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }

  __device__ __forceinline__ float max(float v) const {
    v = lanes_max<G>(v);
    if (W == 1) return v;
    if (lane == 0) s.tops[wave] = v;
    sync();
    v = s.tops[0];
    for (int k = 1; k < W; ++k) v = fmaxf(v, s.tops[k]);
    sync();
    return v;
  }
  // The largest and the least value, and the sum of small numbers.
  __device__ __forceinline__ void range(float* high, float* low, int32_t* number) const {
    float h = lanes_max<G>(*high), l = -lanes_max<G>(-*low);
    int32_t m = lanes_sum<G>(*number);
    if (W > 1) {
      if (lane == 0) {
        s.tops[wave] = h;
        s.lows[wave] = l;
        s.flags[wave] = m;
      }
      sync();
      h = s.tops[0];
      l = s.lows[0];
      m = s.flags[0];
      for (int k = 1; k < W; ++k) {
        h = fmaxf(h, s.tops[k]);
        l = fminf(l, s.lows[k]);
        m += s.flags[k];
      }
      sync();
    }
    *high = h;
    *low = l;
    *number = m;
  }
  __device__ __forceinline__ uint64_t sum(uint64_t v) const {
    v = lanes_sum<G>(v);
    if (W == 1) return v;
    if (lane == 0) s.sums[wave] = v;
    sync();
    v = 0;
    for (int k = 0; k < W; ++k) v += s.sums[k];
    sync();
    return v;
  }
  __device__ __forceinline__ double sum(double v) const {
    v = lanes_sum<G>(v);
    if (W == 1) return v;
    if (lane == 0) s.sums[wave] = (uint64_t)__double_as_longlong(v);
    sync();
    v = 0.0;
    for (int k = 0; k < W; ++k) v += __longlong_as_double((long long)s.sums[k]);
    sync();
    return v;
  }
  // Three sums.
  __device__ __forceinline__ void sum3(double* x, double* y, double* z) const {
    *x = sum(*x);
    *y = sum(*y);
    *z = sum(*z);
  }
  __device__ __forceinline__ bool any(bool v) const {
    uint64_t mine = __ballot(v);
    if (G < 64) mine = mine >> ((threadIdx.x & 63) / G * G) & ((1ull << (G & 63)) - 1);
    if (W == 1) return mine != 0;
    if (lane == 0) s.flags[wave] = mine != 0;
    sync();
    bool r = false;
    for (int k = 0; k < W; ++k) r |= s.flags[k] != 0;
    sync();
    return r;
  }
  // The sum over the lanes before this one, in the wavefront's part: within
  // rows of 16 lanes, then the last lanes of rows added to the rows after them.
  __device__ __forceinline__ uint64_t before(uint64_t v) const {
    uint64_t x = v;
    if (G > 1) x = shifted<0x111, 0xF, 1>(x);
    if (G > 2) x = shifted<0x112, 0xF, 2>(x);
    if (G > 4) x = shifted<0x114, 0xF, 4>(x);
    if (G > 8) x = shifted<0x118, 0xF, 8>(x);
    if (G > 16) x = shifted<0x142, 0xA, 0>(x);
    if (G > 32) x = shifted<0x143, 0xC, 0>(x);
    return x - v;
  }
  template <int CTRL, int ROWS, int D>
  __device__ __forceinline__ uint64_t shifted(uint64_t x) const {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xF, false);
    const uint64_t y = (uint64_t)hi << 32 | lo;
    // (a row of 16 lanes holds several teams)
    return G >= 16 || lane >= D ? x + y : x;
  }

  // The first bin with which the amounts reach P, and the amounts before it.
  // Every wavefront finds it by itself: the lane whose bins reach it, then, with
  // a lane each, which of those (16,384 x 2,048, first 16: 43 us, 50 with the lane
  // reading on alone).  False where all of them do not.
  __device__ __forceinline__ bool find(uint64_t P, int32_t* bin, uint64_t* base) const {
    constexpr int EACH = Shared::BINS / G;
    uint64_t own = 0;
    const int turn = lane * EACH / 32;  // (lanes that share banks begin elsewhere)
    for (int k = 0; k < EACH; ++k) own += s.bins()[lane * EACH + (k + turn) % EACH];
    uint64_t sum = before(own);
    const bool has = sum < P && sum + own >= P;
    int from = holder(has);
    if (from < 0) return false;
    sum = __shfl((unsigned long long)sum, from, G);
    if (EACH <= G) {
      const uint64_t x = lane < EACH ? s.bins()[from * EACH + lane] : 0;
      sum += before(x);
      const int at = holder(sum < P && sum + x >= P);
      *bin = from * EACH + at;
      *base = __shfl((unsigned long long)sum, at, G);
    } else {
      int32_t b = from * EACH;
      for (uint64_t x = s.bins()[b]; sum + x < P; x = s.bins()[++b]) sum += x;
      *bin = b;
      *base = sum;
    }
    return true;
  }
  // The team's first lane of the wavefront for which it holds, or -1.
  __device__ __forceinline__ int holder(bool has) const {
    uint64_t who = __ballot(has);
    if (G < 64) who = who >> ((threadIdx.x & 63) / G * G) & ((1ull << (G & 63)) - 1);
    return __ffsll((unsigned long long)who) - 1;
  }

  __device__ __forceinline__ void clear() const {
    for (int k = t; k < Shared::BINS; k += LANES) s.bins()[k] = 0;
    if (t == 0) {
      s.count = 0;
      s.lo = ~0ull;
      s.hi = 0;
    }
    sync();
  }
  // (without a branch: what is to be in no bin goes to the lane's own place)
  __device__ __forceinline__ void add(int32_t bin, uint64_t x, bool in) const {
    add(in ? bin : Shared::BINS + lane, x);
  }
  __device__ __forceinline__ void add(int32_t bin, uint64_t x) const {
    atomicAdd(reinterpret_cast<unsigned long long*>(&s.bins()[bin]), (unsigned long long)x);
  }
  __device__ __forceinline__ void list(float z, int32_t col, uint64_t x) const {
    // (a count past the list's end need not be exact)
    if (__hip_atomic_load(&s.count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > Shared::LIST)
      return;
    const int32_t at = atomicAdd(&s.count, 1);
    if (at >= Shared::LIST) return;
    s.place()[at] = place(z, col);
    s.amount()[at] = x;
  }
  // The border among the entries listed, `base` being the amounts before them.
  __device__ __forceinline__ Border settle(uint64_t P, uint64_t base) const {
    const int32_t m = s.count;
    for (int32_t i = t; i < m; i += LANES) {
      const uint64_t own = s.place()[i], x = s.amount()[i];
      uint64_t sum = base;
#pragma unroll 4
      for (int32_t j = 0; j < m; ++j) sum += s.place()[j] < own ? s.amount()[j] : 0;
      if (sum < P && sum + x >= P) {
        s.border = {logit_of(own), (int32_t)(uint32_t)own};
      }
    }
    sync();
    return s.border;
  }

  // The border of P, once the amounts are in their bins and the team has met:
  // row.each(f) calls f(z, col) for the lane's entries, amount(z, col) is what
  // one adds, bins are `scale` to a unit of z, from `top` down.  NO_BORDER where
  // the amounts do not reach P.  False where a bin holds more entries than are
  // put in order at once: *bin and *base are for search() then.
  template <typename Row, typename Amount>
  __device__ __forceinline__ bool select(const Row& row, Amount amount, float top, float scale,
                                         uint64_t P, Border* border, int32_t* bin,
                                         uint64_t* base) const {
    if (!find(P, bin, base)) {
      *border = NO_BORDER;
      sync();
      return true;
    }
    if constexpr (Row::CHUNKS > 0) {
      row.each4([&](int32_t col, f4 z) INLINE {
        bool in[4], any = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) any |= in[j] = bin_of(z[j], top, scale) == *bin;
        if (!any) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t x = in[j] ? amount(z[j], col + j) : 0;
          if (x) list(z[j], col + j, x);
        }
      });
    } else {
      row.each([&](float z, int32_t col) INLINE {
        if (bin_of(z, top, scale) != *bin) return;
        const uint64_t x = amount(z, col);
        if (x) list(z, col, x);
      });
    }
    sync();
    if (s.count > Shared::LIST) {
      sync();
      return false;
    }
    *border = settle(P, *base);
    return true;
  }

  __device__ __forceinline__ static int32_t bin_of(float z, float top, float scale) {
    return (int32_t)fminf((top - z) * scale, (float)(Shared::BINS - 1));
  }

  // The border in a bin of many entries: by bins of their places, whose range
  // shrinks BINS times in each turn, at last to one entry.  (The row is one that
  // is read again, so that a row in registers need not be kept for it.  Were it
  // written to meanwhile, the amounts might not reach P any more: that ends the
  // search too.)
  template <typename Row, typename Amount>
  __device__ __forceinline__ Border search(const Row& row, Amount amount, float top, float scale,
                                           int32_t bin, uint64_t P, uint64_t base) const {
    uint64_t lo = 0, hi = ~0ull;
    for (int turn = 0; turn < 64; ++turn) {
      const bool first = turn == 0;
      clear();
      const auto member = [&](float z, int32_t col) INLINE {
        if (first) return bin_of(z, top, scale) == bin;
        const uint64_t at = place(z, col);
        return at >= lo && at <= hi;
      };
      uint64_t least = ~0ull, most = 0;
      row.each([&](float z, int32_t col) INLINE {
        if (!member(z, col) || !amount(z, col)) return;
        const uint64_t at = place(z, col);
        least = at < least ? at : least;
        most = at > most ? at : most;
      });
      if (least <= most) {
        atomicMin(reinterpret_cast<unsigned long long*>(&s.lo), (unsigned long long)least);
        atomicMax(reinterpret_cast<unsigned long long*>(&s.hi), (unsigned long long)most);
      }
      sync();
      const uint64_t from = s.lo, range = s.hi - from;
      const int shift = range < Shared::BINS
                            ? 0 : 64 - __builtin_ctz(Shared::BINS) - __clzll((long long)range);
      row.each([&](float z, int32_t col) INLINE {
        if (!member(z, col)) return;
        const uint64_t x = amount(z, col);
        if (x) add((int32_t)((place(z, col) - from) >> shift), x);
      });
      sync();
      int32_t b;
      uint64_t more = 0;
      if (!find(P - base, &b, &more)) break;
      base += more;
      lo = from + ((uint64_t)b << shift);
      hi = lo + ((1ull << shift) - 1);
      row.each([&](float z, int32_t col) INLINE {
        const uint64_t at = place(z, col);
        if (at < lo || at > hi) return;
        const uint64_t x = amount(z, col);
        if (x) list(z, col, x);
      });
      sync();
      if (s.count <= Shared::LIST) return settle(P, base);
      sync();
    }
    sync();
    return NO_BORDER;
  }
};

// ----------------------------------------------------------------- rows

// A row in the registers of its team: V chunks of four columns a lane, the
// wavefronts' parts one after the other.
template <int G, int W, int V>
struct Held {
  static constexpr int CHUNKS = V, MOST = G * W * V * 4;
  mutable f4 z[V];
  mutable int32_t first;  // column of the lane's first
  int32_t C;

  // The row of `cols` columns, or MOST of them from column `from` on.
  __device__ __forceinline__ void load(const float* row, int32_t cols, int t, int32_t from = 0) {
    C = cols;
    first = from + (t / G) * (G * V * 4) + t % G * 4;
#pragma unroll
    for (int k = 0; k < V; ++k)  // (rows of more than one chunk have at least four columns)
      z[k] = MOST > 4 ? *reinterpret_cast<const f4u*>(row + min(column(k), C - 4))
                      : load_cols(row, column(k), C);
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (column(k) - t % G * 4 + G * 4 > C) z[k] = cut_cols(z[k], column(k), C);
  }
  __device__ __forceinline__ int32_t column(int k) const { return first + k * G * 4; }
  // f(column, its and the next three logits) for the lane's chunks
  template <class F>
  __device__ __forceinline__ void each4(F f) const {
    refresh(first);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      refresh(z[k]);
      f(column(k), z[k]);
      __builtin_amdgcn_sched_barrier(0);  // (what is formed of one chunk only has registers)
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    each4([&](int32_t col, f4 v) INLINE {
#pragma unroll
      for (int j = 0; j < 4; ++j) f(v[j], col + j);
    });
  }
};

// A row that is read again for each pass over it.
template <int G, int W>
struct Reread {
  static constexpr int CHUNKS = 0, MOST = MOST_COLS;
  const float* row;
  int32_t first, C, part;

  // Columns [from, cols) of the row.
  __device__ __forceinline__ void load(const float* at, int32_t cols, int t, int32_t from = 0) {
    row = at;
    C = cols;
    part = (int32_t)ceil_div(ceil_div(C - from, W), G * 4);
    first = from + (t / G) * (part * G * 4) + t % G * 4;
  }
  __device__ __forceinline__ int32_t column(int k) const { return first + k * G * 4; }
  template <class F>
  __device__ __forceinline__ void each4(F f) const {
#pragma unroll 1
    for (int k = 0; k < part; ++k)
      f(column(k), cut_cols(load_cols(row, column(k), C), column(k), C));
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    each4([&](int32_t col, f4 v) INLINE {
#pragma unroll
      for (int j = 0; j < 4; ++j) f(v[j], col + j);
    });
  }
};

// Entries by their places, in any order, from memory (the columns are the
// entries' own).
template <int G, int W>
struct Listed {
  static constexpr int CHUNKS = 0, MOST = MOST_COLS;
  const uint64_t* places;
  int64_t count;
  int32_t t;

  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
    for (int64_t k = t; k < count; k += G * W) f(logit_of(places[k]), (int32_t)(uint32_t)places[k]);
  }
};

// What holds a row of C columns: G lanes of a wavefront or W wavefronts, with V
// chunks each, or one lane (G = 1) with a whole row of up to 32.
struct Shape {
  int32_t G, W, V;
};
// As few lanes as a row takes at four chunks each (eight from 64 lanes on: few
// exchanges between lanes, few lanes past the row's end), more where the rows
// are too few to give the chip's 1,024 vector units two wavefronts each: then a
// row's latency counts.  `places`: entries that each lane compares its share of
// with all the others (a quarter of them is what it gets at most).  `small`:
// columns that a lane takes alone, of rows enough for a wavefront a unit.
// `spread`: rows past 2,048 columns take more wavefronts too where there are few
// (a draw gains what a loss, which has less to do and waits for all of them more
// often, loses: 100 x 16,000 12.5 us in 512 threads, 18.2 in 1,024).
inline Shape shape_of(int32_t n, int32_t C, int32_t places, int32_t small, bool spread) {
  const int32_t q = (int32_t)ceil_div(C, 4);
  if (q <= 2 || (C <= small && n >= 1 << 16))
    return {1, 1, q <= 2 ? q : q <= 4 ? 4 : q <= 6 ? 6 : 8};
  if (!spread && q > 512) n = INT32_MAX;
  if (q > 4096) return {64, 16, q <= 6144 ? 6 : 8};
  if (q > 2048) return n < 256 ? Shape{64, 16, 4} : Shape{64, 8, 8};
  if (q > 1024) return n < 256 ? Shape{64, 16, 2} : n < 512 ? Shape{64, 8, 4} : Shape{64, 4, 8};
  if (q > 512) return n < 512 ? Shape{64, 8, 2} : Shape{64, 4, 4};
  if (q > 256) return n < 1024 ? Shape{64, 4, 2} : Shape{64, 1, q <= 384 ? 6 : 8};
  int32_t G = 4;
  while (G < 64 && 4 * G < std::max(q, places)) G *= 2;
  while (G < 64 && G < q && (int64_t)n * G < 64 * 2048) G *= 2;
  return {G, 1, (int32_t)ceil_div(q, G)};
}

// f.held<G, W, V>() for a shape with G > 1, of rows of at most F::MOST columns,
// spread as F::SPREAD says (no other shapes are built).
template <class F>
auto of_shape(const Shape& s, F f) {
  if constexpr (F::MOST > 16384) {
    static_assert(F::SPREAD, "rows past 16,384 columns take 1,024 threads");
    if (s.W == 16 && s.V == 6) return f.template held<64, 16, 6>();
    if (s.W == 16 && s.V == 8) return f.template held<64, 16, 8>();
  }
  if constexpr (F::SPREAD) {
    if (s.W == 16) return s.V == 2 ? f.template held<64, 16, 2>() : f.template held<64, 16, 4>();
    if (s.W == 8 && s.V == 2) return f.template held<64, 8, 2>();
    if (s.W == 8 && s.V == 4) return f.template held<64, 8, 4>();
  }
  if (s.W == 8) return f.template held<64, 8, 8>();
  if (s.W == 4)
    return s.V == 2   ? f.template held<64, 4, 2>()
           : s.V == 4 ? f.template held<64, 4, 4>()
                      : f.template held<64, 4, 8>();
  const auto few = [&](auto lanes) {
    constexpr int G = decltype(lanes)::value;
    return s.V == 1   ? f.template held<G, 1, 1>()
           : s.V == 2 ? f.template held<G, 1, 2>()
           : s.V == 3 ? f.template held<G, 1, 3>()
                      : f.template held<G, 1, 4>();
  };
  switch (s.G) {
    case 4: return few(std::integral_constant<int, 4>());
    case 8: return few(std::integral_constant<int, 8>());
    case 16: return few(std::integral_constant<int, 16>());
    case 32: return few(std::integral_constant<int, 32>());
  }
  return s.V == 6   ? f.template held<64, 1, 6>()
         : s.V == 8 ? f.template held<64, 1, 8>()
                    : few(std::integral_constant<int, 64>());
}

template <int G, int W>
constexpr int threads_of() {
  return W > 1 ? 64 * W : 256;
}

// (written so that a NaN is refused)
inline bool temperature_ok(double T) { return T >= 1e-6 && T <= 1e6; }

}  // namespace gnnprop
