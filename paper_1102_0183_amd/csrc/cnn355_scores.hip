// Scores of classes and their gradient: what a training or test pass is read with once the sums of its output layer, or
// any others, are there.  For a row x of sums, with m = max x and S = log sum_j exp(x_j - m):
//
//   log p_j = (x_j - m) - S          entropy H = S - sum_j e_j (x_j - m) / sum_j e_j,  e_j = exp(x_j - m)
//   d (g_l log p_l + g_h H) / d x_j = g_l ([j == l] - p_j) - g_h p_j (log p_j + H)
//
// One pass over the row: every lane keeps the largest value m it has seen, s = sum of exp(x - m) and t = sum of
// exp(x - m) (x - m), and takes both to a new m by the factor exp(m - m'): s' = s f, t' = (t + (m - m') s) f.  Lanes,
// wavefronts and workgroups that share a row join their three numbers in the same way.  All of it is held in 32 bits.  (Long rows
// take m in steps, so that most tiles need no factor: at `scan`.)
//
// The best classes ride along.  A wavefront keeps the best so far sorted over its lanes, as 64-bit keys (value, then the
// lower index) whose order is that of whole numbers.  Every 32 tiles it picks out what reaches the n_top-th of its lanes'
// largest values: hardly more than n_top classes, so the price is a maximum and a store to LDS for every 16 classes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"
#include "cnn355_lanes.h"

namespace cnn355 {

namespace {

typedef unsigned long long u64;
constexpr int ST = 256;             // threads of a workgroup
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float LOWEST = -3.402823466e38f;
constexpr float FAR = -256.0f;      // 2^FAR is nothing beside 1: stands in for -inf where it is multiplied by zero

// the largest of three; of values that are no number, at least one of the others
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// ---- keys of values: u64 order is (value, lower index first); 0 is below every key ----
// A key is a double above zero, whose order is the same: 63 bits, and the exponent of +inf's key is 0x7fc.
__device__ __forceinline__ u64 key_of(float v, int index) {
  const unsigned b = __builtin_bit_cast(unsigned, v + 0.0f);   // (-0 as 0)
  return (u64)((int)b < 0 ? ~b : b | 0x80000000u) << 31 | (~index & 0x7fffffff);
}
__device__ __forceinline__ u64 key_of_any(float v, int index) { return v == v ? key_of(v, index) : 0; }   // (0: no number)
__device__ __forceinline__ int index_of(u64 k) { return ~(int)k & 0x7fffffff; }
__device__ __forceinline__ float value_of(u64 k) {
  const unsigned b = (unsigned)(k >> 31);
  return __builtin_bit_cast(float, (int)b < 0 ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ u64 above_value_of(u64 k) { return k + (1ull << 31); }

// a float's order as a whole number's, and back
__device__ __forceinline__ int order_of(float v) {
  const int b = __builtin_bit_cast(int, v);
  return b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float of_order(int o) { return __builtin_bit_cast(float, o ^ (o >> 31 & 0x7fffffff)); }

__device__ __forceinline__ int larger_of(int a, int b) { return a > b ? a : b; }
__device__ __forceinline__ int smaller_of(int a, int b) { return a < b ? a : b; }
// keys as doubles: an operation each (compared as whole numbers, whose outcome goes through the scalar unit, 37 rows of 100003
// classes took 16.1 us, so 15.0, one row of 50000 12.4, so 11.8)
__device__ __forceinline__ u64 larger_of(u64 a, u64 b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(__builtin_bit_cast(double, a)), "v"(__builtin_bit_cast(double, b)));
  return __builtin_bit_cast(u64, r);
}
__device__ __forceinline__ u64 smaller_of(u64 a, u64 b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(__builtin_bit_cast(double, a)), "v"(__builtin_bit_cast(double, b)));
  return __builtin_bit_cast(u64, r);
}

// ---- between lanes, without LDS ----
template <int D>
__device__ __forceinline__ float xor_lane(float v) { return __builtin_bit_cast(float, xor_word<D>(__builtin_bit_cast(unsigned, v))); }
template <int D>
__device__ __forceinline__ int xor_lane(int v) { return (int)xor_word<D>((unsigned)v); }
template <int D>
__device__ __forceinline__ u64 xor_lane(u64 v) { return (u64)xor_word<D>((unsigned)(v >> 32)) << 32 | xor_word<D>((unsigned)v); }

// f(a constant) for 1, 2, 4, .. below LANES
template <int LANES, class F>
__device__ __forceinline__ void for_distances(F f) {
  if constexpr (LANES > 1) f(std::integral_constant<int, 1>());
  if constexpr (LANES > 2) f(std::integral_constant<int, 2>());
  if constexpr (LANES > 4) f(std::integral_constant<int, 4>());
  if constexpr (LANES > 8) f(std::integral_constant<int, 8>());
  if constexpr (LANES > 16) f(std::integral_constant<int, 16>());
  if constexpr (LANES > 32) f(std::integral_constant<int, 32>());
}

// a lane's value and that of lane ^ D, in either order
template <int D, class T>
__device__ __forceinline__ void pair_of(T v, T& a, T& b) {
  if constexpr (D < 16) {
    a = v;
    b = xor_lane<D>(v);
  } else {   // (the swap leaves both halves' values in every lane)
    unsigned w[2 * sizeof(T) / 4];
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 4; ++i) {
      unsigned x;
      if constexpr (sizeof(T) == 8) x = i ? (unsigned)(v >> 32) : (unsigned)v;
      else x = __builtin_bit_cast(unsigned, v);
      const auto r = D == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
      w[i] = r[0];
      w[sizeof(T) / 4 + i] = r[1];
    }
    if constexpr (sizeof(T) == 8) {
      a = (u64)w[1] << 32 | w[0];
      b = (u64)w[3] << 32 | w[2];
    } else {
      a = __builtin_bit_cast(T, w[0]);
      b = __builtin_bit_cast(T, w[1]);
    }
  }
}

// Bitonic sorting: lanes that rise and then fall, or the other way round, in groups of 2 D to fall, or to rise where
// (lane & RISE) != 0 (64: in all of them, 0: in none).
template <int D, int RISE, class T>
__device__ __forceinline__ T merge_lanes(T v) {
  if constexpr (D >= 1) {
    const int lane = threadIdx.x & 63;
    const bool rises = RISE == 64 || (lane & RISE) != 0, larger = ((lane & D) == 0) != rises;
    T a, b;
    pair_of<D>(v, a, b);
    const T most = larger_of(a, b), least = smaller_of(a, b);
    return merge_lanes<D / 2, RISE>(larger ? most : least);
  } else {
    return v;
  }
}
// every group of LANES lanes in falling order; RISE as above
template <int LANES, int RISE, class T>
__device__ __forceinline__ T sort_lanes(T v) {
  if constexpr (LANES > 2) v = sort_lanes<LANES / 2, LANES / 2>(v);
  return merge_lanes<LANES / 2, RISE>(v);
}
// the larger ones of two sorted runs of 64, the first falling and the second rising; sorted
template <int RISE, class T>
__device__ __forceinline__ T best_of(T falling, T rising) { return merge_lanes<32, RISE>(larger_of(falling, rising)); }

// ---- sums of a row ----
struct Sums {
  float m, s, t;   // largest value; sum of 2^d; sum of 2^d d, d = (x - m) / ln 2
};

// to another largest value, which is not smaller
__device__ __forceinline__ void lift(Sums& a, float m) {
  const float d = (a.m - m) * LOG2E, f = __builtin_amdgcn_exp2f(d);
  a.t = fmaf(fmaxf(d, FAR), a.s, a.t) * f;
  a.s *= f;
  a.m = m;
}

template <int LANES>
__device__ __forceinline__ void join_lanes(Sums& a) {
  float m = a.m;
  for_distances<LANES>([&](auto d) { m = fmaxf(m, xor_lane<decltype(d)::value>(m)); });
  lift(a, m);
  for_distances<LANES>([&](auto d) {
    a.s += xor_lane<decltype(d)::value>(a.s);
    a.t += xor_lane<decltype(d)::value>(a.t);
  });
}

// Where one class has most of a row, log p of it is minus the logarithm of 1 + the others' sum, of which the rounding of the sum leaves few
// digits.  Rows of up to 1024 classes whose sum is below SURE are summed again, a lane's 16 places x, the largest value's classes apart
// (for all rows, 100000 of 1000 bf16 classes took 84 us, so 67; longer rows have more others).  The result: s - 1.
constexpr float SURE = 1.5f;
// the rest of a row that `scan` has summed: the largest value's own term is a product of two powers of two there, which may round to
// less than 1 (in row_of, where the other kernels' rows have it too, 100000 rows of 1000 bf16 classes, read from the caches, took 1 % longer)
__device__ __forceinline__ float rest_of(const Sums& a) { return a.s == 0.0f ? -1.0f : fmaxf(a.s - 1.0f, 0.0f); }
template <int LANES, int N>
__device__ __forceinline__ float rest_of(const Sums& a, const float (&x)[N]) {
  float rest = a.s - 1.0f;
  if (__ballot(a.s < SURE)) {
    float others = 0.0f;
    int most = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const bool is = x[k] == a.m;
      others += is ? 0.0f : __builtin_amdgcn_exp2f((x[k] - a.m) * LOG2E);
      most += is;
    }
    for_distances<LANES>([&](auto d) {
      others += xor_lane<decltype(d)::value>(others);
      most += xor_lane<decltype(d)::value>(most);
    });
    if (a.s < SURE) rest = others + (float)(most - 1);
  }
  return rest;
}

// What a row's sums come to; rest: s - 1.  A row without a value above -inf is empty; one with +inf or NaN has no distribution.
struct Row {
  float m, log_s, entropy;
  bool none;
};
__device__ __forceinline__ Row row_of(const Sums& a, float rest) {
  Row r;
  r.none = !(a.s < INFINITY);
  if (r.none) { r.m = r.log_s = r.entropy = __builtin_nanf(""); return r; }
  const bool empty = a.s == 0.0f;
  r.m = empty ? -INFINITY : a.m;
  // log(1 + rest): of u, and where that is small by the share of rest in u - 1 (log1pf: 20000 rows of 64 classes 17.5 us, so 15.1)
  const float u = 1.0f + rest;
  r.log_s = logf(u);
  if (rest < SURE - 1.0f) r.log_s = u == 1.0f ? rest : r.log_s * (rest * __builtin_amdgcn_rcpf(u - 1.0f));
  const float h = r.log_s - LN2 * a.t / a.s;
  r.entropy = empty || h < 0.0f ? 0.0f : h;
  return r;
}
__device__ __forceinline__ float log_prob(const Row& r, float x) { return r.m == -INFINITY ? -INFINITY : (x - r.m) - r.log_s; }

// A row's label and its value, asked for before the row is looked at (two loads one after the other).
struct Label {
  bool is;
  float x;
};
template <int TYPE>
__device__ __forceinline__ Label label_of(const ScoreJob& J, long long row) {
  typedef Element<TYPE> E;
  Label l = {false, 0.0f};
  if (J.log_probs) {
    const int c = J.labels[row];
    l.is = c >= 0 && c < J.classes;
    if (l.is) l.x = E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + c]);
  }
  return l;
}

// Where fewer classes than are asked for are above -inf, the masked ones with the lowest indices follow: fewer than 64 are not
// masked, so of the first 128 there are enough that are.
template <int TYPE>
__device__ __forceinline__ u64 with_masked(const ScoreJob& J, long long row, u64 list) {
  typedef Element<TYPE> E;
  const int lane = threadIdx.x & 63;
  int have = __popcll(__ballot(list != 0));
  for (int first = 0; first < 128 && have < J.n_top; first += 64) {
    const int c = first + lane;
    const bool is = c < J.classes && E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + min(c, J.classes - 1)]) == -INFINITY;
    for (u64 in = __ballot(is); in && have < J.n_top; in &= in - 1, ++have)
      if (lane == have) list = key_of(-INFINITY, first + __builtin_ctzll(in));
  }
  return list;
}

// One lane's share of a row's results: the numbers from one of them,
__device__ __forceinline__ Row give_sums(const ScoreJob& J, long long row, bool gives, const Sums& a, float rest, const Label& l) {
  const Row r = row_of(a, rest);
  if (gives) {
    if (J.log_probs) J.log_probs[row] = l.is ? log_prob(r, l.x) : 0.0f;
    if (J.entropy) J.entropy[row] = r.entropy;
    if (J.normaliser) { J.normaliser[2 * row] = r.m; J.normaliser[2 * row + 1] = r.log_s; }
  }
  return r;
}
// and lane i the i-th of the best.
__device__ __forceinline__ void give_row(const ScoreJob& J, long long row, int lane, const Sums& a, float rest, const Label& l, u64 best) {
  const Row r = give_sums(J, row, lane == 0, a, rest, l);
  if (lane < J.n_top) {
    if (J.top) J.top[row * J.n_top + lane] = r.none ? -1 : index_of(best);
    if (J.top_log_probs) J.top_log_probs[row * J.n_top + lane] = r.none ? r.m : log_prob(r, value_of(best));
  }
}

// ---- the best classes of a wavefront ----
constexpr int SEGMENT = 32;  // tiles after which a wavefront picks out the best
constexpr int HELD = 128;    // keys, or tiles' lanes, waiting in LDS: fewer than 64, and those of one look at every lane

struct Picking {             // LDS of a wavefront
  u64 held[HELD];
  unsigned short where[HELD];          // tile of the segment, lane
  unsigned short largest[SEGMENT][64]; // of every lane's 16 classes of a tile the largest, upper half of a float, rounded up
};

struct Best {
  u64 list;        // lane i: the i-th best so far, 0: none (masked classes, -inf, are none)
  u64 bar;         // a key that can still be among them is above it,
  float bar_value; // and the value of a class of the next tile that can is not below this
  int held;
};

__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
  return (u64)__builtin_amdgcn_readlane((unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)v, lane);
}
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ int place_in(u64 lanes) { return __builtin_amdgcn_mbcnt_hi((unsigned)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)lanes, 0)); }
__device__ __forceinline__ void lds_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }   // (a wavefront's own lanes)

// the 64 (or fewer) keys in front join the list
__device__ __forceinline__ void take_held(Best& b, Picking& L, int n_top) {
  const int lane = threadIdx.x & 63;
  lds_order();
  const u64 mine = lane < b.held ? L.held[lane] : 0, rest = 64 + lane < b.held ? L.held[64 + lane] : 0;
  lds_order();
  L.held[lane] = rest;
  b.held = b.held > 64 ? b.held - 64 : 0;
  b.list = best_of<0>(b.list, sort_lanes<64, 64>(mine));
  const u64 last = lane_of(b.list, n_top - 1);
  if (last > b.bar) {
    // (the classes of the tiles to come have higher indices: of theirs, only larger values are above that key)
    b.bar = last;
    b.bar_value = value_of(above_value_of(last));
  }
}

// Rows are looked at from the 16 bytes on that their first class lies in: place 0 is `lead` classes in front of it, and `end`
// the first place behind the last.  (Loads of 16 bytes at odd addresses cost a row of 131071 bf16 classes 13 %.)
template <int TYPE>
struct RowAt {
  const CNN_GLOBAL typename Element<TYPE>::T* at;   // place 0
  int lead, end;
};
template <int TYPE>
__device__ __forceinline__ RowAt<TYPE> row_at(const ScoreJob& J, long long row) {
  typedef typename Element<TYPE>::T T;
  const CNN_GLOBAL T* x = (const CNN_GLOBAL T*)J.x + row * J.stride;
  const int lead = (int)((unsigned long long)x & 15) / (int)sizeof(T);
  return RowAt<TYPE>{x - lead, lead, J.classes + lead};
}

// The best of a segment: tiles first, first + step, ... of a row, of which place (k / V) 64 V + lane V + k % V is a lane's k-th.
// m0, m1: the largest values of the first and second half of every lane's classes, in this segment and those before it.
//
// As many classes as are asked for reach the n_top-th of the lanes' largest values, so what lies below it is out.  Of G such
// values and n_top best G log(G / (G - n_top)) classes reach it where their order is chance: 24 of 64 for 20, 89 of 128 for 64
// (and 300 of 64).  Their classes are asked for again, one to a lane, 32 lanes' at a time.
// (Looking at every tile as it comes, against the best so far, finds some in every second tile of a row of 131072: 4096 such
// rows with 20 best took 252 us so, 194 without any best.)
template <int TYPE>
__device__ __forceinline__ void pick(Best& b, Picking& L, const RowAt<TYPE>& row, float m0, float m1, int first, int step, int tiles, bool last, int n_top) {
  typedef Element<TYPE> E;
  constexpr int V = E::V;
  const int lane = threadIdx.x & 63;
  const int o0 = order_of(m0), o1 = order_of(m1);
  const float v = of_order(lane_of(n_top <= 24 ? sort_lanes<64, 0>(larger_of(o0, o1)) : best_of<0>(sort_lanes<64, 0>(o0), sort_lanes<64, 64>(o1)), n_top - 1));
  if (v > b.bar_value) {
    b.bar_value = v;
    b.bar = key_of(v, -1);
  }
  int waiting = 0;
#pragma unroll 1
  for (int i = 0; i < tiles; ++i) {
    const u64 in = __ballot(__builtin_bit_cast(float, (unsigned)L.largest[i][lane] << 16) >= b.bar_value);
    if (in) {
      if (in >> lane & 1) L.where[waiting + place_in(in)] = (unsigned short)(i << 6 | lane);
      waiting += __popcll(in);
    }
    if (waiting < 64 && i + 1 < tiles) continue;
    lds_order();
    const bool finish = last && i + 1 == tiles;   // (what is held joins the list here too: its code is there once)
#pragma unroll 1
    for (int w0 = 0; w0 < waiting || (finish && w0 == 0); w0 += 32) {
      u64 key[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int w = w0 + u * 4 + (lane >> 4), k = lane & 15;
        const int at_lane = w < waiting ? L.where[w] : 0;
        const int at = (first + (at_lane >> 6) * step) * SCORE_TILE + (k / V) * 64 * V + (at_lane & 63) * V + k % V;
        key[u] = w < waiting && at >= row.lead && at < row.end ? key_of_any(E::get(row.at[at]), at - row.lead) : 0;
      }
      // all of them where they are few, as they mostly are; else four lanes' at a time
      int n = b.held;
#pragma unroll
      for (int u = 0; u < 8; ++u) n += __popcll(__ballot(key[u] > b.bar));
      const bool few = n <= HELD;
      if (few) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const u64 take = __ballot(key[u] > b.bar);
          if (key[u] > b.bar) L.held[b.held + place_in(take)] = key[u];
          b.held += __popcll(take);
        }
      }
#pragma unroll 1
      for (int u = few ? 7 : 0; u < 8; ++u) {
        if (!few) {
          const u64 k = key[0], take = __ballot(k > b.bar);
#pragma unroll
          for (int j = 0; j < 7; ++j) key[j] = key[j + 1];
          if (k > b.bar) L.held[b.held + place_in(take)] = k;
          b.held += __popcll(take);
        }
        while (b.held >= 64 || (u == 7 && finish && w0 + 32 >= waiting && b.held)) take_held(b, L, n_top);
      }
    }
    waiting = 0;
    lds_order();
  }
}

// ---- the pass over a row ----
template <int TYPE>
__device__ __forceinline__ void load_tile(v4u (&r)[16 / Element<TYPE>::V], const RowAt<TYPE>& row, int tile) {
  constexpr int V = Element<TYPE>::V, N = 16 / V;
  const int lane = threadIdx.x & 63, first = tile * SCORE_TILE;
  const CNN_GLOBAL typename Element<TYPE>::T* at = row.at + first;
  if (first >= row.lead && first + SCORE_TILE <= row.end) {
#pragma unroll
    for (int q = 0; q < N; ++q) r[q] = *(const CNN_GLOBAL v4u*)(at + (q * 64 + lane) * V);
  } else {
#pragma unroll
    for (int q = 0; q < N; ++q) r[q] = load16<TYPE>(at, (q * 64 + lane) * V, row.end - first, row.lead - first);
  }
}

// Tiles first, first + step, ... of a row, below `last`: the wavefront's sums, lane by lane, and its best.
//
// In the usual tile the exponent is one operation, d = x / ln 2 - r, with a lane's r as m / ln 2 was when it was last above r by
// more than GROWTH (then both sums go to the new r): every e is too large by the same 2^(m / ln 2 - r), which is taken out at
// the end.  Not every tile is usual.  A masked class gives 0 (-inf) there, and values near the type's lowest leave the range of d,
// which shows in the sums.  And r is rounded while x / ln 2 is not: from 2^24 on d is off by more than a half for the largest class
// itself, and soon so far that every e is 0 (or all are infinite); so a lane whose r would be no smaller than that makes its sum
// one that shows (FUSED: 11.6 million as a value, more than fp16 holds).  Such a tile is done again with d = (x - m) / ln 2 and the
// product of e and d clamped, and so are those behind it (two operations more for each class).
constexpr float GROWTH = 8.0f;   // (t is off by r's distance from m times the rounding of s)
constexpr float FUSED = 16777216.0f;
template <int TYPE, bool ENTROPY, bool TOP>
__device__ __forceinline__ void scan(const RowAt<TYPE>& row, int first, int step, int last, int n_top, Sums& a, Best& b, Picking* L) {
#pragma clang fp contract(off)   // (r is the rounded product in the difference of two of them, too)
  typedef Element<TYPE> E;
  constexpr int V = E::V, N = 16 / V;
  a = Sums{LOWEST, 0.0f, 0.0f};
  b = Best{0, key_of(-INFINITY, 0), LOWEST, 0};
  float r = -INFINITY;
  float largest[2] = {LOWEST, LOWEST};
  bool rough = false;
  auto settle = [&]() {   // sums of 2^(x / ln 2 - r) to sums of 2^((x - m) / ln 2)
    if (a.s > 0.0f) {
      const float off = fmaf(a.m, LOG2E, -r), f = __builtin_amdgcn_exp2f(-off);
      a.t = fmaf(-off, a.s, a.t) * f;
      a.s *= f;
    }
  };
  int in_segment = 0;
  auto one = [&](v4u (&next)[N], int tile) {   // and asks for the one after the next
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = E::get(next[k / V], k % V);
    if (tile + 2 * step < last) load_tile<TYPE>(next, row, tile + 2 * step);
    float top[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = max3(x[8 * h], x[8 * h + 1], x[8 * h + 2]);
      top[h] = max3(top[h], x[8 * h + 3], x[8 * h + 4]);
      top[h] = max3(top[h], x[8 * h + 5], x[8 * h + 6]);
      top[h] = max3(top[h], x[8 * h + 7], x[8 * h + 7]);
      if (TOP) largest[h] = max3(largest[h], top[h], top[h]);
    }
    const float m = max3(a.m, top[0], top[1]);
    if (!rough) {
      float to = r, s = a.s, t = a.t;
      const bool grown = fmaf(m, LOG2E, -r) > GROWTH;
      if (__ballot(grown)) {
        to = grown ? m * LOG2E : r;
        const float d0 = r - to, f = __builtin_amdgcn_exp2f(d0);
        t = fmaf(fmaxf(d0, FAR), s, t) * f;
        s = fabsf(to) < FUSED ? s * f : __builtin_nanf("");
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float d = fmaf(x[k], LOG2E, -to), e = __builtin_amdgcn_exp2f(d);
        s += e;
        if (ENTROPY) t = fmaf(e, d, t);
      }
      const float sure = ENTROPY ? t + s : s;   // (both: else the sum of all e is put off behind the branch, and every e kept for it)
      if (__ballot(!(sure - sure == 0.0f)) == 0) {
        r = to;
        a = Sums{m, s, t};
      } else {
        rough = true;
        settle();
      }
    }
    if (rough) {
      lift(a, m);
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float d = (x[k] - a.m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
        a.s += e;
        if (ENTROPY) a.t = fmaf(e, fmaxf(d, FAR), a.t);
      }
    }
    if (TOP) {
      const unsigned bits = __builtin_bit_cast(unsigned, max3(top[0], top[1], top[1]));
      L->largest[in_segment++][threadIdx.x & 63] = (unsigned short)((TYPE == ELEMENT_BF16 || (int)bits < 0 ? bits : bits + 0xffffu) >> 16);
    }
  };
  v4u even[N], odd[N];
  if (first < last) load_tile<TYPE>(even, row, first);
  if (first + step < last) load_tile<TYPE>(odd, row, first + step);
  for (int tile = first; tile < last; tile += 2 * step) {
    one(even, tile);
    if (tile + step < last) one(odd, tile + step);
    const bool end = tile + 2 * step >= last;
    if (TOP && (in_segment == SEGMENT || end)) {
      const int begun = tile + (tile + step < last ? step : 0) - (in_segment - 1) * step;
      pick<TYPE>(b, *L, row, largest[0], largest[1], begun, step, in_segment, end, n_top);
      in_segment = 0;
    }
  }
  if (!rough) settle();
}

constexpr int threads_of(int waves) { return waves > ST / 64 ? waves * 64 : ST; }

// Rows of more than 64 classes, WAVES wavefronts a row or, where parts > 1, a part of one.
template <int TYPE, int WAVES, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(threads_of(WAVES)) k_scores(ScoreJob J) {
  constexpr int ROWS = threads_of(WAVES) / 64 / WAVES;
  __shared__ Picking lds_picking[TOP ? threads_of(WAVES) / 64 : 1];
  __shared__ u64 lds_best[TOP && WAVES > 1 ? WAVES : 1][64];
  __shared__ float lds_sums[WAVES][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part_of = WAVES > 1 ? 0 : wave, w = WAVES > 1 ? wave : 0;
  const int part = blockIdx.y;
  for (long long row = (long long)blockIdx.x * ROWS + part_of; row < J.rows; row += (long long)gridDim.x * ROWS) {
    Sums a;
    Best b;
    Label label = {false, 0.0f};
    if (J.parts == 1 && w == 0) label = label_of<TYPE>(J, row);
    const RowAt<TYPE> x = row_at<TYPE>(J, row);
    const int tiles = (x.end + SCORE_TILE - 1) / SCORE_TILE;   // (one more than the parts were planned for, it may be)
    scan<TYPE, ENTROPY, TOP>(x, part * J.part_tiles + w, WAVES, part + 1 == J.parts ? tiles : (part + 1) * J.part_tiles, J.n_top, a, b,
                             &lds_picking[TOP ? wave : 0]);
    join_lanes<64>(a);
    if (WAVES > 1) {
      __syncthreads();   // (what the row before left has been read)
      if (lane == 0) { lds_sums[w][0] = a.m; lds_sums[w][1] = a.s; lds_sums[w][2] = a.t; }
      if (TOP) lds_best[w][lane] = b.list;
      __syncthreads();
      if (TOP && WAVES > 4) {   // two by two
#pragma unroll 1
        for (int half = WAVES / 2; half; half >>= 1) {
          if (wave < half) {
            b.list = best_of<0>(b.list, lds_best[wave + half][63 - lane]);
            lds_best[wave][lane] = b.list;
          }
          __syncthreads();
        }
      }
      if (wave != 0) continue;
      a = Sums{LOWEST, 0.0f, 0.0f};
      if (lane < WAVES) a = Sums{lds_sums[lane][0], lds_sums[lane][1], lds_sums[lane][2]};
      join_lanes<64>(a);
      if (TOP && WAVES <= 4) {
#pragma unroll 1
        for (int o = 1; o < WAVES; ++o) b.list = best_of<0>(b.list, lds_best[o][63 - lane]);
      }
    }
    if (J.parts > 1) {
      const long long at = row * J.parts + part;
      if (lane == 0) {
        CNN_GLOBAL float* p = J.part_sums + at * 4;
        p[0] = a.m; p[1] = a.s; p[2] = a.t;
      }
      if (TOP && lane < J.n_top) J.part_best[at * J.n_top + lane] = b.list;
      continue;
    }
    if (TOP) b.list = with_masked<TYPE>(J, row, b.list);
    float rest = rest_of(a);
    if (WAVES == 1 && J.classes <= SCORE_TILE && __ballot(a.s < SURE)) {   // (from the cache, and from its first class on wherever that
      constexpr int V = Element<TYPE>::V;                                  // lies: a lane has the same 16 of equal rows)
      // (which lanes have which places would be worked out in front of the loop over rows, and kept: 100000 rows of 1000 bf16, 16 best,
      // read from the caches, took 193 us so, 187 like this)
      int end = J.classes;
      asm volatile("" : "+s"(end));
      v4u r[16 / V];
#pragma unroll
      for (int q = 0; q < 16 / V; ++q) r[q] = load16<TYPE>(x.at + x.lead, (q * 64 + lane) * V, end);
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = Element<TYPE>::get(r[k / V], k % V);
      rest = rest_of<64>(a, v);
    }
    give_row(J, row, lane, a, rest, label, b.list);
  }
}

// The parts of rows joined: a workgroup a row.
constexpr int JOINED = 8;   // lists that a wavefront asks for together (all of 128 one after the other: 6.6 us, so 5.1)
template <int TYPE>
__global__ void __launch_bounds__(ST) k_scores_join(ScoreJob J) {
  __shared__ u64 lds_best[ST / 64][64];
  __shared__ float lds_sums[ST / 64][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (long long row = blockIdx.x; row < J.rows; row += gridDim.x) {
    Label label = {false, 0.0f};
    if (wave == 0) label = label_of<TYPE>(J, row);
    Sums a{LOWEST, 0.0f, 0.0f};
    if ((int)threadIdx.x < J.parts) {
      const CNN_GLOBAL float* p = J.part_sums + (row * J.parts + threadIdx.x) * 4;
      a = Sums{p[0], p[1], p[2]};
    }
    join_lanes<64>(a);
    u64 list = 0;
    if (J.n_top)
      for (int p0 = wave; p0 < J.parts; p0 += JOINED * ST / 64) {
        u64 k[JOINED];
#pragma unroll
        for (int u = 0; u < JOINED; ++u) {
          const int part = p0 + u * (ST / 64);
          k[u] = part < J.parts && 63 - lane < J.n_top ? J.part_best[(row * J.parts + part) * J.n_top + 63 - lane] : 0;
        }
        // (unrolled, or joined in pairs: no faster)
#pragma unroll 1
        for (int u = 0; u < JOINED && p0 + u * (ST / 64) < J.parts; ++u) {
          list = best_of<0>(list, k[0]);
#pragma unroll
          for (int i = 0; i + 1 < JOINED; ++i) k[i] = k[i + 1];
        }
      }
    __syncthreads();
    if (lane == 0) { lds_sums[wave][0] = a.m; lds_sums[wave][1] = a.s; lds_sums[wave][2] = a.t; }
    lds_best[wave][lane] = list;
    __syncthreads();
    if (wave != 0) continue;
    a = Sums{LOWEST, 0.0f, 0.0f};
    if (lane < ST / 64) a = Sums{lds_sums[lane][0], lds_sums[lane][1], lds_sums[lane][2]};
    join_lanes<64>(a);
    if (J.n_top) {
#pragma unroll 1
      for (int o = 1; o < ST / 64; ++o) list = best_of<0>(list, lds_best[o][63 - lane]);
    }
    if (J.n_top) list = with_masked<TYPE>(J, row, list);
    give_row(J, row, lane, a, rest_of(a), label, list);
  }
}

// Rows of at most L classes, L = 16, 32 or 64: a lane a class, 64 / L rows a wavefront.
template <int TYPE, int L>
__global__ void __launch_bounds__(ST) k_scores_few(ScoreJob J) {
  typedef Element<TYPE> E;
  const int c = threadIdx.x & (L - 1);
  const long long all = (J.rows + ST / L - 1) / (ST / L) * (ST / L);   // (lanes of a wavefront stay together)
  for (long long row = (long long)blockIdx.x * (ST / L) + threadIdx.x / L; row < all; row += (long long)gridDim.x * (ST / L)) {
    const bool is = row < J.rows && c < J.classes;
    const int l = row < J.rows && J.log_probs ? J.labels[row] : -1;
    const float x = is ? E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + c]) : -INFINITY;
    float m = fmaxf(x, LOWEST);
    for_distances<L>([&](auto d) { m = fmaxf(m, xor_lane<decltype(d)::value>(m)); });
    const float d = (x - m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
    Sums a{m, e, e * fmaxf(d, FAR)};
    for_distances<L>([&](auto o) {
      a.s += xor_lane<decltype(o)::value>(a.s);
      a.t += xor_lane<decltype(o)::value>(a.t);
    });
    u64 k = is ? key_of_any(x, c) : 0;
    if (J.n_top) k = sort_lanes<L, 0>(k);
    Label label = {l >= 0 && l < J.classes, 0.0f};
    label.x = __shfl(x, ((int)threadIdx.x & ~(L - 1) & 63) + (label.is ? l : 0));
    const float one[1] = {x}, rest = rest_of<L>(a, one);
    if (row < J.rows) give_row(J, row, c, a, rest, label, k);
  }
}

// Rows of up to 16 L classes: L lanes a row, 16 classes a lane, place (k / V) L V + l V + k % V lane l's k-th.  The best come one
// by one: the largest value left, its lowest place, which then is no number.
template <int TYPE, int L>
__global__ void __launch_bounds__(ST) k_scores_rows(ScoreJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = 16 / V;
  const int l = threadIdx.x & (L - 1);
  const long long all = (J.rows + ST / L - 1) / (ST / L) * (ST / L);   // (lanes of a wavefront stay together)
  for (long long row = (long long)blockIdx.x * (ST / L) + threadIdx.x / L; row < all; row += (long long)gridDim.x * (ST / L)) {
    const bool is = row < J.rows;
    Label label = {false, 0.0f};
    if (is && l == 0) label = label_of<TYPE>(J, row);
    const CNN_GLOBAL T* from = (const CNN_GLOBAL T*)J.x + (is ? row : 0) * J.stride;
    v4u r[N];
#pragma unroll
    for (int q = 0; q < N; ++q) r[q] = load16<TYPE>(from, (q * L + l) * V, is ? J.classes : 0);
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = E::get(r[k / V], k % V);
    Sums a{LOWEST, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 16; k += 2) a.m = max3(a.m, x[k], x[k + 1]);
    for_distances<L>([&](auto d) { a.m = fmaxf(a.m, xor_lane<decltype(d)::value>(a.m)); });
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float d = (x[k] - a.m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
      a.s += e;
      a.t = fmaf(e, fmaxf(d, FAR), a.t);
    }
    for_distances<L>([&](auto d) {
      a.s += xor_lane<decltype(d)::value>(a.s);
      a.t += xor_lane<decltype(d)::value>(a.t);
    });
    const Row sums = give_sums(J, row, is && l == 0, a, rest_of<L>(a, x), label);
    if (!J.n_top) continue;
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if ((k / V) * L * V + l * V + k % V >= J.classes) x[k] = __builtin_nanf("");
#pragma unroll 1
    for (int i = 0; i < J.n_top; ++i) {
      float best = -INFINITY;
#pragma unroll
      for (int k = 0; k < 16; k += 2) best = max3(best, x[k], x[k + 1]);
      for_distances<L>([&](auto d) { best = fmaxf(best, xor_lane<decltype(d)::value>(best)); });
      int at = 0x7fffffff;
#pragma unroll
      for (int k = 15; k >= 0; --k) at = x[k] == best ? (k / V) * L * V + k % V : at;
      at = at == 0x7fffffff ? at : at + l * V;
      for_distances<L>([&](auto d) { at = min(at, (int)xor_word<decltype(d)::value>((unsigned)at)); });
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = at - l * V == (k / V) * L * V + k % V ? __builtin_nanf("") : x[k];
      if (is && l == 0) {
        if (J.top) J.top[row * J.n_top + i] = sums.none ? -1 : at;
        if (J.top_log_probs) J.top_log_probs[row * J.n_top + i] = sums.none ? sums.m : log_prob(sums, best);
      }
    }
  }
}

// ---- the gradient ----
struct GradRow {
  float m, log_s;
  float a, b;      // -p (a + b log p), a without the label's gradient: b H
  float g_label;
  int label;       // -1: none
  bool empty;
};
__device__ __forceinline__ GradRow grad_row(const ScoreGradJob& J, long long row) {
  GradRow r;
  r.m = J.normaliser[2 * row];
  r.log_s = J.normaliser[2 * row + 1];
  r.empty = r.m == -INFINITY;
  const int label = J.labels && J.g_log_probs ? J.labels[row] : -1;
  const bool has = label >= 0 && label < J.classes;
  r.label = has ? label : -1;
  r.g_label = has ? J.g_log_probs[row] : 0.0f;
  r.b = J.g_entropy ? J.g_entropy[row] : 0.0f;
  r.a = J.g_entropy ? r.b * J.entropy[row] : 0.0f;
  return r;
}
// of one class; a class of probability zero has none but its label's (so has one below 2^-126: the exponential gives no subnormal numbers)
__device__ __forceinline__ float grad_of(const GradRow& r, float with_label, float x) {   // (with_label: a + g_label)
  const float log_p = (x - r.m) - r.log_s, p = __builtin_amdgcn_exp2f(log_p * LOG2E);
  const float g = p == 0.0f ? 0.0f : -p * fmaf(r.b, log_p, with_label);
  return r.empty ? 0.0f : g;
}
// of the label's: 1 - p by its series where p is close to 1 and the difference would keep few digits
__device__ __forceinline__ float grad_of_label(const GradRow& r, float x) {
  const float y = (x - r.m) - r.log_s, p = __builtin_amdgcn_exp2f(y * LOG2E);
  float series = fmaf(y, 1.0f / 720, 1.0f / 120);
  series = fmaf(y, series, 1.0f / 24);
  series = fmaf(y, series, 1.0f / 6);
  series = fmaf(y, series, 0.5f);
  series = fmaf(y, series, 1.0f);
  const float others = y > -0.25f ? -y * series : 1.0f - p;
  const float g = r.g_label * others - (p == 0.0f ? 0.0f : p * fmaf(r.b, y, r.a));
  return r.empty ? 0.0f : g;
}

// of 16 bytes, places c .. of g, which begins with class `first` and ends before place `end`
template <int TYPE>
__device__ __forceinline__ void put_gradients(const GradRow& r, v4u in, CNN_GLOBAL typename Element<TYPE>::T* g, int c, int end, int first) {
  typedef Element<TYPE> E;
  typename E::T e[E::V];
  v4u v = {0, 0, 0, 0};
  const float with_label = r.a + r.g_label;
#pragma unroll
  for (int j = 0; j < E::V; ++j) e[j] = E::make(grad_of(r, with_label, E::get(in, j)));
  const int at = r.label - first - c;
  if (r.label >= 0 && (unsigned)at < (unsigned)E::V) {
    float x = 0.0f;
#pragma unroll
    for (int j = 0; j < E::V; ++j) x = at == j ? E::get(in, j) : x;
    const typename E::T g_label = E::make(grad_of_label(r, x));
#pragma unroll
    for (int j = 0; j < E::V; ++j) e[j] = at == j ? g_label : e[j];
  }
#pragma unroll
  for (int j = 0; j < E::V; ++j) E::put(v, j, e[j]);
  if (c + E::V <= end) *(CNN_GLOBAL v4u_any*)(g + c) = v;
  else {
#pragma unroll
    for (int j = 0; j < E::V; ++j)
      if (c + j < end) g[c + j] = e[j];
  }
}

// L lanes a row of up to 16 L classes, as k_scores_rows
template <int TYPE, int L>
__global__ void __launch_bounds__(ST) k_scores_grad_rows(ScoreGradJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = 16 / V;
  const int l = threadIdx.x & (L - 1);
  for (long long row = (long long)blockIdx.x * (ST / L) + threadIdx.x / L; row < J.rows; row += (long long)gridDim.x * (ST / L)) {
    const CNN_GLOBAL T* x = (const CNN_GLOBAL T*)J.x + row * J.stride;
    CNN_GLOBAL T* g = (CNN_GLOBAL T*)J.grad + row * J.grad_stride;
    v4u in[N];
#pragma unroll
    for (int q = 0; q < N; ++q) in[q] = load16<TYPE>(x, (q * L + l) * V, J.classes);
    const GradRow r = grad_row(J, row);
#pragma unroll
    for (int q = 0; q < N; ++q) put_gradients<TYPE>(r, in[q], g, (q * L + l) * V, J.classes, 0);
  }
}

// A wavefront a tile, row after row.  us with 8192 workgroups that go from row to row, the next one's values under way, / a workgroup
// for four tiles of one row / so: 2000 rows of 50001 fp16 classes 79.4 / 78.1 / 77.9, 2048 of 131072 bf16 193.8 / 180 / 187, of fp32 392 /
// 373 / 373, 20000 of 5000 bf16 101 / 104 / 79, of fp32 186 / 176 / 144, 150000 of 1500 bf16 - / 258 / 192.  (Rows that start at odd
// addresses take 4 % longer, tiles that begin with 16 whole bytes or not.)
template <int TYPE>
__global__ void __launch_bounds__(ST) k_scores_grad(ScoreGradJob J, unsigned tiles, unsigned units) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = 16 / V;
  const int lane = threadIdx.x & 63;
  for (unsigned unit = blockIdx.x * (ST / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += gridDim.x * (ST / 64)) {
    const long long row = unit / tiles;
    const int first = (int)(unit % tiles) * SCORE_TILE, end = J.classes - first;
    const CNN_GLOBAL T* x = (const CNN_GLOBAL T*)J.x + row * J.stride + first;
    CNN_GLOBAL T* g = (CNN_GLOBAL T*)J.grad + row * J.grad_stride + first;
    v4u in[N];
#pragma unroll
    for (int q = 0; q < N; ++q) in[q] = load16<TYPE>(x, (q * 64 + lane) * V, end);
    const GradRow r = grad_row(J, row);
#pragma unroll
    for (int q = 0; q < N; ++q) put_gradients<TYPE>(r, in[q], g, (q * 64 + lane) * V, end, first);
  }
}

constexpr long long GRID_MOST = 1 << 20;   // workgroups of a launch at most: rows beyond are looped over
unsigned grid_of(long long work, long long per) { return (unsigned)std::min((work + per - 1) / per, GRID_MOST); }

int lanes_of(int items) {   // the power of two
  int l = 1;
  while (l < items) l <<= 1;
  return l;
}

// One wavefront a row, four or eight: they share what is read, but each picks out its own best, and the lists have to be joined.
// Eight are for rows that leave compute units idle (16: no faster).
// us of one / four with 20 best, bf16: 512 rows of 8192 classes 12.3 / 10.0, 1000 12.5 / 12.7, 2048 15 / 22, 20000 91 / 186; 4096 rows
// of 32768 65 / 78, 1024 27 / 22; of 131072 4096 rows 209 / 218, 5000 (one of two rounds a fifth full) 305 / 264.  Without best, fp32:
// 20000 rows of 4096 59 / 64, of 8192 113 / 109, of 32768 473 / 437.
// us of four / eight, 20 best of bf16: one row of 8192 7.6 / 7.8, 16384 8.7 / 8.4, 32768 10.9 / 10.1, 50000 14.1 / 11.7; 250 rows of
// 131072 26.7 / 21.8, 512 36.0 / 35.5, 600 43 / 50; one row of 50000 without best 7.7 / 5.7.
int wavefronts_of(const ScoreJob& J) {
  const int tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE;
  if (J.parts > 1) return 4;
  if (tiles <= 4 || (J.n_top && ((tiles <= 8 && J.rows > 512) || (tiles <= 32 && J.rows >= 4096)))) return 1;
  return tiles > 8 && J.rows <= 256 ? 8 : 4;
}

template <int TYPE, int WAVES>
hipError_t launch_scores_waves(hipStream_t stream, const ScoreJob& J) {
  const dim3 grid(grid_of(J.rows, threads_of(WAVES) / 64 / WAVES), (unsigned)J.parts), threads(threads_of(WAVES));
  const bool h = J.entropy, top = J.n_top;
  if (h && top) hipLaunchKernelGGL((k_scores<TYPE, WAVES, true, true>), grid, threads, 0, stream, J);
  else if (h) hipLaunchKernelGGL((k_scores<TYPE, WAVES, true, false>), grid, threads, 0, stream, J);
  else if (top) hipLaunchKernelGGL((k_scores<TYPE, WAVES, false, true>), grid, threads, 0, stream, J);
  else hipLaunchKernelGGL((k_scores<TYPE, WAVES, false, false>), grid, threads, 0, stream, J);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || J.parts == 1) return e;
  hipLaunchKernelGGL(k_scores_join<TYPE>, dim3(grid_of(J.rows, 1)), dim3(ST), 0, stream, J);
  return hipGetLastError();
}

#define CNN355_LANES(kernel, lanes)                                                                                   \
  switch (lanes) {                                                                                                    \
    case 1: hipLaunchKernelGGL((kernel<TYPE, 1>), dim3(grid_of(J.rows, ST)), dim3(ST), 0, stream, J); break;          \
    case 2: hipLaunchKernelGGL((kernel<TYPE, 2>), dim3(grid_of(J.rows, ST / 2)), dim3(ST), 0, stream, J); break;      \
    case 4: hipLaunchKernelGGL((kernel<TYPE, 4>), dim3(grid_of(J.rows, ST / 4)), dim3(ST), 0, stream, J); break;      \
    case 8: hipLaunchKernelGGL((kernel<TYPE, 8>), dim3(grid_of(J.rows, ST / 8)), dim3(ST), 0, stream, J); break;      \
    case 16: hipLaunchKernelGGL((kernel<TYPE, 16>), dim3(grid_of(J.rows, ST / 16)), dim3(ST), 0, stream, J); break;   \
    case 32: hipLaunchKernelGGL((kernel<TYPE, 32>), dim3(grid_of(J.rows, ST / 32)), dim3(ST), 0, stream, J); break;   \
    default: hipLaunchKernelGGL((kernel<TYPE, 64>), dim3(grid_of(J.rows, ST / 64)), dim3(ST), 0, stream, J); break;   \
  }

// Whether the best of rows of up to 1024 classes come one by one (k_scores_rows) or sorted.  One by one they cost a row n_top
// rounds of the lanes that share it, and few rows the rounds' latency.  us one by one / sorted: 100000 rows of 1000 bf16 5 best
// 140 / 175, 16 best 327 / 199; of 100 5 best 22 / 172, fp32 64 best 138 / 247; of 64 16 best 27 / 48, fp32 64 best 89 / 49; of 16 all
// 21 / 11; 300 rows of 300 bf16 16 best 11.6 / 9.1, 5 best the same.
bool one_by_one(const ScoreJob& J) {
  if (J.classes > SCORE_TILE) return false;
  const int round = J.n_top * lanes_of((J.classes + 15) / 16);
  return round <= 512 && (J.n_top <= 8 || (J.rows >= 4096 && 2 * J.classes > 3 * J.n_top));
}

template <int TYPE>
hipError_t launch_scores_type(hipStream_t stream, const ScoreJob& J) {
  if (one_by_one(J)) {
    CNN355_LANES(k_scores_rows, lanes_of((J.classes + 15) / 16))
  } else if (J.classes > 64) {
    switch (wavefronts_of(J)) {
      case 1: return launch_scores_waves<TYPE, 1>(stream, J);
      case 4: return launch_scores_waves<TYPE, 4>(stream, J);
      default: return launch_scores_waves<TYPE, 8>(stream, J);
    }
  } else {
    switch (lanes_of(J.classes)) {   // (more than 8 best)
      case 16: hipLaunchKernelGGL((k_scores_few<TYPE, 16>), dim3(grid_of(J.rows, ST / 16)), dim3(ST), 0, stream, J); break;
      case 32: hipLaunchKernelGGL((k_scores_few<TYPE, 32>), dim3(grid_of(J.rows, ST / 32)), dim3(ST), 0, stream, J); break;
      default: hipLaunchKernelGGL((k_scores_few<TYPE, 64>), dim3(grid_of(J.rows, ST / 64)), dim3(ST), 0, stream, J); break;
    }
  }
  return hipGetLastError();
}

template <int TYPE>
hipError_t launch_scores_grad_type(hipStream_t stream, const ScoreGradJob& J) {
  if (J.classes <= SCORE_TILE) {
    CNN355_LANES(k_scores_grad_rows, lanes_of((J.classes + 15) / 16))
  } else {
    const long long tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE, units = J.rows * tiles;
    if (units > 1ll << 31) return hipErrorInvalidValue;   // (no memory holds so many)
    hipLaunchKernelGGL(k_scores_grad<TYPE>, dim3(grid_of(units, ST / 64)), dim3(ST), 0, stream, J, (unsigned)tiles, (unsigned)units);
  }
  return hipGetLastError();
}

}  // namespace

// How rows are shared where there are too few of them to fill the chip: parts of eight tiles or more, for two workgroups a compute
// unit at most; they cost a second launch that waits for the first.  us in parts / by one workgroup a row, 20 best of bf16: one row
// of 50000 classes 14.1 / 12.6, 65536 13.7 / 12.6, 80000 14.1 / 15.1, 131072 14.2 / 18.5, 1000000 20.6 / 86; of 131072 64 rows 17.0 / 19.5,
// 110 19.1 / 19.6, 180 23.6 / 20.9, 250 25.7 / 21.7.  Without best one row of 50000 takes 9.6 / 8.9, 131072 of fp32 13.1 / 10.9, of bf16
// 22.3 / 25.0 (with the wait for it), 200000 22.3 / 29.0.  Parts of 16 tiles by eight wavefronts: one row of 131072 13.9, 64 17.2.
void score_parts(long long rows, int classes, int n_top, int* parts, int* part_tiles) {
  const int tiles = (classes + SCORE_TILE - 1) / SCORE_TILE;
  *parts = 1;
  *part_tiles = tiles;
  if (rows >= 128 || tiles <= (n_top ? 64 : 100)) return;
  const long long want = std::min<long long>({(512 + rows - 1) / rows, (tiles + 7) / 8, SCORE_PARTS});
  *part_tiles = (int)((tiles + want * 4 - 1) / (want * 4)) * 4;
  *parts = (tiles + *part_tiles - 1) / *part_tiles;
}

hipError_t launch_scores(hipStream_t stream, const ScoreJob& J) {
  switch (J.type) {
    case ELEMENT_F32: return launch_scores_type<ELEMENT_F32>(stream, J);
    case ELEMENT_BF16: return launch_scores_type<ELEMENT_BF16>(stream, J);
    case ELEMENT_F16: return launch_scores_type<ELEMENT_F16>(stream, J);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_scores_grad(hipStream_t stream, const ScoreGradJob& J) {
  switch (J.type) {
    case ELEMENT_F32: return launch_scores_grad_type<ELEMENT_F32>(stream, J);
    case ELEMENT_BF16: return launch_scores_grad_type<ELEMENT_BF16>(stream, J);
    case ELEMENT_F16: return launch_scores_grad_type<ELEMENT_F16>(stream, J);
  }
  return hipErrorInvalidValue;
}

}  // namespace cnn355
