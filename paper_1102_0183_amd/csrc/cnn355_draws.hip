// Classes drawn by their probabilities.  For a row x of sums with m = max x and temperature T: w_j = exp((x_j - m) / T); the
// ranking by x is cut short by top-k (a count), top-p (a share of the mass that top-k leaves) and min-p (a bound of w), and of
// what is left the class is drawn at which the sum of w, in the order of the indices, first is above u times the whole.
//
// A class comes out right only if sums at borders do: among 131072 classes borders lie 1e-5 of the whole apart and closer, so w
// and its sums are double, or whole numbers of 2^-51 where their order is not fixed (an error of 1e-7 would draw another class every hundred rows).  An exponential is a table of 256
// powers of two in LDS and a polynomial of three terms, off by 1.4e-13 at most: 10 operations in double, at the rate of those in
// float.
//
// Rows of up to 64 classes: a lane a class, ranks and masses by looking at every other lane; up to 1024: a wavefront a row, in
// registers.  Longer ones: a workgroup a row.  It goes over the row once and leaves the largest sum of every block of 8 to 512 classes,
// and its mass where all classes count.  Mostly few classes are left: they are among those from a bound on that the blocks' largest
// sums give, are asked for again, and a list of up to 512 is sorted, one of up to 2048 searched.  Where more are left, a second launch
// finds the border by counts.
//
// What bounds it: 512 rows of 131072 bf16 (26 us of memory) take 26 us for the best class alone, 41 with top-k 50 and top-p 0.9, 63 without a
// cut (the exponentials' double operations); top-p 0.9 of steeper and flatter rows 75 and 208; flat rows, of which top-p leaves most
// classes, 403.  Those are gone over four times more, a compute unit each: counts bound by vector issue (17 us a time and row), exponentials (40).
#include <hip/hip_runtime.h>

#include <algorithm>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"
#include "cnn355_lanes.h"

namespace cnn355 {

namespace {

typedef unsigned long long u64;
constexpr double NOTHING = -700.0;   // exp of less counts as 0

// a float's order as a whole number's
__device__ __forceinline__ int order_of(float v) {
  const int b = __builtin_bit_cast(int, v + 0.0f);   // (-0 as 0)
  return b ^ (b >> 31 & 0x7fffffff);
}

// ---- what a row asks for ----
struct Settings {
  double T, c, low;      // temperature, 256 / (T ln 2), x - m below which w is 0
  double p, bound;       // top-p; x - m from which on min-p lets a class stay
  double u;
  int k;                 // classes that top-k lets stay, at most
  bool bad, best;        // no distribution; the best class alone
  bool by_p, by_min;
};

__device__ __forceinline__ Settings settings_of(const DrawJob& J, long long row) {
  Settings s;
  const float T = J.temperature ? J.temperature[row] : 1.f, p = J.top_p ? J.top_p[row] : 1.f, q = J.min_p ? J.min_p[row] : 0.f, u = J.u[row];
  const int k = J.top_k ? J.top_k[row] : 0;
  s.bad = !(T >= 0.f) || p != p || q != q || u != u;
  s.k = k <= 0 || k > J.classes ? J.classes : k;
  s.best = T == 0.f || s.k == 1 || p <= 0.f;
  s.T = T == 0.f || s.bad ? 1.0 : T == __builtin_inff() ? 1e60 : (double)T;   // (infinite: |x - m| / T is nothing beside 1)
  s.c = 256.0 * 1.4426950408889634074 / s.T;
  s.low = NOTHING * s.T;
  s.by_p = p < 1.f;
  s.p = p;
  s.by_min = q > 0.f;
  s.bound = s.by_min ? s.T * log((double)(q < 1.f ? q : 1.f)) : -1e300;
  s.u = u < 0.f ? 0.0 : u < 1.f ? (double)u : 1.0;
  return s;
}

// exp(t / T), NOTHING <= t / T <= 0, added to `sum`: 2^(k / 256) 2^(f / 256) with |f| <= 1/2, the first from a table and an exponent,
// the second by its series
constexpr int POWERS = 256;
__device__ __forceinline__ double exp_of(double t, double c, const double* table, double sum = 0.0) {
  constexpr double MAGIC = 6755399441055744.0;   // 1.5 2^52: what is added to it is rounded to a whole number
  constexpr double L = 0.69314718055994530942 / POWERS;
  const double z = __builtin_fma(t, c, MAGIC);
  const int k = (int)__builtin_bit_cast(u64, z);
  const double f = __builtin_fma(t, c, -(z - MAGIC));
  const double series = __builtin_fma(__builtin_fma(__builtin_fma(f, L * L * L / 6, L * L / 2), f, L), f, 1.0);
  return __builtin_fma(__builtin_ldexp(table[k & (POWERS - 1)], k >> 8), series, sum);
}
__device__ __forceinline__ void fill_table(double* table, int threads) {
  for (int i = threadIdx.x; i < POWERS; i += threads) table[i] = exp2(i / (double)POWERS);
}
__device__ __forceinline__ double weight_of(double t, const Settings& s, const double* table) {
  return t < s.low ? 0.0 : exp_of(t, s.c, table);
}
// A w in units of 2^-51, 1 at least if it is not 0: sums of up to 2048 of them, in any order, are off by 4.5e-13 at most.
constexpr double UNIT = 0x1p-51;
__device__ __forceinline__ u64 units_of(double w) {
  const u64 units = __builtin_bit_cast(u64, __builtin_fma(w, 1 / UNIT, 0x1p52)) & 0xfffffffffffffull;
  return w > 0.0 && !units ? 1 : units;
}

// ---- between lanes ----
template <int D>
__device__ __forceinline__ double xor_lane(double v) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(double, (u64)xor_word<D>((unsigned)(b >> 32)) << 32 | xor_word<D>((unsigned)b));
}
template <int D>
__device__ __forceinline__ u64 xor_lane(u64 v) { return (u64)xor_word<D>((unsigned)(v >> 32)) << 32 | xor_word<D>((unsigned)v); }
template <int D>
__device__ __forceinline__ float xor_lane(float v) { return __builtin_bit_cast(float, xor_word<D>(__builtin_bit_cast(unsigned, v))); }
template <int D>
__device__ __forceinline__ int xor_lane(int v) { return (int)xor_word<D>((unsigned)v); }

// f(v, the other lane's) over groups of 2^log2 lanes
template <class T, class F>
__device__ __forceinline__ T over_lanes(T v, int log2, F f) {
  if (log2 > 0) v = f(v, xor_lane<1>(v));
  if (log2 > 1) v = f(v, xor_lane<2>(v));
  if (log2 > 2) v = f(v, xor_lane<4>(v));
  if (log2 > 3) v = f(v, xor_lane<8>(v));
  if (log2 > 4) v = f(v, xor_lane<16>(v));
  if (log2 > 5) v = f(v, xor_lane<32>(v));
  return v;
}
template <class T> __device__ __forceinline__ T sum_over(T v, int log2 = 6) { return over_lanes(v, log2, [](T a, T b) { return a + b; }); }
template <class T> __device__ __forceinline__ T most_over(T v, int log2 = 6) { return over_lanes(v, log2, [](T a, T b) { return a < b ? b : a; }); }

// v of the lane that CTRL says, 0 where there is none or the lane's row is not among ROWS
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned moved(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true); }
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 v) { return (u64)moved<CTRL, ROWS>((unsigned)(v >> 32)) << 32 | moved<CTRL, ROWS>((unsigned)v); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) { return __builtin_bit_cast(double, moved<CTRL, ROWS>(__builtin_bit_cast(u64, v))); }

// sums over the wavefront's lanes up to this one
template <class T>
__device__ __forceinline__ T sum_up_to(T v) {
  v += moved<0x111, 0xf>(v);   // one lane up in a row of 16, two, four, eight
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);   // the last lane of rows 0 and 2 to rows 1 and 3, and of row 1 to rows 2 and 3
  v += moved<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ double of_lane(double v, int lane) {
  const u64 b = __builtin_bit_cast(u64, v);
  const unsigned hi = __builtin_amdgcn_readlane((int)(b >> 32), lane), lo = __builtin_amdgcn_readlane((int)b, lane);
  return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}
// the sum of the lanes before this one
__device__ __forceinline__ double sum_before_lane(double up_to) {
  const double v = __shfl_up(up_to, 1);
  return (threadIdx.x & 63) == 0 ? 0.0 : v;
}

// ---- rows of up to 64 classes: a lane a class, `lanes` of them (a power of two) a row ----
template <int TYPE>
__global__ __launch_bounds__(256) void k_draw_lanes(DrawJob J, int lanes_log2) {
  typedef Element<TYPE> E;
  const int lanes = 1 << lanes_log2, lane = threadIdx.x & 63, mine = lane & (lanes - 1);
  const long long per = 64 >> lanes_log2, stride = (long long)gridDim.x * (blockDim.x >> 6) * per;
  const u64 group = (lanes == 64 ? ~0ull : (1ull << lanes) - 1) << (lane - mine);
  for (long long r0 = ((long long)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6)) * per; r0 < J.rows; r0 += stride) {
    const long long at = r0 + (lane >> lanes_log2), row = at < J.rows ? at : J.rows - 1;
    const Settings s = settings_of(J, row);
    const bool here = mine < J.classes;
    const float x = here ? E::get(((const CNN_GLOBAL typename E::T*)J.x + row * J.stride)[mine]) : -__builtin_inff();
    const bool bad = s.bad || (__ballot(x != x || x == __builtin_inff()) & group) != 0;
    const float m = most_over(x, lanes_log2);
    const bool empty = m == -__builtin_inff();
    const double t = empty ? -1e300 : (double)x - (double)m, d = t / s.T;
    const double w = d < NOTHING ? 0.0 : exp(d);
    const int first = __ffsll(__ballot(x == m && here) & group) - 1;   // (of the wavefront's lanes)
    bool kept = here && (lane == first || !s.by_min || t >= s.bound);
    if (s.best) kept = lane == first;
    // the lanes ranked before this one, their number and mass
    if (__ballot(!s.best && (s.k < J.classes || s.by_p))) {
      int rank = 0;
      double before = 0.0;
      for (int d = 1; d < lanes; ++d) {
        const int o = lane ^ d;
        const float xo = __shfl(x, o);
        const double wo = __shfl(w, o);
        if (xo > x || (xo == x && o < lane)) {
          ++rank;
          before += wo;
        }
      }
      const double mass = sum_over(here && rank < s.k ? w : 0.0, lanes_log2);
      if (rank >= s.k || (s.by_p && rank > 0 && !(before < s.p * mass))) kept = false;
    }
    const double held = kept ? s.best ? 1.0 : w : 0.0;
    double up_to = held;
    for (int d = 1; d < lanes; d <<= 1) {
      const double o = __shfl_up(up_to, d);
      if (mine >= d) up_to += o;
    }
    const double sum = __shfl(up_to, lane | (lanes - 1));
    const u64 fits = __ballot(held > 0.0 && up_to > s.u * sum) & group, any = __ballot(held > 0.0) & group;
    const int got = fits ? __ffsll(fits) - 1 : any ? 63 - __clzll(any) : lane;
    const double log_p = __shfl(s.best ? 0.0 : d, got) - (s.best ? 0.0 : log(sum));
    if (mine == 0 && at < J.rows) {
      J.drawn[row] = bad || empty ? -1 : got & (lanes - 1);
      if (J.log_probs) J.log_probs[row] = bad ? __builtin_nanf("") : empty ? -__builtin_inff() : (float)log_p;
    }
  }
}

// The order of a value of this type in whole numbers that follow each other more closely: without the bits that it does not have.
template <int TYPE> constexpr int SPARE_BITS = TYPE == ELEMENT_BF16 ? 16 : TYPE == ELEMENT_F16 ? 13 : 0;
template <int TYPE>
__device__ __forceinline__ int rank_of(float v) { return order_of(v) >> SPARE_BITS<TYPE>; }
template <int TYPE>
__device__ __forceinline__ float of_rank(int r) {
  const int o = r < 0 ? ~(~r << SPARE_BITS<TYPE>) : r << SPARE_BITS<TYPE>;
  return __builtin_bit_cast(float, o ^ (o >> 31 & 0x7fffffff));
}
// between two of them: halfway between the values at first, then halfway between the orders
template <int TYPE>
__device__ __forceinline__ int between(int low, int high, int step) {
  const int half = (int)((unsigned)low + ((unsigned)high - (unsigned)low) / 2);
  if (step >= 10) return half;
  const int mid = rank_of<TYPE>(0.5f * of_rank<TYPE>(low) + 0.5f * of_rank<TYPE>(high));
  return mid > low && mid < high ? mid : half;
}

// ---- rows of up to 1024 classes: a wavefront a row, 8 CHUNKS classes a lane, class 512 c + 8 lane + j its number 8 c + j ----
// A border is looked for between the smallest and the largest of the values by halves, with a count (a ballot a class) or a mass of those from
// a bound on, until one class, or one value, is left between the bounds.
template <int TYPE, int CHUNKS>
__global__ __launch_bounds__(256) void k_draw_wave(DrawJob J) {
  typedef Element<TYPE> E;
  constexpr int N = 8 * CHUNKS;
  __shared__ double table[POWERS];
  fill_table(table, 256);
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); row < J.rows; row += (long long)gridDim.x * 4) {
    const CNN_GLOBAL typename E::T* x = (const CNN_GLOBAL typename E::T*)J.x + row * J.stride;
    float v[N];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int h = 0; h < 8; h += E::V) {
        const v4u r = load16<TYPE>(x, c * 512 + lane * 8 + h, J.classes);
#pragma unroll
        for (int j = 0; j < E::V; ++j) v[c * 8 + h + j] = E::get(r, j);
      }
    const Settings s = settings_of(J, row);
    bool bad = false;
    float most = v[0], least = __builtin_inff();
#pragma unroll
    for (int j = 0; j < N; ++j) {
      bad |= v[j] != v[j];
      most = fmaxf(most, v[j]);
      if (v[j] > -__builtin_inff()) least = fminf(least, v[j]);
    }
    most = most_over(most);
    const bool none = s.bad || __ballot(bad) != 0;   // (here, where all lanes are asked)
    if (none || !(__builtin_fabsf(most) < __builtin_inff())) {
      if (lane == 0) {
        J.drawn[row] = -1;
        if (J.log_probs) J.log_probs[row] = !none && most < 0.f ? -__builtin_inff() : __builtin_nanf("");
      }
      continue;
    }
    if (s.best) {
      int got = -0x7fffffff;
#pragma unroll
      for (int j = N - 1; j >= 0; --j)
        if (v[j] == most) got = -(j / 8 * 512 + lane * 8 + j % 8);
      got = -most_over(got);
      if (lane == 0) {
        J.drawn[row] = got;
        if (J.log_probs) J.log_probs[row] = 0.f;
      }
      continue;
    }
    const double m = most;
    double w[N];
#pragma unroll
    for (int j = 0; j < N; ++j) w[j] = weight_of((double)v[j] - m, s, table);
    unsigned left = 0;   // this lane's classes that are left, a bit each
#pragma unroll
    for (int j = 0; j < N; ++j) left |= v[j] > -__builtin_inff() ? 1u << j : 0;
    int n_left = sum_over((int)__popc(left));

    // step 0: top-k, step 1: top-p of what it leaves
    for (int step = 0; step < 2; ++step) {
      if (step == 0 ? s.k >= n_left : !s.by_p) continue;
      auto mass_from = [&](int bound) {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < N; ++j) sum += rank_of<TYPE>(v[j]) >= bound ? w[j] : 0.0;
        return sum_over(sum);
      };
      auto count_from = [&](int bound) {
        int n = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) n += __popcll(__ballot((left >> j & 1) && rank_of<TYPE>(v[j]) >= bound));
        return n;
      };
      // (what is not left has a mass of 0)
      int low = rank_of<TYPE>(-most_over(-least)), high = rank_of<TYPE>(most) + 1, n_low = n_left, n_high = 0;
      double above = 0.0;
      const double need = step ? s.p * mass_from(low) : 0.0;
      for (int i = 0; (unsigned)high - (unsigned)low > 1u && n_low - n_high > 1; ++i) {
        const int mid = between<TYPE>(low, high, i), n = count_from(mid);
        const double mass = step ? mass_from(mid) : 0.0;
        if (step ? mass >= need : n >= s.k) {
          low = mid;
          n_low = n;
        } else {
          high = mid;
          n_high = n;
          above = mass;
        }
      }
      // the value, or the one class, that is left between the bounds, and how many of these stay
      const int same = n_low - n_high;
      int border = -0x7fffffff - 1;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int r = rank_of<TYPE>(v[j]);
        if ((left >> j & 1) && r < high) border = r > border ? r : border;
      }
      border = most_over(border);
      int ties = s.k - n_high;
      if (step) {
        const double weight = weight_of((double)of_rank<TYPE>(border) - m, s, table), q = weight > 0.0 ? ceil((need - above) / weight) : 1.0;
        ties = q < 1.0 ? 1 : q < same ? (int)q : same;
      }
      int before = 0;   // classes of the border's value in front
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        unsigned equal = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) equal |= (left >> (c * 8 + j) & 1) && rank_of<TYPE>(v[c * 8 + j]) == border ? 1u << j : 0;
        const int mine = (int)__popc(equal), up_to = sum_up_to(mine);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = before + up_to - mine + __popc(equal & ((1u << j) - 1));
          const bool stays = (equal >> j & 1) ? at < ties : rank_of<TYPE>(v[c * 8 + j]) > border;
          if (!stays) {
            left &= ~(1u << (c * 8 + j));
            w[c * 8 + j] = 0.0;
          }
        }
        before += __builtin_amdgcn_readlane(up_to, 63);
      }
      n_left = n_high + ties;
    }
    double start = 0.0, before[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      double sum = 0.0;
#pragma unroll
      for (int j = c * 8; j < c * 8 + 8; ++j) {
        if (s.by_min && (double)v[j] - m < s.bound) w[j] = 0.0;
        sum += w[j];
      }
      const double up_to = sum_up_to(sum);
      before[c] = start + sum_before_lane(up_to);
      start += of_lane(up_to, 63);
    }
    const double whole = start, target = s.u * whole;
    int got = 0x7fffffff, last = -1;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      double up_to = before[c];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = c * 512 + lane * 8 + j;
        up_to += w[c * 8 + j];
        if (w[c * 8 + j] > 0.0) {
          last = at;
          if (got == 0x7fffffff && up_to > target) got = at;
        }
      }
    }
    got = -most_over(-got);
    last = most_over(last);
    if (got == 0x7fffffff) got = last;
    if (lane == 0) {
      J.drawn[row] = got;
      if (J.log_probs) J.log_probs[row] = (float)(((double)E::get(x[got]) - m) / s.T - log(whole));
    }
  }
}

// ---- longer rows ----
// What a workgroup shares: counts over values, or a list of classes and their w.
template <int THREADS, int MOST>
struct Shared {
  static constexpr int PARTS = MOST / 16;
  double table[POWERS];
  double wave_sum[THREADS / 64];
  int wave_count[THREADS / 64];
  int wave_ranks[THREADS / 64][2], pair_count[2][THREADS / 64];
  u64 pair_mass[2][THREADS / 64];
  float wave_most[THREADS / 64], wave_least[THREADS / 64];
  double before, aim;
  int chosen, last, listed, blocks;
  u64 above_mass;
  int above_count, bin, found, any;
  int part_count[PARTS], part_steps[PARTS];
  union {
    struct {
      u64 rank_mass[256];
      unsigned rank_count[256];
    };
    unsigned lane_count[PARTS][64];
    struct {
      u64 key[MOST];
      union {
        double weight[MOST];
        int block[2 * MOST];
      };
    };
  };
};

// Eight classes of a row from `at` on, -inf past the end.
template <int TYPE>
__device__ __forceinline__ void eight_of(const CNN_GLOBAL typename Element<TYPE>::T* row, int at, int classes, float (&x)[8]) {
  typedef Element<TYPE> E;
#pragma unroll
  for (int h = 0; h < 8; h += E::V) {
    const v4u r = load16<TYPE>(row, at + h, classes);
#pragma unroll
    for (int j = 0; j < E::V; ++j) x[h + j] = E::get(r, j);
  }
}

// exclusive sum of v over the workgroup's threads, and the whole
template <int THREADS, class T>
__device__ __forceinline__ T sum_before(T v, T* waves, T* whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T up_to = sum_up_to(v);
  __syncthreads();
  if (lane == 63) waves[wave] = up_to;
  __syncthreads();
  T before = __shfl_up(up_to, 1), all = 0;
  if (lane == 0) before = 0;
#pragma unroll
  for (int k = 0; k < THREADS / 64; ++k) {
    if (k == wave) before += all;
    all += waves[k];
  }
  *whole = all;
  return before;
}

// The largest sum of every block from class `begin` to `end` (whole blocks, but at the row's end), +inf where one is no number, and,
// asked for, its mass relative to that.
template <int TYPE, int THREADS, class F>
__device__ __forceinline__ void look(const CNN_GLOBAL typename Element<TYPE>::T* x, int classes, int begin, int end, int block_log2,
                                     bool masses, const Settings& s, const double* table, F result) {
  typedef Element<TYPE> E;
  constexpr int AHEAD = 4, LOADS = 8 / E::V;   // eights asked for together
  const int lanes_log2 = block_log2 - 3;
  const bool first = (threadIdx.x & ((1 << lanes_log2) - 1)) == 0;
  for (int c0 = begin; c0 < end; c0 += AHEAD * THREADS * 8) {
    v4u r[AHEAD][LOADS];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int h = 0; h < LOADS; ++h) {
        const int at = c0 + (i * THREADS + (int)threadIdx.x) * 8 + h * E::V;
        if (c0 + AHEAD * THREADS * 8 <= classes) r[i][h] = *(const CNN_GLOBAL v4u_any*)(x + at);   // (the same for all threads)
        else r[i][h] = load16<TYPE>(x, at, classes);
      }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (c0 + i * THREADS * 8 >= end) break;
      const int at = c0 + (i * THREADS + (int)threadIdx.x) * 8;
      float v[8];
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = E::get(r[i][j / E::V], j % E::V);
      float b = v[0];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        bad |= v[j] != v[j];
        b = fmaxf(b, v[j]);
      }
      b = most_over(bad ? __builtin_inff() : b, lanes_log2);
      double mass = 0.0;
      if (masses) {
        if (b > -__builtin_inff()) {
#pragma unroll
          for (int j = 0; j < 8; ++j) mass = exp_of(fmax((double)v[j] - (double)b, s.low), s.c, table, mass);
        }
        mass = sum_over(mass, lanes_log2);
      }
      if (first && at < end) result(at >> block_log2, b, mass);
    }
  }
}

// f(class, eight values from it on) over a row, the next eight of a thread asked for before; whole wavefronts call it, past the end with -inf
template <int TYPE, int THREADS, class F>
__device__ __forceinline__ void over_row(const CNN_GLOBAL typename Element<TYPE>::T* x, int classes, F f) {
  typedef Element<TYPE> E;
  // (the next loads have no condition, at the end they ask for the last eight again: behind one, the wait for them came before the work)
  constexpr int LOADS = 8 / E::V, STEP = THREADS * 8;
  const int mine = (int)threadIdx.x * 8, whole = classes / STEP, last = classes - 8;
  v4u next[LOADS], tail[LOADS];
#pragma unroll
  for (int h = 0; h < LOADS; ++h) {
    tail[h] = load16<TYPE>(x, whole * STEP + mine + h * E::V, classes);
    next[h] = *(const CNN_GLOBAL v4u_any*)(x + (mine < last ? mine : last) + h * E::V);
  }
  for (int c0 = 0; c0 < classes; c0 += STEP) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = E::get(c0 == whole * STEP ? tail[j / E::V] : next[j / E::V], j % E::V);
    const int at = c0 + STEP + mine;
#pragma unroll
    for (int h = 0; h < LOADS; ++h) next[h] = *(const CNN_GLOBAL v4u_any*)(x + (at < last ? at : last) + h * E::V);
    f(c0 + mine, v);
  }
}

// whether the masses of a row's blocks are asked for: all classes count, or top-p needs the mass of all
__device__ __forceinline__ bool masses_of(const Settings& s, int classes) { return !s.bad && !s.best && s.k == classes && (s.by_p || !s.by_min); }

// rows of few and long rows are looked at by several workgroups each, which leave the blocks' numbers in the scratch memory
template <int TYPE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_draw_look(DrawJob J) {
  __shared__ double table[POWERS];
  const long long row = blockIdx.x / J.parts;
  const int part = blockIdx.x % J.parts;
  const Settings s = settings_of(J, row);
  fill_table(table, THREADS);
  __syncthreads();
  const int each = (J.blocks + J.parts - 1) / J.parts, b0 = part * each, b1 = b0 + each < J.blocks ? b0 + each : J.blocks;
  if (b0 >= b1) return;
  const int begin = b0 << J.block_log2, end = b1 << J.block_log2 < J.classes ? b1 << J.block_log2 : J.classes;
  CNN_GLOBAL float* most = J.part_max + row * J.blocks;
  CNN_GLOBAL double* mass = J.part_mass + row * J.blocks;
  look<TYPE, THREADS>((const CNN_GLOBAL typename Element<TYPE>::T*)J.x + row * J.stride, J.classes, begin, end, J.block_log2,
                      masses_of(s, J.classes), s, table, [&](int b, float v, double w) {
                        most[b] = v;
                        mass[b] = w;
                      });
}

// A class of a list: the larger sum first, then the lower index, as whole numbers that fall.
__device__ __forceinline__ u64 key_of(float v, int index) { return (u64)((unsigned)order_of(v) ^ 0x80000000u) << 32 | (unsigned)~index; }
__device__ __forceinline__ int order_in(u64 key) { return (int)((unsigned)(key >> 32) ^ 0x80000000u); }
__device__ __forceinline__ int index_in(u64 key) { return (int)~(unsigned)key; }
__device__ __forceinline__ float value_of(int order) { return __builtin_bit_cast(float, order ^ (order >> 31 & 0x7fffffff)); }

// The first n of a list's keys in falling order.  Up to a key a thread: every thread counts the larger ones (they are read from LDS by
// all lanes at once); more: a bitonic network.
template <int THREADS, int MOST>
__device__ __forceinline__ void sort_keys(u64* key, int n) {
  const int tid = threadIdx.x;
  if (n <= THREADS) {
    const u64 mine = tid < n ? key[tid] : 0;
    const int whole = (n + 7) & ~7;
    __syncthreads();
    if (tid >= n && tid < whole) key[tid] = 0;
    __syncthreads();
    int larger = 0;
    if ((tid & ~63) < n)
      for (int j = 0; j < whole; j += 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) larger += key[j + i] > mine;
    __syncthreads();
    if (tid < n) key[larger] = mine;
    __syncthreads();
    return;
  }
  int N = 512;
  while (N < n) N *= 2;
  for (int i = n + tid; i < N; i += THREADS) key[i] = 0;
  __syncthreads();
  for (int size = 2; size <= N; size *= 2)
    for (int d = size / 2; d > 0; d /= 2) {
      for (int i = tid; i < N / 2; i += THREADS) {
        const int a = 2 * i - (i & (d - 1)), b = a + d;
        const u64 ka = key[a], kb = key[b];
        if ((ka < kb) == ((a & size) == 0)) {
          key[a] = kb;
          key[b] = ka;
        }
      }
      __syncthreads();
    }
}

// A workgroup a row.  PARTS: other workgroups have looked at it.  MANY: the rows of whose classes the first kernel finds many left (and
// marks so): the code that settles those takes the registers of another workgroup (some 200 vector registers; the first
// kernel has 86, or 111 with 256 threads).  No vector register is spilled (scalar ones go to lanes of vector registers: 59 to 76 in the second), and
// none is to be: bounded so that some were, one kernel for both gave wrong rows, which a second reading of its source did not explain either; a
// test holds the compiler to it.  Without a marked row this launch takes 4 us.
constexpr int MARK = -2;
template <int TYPE, int THREADS, int MOST, bool PARTS, bool MANY>
__global__ __launch_bounds__(THREADS) void k_draw(DrawJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  typedef Shared<THREADS, MOST> Room;
  __shared__ Room S;
  extern __shared__ double block_mass[];                     // [blocks]
  float* block_most = (float*)(block_mass + J.blocks);       // [blocks]
  int* block_ties = (int*)(block_most + J.blocks);           // [blocks]: classes of the border's value, then those in the blocks before
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long row = blockIdx.x;
  const int classes = J.classes, blocks = J.blocks, block_log2 = J.block_log2, lanes_log2 = block_log2 - 3;   // (lanes of a block)
  const CNN_GLOBAL T* x = (const CNN_GLOBAL T*)J.x + row * J.stride;
  if (MANY && J.drawn[row] != MARK) return;
  const Settings s = settings_of(J, row);
  fill_table(S.table, THREADS);
  if (tid == 0) {
    S.last = -1;
    S.chosen = 0x7fffffff;
    S.listed = S.blocks = 0;
  }
  __syncthreads();
  if constexpr (PARTS) {
    for (int b = tid; b < blocks; b += THREADS) {
      block_most[b] = J.part_max[row * blocks + b];
      block_mass[b] = J.part_mass[row * blocks + b];
    }
  } else {
    look<TYPE, THREADS>(x, classes, 0, classes, block_log2, !MANY && masses_of(s, classes), s, S.table, [&](int b, float v, double w) {
      block_most[b] = v;
      block_mass[b] = w;
    });
  }
  __syncthreads();
  float most = -__builtin_inff(), least = __builtin_inff();   // of the blocks' largest sums
  for (int b = tid; b < blocks; b += THREADS) {
    const float v = block_most[b];
    most = fmaxf(most, v);
    if (v > -__builtin_inff()) least = fminf(least, v);
  }
  most = most_over(most);
  least = -most_over(-least);
  if (lane == 0) {
    S.wave_most[wave] = most;
    S.wave_least[wave] = least;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < THREADS / 64; ++k) {
    most = fmaxf(most, S.wave_most[k]);
    least = fminf(least, S.wave_least[k]);
  }
  const bool bad = s.bad || most == __builtin_inff();
  if (!MANY && (bad || most == -__builtin_inff())) {
    if (tid == 0) {
      J.drawn[row] = -1;
      if (J.log_probs) J.log_probs[row] = bad ? __builtin_nanf("") : -__builtin_inff();
    }
    return;
  }

  if (!MANY && s.best) {   // the first class of the largest sum
    for (int b = tid; b < blocks; b += THREADS)
      if (block_most[b] == most) atomicMin(&S.chosen, b);
    __syncthreads();
    if (wave == 0) {
      const int at = (S.chosen << block_log2) + lane * 8;
      float v[8];
      int got = 0x7fffffff;
      if (lane < 1 << lanes_log2) {
        eight_of<TYPE>(x, at, classes, v);
#pragma unroll
        for (int j = 7; j >= 0; --j)
          if (v[j] == most) got = at + j;
      }
      got = -most_over(-got);
      if (lane == 0) {
        J.drawn[row] = got;
        if (J.log_probs) J.log_probs[row] = 0.f;
      }
    }
    return;
  }

  const double m = most;
  const bool all_count = s.k == classes && !s.by_p && !s.by_min;
  double top_mass = 0.0;   // of what top-k leaves
  // (where this kernel looks at the row again, it adds all up with the border's: without masses the look takes half the time)
  constexpr bool LATE = MANY && !PARTS;
  if (!LATE && s.k == classes && s.by_p) {
    double sum = 0.0;
    for (int b = tid; b < blocks; b += THREADS) sum += block_mass[b] * weight_of((double)block_most[b] - m, s, S.table);
    sum_before<THREADS>(sum, S.wave_sum, &top_mass);
  }

  // the classes that are wanted of the blocks that may hold some, by their largest sums, to the list; their number (MOST + 1 where
  // more blocks than `limit` may)
  auto list_of = [&](int limit, auto may_hold, auto wanted) {
    __syncthreads();
    if (tid == 0) S.listed = S.blocks = 0;
    __syncthreads();
    for (int b = tid; b < blocks; b += THREADS)
      if (block_most[b] > -__builtin_inff() && may_hold(block_most[b])) S.block[atomicAdd(&S.blocks, 1)] = b;
    __syncthreads();
    const int n = S.blocks, step = THREADS >> lanes_log2;
    if (n > limit) return MOST + 1;
    for (int i0 = 0; i0 < n; i0 += step) {
      const int i = i0 + (tid >> lanes_log2);
      const int at = (S.block[i < n ? i : n - 1] << block_log2) + (tid & ((1 << lanes_log2) - 1)) * 8;
      float v[8];
      eight_of<TYPE>(x, at, classes, v);
      u64 mask[8];
      int all = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mask[j] = __ballot(i < n && v[j] > -__builtin_inff() && wanted(v[j]));
        all += __popcll(mask[j]);
      }
      if (!all) continue;
      int place = 0;
      if (lane == 0) place = atomicAdd(&S.listed, all);
      place = __builtin_amdgcn_readfirstlane(place);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int to = place + __popcll(mask[j] & ((1ull << lane) - 1));
        if ((mask[j] >> lane & 1) && to < MOST) S.key[to] = key_of(v[j], at + j);
        place += __popcll(mask[j]);
      }
    }
    __syncthreads();
    return S.listed;
  };

  // Few classes left, as mostly: a list of those from a bound on that hardly more than enough classes reach.  The bound: from it on are
  // the largest sums of top_k blocks, or of blocks whose largest sums alone have the mass that top-p asks for.
  const bool by_k = s.k < classes, by_bound = s.by_min && !by_k;   // (min-p leaves nothing below its bound; top-k comes first)
  // What stays, where a row is not settled by a sorted list: classes of a higher rank than `cut`, and the first `ties` of those of this one.
  int cut = -0x7fffffff - 1, ties = 0;
  double tie_weight = 0.0;
  bool masses_there = false;   // of what stays, block by block
  if (!MANY && !all_count) {
    constexpr int PER = DRAW_BLOCKS / THREADS;
    int from = rank_of<TYPE>(-3.4028234663852886e38f), n_from = -1, held = 0;   // (held: blocks that are not switched off)
    if (by_k || s.by_p) {
      int ranks[PER];
      u64 weights[PER];
      const u64 need = (u64)(s.p * top_mass * 0x1p40) + 1;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int b = tid + i * THREADS;
        const float v = b < blocks ? block_most[b] : -__builtin_inff();
        ranks[i] = rank_of<TYPE>(v);
        weights[i] = by_k ? 0 : (u64)(weight_of((double)v - m, s, S.table) * 0x1p40);   // (rounded down: no more than there is)
      }
      // the order's range in 256 parts, the one that the bound lies in again, until it holds few blocks beyond those that are needed
      int low = rank_of<TYPE>(least), n_high = 0;
      unsigned range = (unsigned)rank_of<TYPE>(most) - (unsigned)low;
      u64 mass_high = 0;
      for (;;) {
        const int shift = range < 256 ? 0 : 24 - __clz(range);
        __syncthreads();
        for (int i = tid; i < 256; i += THREADS) {
          S.rank_count[i] = 0;
          S.rank_mass[i] = 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const unsigned at = (unsigned)ranks[k] - (unsigned)low;
          if (tid + k * THREADS < blocks && ranks[k] >= low && at <= range) {
            atomicAdd(&S.rank_count[at >> shift], 1u);
            if (!by_k) atomicAdd(&S.rank_mass[at >> shift], weights[k]);
          }
        }
        __syncthreads();
        if (wave == 0) {   // from the largest part on
          int n[4], n_all = 0;
          u64 w[4], w_all = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            n[i] = (int)S.rank_count[255 - 4 * lane - i];
            w[i] = S.rank_mass[255 - 4 * lane - i];
            n_all += n[i];
            w_all += w[i];
          }
          int count = n_high + sum_up_to(n_all) - n_all;
          u64 mass = mass_high + sum_up_to(w_all) - w_all;
          int found = -1;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (found < 0 && n[i] && (by_k ? count + n[i] >= s.k : mass + w[i] >= need)) {
              found = i;
            }
            if (found < 0) {
              count += n[i];
              mass += w[i];
            }
          }
          const u64 where = __ballot(found >= 0);
          if (where == 0) {
            if (lane == 63) {
              S.found = 0;
              S.above_count = count;
            }
          } else if (lane == __ffsll(where) - 1) {
            S.found = 1;
            S.bin = 255 - 4 * lane - found;
            S.above_count = count;
            S.above_mass = mass;
          }
        }
        __syncthreads();
        if (!S.found) {   // (in the first round only)
          held = S.above_count;
          break;
        }
        low += S.bin << shift;
        range = min(range - ((unsigned)S.bin << shift), (1u << shift) - 1);
        n_high = S.above_count;
        mass_high = S.above_mass;
        from = low;
        n_from = n_high + (int)S.rank_count[S.bin];
        if (shift == 0 || n_from - n_high <= 16 + n_high / 4) break;
      }
      __syncthreads();
    }
    // min-p's bound as a float, or one below
    const float bound = by_bound ? (float)fmax(m + s.bound, -3.4028234663852886e38) : 0.f;
    const bool by_rank = n_from >= 0;
    // (a list that will not do costs a second look: where b of B blocks of many classes hold some, about -B ln(1 - b / B) classes are meant)
    const int limit = classes <= 2 * MOST ? blocks : (int)(blocks * (1.f - expf(-(float)MOST / blocks)));
    const int n = (by_rank && n_from <= MOST) || by_bound || (by_k && !by_rank && held << block_log2 <= 4 * MOST)
                      ? list_of(limit, [&](float v) { return rank_of<TYPE>(v) >= from && !(by_bound && rank_of<TYPE>(v) < rank_of<TYPE>(bound) - 1); },
                                [&](float v) { return rank_of<TYPE>(v) >= from && !(by_bound && (double)v - m < s.bound); })
                      : MOST + 1;
    if (n <= THREADS) {
      sort_keys<THREADS, MOST>(S.key, n);
      for (int r = tid; r < n; r += THREADS) S.weight[r] = weight_of((double)value_of(order_in(S.key[r])) - m, s, S.table);
      __syncthreads();
      const int most_left = n < s.k ? n : s.k, per = (n + THREADS - 1) / THREADS, r0 = tid * per, r1 = r0 + per < most_left ? r0 + per : most_left;
      double sum = 0.0, whole;
      for (int r = r0; r < r1; ++r) sum += S.weight[r];
      double before = sum_before<THREADS>(sum, S.wave_sum, &whole);
      const double need = s.p * (by_k ? whole : top_mass);
      {
        int left = 0;
        for (int r = r0; r < r1; ++r) {
          left += r == 0 || ((!s.by_p || before < need) && (!s.by_min || (double)value_of(order_in(S.key[r])) - m >= s.bound));
          before += S.weight[r];
        }
        int end;
        sum_before<THREADS>(left, S.wave_count, &end);
        // those left, in the order of their indices
        const u64 mine = tid < end ? ~((u64)(unsigned)index_in(S.key[tid]) << 32 | (unsigned)tid) : 0;
        __syncthreads();
        if (tid < end) S.key[tid] = mine;
        __syncthreads();
        sort_keys<THREADS, MOST>(S.key, end);
        const int each = (end + THREADS - 1) / THREADS, a0 = tid * each, a1 = a0 + each < end ? a0 + each : end;
        sum = 0.0;
        for (int a = a0; a < a1; ++a) sum += S.weight[(unsigned)~S.key[a]];
        double up_to = sum_before<THREADS>(sum, S.wave_sum, &whole);
        const double target = s.u * whole;
        int got = 0x7fffffff, last = -1;
        for (int a = a0; a < a1; ++a) {
          const double w = S.weight[(unsigned)~S.key[a]];
          up_to += w;
          if (w > 0.0) {
            last = a;
            if (got == 0x7fffffff && up_to > target) got = a;
          }
        }
        got = -most_over(-got);
        last = most_over(last);
        if (lane == 0 && got != 0x7fffffff) atomicMin(&S.chosen, got);
        if (lane == 0 && last >= 0) atomicMax(&S.last, last);
        __syncthreads();
        if (tid == 0) {
          const u64 key = ~S.key[S.chosen != 0x7fffffff ? S.chosen : S.last];
          const int index = (int)(key >> 32);
          J.drawn[row] = index;
          if (J.log_probs) J.log_probs[row] = (float)(((double)E::get(x[index]) - m) / s.T - log(whole));
        }
        return;
      }
    }
    if (n > THREADS && n <= MOST) {
      // More of them than are sorted quickly: borders by halves, a count or a mass of the list's classes from a bound on at a time, and masses
      // block by block, all as whole numbers: which class comes to which thread is the wavefronts' race, and does not matter to their sums (37 rows of 50001 with top-p 0.9, mostly such lists, 53 us with two bitonic
      // sorts, so 42; 2000 of 4000 102 and 90).
      constexpr int EACH = MOST / THREADS;
      int ranks[EACH], index[EACH], lowest = 0x7fffffff;
      u64 w[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const bool in = tid + i * THREADS < n;
        const u64 key = S.key[in ? tid + i * THREADS : 0];
        const float v = value_of(order_in(key));
        ranks[i] = in ? rank_of<TYPE>(v) : -0x7fffffff;   // (below all; its negative is a whole number too)
        index[i] = index_in(key);
        w[i] = in ? units_of(weight_of((double)v - m, s, S.table)) : 0;
        lowest = in ? min(lowest, ranks[i]) : lowest;
      }
      auto least_of_all = [&](int v) {
        v = -most_over(-v);
        __syncthreads();
        if (lane == 0) S.wave_ranks[wave][0] = v;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < THREADS / 64; ++k) v = min(v, S.wave_ranks[k][0]);
        return v;
      };
      lowest = least_of_all(lowest);
      cut = lowest - 1;   // (no border: all of the list stay, and nothing below it, where top-k asked for just as many)
      double left_mass = top_mass;
      int same = 0;
      for (int step = 0; step < 2; ++step) {   // top-k, top-p
        if (step == 0 ? s.k >= n : !s.by_p) continue;
        if (step == 1 && by_k && s.k >= n) {   // (all of the list are what top-k leaves)
          u64 sum = 0;
#pragma unroll
          for (int i = 0; i < EACH; ++i) sum += w[i];
          sum_before<THREADS>(sum, S.pair_mass[1], &sum);   // (the first halving writes the other one)
          left_mass = (double)sum * UNIT;
        }
        const double need = s.p * left_mass;
        int low = lowest, high = rank_of<TYPE>(most) + 1, n_low = n, n_high = 0;
        double above = 0.0;
        for (int i = 0; (unsigned)high - (unsigned)low > 1u && n_low - n_high > 1; ++i) {
          const int mid = between<TYPE>(low, high, i);
          int count = 0;
          u64 units = 0;
#pragma unroll
          for (int k = 0; k < EACH; ++k) {
            count += __popcll(__ballot(ranks[k] >= mid));
            units += ranks[k] >= mid ? w[k] : 0;
          }
          units = sum_over(units);
          if (lane == 0) {
            S.pair_count[i & 1][wave] = count;
            S.pair_mass[i & 1][wave] = units;
          }
          __syncthreads();
          count = 0;
          units = 0;
#pragma unroll
          for (int k = 0; k < THREADS / 64; ++k) {
            count += S.pair_count[i & 1][k];
            units += S.pair_mass[i & 1][k];
          }
          const double mass = (double)units * UNIT;
          if (step ? mass >= need : count >= s.k) {
            low = mid;
            n_low = count;
          } else {
            high = mid;
            n_high = count;
            above = mass;
          }
        }
        int border = -0x7fffffff;   // the value, or the one class, that is left between the bounds
#pragma unroll
        for (int i = 0; i < EACH; ++i) border = ranks[i] < high ? max(border, ranks[i]) : border;
        border = -least_of_all(-border);
        const double weight = weight_of((double)of_rank<TYPE>(border) - m, s, S.table);
        const double q = weight > 0.0 ? ceil((need - above) / weight) : 1.0;
        const int all = n_low - n_high, some = step ? q < 1.0 ? 1 : q < all ? (int)q : all : s.k - n_high;
        if (step == 0) left_mass = above + some * weight;
        if (step && same && (border < cut || (border == cut && some >= ties))) continue;   // (within rounding of all that top-k leaves)
        cut = border;
        ties = some;
        same = all;
        tie_weight = weight;
      }
      if (same && ties == same) {   // all of them
        ties = 0;
        --cut;
      }
      if (s.by_min && ties && (double)of_rank<TYPE>(cut) - m < s.bound) ties = 0;
      u64* fixed = (u64*)block_mass;
      __syncthreads();
      for (int b = tid; b < blocks; b += THREADS) {
        fixed[b] = 0;
        block_ties[b] = 0;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (tid + i * THREADS >= n || (s.by_min && (double)of_rank<TYPE>(ranks[i]) - m < s.bound)) continue;
        if (ranks[i] > cut && w[i]) atomicAdd(&fixed[index[i] >> block_log2], w[i]);
        if (ties && ranks[i] == cut) atomicAdd(&block_ties[index[i] >> block_log2], 1);
      }
      __syncthreads();
      for (int b = tid; b < blocks; b += THREADS) block_mass[b] = (double)fixed[b] * UNIT;
      masses_there = true;
    }
  }

  if (!MANY && !masses_there && (by_k || s.by_p)) {   // the other kernel's
    if (tid == 0) J.drawn[row] = MARK;
    return;
  }
  // Many classes left.
  // step 0: the border of top-k; step 1: that of top-p
  for (int step = MANY ? 0 : 2; step < 2; ++step) {
    if (step == 0 ? !by_k : !s.by_p) continue;
    const bool counts = step == 0;
    double need = counts ? (double)s.k : s.p * top_mass;   // (LATE: of all classes, when they have been added up)
    // Counts over parts of m - x, and over parts of the one that the border lies in with those beside it, say closely where it is; the mass of
    // the classes above a few parts is added up and the classes in those are listed, which settles it.  A lane counts in a column of its own,
    // without conflicts (masses added to shared bins of LDS: 100 clocks of a wavefront for a class a lane).  A count is 16 bits, and 16 are the sum
    // of the places in the part.
    constexpr int PARTS_ = Room::PARTS, PER = PARTS_ / 64;
    const float spread = (float)fmin(fmax(fmin(40.0 * s.T, 4.0 * (m - (double)least)), 1e-30), 1e37), fine = PARTS_ / spread;
    int steps_log2 = 0;
    while (steps_log2 < 6 && (classes >> 6) + 8 <= 65535 >> (steps_log2 + 1)) ++steps_log2;
    const float steps = (float)(1 << steps_log2);
    const float end_place = (float)(PARTS_ << steps_log2);
    int c0 = 0, c1 = PARTS_ - 1, found = 0;   // coarse parts that are cut again; the part that holds the border
    float again = 1.f, scale = fine * steps, shift = 0.f, most_place = end_place - 1.f;
    bool any = true;
    // the place among the parts, in steps: below 0 above them, from end_place on below them (to the last part go all that are smaller, if there is
    // no part below it)
    auto place_of = [&](float v) { return __builtin_amdgcn_fmed3f(__builtin_fmaf(most - v, scale, -shift), -__builtin_inff(), most_place); };
    const float last_place = value_of(order_of(end_place) - 1);
    double base = 0.0, aim = need;
    for (int round = 0; round < 2 && any; ++round) {
      __syncthreads();
      for (int i = tid; i < PARTS_ * 64; i += THREADS) S.lane_count[i / 64][i % 64] = 0;
      __syncthreads();
      over_row<TYPE, THREADS>(x, classes, [&](int, const float (&v)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // (no branches: others count 0 at either end)
          const float place = place_of(v[j]), among = __builtin_amdgcn_fmed3f(place, 0.f, last_place);
          const int q = (int)among;
          const bool counted = v[j] > -__builtin_inff() && place == among;
          atomicAdd(&S.lane_count[q >> steps_log2][lane], counted ? 0x10000u + (q & ((1 << steps_log2) - 1)) : 0u);
        }
      });
      __syncthreads();
      for (int b = wave; b < PARTS_; b += THREADS / 64) {
        const unsigned here = S.lane_count[b][lane];
        const int n = sum_over((int)(here >> 16)), sums = sum_over((int)(here & 0xffff));
        if (lane == 0) {
          S.part_count[b] = n;
          S.part_steps[b] = sums;
        }
      }
      __syncthreads();
      if (wave == 0) {   // the part at which counts, or masses, reach what is aimed at
        double w[PER], sum = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          // the mass of a part's classes: that of all at their mean, and what they lie apart of it (evenly, their mean aside) adds
          const int b = lane * PER + i;
          const double n = S.part_count[b], at = b + (n > 0.0 ? S.part_steps[b] / n + 0.5 : 0.5) / steps;
          const double width = 1.0 / (fine * s.T * again), t = fmax(-(c0 + at / again) / fine, s.low);
          w[i] = counts ? n : n > 0.0 ? (n + (n - 1.0) * fmin(width * width, 6.0) / 24) * weight_of(t, s, S.table) : 0.0;
          sum += w[i];
        }
        const double up_to = sum_up_to(sum), all = of_lane(up_to, 63);
        if (round == 0 && !counts && !by_k) aim = s.p * all;
        const double start = base + (up_to - sum);
        double before = start;
        int mine = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (mine == 0x7fffffff && w[i] > 0.0 && before + w[i] >= aim) mine = lane * PER + i;
          before += w[i];
        }
        int first = -most_over(-mine);
        if (lane == 0) S.any = round || !counts || first != 0x7fffffff;
        if (first == 0x7fffffff) first = PARTS_ - 1;
        before = start;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (lane * PER + i == max(first - 1, 0)) S.before = before;   // of the part before it
          before += w[i];
        }
        if (lane == 0) {
          S.found = first;
          S.aim = aim;
        }
      }
      __syncthreads();
      any = S.any;
      found = S.found;
      aim = S.aim;
      if (round == 0) {   // it again, with the parts beside it
        base = S.before;
        c0 = found > 0 ? found - 1 : 0;
        c1 = found < PARTS_ - 1 ? found + 1 : found;
        again = (float)PARTS_ / (float)(c1 + 1 - c0);
        scale = fine * again * steps;
        shift = c0 * again * steps;
        most_place = c1 == PARTS_ - 1 ? end_place - 1.f : 2.f * end_place;
      }
    }
    if (!any) {   // fewer classes than top-k asks for: all of them
      if (s.by_p) {
        double sum = 0.0;
        over_row<TYPE, THREADS>(x, classes, [&](int, const float (&v)[8]) {
#pragma unroll
          for (int j = 0; j < 8; ++j) sum += v[j] > -__builtin_inff() ? weight_of((double)v[j] - m, s, S.table) : 0.0;
        });
        sum_before<THREADS>(sum, S.wave_sum, &top_mass);
      }
      continue;
    }

    // The border lies at a rank from `low` on, below `high`.  The part, and parts on both sides as long as the list is short; where it is not in
    // these, those beside them; then half of what is left at a time.
    const int lowest = rank_of<TYPE>(-3.4028234663852886e38f);
    int low = lowest, high = rank_of<TYPE>(most) + 1;
    int p0 = found, p1 = found, first_part = 0, last_part = PARTS_ - 1;
    for (int attempt = 0;; ++attempt) {
      int in_from = low, over_from = high;   // ranks: what is listed, and what is above it
      const bool by_parts = attempt < 4 && first_part <= last_part;
      if (by_parts) {
        if (attempt) {
          const bool below = found < first_part;
          p0 = below ? first_part : last_part;
          while (S.part_count[p0] == 0 && (below ? p0 < last_part : p0 > first_part)) p0 += below ? 1 : -1;
          p1 = p0;
        }
        int n = S.part_count[p0];
        for (int i = 0; i < 12; ++i) {
          if (p0 > first_part && n + S.part_count[p0 - 1] <= 400) n += S.part_count[--p0];
          if (p1 < last_part && n + S.part_count[p1 + 1] <= 400) n += S.part_count[++p1];
        }
        auto smallest_until = [&](int part) {   // the smallest rank whose part is this one or above: 64 of them looked at together
          int not_it = lowest - 1, it = high;
          const float until = (float)((part + 1) << steps_log2);
          while ((unsigned)it - (unsigned)not_it > 1u) {
            const unsigned range = (unsigned)it - (unsigned)not_it;
            const int by = range > 64 ? 26 - __clz(range - 1) : 0;
            const unsigned away = (unsigned)(lane + 1) << by;
            // (the last one's is `it` or beyond, and may be 2^32 away)
            const int first = __ffsll(__ballot(lane == 63 || away >= range || place_of(of_rank<TYPE>((int)((unsigned)not_it + away))) < until)) - 1;
            if (first < 63 && ((unsigned)(first + 1) << by) < range) it = (int)((unsigned)not_it + ((unsigned)(first + 1) << by));
            not_it = (int)((unsigned)not_it + ((unsigned)first << by));
          }
          return it;
        };
        over_from = smallest_until(p0 - 1);
        in_from = smallest_until(p1);
      } else if ((unsigned)high - (unsigned)low > 1u) {
        in_from = (int)((unsigned)low + ((unsigned)high - (unsigned)low) / 2);
      }
      const float in_value = of_rank<TYPE>(in_from), over_value = over_from > rank_of<TYPE>(most) ? __builtin_inff() : of_rank<TYPE>(over_from);
      float heavy = (float)fmax(m + s.low, -3.4028234663852886e38);   // from here on w is not 0
      if ((double)heavy - m < s.low) heavy = value_of(order_of(heavy) + 1);
      const float heavy_above = fmaxf(heavy, over_value);
      __syncthreads();
      if (tid == 0) S.listed = 0;
      __syncthreads();
      int first_rank = 0x7fffffff, last_rank = -0x7fffffff - 1, n_above = 0;
      double inside = 0.0, all_mass = 0.0;
      over_row<TYPE, THREADS>(x, classes, [&](int at, const float (&v)[8]) {
        // (no branches: the exponentials are under way together)
        double mass = 0.0;
        unsigned mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool over = v[j] >= over_value, in = v[j] >= in_value && !over;
          const double w = exp_of((double)v[j] - m, s.c, S.table);   // (of others not looked at)
          mass += v[j] >= heavy_above ? w : 0.0;
          if (LATE) all_mass += v[j] >= heavy ? w : 0.0;
          n_above += over;
          mine |= in ? 1u << j : 0;
        }
        const int n = sum_over((int)__popc(mine), lanes_log2);
        mass = sum_over(mass, lanes_log2);
        if ((lane & ((1 << lanes_log2) - 1)) == 0 && at < classes) {
          block_mass[at >> block_log2] = mass;
          block_ties[at >> block_log2] = n;
        }
        if (!__ballot(mine != 0)) return;
        const int up_to = sum_up_to((int)__popc(mine));
        int place = 0;
        if (lane == 63) place = atomicAdd(&S.listed, up_to);
        place = __builtin_amdgcn_readlane(place, 63) + up_to - (int)__popc(mine);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (mine >> j & 1) {
            if (place < MOST) S.key[place] = key_of(v[j], at + j);
            ++place;
            inside += weight_of((double)v[j] - m, s, S.table);
            first_rank = min(first_rank, rank_of<TYPE>(v[j]));
            last_rank = max(last_rank, rank_of<TYPE>(v[j]));
          }
      });
      first_rank = -most_over(-first_rank);
      last_rank = most_over(last_rank);
      if (lane == 0) {
        S.wave_ranks[wave][0] = first_rank;
        S.wave_ranks[wave][1] = last_rank;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < THREADS / 64; ++k) {
        first_rank = min(first_rank, S.wave_ranks[k][0]);
        last_rank = max(last_rank, S.wave_ranks[k][1]);
      }
      const int n = S.listed;
      double above = 0.0, whole;
      for (int b = tid; b < blocks; b += THREADS) above += block_mass[b];
      {
        double sum;
        sum_before<THREADS>(above, S.wave_sum, &sum);
        above = sum;
        sum_before<THREADS>(inside, S.wave_sum, &whole);
        if (LATE && !counts && !by_k) {
          sum_before<THREADS>(all_mass, S.wave_sum, &top_mass);
          need = s.p * top_mass;
        }
        int all;
        sum_before<THREADS>(n_above, S.wave_count, &all);
        n_above = all;
      }
      const bool last = !by_parts && (unsigned)high - (unsigned)low <= 1u;   // (one value: it is the border, however sums are rounded)
      if (!last && (counts ? n_above >= s.k : above >= need)) {   // it is above the list
        low = over_from;
        last_part = p0 - 1;
        continue;
      }
      if (!last && (counts ? n_above + n < s.k : above + whole < need)) {   // it is below
        high = in_from;
        first_part = p1 + 1;
        continue;
      }
      if (n == 0) {   // the sums of two passes lie on either side of the border, by their rounding: what is above the empty list stays, and no more
        cut = over_from - 1;
        ties = 0;
        break;
      }
      if (first_rank == last_rank) {   // all of the list have the same value (block_ties has their numbers)
        cut = first_rank;
        tie_weight = weight_of((double)of_rank<TYPE>(cut) - m, s, S.table);
        const double q = tie_weight > 0.0 ? ceil((need - above) / tie_weight) : 1.0;
        ties = counts ? s.k - n_above : q < 1.0 ? 1 : q < n ? (int)q : n;
        top_mass = counts ? above + ties * tie_weight : top_mass;
        break;
      }
      if (n > MOST) {
        low = in_from;
        high = over_from;
        first_part = PARTS_;   // (no more by parts)
        continue;
      }
      sort_keys<THREADS, MOST>(S.key, n);
      for (int r = tid; r < n; r += THREADS) S.weight[r] = weight_of((double)value_of(order_in(S.key[r])) - m, s, S.table);
      __syncthreads();
      const int per = (n + THREADS - 1) / THREADS, r0 = tid * per, r1 = r0 + per < n ? r0 + per : n;
      int end = s.k - n_above;   // of the list's classes in their ranking, so many stay
      double sum = 0.0;
      for (int r = r0; r < r1; ++r) sum += !counts || r < end ? S.weight[r] : 0.0;
      double before = sum_before<THREADS>(sum, S.wave_sum, &whole) + above;
      if (counts) {
        top_mass = above + whole;
      } else {
        int left = 0;
        for (int r = r0; r < r1; ++r) {
          left += before < need;
          before += S.weight[r];
        }
        sum_before<THREADS>(left, S.wave_count, &end);
        end = end < 1 ? 1 : end;
      }
      const int order = order_in(S.key[end - 1]);
      int larger = 0;
      for (int r = tid; r < n; r += THREADS) larger += order_in(S.key[r]) > order;
      int sums;
      sum_before<THREADS>(larger, S.wave_count, &sums);
      larger = sums;
      cut = rank_of<TYPE>(value_of(order));
      ties = end - larger;
      tie_weight = weight_of((double)value_of(order) - m, s, S.table);
      for (int b = tid; b < blocks; b += THREADS) block_ties[b] = 0;
      __syncthreads();
      for (int r = larger + tid; r < n; r += THREADS)
        if (order_in(S.key[r]) == order) atomicAdd(&block_ties[index_in(S.key[r]) >> block_log2], 1);
      // those above it to their blocks, in the order of their indices
      u64 mine[(MOST + THREADS - 1) / THREADS];
#pragma unroll
      for (int i = 0; i < (MOST + THREADS - 1) / THREADS; ++i) {
        const int r = tid + i * THREADS;
        mine[i] = r < larger ? ~((u64)(unsigned)index_in(S.key[r]) << 32 | (unsigned)r) : 0;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < (MOST + THREADS - 1) / THREADS; ++i)
        if (tid + i * THREADS < larger) S.key[tid + i * THREADS] = mine[i];
      __syncthreads();
      sort_keys<THREADS, MOST>(S.key, larger);
      for (int i = tid; i < larger; i += THREADS) {
        const int block = (int)(~S.key[i] >> 32) >> block_log2;
        if (i && (int)(~S.key[i - 1] >> 32) >> block_log2 == block) continue;   // (the first of a block adds all of its)
        double sum = block_mass[block];
        for (int k = i; k < larger && (int)(~S.key[k] >> 32) >> block_log2 == block; ++k) sum += S.weight[(unsigned)~S.key[k]];
        block_mass[block] = sum;
      }
      break;
    }
    masses_there = true;
    __syncthreads();
  }
  // (what is left by top-p ends above min-p's bound, or min-p's bound is all)
  if (MANY && s.by_min && masses_there && (double)of_rank<TYPE>(cut) - m < s.bound) {
    masses_there = false;
    cut = -0x7fffffff - 1;
    ties = 0;
  }
  if (!all_count && !masses_there) {
    // no border, or min-p's alone: the mass of what is above its bound, block by block
    over_row<TYPE, THREADS>(x, classes, [&](int at, const float (&v)[8]) {
      double mass = 0.0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double t = (double)v[j] - m, w = exp_of(t, s.c, S.table);
        mass += t >= fmax(s.bound, s.low) ? w : 0.0;
      }
      mass = sum_over(mass, lanes_log2);
      if ((lane & ((1 << lanes_log2) - 1)) == 0 && at < classes) block_mass[at >> block_log2] = mass;
    });
  } else if (all_count) {
    for (int b = tid; b < blocks; b += THREADS) block_mass[b] *= weight_of((double)block_most[b] - m, s, S.table);
  }
  __syncthreads();

  // the block at which the sum is above u times the whole
  const int per = (blocks + THREADS - 1) / THREADS, b0 = tid * per, b1 = b0 + per < blocks ? b0 + per : blocks;
  if (ties) {
    int n = 0, whole;
    for (int b = b0; b < b1; ++b) n += block_ties[b];
    n = sum_before<THREADS>(n, S.wave_count, &whole);
    for (int b = b0; b < b1; ++b) {
      const int k = block_ties[b], left = ties - n < 0 ? 0 : ties - n < k ? ties - n : k;
      block_mass[b] += left * tie_weight;
      block_ties[b] = n;
      n += k;
    }
  }
  double sum = 0.0, whole;
  for (int b = b0; b < b1; ++b) sum += block_mass[b];
  const double before = sum_before<THREADS>(sum, S.wave_sum, &whole), target = s.u * whole;
  double at = before;
  int mine = 0x7fffffff, last = -1;
  for (int b = b0; b < b1; ++b) {
    const double w = block_mass[b];
    if (w > 0.0) {
      last = b;
      if (mine == 0x7fffffff && at + w > target) mine = b;
    }
    at += w;
  }
  mine = -most_over(-mine);
  last = most_over(last);
  if (lane == 0 && mine != 0x7fffffff) atomicMin(&S.chosen, mine);
  if (lane == 0 && last >= 0) atomicMax(&S.last, last);
  __syncthreads();
  const int chosen = S.chosen != 0x7fffffff ? S.chosen : S.last;
  if (chosen >= b0 && chosen < b1) {
    double a = before;
    for (int b = b0; b < chosen; ++b) a += block_mass[b];
    S.before = a;
  }
  __syncthreads();

  // and the class
  if (wave == 0) {
    const int at0 = (chosen << block_log2) + lane * 8;
    float v[8];
    double w[8], lane_sum = 0.0;
    int n = 0;
    const bool in = lane < 1 << lanes_log2;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = -__builtin_inff();
    if (in) eight_of<TYPE>(x, at0, classes, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) n += ties && rank_of<TYPE>(v[j]) == cut;
    int rank = (ties ? block_ties[chosen] : 0) + sum_up_to(n) - n;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = rank_of<TYPE>(v[j]);
      const double t = (double)v[j] - m;
      w[j] = 0.0;
      if (v[j] == -__builtin_inff() || (s.by_min && t < s.bound)) continue;
      if (r > cut) w[j] = weight_of(t, s, S.table);
      else if (ties && r == cut) w[j] = rank++ < ties ? tie_weight : 0.0;
      lane_sum += w[j];
    }
    double up_to = S.before + sum_before_lane(sum_up_to(lane_sum));
    int got = 0x7fffffff, final = -1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      up_to += w[j];
      if (w[j] > 0.0) {
        final = at0 + j;
        if (got == 0x7fffffff && up_to > target) got = at0 + j;
      }
    }
    got = -most_over(-got);
    final = most_over(final);
    if (got == 0x7fffffff) got = final;
    if (lane == 0) {
      J.drawn[row] = got;
      if (J.log_probs) J.log_probs[row] = (float)(((double)E::get(x[got]) - m) / s.T - log(whole));
    }
  }
}

constexpr int LOOK_THREADS = 256;

template <int TYPE, int THREADS, int MOST, bool PARTS, bool MANY>
hipError_t launch_kernel(hipStream_t stream, const DrawJob& J) {
  const size_t lds = (size_t)J.blocks * 16;
  if (sizeof(Shared<THREADS, MOST>) + lds > 64 << 10) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_draw<TYPE, THREADS, MOST, PARTS, MANY>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             DRAW_BLOCKS * 16);   // (the same for every call: others may be under way)
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_draw<TYPE, THREADS, MOST, PARTS, MANY>), dim3((unsigned)J.rows), dim3(THREADS), lds, stream, J);
  return hipGetLastError();
}

template <int TYPE, int THREADS, bool PARTS>
hipError_t launch_rows(hipStream_t stream, const DrawJob& J) {
  for (long long r = 0; r < J.rows; r += 1 << 20) {   // (a grid has fewer than 2^32 threads)
    DrawJob P = J;
    P.x = (const CNN_GLOBAL char*)J.x + r * J.stride * (long long)element_bytes(J.type);
    if (P.temperature) P.temperature += r;
    if (P.top_k) P.top_k += r;
    if (P.top_p) P.top_p += r;
    if (P.min_p) P.min_p += r;
    P.u += r;
    P.drawn += r;
    if (P.log_probs) P.log_probs += r;
    P.rows = std::min(J.rows - r, 1ll << 20);
    if (PARTS) hipLaunchKernelGGL((k_draw_look<TYPE, LOOK_THREADS>), dim3((unsigned)(P.rows * P.parts)), dim3(LOOK_THREADS), 0, stream, P);
    hipError_t e = launch_kernel<TYPE, THREADS, THREADS * 4, PARTS, false>(stream, P);
    if (e == hipSuccess && (P.top_k || P.top_p)) e = launch_kernel<TYPE, THREADS, THREADS * 4, PARTS, true>(stream, P);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Which form (10000 rows, us without a cut / with top-k 50 and top-p 0.9): a lane a class up to 64 of them 9.6 / 30 (a wavefront a row 17.1 / 53);
// a wavefront a row up to 1024, 1000 bf16 30 / 103 (a workgroup 65 / 142; 2000 in registers 91 / 415, a workgroup 71 / 143); then 256 threads,
// 2000 rows of 4000 20.7 / 34 (512 threads 31 / 58), or 512, 1000 rows of 32768 36.9 / 43.1 (256 41.7 / 43.2; at 16384 26.5 / 38.6, 28.5 / 36.9).
template <int TYPE>
hipError_t launch_type(hipStream_t stream, const DrawJob& J) {
  if (J.classes <= 64) {
    int log2 = 1;
    while (1 << log2 < J.classes) ++log2;
    const long long waves = (J.rows + (64 >> log2) - 1) / (64 >> log2);
    hipLaunchKernelGGL((k_draw_lanes<TYPE>), dim3((unsigned)std::min((waves + 3) / 4, 1ll << 16)), dim3(256), 0, stream, J, log2);
    return hipGetLastError();
  }
  if (J.classes <= 1024) {
    const dim3 grid((unsigned)std::min((J.rows + 3) / 4, 1ll << 16));
    if (J.classes <= 512) hipLaunchKernelGGL((k_draw_wave<TYPE, 1>), grid, dim3(256), 0, stream, J);
    else hipLaunchKernelGGL((k_draw_wave<TYPE, 2>), grid, dim3(256), 0, stream, J);
    return hipGetLastError();
  }
  if (J.parts > 1) return launch_rows<TYPE, 512, true>(stream, J);
  return J.classes <= 16384 ? launch_rows<TYPE, 256, false>(stream, J) : launch_rows<TYPE, 512, false>(stream, J);
}

}  // namespace

// How a row is cut into blocks (8 to 512 classes, some 2048 of them at most: up to 4096 beyond 2^20 classes), and how many workgroups
// look at a row first.  They help where rows alone leave compute units idle and are long enough for a launch more (us without a cut / with
// top-k 50 and top-p 0.9): one row of 131072 bf16 in 32 parts 12.0 / 19.7 (not in parts 35.1 / 25.9), 64 in 16 17.9 / 22.5 (36.0 / 26.2), 160
// in 8 25.9 / 26.8 (37.9 / 28.5), 37 of 50001 fp32 in 12 14.9 / 20.8 (19.4 / 20.2), 250 of 300000 in 5 69 / 49 (87 / 56), one of 2^21 in 512 15.8 / 31
// (542 / 246).  Not for rows of 32768, 16 of them in 8 12.5 / 20.3 (13.9 / 17.7), nor for many of 131072, 256 in 5 35.8 / 32.0 (38.8 / 29.7).
void draw_blocks(long long rows, int classes, int* block_log2, int* blocks, int* parts) {
  *block_log2 = 3;
  while (*block_log2 < 9 && (classes + (1 << *block_log2) - 1) >> *block_log2 > DRAW_BLOCKS / 2) ++*block_log2;
  *blocks = (classes + (1 << *block_log2) - 1) >> *block_log2;
  *parts = (int)std::min((long long)classes / 4096, 1280 / std::max(1ll, rows));
  if (classes < 36864 || *parts < (classes < 1 << 18 ? 8 : 4)) *parts = 1;
}

hipError_t launch_draws(hipStream_t stream, const DrawJob& J) {
  switch (J.type) {
    case ELEMENT_F32: return launch_type<ELEMENT_F32>(stream, J);
    case ELEMENT_BF16: return launch_type<ELEMENT_BF16>(stream, J);
    case ELEMENT_F16: return launch_type<ELEMENT_F16>(stream, J);
  }
  return hipErrorInvalidValue;
}

}  // namespace cnn355
