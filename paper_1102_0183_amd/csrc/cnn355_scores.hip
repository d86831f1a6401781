// Scores of classes and their gradient: what a training or test pass is read with once the sums of its output layer, or
// any others, are there.  For a row x of sums, with m = max x and S = log sum_j exp(x_j - m):
//
//   log p_j = (x_j - m) - S          entropy H = S - sum_j e_j (x_j - m) / sum_j e_j,  e_j = exp(x_j - m)
//   d (g_l log p_l + g_h H) / d x_j = g_l ([j == l] - p_j) - g_h p_j (log p_j + H)
//
// One pass over the row: every lane keeps the largest value m it has seen, s = sum of exp(x - m) and t = sum of
// exp(x - m) (x - m), and takes both to a new m by the factor exp(m - m'): s' = s f, t' = (t + (m - m') s) f.  Lanes,
// wavefronts and workgroups that share a row join their three numbers in the same way.  All of it is held in 32 bits.
//
// The best classes ride along.  A wavefront keeps the best so far sorted over its lanes, as 64-bit keys (value, then the
// lower index) whose order is that of whole numbers; a class is looked at only if its value reaches that of the last one
// kept, which after the first few tiles hardly any does, so the price is a comparison for every 16 classes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"

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
__device__ __forceinline__ u64 key_of(float v, int index) {
  const unsigned b = __builtin_bit_cast(unsigned, v + 0.0f);   // (-0 as 0)
  return (u64)((int)b < 0 ? ~b : b | 0x80000000u) << 32 | (unsigned)~index;
}
__device__ __forceinline__ int index_of(u64 k) { return (int)~(unsigned)k; }
__device__ __forceinline__ float value_of(u64 k) {
  const unsigned b = (unsigned)(k >> 32);
  return __builtin_bit_cast(float, (int)b < 0 ? b & 0x7fffffffu : ~b);
}

template <class T>
__device__ __forceinline__ T larger(T a, T b) { return a < b ? b : a; }
template <class T>
__device__ __forceinline__ T smaller(T a, T b) { return a < b ? a : b; }

// Values of `lanes` lanes side by side (a power of two) in descending order; `from` > 2: they already are in two runs of
// lanes, rising and falling or the other way round, of which only the merge is left (from = lanes).
template <class T>
__device__ __forceinline__ T sort_lanes(T v, int lanes, int from = 2) {
  const int lane = threadIdx.x & 63;
  for (int size = from; size <= lanes; size <<= 1)
    for (int d = size >> 1; d; d >>= 1) {
      const T o = __shfl_xor(v, d);
      const bool first = (lane & d) == 0, down = size == lanes || (lane & size) == 0;
      v = first == down ? larger(v, o) : smaller(v, o);
    }
  return v;
}

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

__device__ __forceinline__ void join_lanes(Sums& a, int lanes) {
  float m = a.m;
  for (int d = 1; d < lanes; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  lift(a, m);
  for (int d = 1; d < lanes; d <<= 1) { a.s += __shfl_xor(a.s, d); a.t += __shfl_xor(a.t, d); }
}

// What a row's sums come to.  A row without a value above -inf is empty; one with +inf or NaN has no distribution.
struct Row {
  float m, log_s, entropy;
  bool none;
};
__device__ __forceinline__ Row row_of(const Sums& a) {
  Row r;
  r.none = !(a.s < INFINITY);
  if (r.none) { r.m = r.log_s = r.entropy = __builtin_nanf(""); return r; }
  const bool empty = a.s == 0.0f;
  r.m = empty ? -INFINITY : a.m;
  r.log_s = logf(a.s);
  const float h = r.log_s - LN2 * a.t / a.s;
  r.entropy = empty || h < 0.0f ? 0.0f : h;
  return r;
}
__device__ __forceinline__ float log_prob(const Row& r, float x) { return r.m == -INFINITY ? -INFINITY : (x - r.m) - r.log_s; }

// One lane's share of a row's results: lane 0 the numbers, lane i the i-th of the best.
template <int TYPE>
__device__ __forceinline__ void give_row(const ScoreJob& J, long long row, int lane, const Sums& a, u64 best) {
  typedef Element<TYPE> E;
  const Row r = row_of(a);
  if (lane == 0) {
    if (J.log_probs) {
      const int l = J.labels[row];
      float v = 0.0f;
      if (l >= 0 && l < J.classes) v = log_prob(r, E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + l]));
      J.log_probs[row] = v;
    }
    if (J.entropy) J.entropy[row] = r.entropy;
    if (J.normaliser) { J.normaliser[2 * row] = r.m; J.normaliser[2 * row + 1] = r.log_s; }
  }
  if (lane < J.n_top) {
    if (J.top) J.top[row * J.n_top + lane] = r.none ? -1 : index_of(best);
    if (J.top_log_probs) J.top_log_probs[row * J.n_top + lane] = r.none ? r.m : log_prob(r, value_of(best));
  }
}

// ---- the best classes of a wavefront ----
constexpr int HELD = 128;   // keys waiting in LDS: fewer than 64, and those of one look at every lane

struct Best {
  u64 list;        // lane i: the i-th best so far, 0: none
  u64 bar;         // a key that can still be among them is above it,
  float bar_value; // and the value of a class of the next tile that can is not below this
  int held;
};

__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
  return (u64)__builtin_amdgcn_readlane((unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)v, lane);
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// the 64 (or fewer) keys in front join the list
__device__ __forceinline__ void take_held(Best& b, u64* held, int n_top) {
  const int lane = threadIdx.x & 63;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const u64 mine = lane < b.held ? held[lane] : 0, rest = 64 + lane < b.held ? held[64 + lane] : 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  held[lane] = rest;
  b.held = b.held > 64 ? b.held - 64 : 0;
  const u64 sorted = sort_lanes(mine, 64);
  b.list = sort_lanes(larger(b.list, (u64)__shfl(sorted, 63 - lane)), 64, 64);
  const u64 last = lane_of(b.list, n_top - 1);
  // (the classes of the tiles to come have higher indices: of theirs, only larger values are above that key)
  if (last > b.bar) { b.bar = last; b.bar_value = value_of(last + (1ull << 32)); }
}

// A tile of a wavefront, x[k] of class first + (k / V) 64 V + lane V + k % V, `largest` the lane's largest, `end` the
// first class that is not the row's (or its part's).
template <int TYPE>
__device__ __forceinline__ void look(Best& b, u64* held, const CNN_GLOBAL typename Element<TYPE>::T* row, const float (&x)[16],
                                     float largest, int first, int end, int n_top) {
  typedef Element<TYPE> E;
  constexpr int V = E::V;
  const u64 any = __ballot(largest >= b.bar_value);
  if (!any) return;
  const int lane = threadIdx.x & 63;
  // Many lanes at once, as in a wavefront's first tile or where values rise along the row: as many classes as are asked for
  // reach the n_top-th of the lanes' largest values, so what lies below it is out.
  if (b.bar == 0 || __popcll(any) > n_top) {
    const float v = lane_of(sort_lanes(largest, 64), n_top - 1);
    if (v > b.bar_value) { b.bar_value = v; b.bar = key_of(v, -1); }
  }
  unsigned hits = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) hits |= x[k] >= b.bar_value ? 1u << k : 0u;
  while (__ballot(hits != 0)) {
    const int k = __builtin_ctz(hits | 0x10000u), at = first + (k / V) * 64 * V + lane * V + k % V;
    u64 key = 0;
    if (hits && at < end) key = key_of(E::get(row[at]), at);   // (asked for again: it has just been read)
    hits &= hits - 1;
    const u64 in = __ballot(key > b.bar);
    if (key > b.bar) held[b.held + __builtin_amdgcn_mbcnt_hi((unsigned)(in >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in, 0))] = key;
    b.held += __popcll(in);
    if (b.held >= 64) take_held(b, held, n_top);
  }
}

// ---- the pass over a row ----
// Tiles first, first + step, ... of a row, below `last`: the wavefront's sums, lane by lane, and its best.
template <int TYPE, bool ENTROPY, bool TOP>
__device__ __forceinline__ void scan(const ScoreJob& J, const CNN_GLOBAL typename Element<TYPE>::T* row, int first, int step, int last,
                                     Sums& a, Best& b, u64* held) {
  typedef Element<TYPE> E;
  constexpr int V = E::V, N = 16 / V;
  const int lane = threadIdx.x & 63, end = J.classes;
  a = Sums{LOWEST, 0.0f, 0.0f};
  b = Best{0, 0, -INFINITY, 0};
  v4u next[N];
  if (first < last) {
#pragma unroll
    for (int q = 0; q < N; ++q) next[q] = load16<TYPE>(row, first * SCORE_TILE + q * 64 * V + lane * V, end);
  }
  for (int tile = first; tile < last; tile += step) {
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = E::get(next[k / V], k % V);
    if (tile + step < last) {
#pragma unroll
      for (int q = 0; q < N; ++q) next[q] = load16<TYPE>(row, (tile + step) * SCORE_TILE + q * 64 * V + lane * V, end);
    }
    float largest = max3(x[0], x[1], x[2]);
#pragma unroll
    for (int k = 3; k < 15; k += 2) largest = max3(largest, x[k], x[k + 1]);
    largest = max3(largest, x[15], x[15]);
    lift(a, max3(a.m, largest, largest));
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float d = (x[k] - a.m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
      a.s += e;
      if (ENTROPY) a.t = fmaf(e, fmaxf(d, FAR), a.t);
    }
    if (TOP) look<TYPE>(b, held, row, x, largest, tile * SCORE_TILE, end, J.n_top);
  }
  if (TOP && b.held) take_held(b, held, J.n_top);
}

// Rows of more than 64 classes, WAVES wavefronts a row or, where parts > 1, a part of one.
template <int TYPE, int WAVES, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(ST) k_scores(ScoreJob J) {
  constexpr int ROWS = ST / 64 / WAVES;
  __shared__ u64 lds_held[TOP ? ST / 64 : 1][HELD];
  __shared__ u64 lds_best[TOP && WAVES > 1 ? WAVES : 1][64];
  __shared__ float lds_sums[WAVES][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part_of = WAVES > 1 ? 0 : wave, w = WAVES > 1 ? wave : 0;
  const int part = blockIdx.y, tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE;
  for (long long row = (long long)blockIdx.x * ROWS + part_of; row < J.rows; row += (long long)gridDim.x * ROWS) {
    Sums a;
    Best b;
    scan<TYPE, ENTROPY, TOP>(J, (const CNN_GLOBAL typename Element<TYPE>::T*)J.x + row * J.stride, part * J.part_tiles + w, WAVES,
                             min(tiles, (part + 1) * J.part_tiles), a, b, lds_held[TOP ? wave : 0]);
    join_lanes(a, 64);
    if (WAVES > 1) {
      __syncthreads();   // (what the row before left has been read)
      if (lane == 0) { lds_sums[w][0] = a.m; lds_sums[w][1] = a.s; lds_sums[w][2] = a.t; }
      if (TOP) lds_best[w][lane] = b.list;
      __syncthreads();
      if (wave != 0) continue;
      a = Sums{LOWEST, 0.0f, 0.0f};
      if (lane < WAVES) a = Sums{lds_sums[lane][0], lds_sums[lane][1], lds_sums[lane][2]};
      join_lanes(a, 64);
      if (TOP)
        for (int o = 1; o < WAVES; ++o) b.list = sort_lanes(larger(b.list, lds_best[o][63 - lane]), 64, 64);
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
    give_row<TYPE>(J, row, lane, a, b.list);
  }
}

// The parts of rows joined: a workgroup a row.
template <int TYPE>
__global__ void __launch_bounds__(ST) k_scores_join(ScoreJob J) {
  __shared__ u64 lds_best[ST / 64][64];
  __shared__ float lds_sums[ST / 64][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (long long row = blockIdx.x; row < J.rows; row += gridDim.x) {
    Sums a{LOWEST, 0.0f, 0.0f};
    if ((int)threadIdx.x < J.parts) {
      const CNN_GLOBAL float* p = J.part_sums + (row * J.parts + threadIdx.x) * 4;
      a = Sums{p[0], p[1], p[2]};
    }
    join_lanes(a, 64);
    u64 list = 0;
    if (J.n_top)
      for (int part = wave; part < J.parts; part += ST / 64) {
        const u64 k = 63 - lane < J.n_top ? J.part_best[(row * J.parts + part) * J.n_top + 63 - lane] : 0;
        list = sort_lanes(larger(list, k), 64, 64);
      }
    __syncthreads();
    if (lane == 0) { lds_sums[wave][0] = a.m; lds_sums[wave][1] = a.s; lds_sums[wave][2] = a.t; }
    lds_best[wave][lane] = list;
    __syncthreads();
    if (wave != 0) continue;
    a = Sums{LOWEST, 0.0f, 0.0f};
    if (lane < ST / 64) a = Sums{lds_sums[lane][0], lds_sums[lane][1], lds_sums[lane][2]};
    join_lanes(a, 64);
    if (J.n_top)
      for (int o = 1; o < ST / 64; ++o) list = sort_lanes(larger(list, lds_best[o][63 - lane]), 64, 64);
    give_row<TYPE>(J, row, lane, a, list);
  }
}

// Rows of at most 64 classes: a lane a class, 64 / L rows a wavefront.
template <int TYPE, int L>
__global__ void __launch_bounds__(ST) k_scores_few(ScoreJob J) {
  typedef Element<TYPE> E;
  const int c = threadIdx.x & (L - 1);
  const long long all = (J.rows + ST / L - 1) / (ST / L) * (ST / L);   // (lanes of a wavefront stay together)
  for (long long row = (long long)blockIdx.x * (ST / L) + threadIdx.x / L; row < all; row += (long long)gridDim.x * (ST / L)) {
    const bool is = row < J.rows && c < J.classes;
    const float x = is ? E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + c]) : -INFINITY;
    float m = fmaxf(x, LOWEST);
    for (int d = 1; d < L; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    const float d = (x - m) * LOG2E, e = __builtin_amdgcn_exp2f(d);
    Sums a{m, e, e * fmaxf(d, FAR)};
    for (int o = 1; o < L; o <<= 1) { a.s += __shfl_xor(a.s, o); a.t += __shfl_xor(a.t, o); }
    u64 k = is && x == x ? key_of(x, c) : 0;
    if (J.n_top) k = sort_lanes(k, L);
    if (row < J.rows) give_row<TYPE>(J, row, c, a, k);
  }
}

// ---- the gradient ----
struct GradRow {
  float m, log_s;
  float a, b;      // -p (a + b log p)
  float g_label;
  int label;
  bool empty;
};
__device__ __forceinline__ GradRow grad_row(const ScoreGradJob& J, long long row) {
  GradRow r;
  r.m = J.normaliser[2 * row];
  r.log_s = J.normaliser[2 * row + 1];
  r.empty = r.m == -INFINITY;
  r.label = J.labels ? J.labels[row] : -1;
  const bool has = r.label >= 0 && r.label < J.classes && J.g_log_probs;
  r.g_label = has ? J.g_log_probs[row] : 0.0f;
  r.b = J.g_entropy ? J.g_entropy[row] : 0.0f;
  r.a = J.g_entropy ? fmaf(r.b, J.entropy[row], r.g_label) : r.g_label;
  return r;
}
// of one class; a class of probability zero has none but its label's
__device__ __forceinline__ float grad_of(const GradRow& r, float x, int c) {
  const float log_p = (x - r.m) - r.log_s, p = __builtin_amdgcn_exp2f(log_p * LOG2E);
  const float g = (c == r.label ? r.g_label : 0.0f) - (p == 0.0f ? 0.0f : p * fmaf(r.b, log_p, r.a));
  return r.empty ? 0.0f : g;
}

template <int TYPE, int L>
__global__ void __launch_bounds__(ST) k_scores_grad_few(ScoreGradJob J) {
  typedef Element<TYPE> E;
  const int c = threadIdx.x & (L - 1);
  if (c >= J.classes) return;
  for (long long row = (long long)blockIdx.x * (ST / L) + threadIdx.x / L; row < J.rows; row += (long long)gridDim.x * (ST / L)) {
    const GradRow r = grad_row(J, row);
    const float x = E::get(((const CNN_GLOBAL typename E::T*)J.x)[row * J.stride + c]);
    ((CNN_GLOBAL typename E::T*)J.grad)[row * J.grad_stride + c] = E::make(grad_of(r, x, c));
  }
}

// a wavefront a tile
template <int TYPE>
__global__ void __launch_bounds__(ST) k_scores_grad(ScoreGradJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int V = E::V, N = 16 / V;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE;
  const long long n = J.rows * tiles;
  for (long long at = (long long)blockIdx.x * (ST / 64) + wave; at < n; at += (long long)gridDim.x * (ST / 64)) {
    const long long row = at / tiles;
    const int first = (int)(at - row * tiles) * SCORE_TILE;
    const CNN_GLOBAL T* x = (const CNN_GLOBAL T*)J.x + row * J.stride;
    CNN_GLOBAL T* g = (CNN_GLOBAL T*)J.grad + row * J.grad_stride;
    v4u in[N];
#pragma unroll
    for (int q = 0; q < N; ++q) in[q] = load16<TYPE>(x, first + q * 64 * V + lane * V, J.classes);
    const GradRow r = grad_row(J, row);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int c = first + q * 64 * V + lane * V;
      union { v4u v; T e[V]; } out;
#pragma unroll
      for (int j = 0; j < V; ++j) out.e[j] = E::make(grad_of(r, E::get(in[q], j), c + j));
      if (c + V <= J.classes) *(CNN_GLOBAL v4u_any*)(g + c) = out.v;
      else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (c + j < J.classes) g[c + j] = out.e[j];
      }
    }
  }
}

constexpr long long GRID_MOST = 1 << 20;   // workgroups of a launch at most: rows beyond are looped over
unsigned grid_of(long long work, long long per) { return (unsigned)std::min((work + per - 1) / per, GRID_MOST); }

int lanes_of(int classes) {
  int l = 4;
  while (l < classes) l <<= 1;
  return l;
}

template <int TYPE, int WAVES>
hipError_t launch_scores_waves(hipStream_t stream, const ScoreJob& J) {
  const dim3 grid(grid_of(J.rows, ST / 64 / WAVES), (unsigned)J.parts);
  const bool h = J.entropy, top = J.n_top;
  if (h && top) hipLaunchKernelGGL((k_scores<TYPE, WAVES, true, true>), grid, dim3(ST), 0, stream, J);
  else if (h) hipLaunchKernelGGL((k_scores<TYPE, WAVES, true, false>), grid, dim3(ST), 0, stream, J);
  else if (top) hipLaunchKernelGGL((k_scores<TYPE, WAVES, false, true>), grid, dim3(ST), 0, stream, J);
  else hipLaunchKernelGGL((k_scores<TYPE, WAVES, false, false>), grid, dim3(ST), 0, stream, J);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || J.parts == 1) return e;
  hipLaunchKernelGGL(k_scores_join<TYPE>, dim3(grid_of(J.rows, 1)), dim3(ST), 0, stream, J);
  return hipGetLastError();
}

#define CNN355_LANES(kernel)                                                                                                   \
  switch (lanes_of(J.classes)) {                                                                                               \
    case 4: hipLaunchKernelGGL((kernel<TYPE, 4>), dim3(grid_of(J.rows, ST / 4)), dim3(ST), 0, stream, J); break;               \
    case 8: hipLaunchKernelGGL((kernel<TYPE, 8>), dim3(grid_of(J.rows, ST / 8)), dim3(ST), 0, stream, J); break;               \
    case 16: hipLaunchKernelGGL((kernel<TYPE, 16>), dim3(grid_of(J.rows, ST / 16)), dim3(ST), 0, stream, J); break;            \
    case 32: hipLaunchKernelGGL((kernel<TYPE, 32>), dim3(grid_of(J.rows, ST / 32)), dim3(ST), 0, stream, J); break;            \
    default: hipLaunchKernelGGL((kernel<TYPE, 64>), dim3(grid_of(J.rows, ST / 64)), dim3(ST), 0, stream, J); break;            \
  }

template <int TYPE>
hipError_t launch_scores_type(hipStream_t stream, const ScoreJob& J) {
  if (J.classes > 64) {
    const int tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE;
    return tiles <= 2 ? launch_scores_waves<TYPE, 1>(stream, J) : launch_scores_waves<TYPE, 4>(stream, J);
  }
  CNN355_LANES(k_scores_few)
  return hipGetLastError();
}

template <int TYPE>
hipError_t launch_scores_grad_type(hipStream_t stream, const ScoreGradJob& J) {
  if (J.classes > 64) {
    const long long tiles = (J.classes + SCORE_TILE - 1) / SCORE_TILE;
    hipLaunchKernelGGL(k_scores_grad<TYPE>, dim3(grid_of(J.rows * tiles, ST / 64)), dim3(ST), 0, stream, J);
  } else {
    CNN355_LANES(k_scores_grad_few)
  }
  return hipGetLastError();
}

}  // namespace

// How rows are shared: parts of whole rounds of a workgroup's tiles where the rows alone do not fill the chip.
void score_parts(long long rows, int classes, int* parts, int* part_tiles) {
  const int tiles = (classes + SCORE_TILE - 1) / SCORE_TILE;
  *parts = 1;
  *part_tiles = tiles;
  if (rows >= 512 || tiles <= 4) return;
  const long long want = std::min<long long>({(512 + rows - 1) / rows, (tiles + 3) / 4, SCORE_PARTS});
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
