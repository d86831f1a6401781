// The 2-norm of all gradients of a step, gradients clipped by it, and the update with clipped gradients:
//
//   N = sqrt(sum over tensors, elements of g^2),  f = max_norm / N where N > max_norm, else 1
//   clipped: g f        update: w - lr f g        (N infinite or no number: g, and w, as they are)
//
// Two launches: every workgroup of the first leaves the sum of its chunks in memory, every workgroup of the second adds all
// those sums (the same way, so that all agree on N to the last bit and a call gives the same bits again) and goes over its
// chunks.  Squares and sums are doubles: no gradient that a float holds overflows or vanishes in its square, and the order of
// a thousand million terms does not show.  So is an update's product with the factor, rounded once with the difference.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"
#include "cnn355_lanes.h"

namespace cnn355 {

namespace {

constexpr int GT = 256;   // threads of a workgroup

typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v2u_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

template <int D>
__device__ __forceinline__ double add_lane(double s) {   // and that of the lane whose number differs by D
  const unsigned long long b = __builtin_bit_cast(unsigned long long, s);
  return s + __builtin_bit_cast(double, (unsigned long long)xor_word<D>((unsigned)(b >> 32)) << 32 | xor_word<D>((unsigned)b));
}
// the sum of a double of every thread, in every thread
template <int THREADS>
__device__ __forceinline__ double sum_of_workgroup(double s, double* lds) {
  s = add_lane<1>(add_lane<2>(add_lane<4>(add_lane<8>(add_lane<16>(add_lane<32>(s))))));
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) lds[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
  return s;
}

// ---- chunks ----
constexpr int NV = LIST_CHUNK / GT / 16;   // loads of 16 bytes a lane

struct Piece {   // a chunk of a tensor
  const CNN_GLOBAL char* from;
  CNN_GLOBAL void* to;             // the tensor's beginning,
  unsigned long long begin;        // its first element in it
  int n, type;                     // elements (0: no chunk)
};

__device__ __forceinline__ Piece piece_from(unsigned long long from, unsigned long long to, unsigned long long n, unsigned first, int type, unsigned c) {
  Piece p;
  const unsigned long long at = (unsigned long long)(c - first) * LIST_CHUNK;
  const int shift = type == ELEMENT_F32 ? 2 : 1;
  p.from = (const CNN_GLOBAL char*)(from + at);
  p.to = (CNN_GLOBAL void*)to;
  p.type = type;
  p.begin = at >> shift;
  p.n = (int)min(n - p.begin, (unsigned long long)(LIST_CHUNK >> shift));
  return p;
}

// Where chunks lie.  A list in a kernel's argument: a lane an entry (or two), all asked for together at the start; the last whose first
// chunk is not behind c is the number of lanes that hold such a one, and its entry is read from its lane.  (Looked for in the argument by
// halves, a dependent load each, eight tensors of 40 KB together took an update 7.7 us, one of them 5.9.)
template <bool FAR, bool DOWN, class JOB>
struct Finder {
  static constexpr int SETS = (JOB::MOST + 63) / 64;
  unsigned long long from[SETS], to[SETS], n[SETS];
  unsigned first[SETS];
  int type[SETS];

  __device__ __forceinline__ explicit Finder(const JOB& J) {
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      const int k = s * 64 + (threadIdx.x & 63);
      from[s] = to[s] = n[s] = 0;
      first[s] = 0xffffffffu;
      type[s] = 0;
      if (k < J.tensors) {
        const TensorEntry& e = J.e[k];
        from[s] = (unsigned long long)e.from; to[s] = (unsigned long long)e.to; n[s] = e.n; first[s] = e.chunk; type[s] = e.type;
      }
    }
  }
  static __device__ __forceinline__ unsigned long long word(unsigned long long v, int lane) {
    return (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
  }
  __device__ __forceinline__ Piece of(int s, int lane, unsigned c) const {
    return piece_from(word(from[s], lane), word(to[s], lane), word(n[s], lane), (unsigned)__builtin_amdgcn_readlane((int)first[s], lane),
                      __builtin_amdgcn_readlane(type[s], lane), c);
  }
  __device__ __forceinline__ Piece operator()(const JOB& J, unsigned i) {
    if (i >= J.chunks) return Piece{nullptr, nullptr, 0, 0, 0};
    const unsigned c = DOWN ? J.chunks - 1 - i : i;
    int t = -1;
#pragma unroll
    for (int s = 0; s < SETS; ++s) t += __popcll(__ballot(first[s] <= c));
    return SETS == 1 || t < 64 ? of(0, t & 63, c) : of(SETS - 1, t & 63, c);
  }
};
// A list in memory: by halves between the tensor that was looked up before and the end that chunks go towards.
template <bool DOWN, class JOB>
struct Finder<true, DOWN, JOB> {
  int t;

  __device__ __forceinline__ explicit Finder(const JOB& J) : t(DOWN ? J.tensors - 1 : 0) {}
  __device__ __forceinline__ Piece operator()(const JOB& J, unsigned i) {
    if (i >= J.chunks) return Piece{nullptr, nullptr, 0, 0, 0};
    const unsigned c = DOWN ? J.chunks - 1 - i : i;
    int lo = DOWN ? 0 : t, hi = DOWN ? t + 1 : J.tensors;
    while (hi - lo > 1) {   // first chunk of lo <= c, and c in front of that of hi where there is one
      const int mid = (lo + hi) >> 1;
      if (J.table[mid].chunk <= c) lo = mid; else hi = mid;
    }
    t = lo;
    const CNN_GLOBAL TensorEntry* e = J.table + t;
    return piece_from((unsigned long long)e->from, (unsigned long long)e->to, e->n, e->chunk, e->type, c);
  }
};
__device__ __forceinline__ bool whole(const Piece& p) { return p.n << (p.type == ELEMENT_F32 ? 2 : 1) == LIST_CHUNK; }

// GT threads and which of all chunks are theirs: every step-th, so that what is read side by side lies side by side.
struct Share {
  unsigned first, step;
  int thread;
};
__device__ __forceinline__ Share share_of_workgroup() { return Share{blockIdx.x, gridDim.x, (int)threadIdx.x}; }

// The chunks of a share (DOWN: from the last one on): full(piece, its elements, 16 bytes a lane and load) or part(piece).  The next
// one is looked up while the loads of a chunk are under way (its loads too: no faster, and clipping of 320 tensors 288 us -> 304).
// FOURS: types of 16 bits in loads of 8 bytes, two in the place of one of 16, so that the fp32 values that belong to a wavefront's
// load lie side by side too.
// early(piece): what else a whole chunk wants loaded; goes_on(): called behind the loads of every chunk, with whole workgroups, so that
// what has to be known first (a norm) is waited for together with them; the loop ends where it says no.
template <bool FAR, bool DOWN, bool FOURS, class JOB, class Early, class GoesOn, class Full, class Part>
__device__ __forceinline__ void for_chunks(const JOB& J, Share at, Early early, GoesOn goes_on, Full full, Part part) {
  Finder<FAR, DOWN, JOB> piece(J);
  Piece p = piece(J, at.first);
  for (unsigned i = at.first; i < J.chunks; i += at.step) {
    Piece next;
    if (whole(p)) {
      v4u r[NV];
      if (FOURS && p.type != ELEMENT_F32) {
#pragma unroll
        for (int q = 0; q < 2 * NV; ++q) {
          const v2u v = *(const CNN_GLOBAL v2u_any*)(p.from + (q * GT + at.thread) * 8);
          r[q >> 1][(q & 1) * 2] = v[0];
          r[q >> 1][(q & 1) * 2 + 1] = v[1];
        }
      } else {
#pragma unroll
        for (int q = 0; q < NV; ++q) r[q] = *(const CNN_GLOBAL v4u_any*)(p.from + (q * GT + at.thread) * 16);
      }
      early(p);
      next = piece(J, i + at.step);
      if (!goes_on()) return;
      full(p, r);
    } else {
      next = piece(J, i + at.step);
      if (!goes_on()) return;
      part(p);
    }
    p = next;
  }
}

// f(a constant of the type)
template <class F>
__device__ __forceinline__ void by_type(int type, F f) {
  switch (type) {
    case ELEMENT_F32: f(std::integral_constant<int, ELEMENT_F32>()); break;
    case ELEMENT_BF16: f(std::integral_constant<int, ELEMENT_BF16>()); break;
    default: f(std::integral_constant<int, ELEMENT_F16>()); break;
  }
}

// ---- the sum of squares ----
template <bool FAR, class JOB>
__device__ __forceinline__ double squares_of(const JOB& J, Share at) {
  double s = 0.0;
  for_chunks<FAR, false, false>(
      J, at, [](const Piece&) {}, []() { return true; },
      [&](const Piece& p, const v4u (&r)[NV]) {
        by_type(p.type, [&](auto type) {
          typedef Element<decltype(type)::value> E;
#pragma unroll
          for (int q = 0; q < NV; ++q)
#pragma unroll
            for (int j = 0; j < E::V; ++j) { const double v = E::get(r[q], j); s = fma(v, v, s); }
        });
      },
      [&](const Piece& p) {
        by_type(p.type, [&](auto type) {
          typedef Element<decltype(type)::value> E;
          const CNN_GLOBAL typename E::T* g = (const CNN_GLOBAL typename E::T*)p.from;
          const int n = p.n / E::V, last = n * E::V + at.thread;
          float rest = 0.0f;
          if (last < p.n) rest = E::get(g[last]);
          v4u r[NV];
#pragma unroll
          for (int q = 0; q < NV; ++q) {
            if (q * GT >= n) break;
            r[q] = v4u{0, 0, 0, 0};
            if (q * GT + at.thread < n) r[q] = *(const CNN_GLOBAL v4u_any*)(g + (q * GT + at.thread) * E::V);
          }
#pragma unroll
          for (int q = 0; q < NV; ++q) {
            if (q * GT >= n) break;
#pragma unroll
            for (int j = 0; j < E::V; ++j) { const double v = E::get(r[q], j); s = fma(v, v, s); }
          }
          s = fma((double)rest, (double)rest, s);
        });
      });
  return s;
}

template <class JOB, bool FAR>
__global__ void __launch_bounds__(GT) k_squares(JOB J, CNN_GLOBAL double* sums) {
  __shared__ double lds[GT / 64];
  const double s = sum_of_workgroup<GT>(squares_of<FAR>(J, share_of_workgroup()), lds);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// entries that fit no kernel's argument, to memory
__global__ void __launch_bounds__(128) k_table(TensorJob J, CNN_GLOBAL TensorEntry* at) {
  if ((int)threadIdx.x >= J.tensors) return;
  const TensorEntry& e = J.e[threadIdx.x];
  CNN_GLOBAL TensorEntry* o = at + threadIdx.x;
  o->from = e.from; o->to = e.to; o->n = e.n; o->chunk = e.chunk; o->type = e.type;
}

// the sums, asked for, and the root of what they come to
struct Sums {
  double v[LIST_SUMS / GT];
};
__device__ __forceinline__ Sums load_sums(const CNN_GLOBAL double* sums, int n) {
  Sums r;
#pragma unroll
  for (int k = 0; k < LIST_SUMS / GT; ++k) r.v[k] = (int)threadIdx.x + k * GT < n ? sums[threadIdx.x + k * GT] : 0.0;
  return r;
}
__device__ __forceinline__ double norm_of(const Sums& sums, double* lds) {
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < LIST_SUMS / GT; ++k) s += sums.v[k];
  return sqrt(sum_of_workgroup<GT>(s, lds));
}

__global__ void __launch_bounds__(GT) k_norm(const CNN_GLOBAL double* sums, int n, CNN_GLOBAL float* norm) {
  __shared__ double lds[GT / 64];
  const double v = norm_of(load_sums(sums, n), lds);
  if (threadIdx.x == 0) *norm = (float)v;
}

// ---- what is done with it ----
// A gradient times the factor, to its type.  fp32: the product in double.  Types of 16 bits: in float, the factor as the sum of
// two of them times a power of two, which keeps its 48 bits whatever its size (conversions to double and back bound fp16:
// 145 us for 100 M elements, bf16 108).
struct Factor {
  double f;
  float high, low;   // f = (high + low) 2^e, 0.5 <= high + low < 1
  int e;
};
__device__ __forceinline__ Factor factor_of(double f) {
  Factor r;
  r.f = f;
  const double m = frexp(f, &r.e);
  r.high = (float)m;
  r.low = (float)(m - r.high);
  return r;
}
template <int TYPE>
__device__ __forceinline__ typename Element<TYPE>::T times(float g, const Factor& f) {
  if (TYPE == ELEMENT_F32) return Element<TYPE>::make((float)(g * f.f));
  return Element<TYPE>::make(ldexpf(fmaf(g, f.high, g * f.low), f.e));
}

template <int TYPE>
__device__ __forceinline__ v4u times(v4u r, const Factor& f) {
  typedef Element<TYPE> E;
  v4u v;
#pragma unroll
  for (int j = 0; j < E::V; ++j) E::put(v, j, times<TYPE>(E::get(r, j), f));
  return v;
}

// to = f g of a share's chunks, f = max_norm / v where that is less than 1; to may be the gradients themselves (in_place: all are).
// norm(): v
template <bool FAR, class JOB, class Norm>
__device__ __forceinline__ void scale(const JOB& J, Share at, Norm norm, double max_norm, int in_place) {
  bool known = false, clips = false;
  Factor f;
  auto goes_on = [&]() {
    if (!known) {
      const double v = norm();
      clips = v < __builtin_inf() && v > max_norm;
      f = factor_of(clips ? max_norm / v : 1.0);
      known = true;
    }
    return clips || !in_place;
  };
  // the last chunks first: they are the ones that the launch before read last, and may still be in a cache
  for_chunks<FAR, true, false>(
      J, at, [](const Piece&) {}, goes_on,
      [&](const Piece& p, const v4u (&r)[NV]) {
        by_type(p.type, [&](auto type) {
          constexpr int TYPE = decltype(type)::value;
          CNN_GLOBAL typename Element<TYPE>::T* o = (CNN_GLOBAL typename Element<TYPE>::T*)p.to + p.begin;
#pragma unroll
          for (int q = 0; q < NV; ++q)
            __builtin_nontemporal_store(clips ? times<TYPE>(r[q], f) : r[q], (CNN_GLOBAL v4u_any*)(o + (q * GT + at.thread) * Element<TYPE>::V));
        });
      },
      [&](const Piece& p) {
        by_type(p.type, [&](auto type) {
          constexpr int TYPE = decltype(type)::value, V = Element<TYPE>::V;
          typedef typename Element<TYPE>::T T;
          const CNN_GLOBAL T* g = (const CNN_GLOBAL T*)p.from;
          CNN_GLOBAL T* o = (CNN_GLOBAL T*)p.to + p.begin;
          const int n = p.n / V, last = n * V + at.thread;
          T rest = {};
          if (last < p.n) rest = g[last];
          v4u r[NV];
#pragma unroll
          for (int q = 0; q < NV; ++q) {
            r[q] = v4u{0, 0, 0, 0};
            if (q * GT + at.thread < n) r[q] = *(const CNN_GLOBAL v4u_any*)(g + (q * GT + at.thread) * V);
          }
#pragma unroll
          for (int q = 0; q < NV; ++q)
            if (q * GT + at.thread < n)
              __builtin_nontemporal_store(clips ? times<TYPE>(r[q], f) : r[q], (CNN_GLOBAL v4u_any*)(o + (q * GT + at.thread) * V));
          if (last < p.n) o[last] = clips ? times<TYPE>(Element<TYPE>::get(rest), f) : rest;
        });
      });
  if (!known) goes_on();
}

// to (weights) -= lr f g; norm(): v
template <bool FAR, class JOB, class Norm>
__device__ __forceinline__ void update(const JOB& J, Share at, Norm norm, double max_norm, double lr) {
  bool known = false, finite = false;
  double f = 0.0;
  auto goes_on = [&]() {
    if (!known) {
      const double v = norm();
      finite = v < __builtin_inf();
      f = -lr * (v > max_norm ? max_norm / v : 1.0);
      known = true;
    }
    return finite;
  };
  auto one = [&](float w, float g) { return (float)fma(f, (double)g, (double)w); };
  v4f o[2 * NV];
  for_chunks<FAR, true, true>(
      J, at,
      [&](const Piece& p) {
        const CNN_GLOBAL float* w = (const CNN_GLOBAL float*)p.to + p.begin;
#pragma unroll
        for (int q = 0; q < NV; ++q) o[q] = __builtin_nontemporal_load((const CNN_GLOBAL v4f_any*)(w + (q * GT + at.thread) * 4));
        if (p.type != ELEMENT_F32) {
#pragma unroll
          for (int q = NV; q < 2 * NV; ++q) o[q] = __builtin_nontemporal_load((const CNN_GLOBAL v4f_any*)(w + (q * GT + at.thread) * 4));
        }
      },
      goes_on,
      [&](const Piece& p, const v4u (&r)[NV]) {
        by_type(p.type, [&](auto type) {
          typedef Element<decltype(type)::value> E;
          CNN_GLOBAL float* w = (CNN_GLOBAL float*)p.to + p.begin;
          constexpr int N = E::V == 4 ? NV : 2 * NV;
#pragma unroll
          for (int q = 0; q < N; ++q) {
            v4f v = o[q];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = one(v[j], E::V == 4 ? E::get(r[q], j) : E::get(r[q >> 1], (q & 1) * 4 + j));
            __builtin_nontemporal_store(v, (CNN_GLOBAL v4f_any*)(w + (q * GT + at.thread) * 4));
          }
        });
      },
      [&](const Piece& p) {
        by_type(p.type, [&](auto type) {
          typedef Element<decltype(type)::value> E;
          const CNN_GLOBAL typename E::T* g = (const CNN_GLOBAL typename E::T*)p.from;
          CNN_GLOBAL float* w = (CNN_GLOBAL float*)p.to + p.begin;
          const int fours = p.n >> 2, rest = (p.n & ~3) + at.thread;
          float w_rest = 0.0f, g_rest = 0.0f;
          if (rest < p.n) {
            w_rest = w[rest];
            g_rest = E::get(g[rest]);
          }
#pragma unroll 1
          for (int i0 = at.thread; i0 < fours; i0 += NV * GT) {   // (a float at a time, the widest colour net took 17.3 us in fp16, so 12.6)
            v4f u[NV];
            v4u r[NV];
#pragma unroll
            for (int q = 0; q < NV; ++q) {
              u[q] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
              r[q] = v4u{0, 0, 0, 0};
              const int i = i0 + q * GT;
              if (i >= fours) continue;
              u[q] = __builtin_nontemporal_load((const CNN_GLOBAL v4f_any*)(w + i * 4));
              if constexpr (E::V == 4) {
                r[q] = *(const CNN_GLOBAL v4u_any*)(g + i * 4);
              } else {
                const v2u v = *(const CNN_GLOBAL v2u_any*)(g + i * 4);
                r[q][0] = v[0];
                r[q][1] = v[1];
              }
            }
#pragma unroll
            for (int q = 0; q < NV; ++q) {
              const int i = i0 + q * GT;
              if (i >= fours) continue;
#pragma unroll
              for (int j = 0; j < 4; ++j) u[q][j] = one(u[q][j], E::get(r[q], j));
              __builtin_nontemporal_store(u[q], (CNN_GLOBAL v4f_any*)(w + i * 4));
            }
          }
          if (rest < p.n) w[rest] = one(w_rest, g_rest);
        });
      });
  if (!known) goes_on();
}

// v, and where it is wanted
__device__ __forceinline__ double give_norm(double v, CNN_GLOBAL float* norm) {
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
  return v;
}

// Whether the gradients are of an image that is passed over for its label (its norm is 0)
__device__ __forceinline__ bool passed_over(const TensorHead& J, CNN_GLOBAL float* norm) {
  if (!J.label || (J.label[0] >= 0 && J.label[0] < J.classes)) return false;
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = 0.0f;
  return true;
}

template <class JOB, bool FAR>
__global__ void __launch_bounds__(GT) k_scale(JOB J, const CNN_GLOBAL double* sums, double max_norm, CNN_GLOBAL float* norm, int in_place) {
  __shared__ double lds[GT / 64];
  const Sums all = load_sums(sums, J.sums);
  scale<FAR>(J, share_of_workgroup(), [&]() { return give_norm(norm_of(all, lds), norm); }, max_norm, in_place);
}

template <class JOB, bool FAR>
__global__ void __launch_bounds__(GT) k_update(JOB J, const CNN_GLOBAL double* sums, double max_norm, double lr, CNN_GLOBAL float* norm) {
  __shared__ double lds[GT / 64];
  if (passed_over(J, norm)) return;
  const Sums all = load_sums(sums, J.sums);
  update<FAR>(J, share_of_workgroup(), [&]() { return give_norm(norm_of(all, lds), norm); }, max_norm, lr);
}

// Small lists in one launch: every workgroup, four groups of GT threads, adds the squares of all chunks for itself (the same way, so
// that they agree) and goes over its own.  OP 0: the norm alone, 1: scale (not in place: another workgroup may still read what
// one has written), 2: update.
constexpr int SMALL_GROUPS = 4;
template <class JOB, int OP>
__global__ void __launch_bounds__(GT * SMALL_GROUPS) k_small(JOB J, double max_norm, double lr, CNN_GLOBAL float* norm) {
  __shared__ double lds[SMALL_GROUPS * GT / 64];
  if (passed_over(J, norm)) return;
  const unsigned group = __builtin_amdgcn_readfirstlane(threadIdx.x / GT);
  const int thread = threadIdx.x % GT;
  const double v = give_norm(sqrt(sum_of_workgroup<GT * SMALL_GROUPS>(squares_of<false>(J, Share{group, SMALL_GROUPS, thread}), lds)), norm);
  const Share own = {blockIdx.x * SMALL_GROUPS + group, gridDim.x * SMALL_GROUPS, thread};
  if (OP == 1) scale<false>(J, own, [&]() { return v; }, max_norm, 0);
  if (OP == 2) update<false>(J, own, [&]() { return v; }, max_norm, lr);
}

constexpr unsigned APPLY_GRID = 2048;

// f(the argument that a kernel takes, whether its entries lie in memory)
template <class F>
hipError_t with_job(const TensorJob& J, F f) {
  if (!J.table && J.tensors > LIST_FEW) {
    f(J, std::false_type());
  } else {
    TensorJobFew few;
    static_cast<TensorHead&>(few) = J;
    if (J.table) {
      f(few, std::true_type());
    } else {
      for (int t = 0; t < J.tensors; ++t) few.e[t] = J.e[t];
      f(few, std::false_type());
    }
  }
  return hipGetLastError();
}

unsigned apply_grid(const TensorJob& J) { return std::max(1u, std::min(J.chunks, APPLY_GRID)); }

}  // namespace

hipError_t launch_table(hipStream_t stream, const TensorJob& J, TensorEntry* at) {
  hipLaunchKernelGGL(k_table, dim3(1), dim3(128), 0, stream, J, (CNN_GLOBAL TensorEntry*)at);
  return hipGetLastError();
}

hipError_t launch_squares(hipStream_t stream, const TensorJob& J, double* sums) {
  return with_job(J, [&](const auto& job, auto far) {
    hipLaunchKernelGGL((k_squares<std::decay_t<decltype(job)>, decltype(far)::value>), dim3((unsigned)J.sums), dim3(GT), 0, stream, job, (CNN_GLOBAL double*)sums);
  });
}

// Whether one launch does it (k_small; not where anything is in place).  Its time grows with the chunks: those of 16-bit types hold twice
// the elements and count half more or, where an update's weights go with them, twice.  us in one / two launches, a call through Python:
// fp32 norm of 14 chunks 5.6 / 8.8, 36 7.5 / 8.8, 44 8.6 / 8.9 (in eight tensors 9.7 / 8.8); clipped 18 6.9 / 9.3, 30 8.7 / 9.7, 36 9.6 / 9.8
// (10.4 / 9.8); updated 30 9.1 / 9.7, 36 10.2 / 9.8; bf16 norm of 22 7.6 / 8.8, 30 9.5 / 8.9; clipped 18 9.2 / 9.8, 22 10.2 / 9.8; updated
// 14 9.6 / 9.8, 18 10.7 / 9.9.
bool list_is_small(const TensorJob& J, int op) {
  constexpr unsigned MOST[3] = {80, 64, 60};   // twice the chunks of fp32
  if (J.table || 2 * J.chunks > MOST[op]) return false;
  unsigned cost = 2 * J.chunks;
  for (int t = 0; t < J.tensors; ++t) {
    const unsigned end = t + 1 < J.tensors ? J.e[t + 1].chunk : J.chunks;
    if (J.e[t].type != ELEMENT_F32) cost += (op == 2 ? 2 : 1) * (end - J.e[t].chunk);
  }
  return cost <= MOST[op];
}

hipError_t launch_small(hipStream_t stream, const TensorJob& J, int op, double max_norm, double lr, float* norm) {
  const dim3 grid(op == 0 ? 1 : std::max(1u, (J.chunks + SMALL_GROUPS - 1) / SMALL_GROUPS)), threads(GT * SMALL_GROUPS);
  CNN_GLOBAL float* n = (CNN_GLOBAL float*)norm;
  return with_job(J, [&](const auto& job, auto) {
    typedef std::decay_t<decltype(job)> JOB;
    if (op == 0) hipLaunchKernelGGL((k_small<JOB, 0>), grid, threads, 0, stream, job, max_norm, lr, n);
    else if (op == 1) hipLaunchKernelGGL((k_small<JOB, 1>), grid, threads, 0, stream, job, max_norm, lr, n);
    else hipLaunchKernelGGL((k_small<JOB, 2>), grid, threads, 0, stream, job, max_norm, lr, n);
  });
}

hipError_t launch_norm(hipStream_t stream, const double* sums, int n, float* norm) {
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(GT), 0, stream, (const CNN_GLOBAL double*)sums, n, (CNN_GLOBAL float*)norm);
  return hipGetLastError();
}

hipError_t launch_scale(hipStream_t stream, const TensorJob& J, const double* sums, double max_norm, float* norm, int in_place) {
  return with_job(J, [&](const auto& job, auto far) {
    hipLaunchKernelGGL((k_scale<std::decay_t<decltype(job)>, decltype(far)::value>), dim3(apply_grid(J)), dim3(GT), 0, stream, job,
                       (const CNN_GLOBAL double*)sums, max_norm, (CNN_GLOBAL float*)norm, in_place);
  });
}

hipError_t launch_update(hipStream_t stream, const TensorJob& J, const double* sums, double max_norm, double lr, float* norm) {
  return with_job(J, [&](const auto& job, auto far) {
    hipLaunchKernelGGL((k_update<std::decay_t<decltype(job)>, decltype(far)::value>), dim3(apply_grid(J)), dim3(GT), 0, stream, job,
                       (const CNN_GLOBAL double*)sums, max_norm, lr, (CNN_GLOBAL float*)norm);
  });
}

}  // namespace cnn355
