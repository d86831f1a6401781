// Elements of a caller's tensors, fp32, bf16 or fp16, 16 bytes a lane: arithmetic is fp32 or wider whatever the type.
// (Device code; included behind the definition of CNN_GLOBAL.)
#pragma once
#include "cnn355_ops.h"

namespace cnn355 {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
// 16 bytes at any element: rows and tensors start where they do, and the hardware takes an address of any alignment
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));

template <int TYPE> struct Element;
template <> struct Element<ELEMENT_F32> {
  typedef float T;
  static constexpr int V = 4;                       // elements of 16 bytes
  static constexpr unsigned MASKED = 0xff800000u;   // -inf
  static __device__ __forceinline__ float get(v4u r, int j) {
    const unsigned b = r[j];   // (a bit cast of an element in its vector would take the first)
    return __builtin_bit_cast(float, b);
  }
  static __device__ __forceinline__ float get(T v) { return v; }
  static __device__ __forceinline__ T make(float v) { return v; }
  static __device__ __forceinline__ void put(v4u& r, int j, T v) { r[j] = __builtin_bit_cast(unsigned, v); }
};
struct Element16 {   // what the two types of 16 bits have in common
  static constexpr int V = 8;
  static __device__ __forceinline__ unsigned short bits(v4u r, int j) { return (unsigned short)(j & 1 ? r[j >> 1] >> 16 : r[j >> 1]); }
  static __device__ __forceinline__ void put_bits(v4u& r, int j, unsigned v) {
    r[j >> 1] = j & 1 ? (r[j >> 1] & 0xffffu) | v << 16 : (r[j >> 1] & 0xffff0000u) | v;
  }
};
template <> struct Element<ELEMENT_BF16> : Element16 {
  typedef unsigned short T;
  static constexpr unsigned MASKED = 0xff80ff80u;
  static __device__ __forceinline__ float get(v4u r, int j) {
    return __builtin_bit_cast(float, j & 1 ? r[j >> 1] & 0xffff0000u : r[j >> 1] << 16);
  }
  static __device__ __forceinline__ float get(T v) { return __builtin_bit_cast(float, (unsigned)v << 16); }
  static __device__ __forceinline__ T make(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }   // to the nearest
  static __device__ __forceinline__ void put(v4u& r, int j, T v) { put_bits(r, j, v); }
};
template <> struct Element<ELEMENT_F16> : Element16 {
  typedef _Float16 T;
  static constexpr unsigned MASKED = 0xfc00fc00u;
  static __device__ __forceinline__ float get(v4u r, int j) { return (float)__builtin_bit_cast(_Float16, bits(r, j)); }
  static __device__ __forceinline__ float get(T v) { return (float)v; }
  static __device__ __forceinline__ T make(float v) { return (_Float16)v; }
  static __device__ __forceinline__ void put(v4u& r, int j, T v) { put_bits(r, j, __builtin_bit_cast(unsigned short, v)); }
};

// 16 bytes from element `at` on of a row, -inf from element `end` on and in front of `begin`
template <int TYPE>
__device__ __forceinline__ v4u load16(const CNN_GLOBAL typename Element<TYPE>::T* row, int at, int end, int begin = 0) {
  typedef Element<TYPE> E;
  if (at >= begin && at + E::V <= end) return *(const CNN_GLOBAL v4u_any*)(row + at);
  v4u r = {E::MASKED, E::MASKED, E::MASKED, E::MASKED};
#pragma unroll
  for (int j = 0; j < E::V; ++j)
    if (at + j >= begin && at + j < end) E::put(r, j, row[at + j]);
  return r;
}

}  // namespace cnn355
