// Fully connected layers (Sec. 2.4) whose weights are held in 4 bits, a scale for every group of them:
//
//   y[row][o] = bias[o] + sum over groups g of scale[o][g] * sum over i in g of x[row][i] * value(code[o][i])
//
// The inner sums are products on the matrix cores (v_mfma_f32_16x16x32_bf16 / _f16): 16 rows of x times 16 outputs, 32 columns
// at a time.  Values of codes are exact in 16 bits, so are the products, and a group's scale is applied to the sum in fp32:
// nothing of a weight is rounded again.  fp32 rows go in as three rows of bf16 that add up to them exactly (24 bits in three times 8),
// and their three sums are added at the end.
//
// For few rows the codes are what is read: half a byte a weight, once.  A wavefront takes 128 columns of 16 outputs at a time
// (a slab: 16 bytes a lane), the wavefronts of a workgroup one in turn each, and their sums meet in LDS at the end, always in the same
// order.  Many rows (k_product_tile) have their rows in LDS, for four wavefronts on outputs of their own.
//
// 4096 x 4096 weights times one bf16 row 5.2 us (chains of loads), 131072 x 4096 times 16 rows 72 (4.0 TB/s of codes, scales and sums),
// 8192 x 8192 times 256 rows 55 (625 TFLOP/s: two wavefronts a SIMD, for their registers, and a barrier a slab, so that a third of their clocks are
// waits; vector instructions, which make values of codes, issue in half of the clocks, the matrix cores are busy in 22 %).  Groups of 32 spill in
// that form: 79 (bf16 68).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#define CNN_GLOBAL __attribute__((address_space(1)))
#include "cnn355_ops.h"
#include "cnn355_elements.h"

namespace cnn355 {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

// rows of x that a tile of 16 rows of the product holds, and parts of each
template <int TYPE> constexpr int PIECES = TYPE == ELEMENT_F32 ? 3 : 1;
template <int TYPE> constexpr int TILE_ROWS = 16 / PIECES<TYPE>;

template <int TYPE>
__device__ __forceinline__ f4 multiply(v4u a, v4u b, f4 c) {
  if constexpr (TYPE == ELEMENT_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// The values of the eight codes of a word, 16 bits each, in order.  INT4: a sixteenth of them (the instruction's own scale).
template <int TYPE, int KIND>
__device__ __forceinline__ v4u values_of(unsigned w) {
  v4u r;
  if constexpr (KIND == CODES_E2M1) {
    if constexpr (TYPE == ELEMENT_F16) {
      r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
      r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
      r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
      r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
    } else {
      r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
      r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
      r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
      r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
    }
  } else {
    w ^= 0x88888888u;   // two's complement
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = __builtin_amdgcn_cvt_off_f32_i4(w >> (8 * j)), b = __builtin_amdgcn_cvt_off_f32_i4(w >> (8 * j + 4));
      if constexpr (TYPE == ELEMENT_F16) r[j] = __builtin_bit_cast(unsigned, h2{(_Float16)a, (_Float16)b});
      else r[j] = __builtin_bit_cast(unsigned, bf2{(__bf16)a, (__bf16)b});
    }
  }
  return r;
}

// Piece 0, 1 or 2 of a float in bf16 (in the upper half of the word), cut off and not rounded: 8 bits each, together all of them.
// Infinities and NaN are in the first alone.
__device__ __forceinline__ unsigned piece_of(float v, int piece) {
  const unsigned first = piece > 0 ? 0xffff0000u : 0, second = piece > 1 ? 0xffff0000u : 0;
  float r = piece == 0 || __builtin_fabsf(v) < __builtin_inff() ? __builtin_canonicalizef(v) : 0.f;
  r -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, r) & first);
  r -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, r) & second);
  return __builtin_bit_cast(unsigned, r);
}

// Eight columns of a row from `at` on, those from n_in on 0 (WHOLE: there are none).
template <int TYPE, bool WHOLE>
__device__ __forceinline__ v4u columns_of(const CNN_GLOBAL typename Element<TYPE>::T* row, int at, int n_in, int piece) {
  typedef Element<TYPE> E;
  v4u r = {0, 0, 0, 0};
  if constexpr (TYPE != ELEMENT_F32) {
    if (WHOLE || at + 8 <= n_in) return *(const CNN_GLOBAL v4u_any*)(row + at);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (at + j < n_in) E::put(r, j, row[at + j]);
  } else {
    v4u a = r, b = r;
    if (WHOLE || at + 8 <= n_in) {
      a = *(const CNN_GLOBAL v4u_any*)(row + at);
      b = *(const CNN_GLOBAL v4u_any*)(row + at + 4);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (at + j < n_in) E::put(j < 4 ? a : b, j & 3, row[at + j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 2 * (j & 1);
      const float low = j < 2 ? E::get(a, i) : E::get(b, i), high = j < 2 ? E::get(a, i + 1) : E::get(b, i + 1);
      r[j] = __builtin_amdgcn_perm(piece_of(high, piece), piece_of(low, piece), 0x07060302);   // their upper halves
    }
  }
  return r;
}

// 16 bytes of a row of codes from byte `at` on, those from `bytes` on 0 (WHOLE: there are none).
template <bool WHOLE>
__device__ __forceinline__ v4u codes_of(const CNN_GLOBAL unsigned char* row, long long at, long long bytes) {
  typedef unsigned v4u_byte __attribute__((ext_vector_type(4), aligned(1)));
  if (WHOLE || at + 16 <= bytes) return *(const CNN_GLOBAL v4u_byte*)(row + at);
  v4u r = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (at + j < bytes) r[j >> 2] |= (unsigned)row[at + j] << (8 * (j & 3));
  return r;
}

// A 4 x 4 transpose of words between a lane's registers and the wavefront's quarters: word t of quarter q becomes word q of
// quarter t.  A lane asks for 16 bytes of its row that follow each other, which belong to 32 columns; the matrix cores take 32
// columns of all quarters, 8 each.
__device__ __forceinline__ v4u across_quarters(v4u w) {
  auto p = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto q = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto a = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false);
  auto b = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
  return v4u{a[0], a[1], b[0], b[1]};
}

// 16 rows of 64 bytes are asked for with four lanes beside each other on a row, 16 bytes each (a lane a row, with the lanes beside it on
// other rows, costs the caches four times as many accesses: 256 rows times 8192 x 8192 codes took 61 us, so 52), and the matrix cores want
// lane 16 q + r to hold the 16 bytes q of row r: they pass through a place of the wavefront's own in LDS, 16 bytes q of row r at
// 4 r + (q ^ r / 4), so that both sides meet all banks.
__device__ __forceinline__ v4u turned(v4u* place, v4u v) {
  const int lane = threadIdx.x & 63, column = lane & 15, quarter = lane >> 4;
  place[(lane & ~3) | ((lane & 3) ^ (lane >> 4))] = v;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const v4u r = place[column * 4 + (quarter ^ (column >> 2))];
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  return r;
}

// What a wavefront asks for together: the codes and rows of a slab.
template <int RT, int OT>
struct Slab {
  v4u codes[OT], x[RT][4];
};

// The scales of four slabs, one for every STEPS products of 32 columns.  A quarter of the wavefront asks for those of one slab, which lie
// side by side, and every lane gets all of them from its output's lanes of the quarters: asked for one by one, 131072 x 4096 codes in
// groups of 64 took 96 us.
template <int TYPE, int STEPS>
struct Scales {
  static constexpr int N = 4 / STEPS, BYTES = N * (int)element_bytes(TYPE), WORDS = (BYTES + 3) / 4;
  unsigned words[WORDS];
  __device__ __forceinline__ void ask(const CNN_GLOBAL typename Element<TYPE>::T* row, int slab, int group_log2) {
    typedef unsigned word_any __attribute__((aligned(2)));
    typedef unsigned v2u_any __attribute__((ext_vector_type(2), aligned(2)));
    const CNN_GLOBAL typename Element<TYPE>::T* at = row + ((slab * PRODUCT_SLAB) >> group_log2);
    if constexpr (BYTES == 2) {
      words[0] = __builtin_bit_cast(unsigned short, at[0]);
    } else if constexpr (BYTES == 4) {
      words[0] = *(const CNN_GLOBAL word_any*)at;
    } else if constexpr (BYTES == 8) {
      const v2u_any r = *(const CNN_GLOBAL v2u_any*)at;
      words[0] = r[0];
      words[1] = r[1];
    } else {
      const v4u r = *(const CNN_GLOBAL v4u_any*)at;
#pragma unroll
      for (int j = 0; j < 4; ++j) words[j] = r[j];
    }
  }
  // those of slab i
  __device__ __forceinline__ Scales of(int i) const {
    Scales r;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const auto a = __builtin_amdgcn_permlane16_swap(words[w], words[w], false, false);   // the even quarters' twice, the odd ones' twice
      const auto b = __builtin_amdgcn_permlane32_swap(a[i & 1], a[i & 1], false, false);
      r.words[w] = b[i >> 1];
    }
    return r;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (TYPE == ELEMENT_F32) return __builtin_bit_cast(float, words[i]);
    else if constexpr (TYPE == ELEMENT_BF16) return __builtin_bit_cast(float, i & 1 ? words[i / 2] & 0xffff0000u : words[i / 2] << 16);
    else return (float)__builtin_bit_cast(_Float16, (unsigned short)(i & 1 ? words[i / 2] >> 16 : words[i / 2]));
  }
};

// wavefronts of a workgroup at most: as many as there are registers for
template <int RT, int OT> constexpr int WAVES = RT * OT >= 4 ? 8 : 16;

// RT tiles of rows times OT tiles of 16 outputs a workgroup; a scale for every STEPS products of 32 columns (4: one or less a slab).
// TURN: rows pass through LDS like codes (of up to four rows, lanes beside each other ask for the same 16 bytes).
template <int TYPE, int KIND, int RT, int OT, int STEPS, bool TURN>
__global__ __launch_bounds__((64 * WAVES<RT, OT>)) void k_product(ProductJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int PC = PIECES<TYPE>, TR = TILE_ROWS<TYPE>;
  extern __shared__ v4u lds[];   // a place of 1 KB for each wavefront; at the end [wavefront][RT][OT][16 rows][16 outputs] of float
  float* red = (float*)lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int column = lane & 15, quarter = lane >> 4;
  const int out0 = blockIdx.x * (16 * OT);
  const long long row0 = (long long)blockIdx.y * (TR * RT);
  const int whole = J.n_in / PRODUCT_SLAB;
  const long long bytes = ((long long)J.n_in + 1) / 2;
  v4u* place = lds + wave * 64;

  // what is past the last row or output reads the last one's, and is not stored
  const CNN_GLOBAL T* x[RT];
  const int x_row = TURN ? lane >> 2 : column, x_part = TURN ? lane & 3 : quarter, piece = PC == 1 ? 0 : x_row % PC;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const long long row = row0 + r * TR + (PC == 1 ? x_row : x_row / PC < TR ? x_row / PC : TR - 1);
    x[r] = (const CNN_GLOBAL T*)J.x + (row < J.rows ? row : J.rows - 1) * J.x_stride;
  }
  const CNN_GLOBAL unsigned char* codes[OT];
  const CNN_GLOBAL T* scales[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) {
    const int out = out0 + o * 16, asked = out + (lane >> 2), mine = out + column;
    codes[o] = J.codes + (long long)(asked < J.n_out ? asked : J.n_out - 1) * J.code_stride;
    scales[o] = (const CNN_GLOBAL T*)J.scales + (long long)(mine < J.n_out ? mine : J.n_out - 1) * J.groups;
  }
  f4 sum[RT][OT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int o = 0; o < OT; ++o) sum[r][o] = f4{0.f, 0.f, 0.f, 0.f};

  auto ask = [&](auto all, int slab, Slab<RT, OT>& s) {
    const int k0 = slab * PRODUCT_SLAB;
#pragma unroll
    for (int o = 0; o < OT; ++o) s.codes[o] = codes_of<all>(codes[o], k0 / 2 + (lane & 3) * 16, bytes);
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int t = 0; t < 4; ++t) s.x[r][t] = columns_of<TYPE, all>(x[r], k0 + t * 32 + x_part * 8, J.n_in, piece);
  };
  auto add = [&](Slab<RT, OT>& s, auto scale_of) {
    if constexpr (TURN) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < 4; ++t) s.x[r][t] = turned(place, s.x[r][t]);
    }
#pragma unroll
    for (int o = 0; o < OT; ++o) {
      const v4u w = across_quarters(turned(place, s.codes[o]));
      f4 part[RT];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const v4u b = values_of<TYPE, KIND>(w[t]);
        const float scale = scale_of(o, t / STEPS);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          part[r] = multiply<TYPE>(s.x[r][t], b, t % STEPS ? part[r] : f4{0.f, 0.f, 0.f, 0.f});
          if ((t + 1) % STEPS == 0) sum[r][o] += part[r] * scale;
        }
      }
    }
  };
  // The wavefront's whole slabs, `waves` apart: the next one is asked for before one is worked on, scales of four before they are needed.
  typedef std::true_type All;
  const int mine = whole > wave ? (whole - wave + waves - 1) / waves : 0, last = wave + (mine - 1) * waves;
  auto slab_of = [&](int i) { return wave + i * waves; };
  Slab<RT, OT> slab[2];
  Scales<TYPE, STEPS> now[OT], next[OT];
  auto ask_scales = [&](int i) {
    const int s = slab_of(i + quarter);
#pragma unroll
    for (int o = 0; o < OT; ++o) next[o].ask(scales[o], s < last ? s : last, J.group_log2);
  };
  if (mine > 0) {
    ask(All(), slab_of(0), slab[0]);
    ask_scales(0);
  }
  for (int i0 = 0; i0 < mine; i0 += 4) {
#pragma unroll
    for (int o = 0; o < OT; ++o) now[o] = next[o];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int i = i0 + d;
      if (i >= mine) break;
      if (i + 1 < mine) ask(All(), slab_of(i + 1), slab[(d + 1) & 1]);
      if (d == 0 && i0 + 4 < mine) ask_scales(i0 + 4);
      Scales<TYPE, STEPS> scale[OT];
#pragma unroll
      for (int o = 0; o < OT; ++o) scale[o] = now[o].of(d);
      add(slab[d & 1], [&](int o, int step) { return scale[o].get(step); });
    }
  }
  if (whole * PRODUCT_SLAB < J.n_in && whole % waves == wave) {   // columns that end inside a slab
    ask(std::false_type(), whole, slab[0]);
    add(slab[0], [&](int o, int step) {
      const int g = (whole * PRODUCT_SLAB + step * STEPS * 32) >> J.group_log2;
      const float scale = E::get(scales[o][g < J.groups ? g : J.groups - 1]);
      return g < J.groups ? scale : 0.f;   // (past the columns: an infinite scale times none of them is nothing)
    });
  }
  __syncthreads();

  // lane: output `column`, rows 4 quarter + i of each tile
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int o = 0; o < OT; ++o)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[(((wave * RT + r) * OT + o) * 16 + quarter * 4 + i) * 16 + column] = sum[r][o][i];
  __syncthreads();
  for (int at = threadIdx.x; at < RT * TR * OT * 16; at += blockDim.x) {
    const int c = at % 16, o = at / 16 % OT, r = at / (16 * OT);
    const int out = out0 + o * 16 + c;
    const long long row = row0 + r;
    if (out >= J.n_out || row >= J.rows) continue;
    float v = 0.f;
#pragma unroll
    for (int p = 0; p < PC; ++p) {
      const float before = v;
      for (int k = 0; k < waves; ++k) v += red[(((k * RT + r / TR) * OT + o) * 16 + r % TR * PC + p) * 16 + c];
      if (p && __builtin_isinf(before)) v = before;   // (an infinite scale's: it makes NaN of the other pieces' sums, nothing mostly)
    }
    if (KIND == CODES_INT4) v *= 16.f;
    if (J.bias) v += J.bias[out];
    if (J.y_type == ELEMENT_F32) ((CNN_GLOBAL float*)J.y)[row * J.y_stride + out] = v;
    else ((CNN_GLOBAL T*)J.y)[row * J.y_stride + out] = E::make(v);
  }
}

// Many rows: 64 rows (of pieces) times 128 outputs a workgroup of eight wavefronts: four of them 32 outputs each, on either half of the
// columns.  A slab of the rows is in LDS for the four, twice: the next one is written while one is worked on.  16 bytes c of row r
// are at place c ^ (r % 16) of the row, so that the 16 rows of a tile are read from all banks.  Slabs are asked for two before they are
// worked on.
constexpr int TILE_R = 4, TILE_O = 2, TILE_GROUPS = 4, TILE_HALVES = 2, TILE_THREADS = 64 * TILE_GROUPS * TILE_HALVES;
constexpr int TILE_OUTS = 16 * TILE_O * TILE_GROUPS, TILE_LDS = TILE_HALVES * 2 * TILE_R * 16 * 2 * PRODUCT_SLAB + TILE_THREADS * 16;

template <int TYPE, int KIND, int STEPS>
__global__ __launch_bounds__(TILE_THREADS) void k_product_tile(ProductJob J) {
  typedef Element<TYPE> E;
  typedef typename E::T T;
  constexpr int PC = PIECES<TYPE>, TR = TILE_ROWS<TYPE>, RT = TILE_R, OT = TILE_O;
  extern __shared__ v4u lds[];   // [half][2][64 rows][16 places], 1 KB for each wavefront; at the end [64 rows][128 outputs] of float
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = wave / TILE_GROUPS, column = lane & 15, quarter = lane >> 4, in_half = tid % (64 * TILE_GROUPS);
  const int block0 = blockIdx.x * TILE_OUTS, out0 = block0 + wave % TILE_GROUPS * (16 * OT);
  const long long row0 = (long long)blockIdx.y * (TR * RT);
  const int whole = J.n_in / PRODUCT_SLAB, steps = (whole + 1) / 2;   // (the second half's last step may have nothing)
  const int first = half ? steps : 0, end = half ? whole : steps;
  const long long bytes = ((long long)J.n_in + 1) / 2;
  v4u* const stage = lds + half * (2 * RT * 16 * 16);
  v4u* const turning = lds + TILE_HALVES * 2 * RT * 16 * 16 + wave * 64;

  // what this thread brings of a slab: 16 bytes of rows t, 16 + t, ...
  const int place = in_half & 15, row16 = in_half >> 4, piece = PC == 1 ? 0 : row16 % PC;
  const CNN_GLOBAL T* x[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const long long row = row0 + r * TR + (PC == 1 ? row16 : row16 / PC < TR ? row16 / PC : TR - 1);
    x[r] = (const CNN_GLOBAL T*)J.x + (row < J.rows ? row : J.rows - 1) * J.x_stride;
  }
  const CNN_GLOBAL unsigned char* codes[OT];
  const CNN_GLOBAL T* scales[OT];
#pragma unroll
  for (int o = 0; o < OT; ++o) {
    const int asked = out0 + o * 16 + (lane >> 2), mine = out0 + o * 16 + column;
    codes[o] = J.codes + (long long)(asked < J.n_out ? asked : J.n_out - 1) * J.code_stride;
    scales[o] = (const CNN_GLOBAL T*)J.scales + (long long)(mine < J.n_out ? mine : J.n_out - 1) * J.groups;
  }
  struct Asked {
    v4u x[RT], codes[OT];
  };
  Asked asked[2];
  Scales<TYPE, STEPS> now[OT], next[OT];   // of four slabs
  auto ask_scales = [&](int slab) {
#pragma unroll
    for (int o = 0; o < OT; ++o) next[o].ask(scales[o], slab + quarter < end ? slab + quarter : end - 1, J.group_log2);
  };
  auto ask = [&](int slab, Asked& next) {
    const int k0 = slab * PRODUCT_SLAB;
#pragma unroll
    for (int o = 0; o < OT; ++o) next.codes[o] = codes_of<true>(codes[o], k0 / 2 + (lane & 3) * 16, bytes);
#pragma unroll
    for (int r = 0; r < RT; ++r) next.x[r] = columns_of<TYPE, true>(x[r], k0 + place * 8, J.n_in, piece);
  };
  auto put = [&](int buffer, const Asked& next) {
#pragma unroll
    for (int r = 0; r < RT; ++r) stage[buffer * (RT * 256) + (r * 16 + row16) * 16 + (place ^ row16)] = next.x[r];
  };

  f4 sum[RT][OT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int o = 0; o < OT; ++o) sum[r][o] = f4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](int buffer, const v4u (&w)[OT], auto scale_of) {
    const v4u* rows = stage + buffer * (RT * 256) + column * 16;
    f4 part[RT][OT];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v4u a[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) a[r] = rows[r * 256 + ((t * 4 + quarter) ^ column)];
#pragma unroll
      for (int o = 0; o < OT; ++o) {
        const v4u b = values_of<TYPE, KIND>(w[o][t]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          part[r][o] = multiply<TYPE>(a[r], b, t % STEPS ? part[r][o] : f4{0.f, 0.f, 0.f, 0.f});
          if ((t + 1) % STEPS == 0) sum[r][o] += part[r][o] * scale_of(o, t / STEPS);
        }
      }
    }
  };
  if (first < end) {
    ask(first, asked[0]);
    ask_scales(first);
    if (first + 1 < end) ask(first + 1, asked[1]);
    put(0, asked[0]);
  }
  for (int i0 = 0; i0 < steps; i0 += 4) {
#pragma unroll
    for (int o = 0; o < OT; ++o) now[o] = next[o];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int i = i0 + d, slab = first + i;
      if (i >= steps) break;
      __syncthreads();
      if (slab >= end) continue;
      v4u w[OT];
      Scales<TYPE, STEPS> scale[OT];
#pragma unroll
      for (int o = 0; o < OT; ++o) {
        w[o] = across_quarters(turned(turning, asked[d & 1].codes[o]));
        scale[o] = now[o].of(d);
      }
      if (slab + 2 < end) ask(slab + 2, asked[d & 1]);
      if (d == 0 && slab + 4 < end) ask_scales(slab + 4);
      add(i & 1, w, [&](int o, int step) { return scale[o].get(step); });
      if (slab + 1 < end) put((i + 1) & 1, asked[(d + 1) & 1]);
    }
  }
  if (whole * PRODUCT_SLAB < J.n_in) {   // columns that end inside a slab: the first half's
    const int k0 = whole * PRODUCT_SLAB;
    v4u w[OT];
    __syncthreads();
    if (!half) {
#pragma unroll
      for (int r = 0; r < RT; ++r) asked[0].x[r] = columns_of<TYPE, false>(x[r], k0 + place * 8, J.n_in, piece);
      put(0, asked[0]);
#pragma unroll
      for (int o = 0; o < OT; ++o) w[o] = across_quarters(turned(turning, codes_of<false>(codes[o], k0 / 2 + (lane & 3) * 16, bytes)));
    }
    __syncthreads();
    if (!half)
      add(0, w, [&](int o, int step) {
        const int g = (k0 + step * STEPS * 32) >> J.group_log2;
        const float scale = E::get(scales[o][g < J.groups ? g : J.groups - 1]);
        return g < J.groups ? scale : 0.f;
      });
  }
  __syncthreads();
  float* red = (float*)lds;
  auto at = [&](int r, int o, int i) -> float& { return red[(r * 16 + quarter * 4 + i) * TILE_OUTS + (out0 - block0) + o * 16 + column]; };
  if (half) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i) at(r, o, i) = sum[r][o][i];
  }
  __syncthreads();
  if (!half) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int o = 0; o < OT; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i) at(r, o, i) += sum[r][o][i];
  }
  __syncthreads();
  for (int i = tid; i < RT * TR * TILE_OUTS; i += TILE_THREADS) {
    const int o = i % TILE_OUTS, r = i / TILE_OUTS, out = block0 + o;
    const long long row = row0 + r;
    if (out >= J.n_out || row >= J.rows) continue;
    float v = 0.f;
#pragma unroll
    for (int p = 0; p < PC; ++p) {
      const float before = v;
      v += red[(r / TR * 16 + r % TR * PC + p) * TILE_OUTS + o];
      if (p && __builtin_isinf(before)) v = before;   // (an infinite scale's)
    }
    if (KIND == CODES_INT4) v *= 16.f;
    if (J.bias) v += J.bias[out];
    if (J.y_type == ELEMENT_F32) ((CNN_GLOBAL float*)J.y)[row * J.y_stride + out] = v;
    else ((CNN_GLOBAL T*)J.y)[row * J.y_stride + out] = E::make(v);
  }
}

// launch(J, workgroups over the rows) for as many rows at a time as a grid's second axis has workgroups
template <class F>
hipError_t over_rows(const ProductJob& J, int rows_each, F launch) {
  const long long down = (J.rows + rows_each - 1) / rows_each;
  for (long long d = 0; d < down; d += 65535) {
    ProductJob P = J;
    const long long first = d * rows_each;
    P.x = (const CNN_GLOBAL char*)J.x + first * J.x_stride * (long long)element_bytes(J.type);
    P.y = (CNN_GLOBAL char*)J.y + first * J.y_stride * (long long)element_bytes(J.y_type);
    P.rows = J.rows - first;
    launch(P, (unsigned)std::min(down - d, 65535ll));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int TYPE, int KIND, int RT, int OT, bool TURN>
hipError_t launch_few(hipStream_t stream, const ProductJob& J, int waves) {
  const unsigned across = (unsigned)((J.n_out + 16 * OT - 1) / (16 * OT));
  const size_t lds = (size_t)waves * RT * OT * 1024;
  return over_rows(J, TILE_ROWS<TYPE> * RT, [&](const ProductJob& P, unsigned down) {
    if (J.group_log2 >= 7) hipLaunchKernelGGL((k_product<TYPE, KIND, RT, OT, 4, TURN>), dim3(across, down), dim3(64 * waves), lds, stream, P);
    else if (J.group_log2 == 6) hipLaunchKernelGGL((k_product<TYPE, KIND, RT, OT, 2, TURN>), dim3(across, down), dim3(64 * waves), lds, stream, P);
    else hipLaunchKernelGGL((k_product<TYPE, KIND, RT, OT, 1, TURN>), dim3(across, down), dim3(64 * waves), lds, stream, P);
  });
}

template <int TYPE, int KIND, int STEPS>
hipError_t launch_tiles(hipStream_t stream, const ProductJob& J) {
  const unsigned across = (unsigned)((J.n_out + TILE_OUTS - 1) / TILE_OUTS);
  const hipError_t e = hipFuncSetAttribute((const void*)k_product_tile<TYPE, KIND, STEPS>, hipFuncAttributeMaxDynamicSharedMemorySize, TILE_LDS);
  if (e != hipSuccess) return e;
  return over_rows(J, TILE_ROWS<TYPE> * TILE_R, [&](const ProductJob& P, unsigned down) {
    hipLaunchKernelGGL((k_product_tile<TYPE, KIND, STEPS>), dim3(across, down), dim3(TILE_THREADS), TILE_LDS, stream, P);
  });
}

template <int TYPE, int KIND>
hipError_t launch_many(hipStream_t stream, const ProductJob& J) {
  if (J.group_log2 >= 7) return launch_tiles<TYPE, KIND, 4>(stream, J);
  return J.group_log2 == 6 ? launch_tiles<TYPE, KIND, 2>(stream, J) : launch_tiles<TYPE, KIND, 1>(stream, J);
}

// Which form (us, both sides measured, columns x outputs):
// - tiles of 64 rows where there are workgroups of them for most of the chip: 64 rows of 4096 x 32768 31.6 (44 otherwise), 96 of 4096 x
//   16384 28.8 (32.9); with workgroups for half of it, 256 rows of 4096 x 4096 30.9 (26.8)
// - few rows, one tile: two tiles of outputs a workgroup from 16384 outputs on, 8192 x 32768 37.5 (one 40.9, four 40.1), four from 65536
//   on, 4096 x 131072 16 rows 69.7 (two 77.8); 4096 x 4096 4.9 (two 6.0)
// - more tiles: two at a time, and as many of outputs as leave workgroups for the chip: 200 rows of 2048 x 2048 8.0 with four (two 9.9), 64
//   of 4096 x 4096 9.6 with two (four 12.1)
// - wavefronts that share the columns: eight, or four where workgroups are many: 128 rows of 8192 x 8192 45.3 (eight 47.5), 64 26.4 (four
//   32.3); sixteen of one tile for many columns, 14336 x 4096 11.9 (eight 13.1)
template <int TYPE, int KIND>
hipError_t launch_kind(hipStream_t stream, const ProductJob& J) {
  const long long tiles = (J.rows + TILE_ROWS<TYPE> - 1) / TILE_ROWS<TYPE>, outs = (J.n_out + 15) / 16;
  const int slabs = (J.n_in + PRODUCT_SLAB - 1) / PRODUCT_SLAB;
  if ((tiles + TILE_R - 1) / TILE_R * ((J.n_out + TILE_OUTS - 1) / TILE_OUTS) >= 192 && tiles >= TILE_R) return launch_many<TYPE, KIND>(stream, J);
  auto waves = [&](int n) {
    while (n > slabs) n /= 2;
    return n;
  };
  if (tiles > 1) {
    const long long pairs = (tiles + 1) / 2, by_four = (outs + 3) / 4 * pairs, by_two = (outs + 1) / 2 * pairs;
    if (by_four >= 150) return launch_few<TYPE, KIND, 2, 4, true>(stream, J, waves(by_four >= 400 ? 4 : 8));
    if (by_two >= 150) return launch_few<TYPE, KIND, 2, 2, true>(stream, J, waves(8));
    return launch_few<TYPE, KIND, 2, 1, true>(stream, J, waves(8));
  }
  const int form = outs >= 4096 ? 2 : outs >= 1024 && slabs >= 16 ? 1 : 0, most = form == 2 ? 4 : form == 1 ? 8 : slabs >= 64 || outs < 128 ? 16 : 8;
  if (J.rows <= 4)
    switch (form) {
      case 2: return launch_few<TYPE, KIND, 1, 4, false>(stream, J, waves(most));
      case 1: return launch_few<TYPE, KIND, 1, 2, false>(stream, J, waves(most));
      default: return launch_few<TYPE, KIND, 1, 1, false>(stream, J, waves(most));
    }
  switch (form) {
    case 2: return launch_few<TYPE, KIND, 1, 4, true>(stream, J, waves(most));
    case 1: return launch_few<TYPE, KIND, 1, 2, true>(stream, J, waves(most));
    default: return launch_few<TYPE, KIND, 1, 1, true>(stream, J, waves(most));
  }
}

template <int TYPE>
hipError_t launch_type(hipStream_t stream, const ProductJob& J) {
  return J.kind == CODES_INT4 ? launch_kind<TYPE, CODES_INT4>(stream, J) : launch_kind<TYPE, CODES_E2M1>(stream, J);
}

}  // namespace

hipError_t launch_product(hipStream_t stream, const ProductJob& J) {
  switch (J.type) {
    case ELEMENT_F32: return launch_type<ELEMENT_F32>(stream, J);
    case ELEMENT_BF16: return launch_type<ELEMENT_BF16>(stream, J);
    case ELEMENT_F16: return launch_type<ELEMENT_F16>(stream, J);
  }
  return hipErrorInvalidValue;
}

}  // namespace cnn355
