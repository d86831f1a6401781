// What a lane of a wavefront gets from another one without LDS.  (Device code.)
#pragma once

namespace cnn355 {

// a word of the lane whose number differs by D (a power of two)
template <int D>
__device__ __forceinline__ unsigned xor_word(unsigned v) {
  if constexpr (D == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);        // quad_perm [1, 0, 3, 2]
  else if constexpr (D == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);   // quad_perm [2, 3, 0, 1]
  else if constexpr (D == 4)                                                             // row_half_mirror, quad_perm [3, 2, 1, 0]
    return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
  else if constexpr (D == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);  // row_ror:8
  else if constexpr (D == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
}  // namespace cnn355
