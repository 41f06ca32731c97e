// Sums and maxima over neighbouring lanes of a wave, the same bits in every lane
// (block_norm.hip, layer_norm.hip, graph_attention.hip): four exchanges inside a row of 16 lanes
// by data-parallel moves and two across rows by permlane swaps, none of which
// goes through the LDS.
#pragma once

#include <hip/hip_runtime.h>

namespace e2f {

// the value of lane l ^ 1, l ^ 2, and, where quads (halves of a row) already agree, of the other quad (half)
template <int STEP>
__device__ __forceinline__ float lane_other(float v) {
  constexpr int ctrl = STEP == 1 ? 0xb1 /* quad_perm 1 0 3 2 */
                     : STEP == 2 ? 0x4e /* quad_perm 2 3 0 1 */
                     : STEP == 4 ? 0x141 /* row_half_mirror */
                                 : 0x140 /* row_mirror */;
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, true));
}
typedef unsigned lane_pair __attribute__((ext_vector_type(2)));
// the values of the two rows of 16 lanes of a half wave (16), of the two half waves (32)
template <int STEP>
__device__ __forceinline__ void lane_halves(float v, float& a, float& b) {
  const unsigned u = __float_as_uint(v);
  lane_pair p;
  if constexpr (STEP == 16)
    p = __builtin_bit_cast(lane_pair, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  else
    p = __builtin_bit_cast(lane_pair, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  a = __uint_as_float(p.x), b = __uint_as_float(p.y);
}

// f over groups of `n` neighbouring lanes (a power of two up to 64, the same for the wave)
template <typename F>
__device__ __forceinline__ float lanes_all(float v, int n, F f) {
  float a, b;
  if (n > 1) v = f(v, lane_other<1>(v));
  if (n > 2) v = f(v, lane_other<2>(v));
  if (n > 4) v = f(v, lane_other<4>(v));
  if (n > 8) v = f(v, lane_other<8>(v));
  if (n > 16) lane_halves<16>(v, a, b), v = f(a, b);
  if (n > 32) lane_halves<32>(v, a, b), v = f(a, b);
  return v;
}
__device__ __forceinline__ float lanes_sum(float v, int n = 64) {
  return lanes_all(v, n, [](float a, float b) { return a + b; });
}

// f over the lanes l, l + n, l + 2n .. of each of n classes (a power of two up to 64)
template <typename F>
__device__ __forceinline__ float classes_all(float v, int n, F f) {
  float a, b;
  if (n <= 32) lane_halves<32>(v, a, b), v = f(a, b);
  if (n <= 16) lane_halves<16>(v, a, b), v = f(a, b);
  if (n <= 8) v = f(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128 /* row_ror 8 */, 0xf, 0xf, true)));
  if (n <= 4) v = f(v, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124 /* row_ror 4 */, 0xf, 0xf, true)));
  if (n <= 2) v = f(v, lane_other<2>(v));
  if (n <= 1) v = f(v, lane_other<1>(v));
  return v;
}

}  // namespace e2f
