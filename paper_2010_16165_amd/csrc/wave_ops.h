// Internal: exchanges between the lanes of a wave by DPP, a few clocks each where a permutation through LDS takes a hundred.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace fupr {

template <int CONTROL>
__device__ __forceinline__ int dpp_move(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CONTROL, 0xf, 0xf, true);
}

// The value of lane ^ D, for the steps D = 1, 2, 4, ... of a reduction: once groups of D lanes agree, the mirror image
// within 2 D lanes is as good as lane ^ D.
template <int D>
__device__ __forceinline__ int fold_partner(int v) {
  if constexpr (D == 1) return dpp_move<0xB1>(v);         // quad_perm 1 0 3 2
  else if constexpr (D == 2) return dpp_move<0x4E>(v);    // quad_perm 2 3 0 1
  else if constexpr (D == 4) return dpp_move<0x141>(v);   // row_half_mirror
  else if constexpr (D == 8) return dpp_move<0x140>(v);   // row_mirror
  else return __shfl_xor(v, D);
}
template <int D>
__device__ __forceinline__ uint32_t fold_partner(uint32_t v) {
  return (uint32_t)fold_partner<D>((int)v);
}
template <int D>
__device__ __forceinline__ float fold_partner(float v) {
  return __int_as_float(fold_partner<D>(__float_as_int(v)));
}
template <int D>
__device__ __forceinline__ uint64_t fold_partner(uint64_t v) {
  return (uint64_t)fold_partner<D>((uint32_t)(v >> 32)) << 32 | fold_partner<D>((uint32_t)v);
}
template <int D>
__device__ __forceinline__ double fold_partner(double v) {
  return __longlong_as_double((long long)fold_partner<D>((uint64_t)__double_as_longlong(v)));
}

// f(v, partner's v) over groups of LPT lanes; f must not care for the order.
template <int LPT, int D = 1, class T, class F>
__device__ __forceinline__ T group_fold(T v, F f) {
  if constexpr (D < LPT) return group_fold<LPT, D * 2>(f(v, fold_partner<D>(v)), f);
  else return v;
}

// Sums over the lanes up to the own one; all 64 lanes take part.
__device__ __forceinline__ int wave_prefix(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8: within 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
  return v;
}

}  // namespace fupr
