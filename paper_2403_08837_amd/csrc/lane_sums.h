// Sums over lanes of a wavefront, without LDS.
#pragma once
#include <hip/hip_runtime.h>

namespace cdp {

template <int CTRL> __device__ __forceinline__ float lanes_dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lanes_swap16(float v) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}
__device__ __forceinline__ float lanes_swap32(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}
// Over groups of L neighbouring lanes, in every one of them.
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (L >= 2) v += lanes_dpp<0xB1>(v);    // neighbours
  if constexpr (L >= 4) v += lanes_dpp<0x4E>(v);    // pairs
  if constexpr (L >= 8) v += lanes_dpp<0x141>(v);   // the other four of eight (mirrored)
  if constexpr (L >= 16) v += lanes_dpp<0x140>(v);
  if constexpr (L >= 32) v = lanes_swap16(v);
  if constexpr (L >= 64) v = lanes_swap32(v);
  return v;
}
// Their maximum (of what is not NaN), likewise.
template <int L> __device__ __forceinline__ float lanes_max(float v) {
  if constexpr (L >= 2) v = fmaxf(v, lanes_dpp<0xB1>(v));
  if constexpr (L >= 4) v = fmaxf(v, lanes_dpp<0x4E>(v));
  if constexpr (L >= 8) v = fmaxf(v, lanes_dpp<0x141>(v));
  if constexpr (L >= 16) v = fmaxf(v, lanes_dpp<0x140>(v));
  if constexpr (L >= 32) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  }
  if constexpr (L >= 64) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  }
  return v;
}
// Over the lanes that are a multiple of L apart, in every one of them.
template <int L> __device__ __forceinline__ float groups_sum(float v) {
  if constexpr (L <= 4) v += lanes_dpp<0x124>(v);   // (four on, around sixteen)
  if constexpr (L <= 8) v += lanes_dpp<0x128>(v);   // (eight on)
  if constexpr (L <= 16) v = lanes_swap16(v);
  if constexpr (L <= 32) v = lanes_swap32(v);
  return v;
}

}  // namespace cdp
