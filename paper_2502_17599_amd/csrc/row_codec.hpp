// Rows of a cache as the 16-byte pieces that lanes hold, and their 8-bit form (per row: scale = max|x| / 448, codes in
// E4M3), shared by the kernels that store rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "device_utils.hpp"
#include "fp8.hpp"

namespace meda {

template <typename T>
struct RowPiece;   // the 16 bytes of a row one lane handles
template <>
struct RowPiece<bf16_t> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint4 o;
    o.x = float_to_bf16_rne(f[0]) | (float_to_bf16_rne(f[1]) << 16);
    o.y = float_to_bf16_rne(f[2]) | (float_to_bf16_rne(f[3]) << 16);
    o.z = float_to_bf16_rne(f[4]) | (float_to_bf16_rne(f[5]) << 16);
    o.w = float_to_bf16_rne(f[6]) | (float_to_bf16_rne(f[7]) << 16);
    return o;
  }
};
template <>
struct RowPiece<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

// Maximum over the LPR (8, 16 or 32) lanes that hold one row (data-parallel primitives: no LDS traffic).
template <int LPR>
__device__ __forceinline__ float row_max(float v) {
  auto dpp = [](float x, auto ctrl) {
    const int i = __float_as_int(x);
    return __int_as_float(__builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, true));
  };
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0xB1>()));    // neighbours
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x4E>()));    // pairs of a quad
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x141>()));   // quads of a half row (mirrored)
  if constexpr (LPR >= 16) v = fmaxf(v, dpp(v, std::integral_constant<int, 0x140>()));  // halves of a row (mirrored)
  if constexpr (LPR >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return v;
}

// x / s, correctly rounded, for a divisor whose reciprocal y (one Newton step behind the hardware's) is shared by
// many quotients: quotient estimate and two exact-remainder corrections, five multiply-adds (which lose the sign of a
// zero: it is put back).  No intermediate may leave the normal range, which the caller checks.
__device__ __forceinline__ float refined_rcp(float s) {
  const float y = __builtin_amdgcn_rcpf(s);
  return fmaf(fmaf(-s, y, 1.0f), y, y);
}
__device__ __forceinline__ float quotient(float x, float s, float y) {
  float q = x * y;
  q = fmaf(fmaf(-s, q, x), y, q);
  return copysignf(fmaf(fmaf(-s, q, x), y, q), x);
}

// The scale of a row held by LPR lanes (E elements each) and this lane's codes; f is clobbered.
// Division and rounding to E4M3 written out element by element
// (a division instruction sequence and some ten integer instructions each) bound the quantiser at 3.8 TB/s: now one
// reciprocal per row, the correctly rounded quotients from it (`quotient`; rows whose scale could leave the normal
// range divide) and the hardware's conversion, which rounds to nearest even.
template <int E, int LPR>
__device__ __forceinline__ float quantize_row(float (&f)[E], uint32_t (&w)[E / 4]) {
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) amax = fmaxf(amax, fabsf(f[i]));
  amax = row_max<LPR>(amax);
  float scale;
  // quotients of elements far below the row's maximum may be subnormal: they round to the code of zero either way
  const bool plain = amax > 0x1p-80f && amax < 0x1p80f;
  if (__ballot(plain) == ~0ull) {
    scale = quotient(amax, kE4M3Max, 1.0f / kE4M3Max);
    const float y = refined_rcp(scale);
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = __builtin_amdgcn_fmed3f(quotient(f[i], scale, y), -kE4M3Max, kE4M3Max);
#pragma unroll
    for (int i = 0; i < E / 4; ++i) w[i] = floats_to_e4m3x4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
  } else {
    scale = amax > 0.f ? amax / kE4M3Max : 1.0f;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      w[i] = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[i] |= float_to_e4m3(fminf(fmaxf(f[4 * i + k] / scale, -kE4M3Max), kE4M3Max)) << (8 * k);
    }
  }
  return scale;
}

}  // namespace meda
