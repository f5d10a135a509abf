// Wave-level building blocks of the kernels in which one query row attends over many cached rows: sums and maxima over
// groups of lanes without LDS traffic, streaming loads, weights as sums of bf16 numbers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.hpp"

namespace meda {

// Inclusive sum over the lanes of the wave (data-parallel primitives, no LDS traffic).
__device__ __forceinline__ int wave_inclusive_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8: inside the rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 of rows 0, 2 to rows 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2, 3
  return v;
}

// 8-byte load of data that is read once (see load16_stream)
__device__ __forceinline__ uint2 load8_stream(const void* p) {
  typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
  const u32x2_t t = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p));
  return make_uint2(t.x, t.y);
}

__device__ __forceinline__ void store_elem(char* dst, float x, bf16_t) {
  *reinterpret_cast<uint16_t*>(dst) = (uint16_t)float_to_bf16_rne(x);
}
__device__ __forceinline__ void store_elem(char* dst, float x, float) { *reinterpret_cast<float*>(dst) = x; }

__device__ __forceinline__ void unpack4(const uint4& v, float (&f)[4]) {
  f[0] = __uint_as_float(v.x);
  f[1] = __uint_as_float(v.y);
  f[2] = __uint_as_float(v.z);
  f[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ float dot4(const uint4& a, const uint4& b) {
  float d = __uint_as_float(a.x) * __uint_as_float(b.x);
  d = fmaf(__uint_as_float(a.y), __uint_as_float(b.y), d);
  d = fmaf(__uint_as_float(a.z), __uint_as_float(b.z), d);
  return fmaf(__uint_as_float(a.w), __uint_as_float(b.w), d);
}

// Value of a partner lane whose lane-index bit X differs (X = 1, 2, 4, 8 inside a row of 16 lanes: data-parallel
// primitives, no LDS traffic; the partners of 4 and 8 are the mirrored lanes of the half row / row, which differ
// in the lower bits too; X = 16: the lane 16 away).
template <int X>
__device__ __forceinline__ float lane_partner(float v) {
  const int i = __float_as_int(v);
  if constexpr (X == 1) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0xB1, 0xF, 0xF, true));        // quad_perm 1,0,3,2
  else if constexpr (X == 2) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x4E, 0xF, 0xF, true));   // quad_perm 2,3,0,1
  else if constexpr (X == 4) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x141, 0xF, 0xF, true));  // row_half_mirror
  else if constexpr (X == 8) return __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x140, 0xF, 0xF, true));  // row_mirror
  else return __shfl_xor(v, X, kWave);
}

// The LPR lanes that read one row each hold, for every query head of the group, a partial dot product.
// RowReduceScatter sums them over the lanes and leaves in v[0] the total of ONE head per lane (the head
// row_head() names: the upper lane-index bits choose it), at GP + log2(LPR) - 1 exchanges instead of
// GP * log2(LPR); RowAllGather is the inverse: from one value per lane for that lane's head to all GP
// values in every lane.  N: values still held, X: bit in which the partner differs.  All array indices
// are compile-time constants (the arrays live in registers).
template <int GP, int N, int X>
struct RowReduceScatter {
  static __device__ __forceinline__ void run(float (&v)[GP], int cc) {
    if constexpr (X >= 1) {
      if constexpr (N > 1) {
        const bool up = (cc & X) != 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float keep = up ? v[i + N / 2] : v[i], send = up ? v[i] : v[i + N / 2];
          v[i] = keep + lane_partner<X>(send);
        }
        RowReduceScatter<GP, N / 2, X / 2>::run(v, cc);
      } else {
        v[0] += lane_partner<X>(v[0]);
        RowReduceScatter<GP, 1, X / 2>::run(v, cc);
      }
    }
  }
};
template <int GP, int LPR>
__device__ __forceinline__ int row_head(int cc) {
  int h = 0, n = GP;
#pragma unroll
  for (int x = LPR / 2; x >= 1; x >>= 1) {
    if (n > 1) {
      n >>= 1;
      h += (cc & x) ? n : 0;
    }
  }
  return h;
}
// N: values held so far (w[0..N)), X: partner bit of this step; the steps run from the last halving
// distance of the reduce-scatter back up to LPR / 2.
template <int GP, int N, int X>
struct RowAllGather {
  static __device__ __forceinline__ void run(float (&w)[GP], int cc) {
    if constexpr (N < GP) {
      const bool up = (cc & X) != 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float other = lane_partner<X>(w[i]);
        w[i + N] = up ? w[i] : other;
        w[i] = up ? other : w[i];
      }
      RowAllGather<GP, 2 * N, 2 * X>::run(w, cc);
    }
  }
};
template <int GP, int LPR>
__device__ __forceinline__ void row_reduce_scatter(float (&v)[GP], int cc) {
  RowReduceScatter<GP, GP, LPR / 2>::run(v, cc);
}
template <int GP, int LPR>
__device__ __forceinline__ void row_all_gather(float mine, float (&w)[GP], int cc) {
  w[0] = mine;
  RowAllGather<GP, 1, LPR / GP>::run(w, cc);   // the last halving step of the reduce-scatter had distance LPR / GP
}

typedef __attribute__((ext_vector_type(4))) float f32x4_t;

// out[i] = the value of lane FIRST + i of this lane's row of 16 lanes, i = 0..7 (0x150 + n: broadcast of lane n)
template <int FIRST>
__device__ __forceinline__ void row_broadcast(float v, float (&out)[8]) {
  const int i = __float_as_int(v);
  out[0] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 0, 0xF, 0xF, true));
  out[1] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 1, 0xF, 0xF, true));
  out[2] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 2, 0xF, 0xF, true));
  out[3] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 3, 0xF, 0xF, true));
  out[4] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 4, 0xF, 0xF, true));
  out[5] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 5, 0xF, 0xF, true));
  out[6] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 6, 0xF, 0xF, true));
  out[7] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x150 + FIRST + 7, 0xF, 0xF, true));
}

__device__ __forceinline__ float group_max(float v) {  // over the four lane groups of 16
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float group_sum(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The upper part of a positive weight: the largest bf16 number BELOW it (0 for 0).  What remains is then exact and
// never zero: after two parts it has 8 significant bits or less.
__device__ __forceinline__ float weight_part(float w) {
  return __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(w), 1u) & 0xffff0000u);
}

// N bytes of a row that is read once, as dwords (see load16_stream)
template <int N>
__device__ __forceinline__ void load_piece(const char* p, uint32_t (&w)[N / 4]) {
  if constexpr (N == 16) {
    const uint4 v = load16_stream(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 8) {
    const uint2 v = load8_stream(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
  }
}


}  // namespace meda
