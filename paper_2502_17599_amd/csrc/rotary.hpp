// Rotary positions, for rows held by LPR = D / E lanes of 16 bytes each.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "row_codec.hpp"

namespace meda {

struct RotaryPlan {
  const int32_t* positions;   // [axes][tokens]
  const double* inv_freq;     // [half]
  const uint8_t* axis;        // [half] or null
  long long pos_stride;
  int half, axes;             // pairs that are turned (0: none), position axes
  int interleaved;
  float sign;                 // of the sine: -1 turns back
};

// (cos, sin) of pair `pair` at token t.
// The angle in turns, reduced to [-1/2, 1/2], is a product of doubles: with 32 bits the position 100000 would leave an
// error of 0.006 rad.  Its error here is 2^-52 of the number of turns.  The sine and cosine are those of the angle x rounded
// to 32 bits; what that leaves, d (2^-26 turns at most), enters by their derivatives, cos(x + d) = cos x - d sin x and
// sin(x + d) = sin x + d cos x up to d^2 / 2 < 2^-47: two multiply-adds, after which the 32-bit results are those of the 64-bit
// angle.  (Without them sines and cosines were off by 2^-23.4 rad, and those near zero by far more than a rounding.)
__device__ __forceinline__ float2 rotary_pair(const RotaryPlan& p, long long t, int pair) {
  const int ax = p.axis ? min((int)p.axis[pair], p.axes - 1) : 0;
  double turns = (double)p.positions[ax * p.pos_stride + t] * p.inv_freq[pair] * 0.15915494309189533577;
  turns -= rint(turns);
  const float x = (float)turns, d = (float)(turns - (double)x) * 6.2831853071795864769f;
  float sn, cs;
  sincospif(2.0f * x, &sn, &cs);
  return make_float2(fmaf(-d, sn, cs), fmaf(d, cs, sn) * p.sign);
}

// Factors of element e of a row, from its token's pairs: out = x * c + partner * s; (1, 0) past the turned elements.
__device__ __forceinline__ void rotary_factors(const RotaryPlan& p, const float2* pairs, int e, float& c, float& s) {
  c = 1.f;
  s = 0.f;
  if (e >= 2 * p.half) return;
  const bool first = p.interleaved ? (e & 1) == 0 : e < p.half;
  const float2 cs = pairs[p.interleaved ? e >> 1 : (first ? e : e - p.half)];
  c = cs.x;
  s = first ? -cs.y : cs.y;
}

__device__ __forceinline__ uint4 pack_row(const float (&f)[8]) {
  return make_uint4(floats_to_bf16x2(f[0], f[1]), floats_to_bf16x2(f[2], f[3]), floats_to_bf16x2(f[4], f[5]), floats_to_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ uint4 pack_row(const float (&f)[4]) { return RowPiece<float>::pack(f); }

// Turns this lane's piece x of a row by its factors (rotary_factors) and leaves the result in f.  The halves of the pairs
// lie in the same piece (interleaved), in the piece of one other lane, which is exchanged as it was read, or, where half is
// no multiple of the piece's E elements, in two other lanes: then the row goes through `lds`, D floats of its own.
template <typename T, int LPR>
__device__ __forceinline__ void rotary_turn(const RotaryPlan& p, int cc, const uint4& x, const float (&c)[RowPiece<T>::kElems],
                                            const float (&s)[RowPiece<T>::kElems], float (&f)[RowPiece<T>::kElems], float* lds) {
  constexpr int E = RowPiece<T>::kElems;
  float o[E];
  RowPiece<T>::unpack(x, f);
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = f[i ^ 1];
  } else if (p.half % E == 0) {
    const int step = p.half / E;   // lanes between the two halves
    const int lane = (int)(threadIdx.x & 63) + (cc < step ? step : (cc < 2 * step ? -step : 0));
    uint4 y;
    y.x = (unsigned)__builtin_amdgcn_ds_bpermute(4 * lane, (int)x.x);
    y.y = (unsigned)__builtin_amdgcn_ds_bpermute(4 * lane, (int)x.y);
    y.z = (unsigned)__builtin_amdgcn_ds_bpermute(4 * lane, (int)x.z);
    y.w = (unsigned)__builtin_amdgcn_ds_bpermute(4 * lane, (int)x.w);
    RowPiece<T>::unpack(y, o);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) lds[cc * E + i] = f[i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = cc * E + i;
      o[i] = lds[e < p.half ? e + p.half : (e < 2 * p.half ? e - p.half : e)];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  if (2 * p.half == E * LPR) {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = fmaf(f[i], c[i], o[i] * s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)   // elements past the turned ones stay as they are (infinity * 0 would not)
      f[i] = cc * E + i < 2 * p.half ? fmaf(f[i], c[i], o[i] * s[i]) : f[i];
  }
}

}  // namespace meda
