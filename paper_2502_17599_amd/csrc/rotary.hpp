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

// cos and sin of the pair that element e of a row belongs to at token t, with the sign of the element's own term:
// out = x * c + partner * s.  (1, 0) past the turned elements.
// The angle in turns, reduced to [-1/2, 1/2], is a product of doubles: with 32 bits the position 100000 would leave an
// error of 0.006 rad.  Its error here is 2^-52 of the number of turns.
__device__ __forceinline__ void rotary_factors(const RotaryPlan& p, long long t, int e, float& c, float& s) {
  c = 1.f;
  s = 0.f;
  if (e >= 2 * p.half) return;
  const int pair = p.interleaved ? e >> 1 : (e < p.half ? e : e - p.half);
  const bool first = p.interleaved ? (e & 1) == 0 : e < p.half;
  const int ax = p.axis ? min((int)p.axis[pair], p.axes - 1) : 0;
  double turns = (double)p.positions[ax * p.pos_stride + t] * p.inv_freq[pair] * 0.15915494309189533577;
  turns -= rint(turns);
  float sn, cs;
  sincospif(2.0f * (float)turns, &sn, &cs);
  c = cs;
  s = first ? -sn * p.sign : sn * p.sign;
}

// The values that this lane's elements are paired with, from the lanes that hold them.  `lds`: D floats of this row's
// own, only used where the partners do not lie in one lane (a half that is no multiple of E).
template <int E, int LPR>
__device__ __forceinline__ void rotary_partners(const RotaryPlan& p, int cc, const float (&f)[E], float (&q)[E], float* lds) {
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < E; ++i) q[i] = f[i ^ 1];
  } else if (p.half % E == 0) {
    const int step = p.half / E;   // lanes between the two halves
    const int from = cc < step ? cc + step : (cc < 2 * step ? cc - step : cc);
    const int lane = (int)(threadIdx.x & 63) - cc + from;
#pragma unroll
    for (int i = 0; i < E; ++i) q[i] = __shfl(f[i], lane, kWave);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) lds[cc * E + i] = f[i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = cc * E + i;
      q[i] = lds[e < p.half ? e + p.half : (e < 2 * p.half ? e - p.half : e)];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
}

}  // namespace meda
