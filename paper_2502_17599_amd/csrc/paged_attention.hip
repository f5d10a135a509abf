// Attention of one new token per row over its pages: out = Softmax(q K^T / sqrt(d)) V.
//
// Every cached key and value is read once and takes 4 * G * d flops per pair (G query heads share a kv head), so the step
// is bound by HBM where it is long and by latency where it is short.  The work is numbered in units of 32 positions (fp32: 16),
// row after row and kv head after kv head, and cut into contiguous shares of equal size, one per workgroup, on the device:
// lengths that differ by a factor of a thousand and a single long request all fill the chip, and empty rows take no share.  (They
// do take time where a wave goes on from one row to the next: see where it does.)  A (row, kv head) that lies in one share is
// finished by its workgroup; one that is cut leaves, per share, a running maximum, a normaliser and a weighted value sum,
// which a second kernel joins.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/meda.h"
#include "fp8.hpp"
#include "paged.hpp"

namespace meda {

constexpr int kAttThreads = kLocateThreads, kAttWaves = kAttThreads / 64;
constexpr int kBlock = 16;        // positions of one matrix instruction; they lie in one page
constexpr int kMinUnits = 4;      // a workgroup's share, at least: a step per wave
constexpr int kMaxGroup = 16;     // query heads per kv head
// positions of a unit, a step of one wave: two blocks, of 4-byte rows one (as many bytes)
constexpr int unit_positions(int bytes) { return bytes == 4 ? kBlock : 2 * kBlock; }

struct PagedArgs {
  Pool pool;
  const char* q;
  char* out;
  const int32_t* table;
  const int32_t* lens;
  float* part;             // [2 * groups][G][d]: value sums of the pieces
  float2* part_mz;         // [2 * groups][G]: their maximum (unscaled logits) and normaliser
  int2* cut;               // which (row, kv head) is cut: see below
  long long q_stride, out_stride;   // bytes
  long long table_stride, len_stride;
  int R, Hq, Hkv, G, max_blocks;
  int cut_by_pair;
  float scale_log2;
};

__device__ __forceinline__ int row_len(const PagedArgs& a, int r) {
  return min(max(a.lens[r * a.len_stride], 0), a.max_blocks << a.pool.page_log2);
}

// A maximum starts at the least finite number, not at -infinity: every finite logit replaces or equals it, a logit of
// -infinity has the weight exp2(-inf) = 0 under it, and differences of maxima are never inf - inf.
constexpr float kLeast = -__FLT_MAX__;
// The weight of logit x under maximum `top`.  Logits and maxima are kept unscaled: the difference of two near ones is exact,
// and that of a maximum and itself is zero, however large they are.
__device__ __forceinline__ float weight_under(float x, float top, float scale_log2) {
  return __builtin_amdgcn_exp2f((x - top) * scale_log2);
}

// The pages of the 64 / BLOCKS units from u on: lane BLOCKS i + b holds that of block b of the i-th.  One load for many
// steps: a load of its own in every step would have to be waited for, and with it, as loads come back in order, for all
// rows that are on their way.
template <int BLOCKS>
__device__ __forceinline__ int load_pages(const PagedArgs& a, const int32_t* table, int u, int u1, int len) {
  const int lane = threadIdx.x & 63;
  const int pos = min(u + lane / BLOCKS, u1 - 1) * (BLOCKS * kBlock);   // (units past the last one repeat it)
  const int p = pos + kBlock * (lane % BLOCKS);
  return table[(p < len ? p : pos) >> a.pool.page_log2];                // a block behind the end repeats the first one
}

// Where a unit's blocks lie, as byte offsets of (page, head, place) and scale indexes.
template <int BLOCKS>
struct UnitPages {
  size_t at[BLOCKS];
  size_t scale[BLOCKS];
  bool ok[BLOCKS];      // the page exists
  bool full;            // all positions count
};
template <int ROW_BYTES, int BLOCKS>
__device__ __forceinline__ UnitPages<BLOCKS> unit_pages(const PagedArgs& a, int pages, int step, int head, int pos, int len) {
  UnitPages<BLOCKS> u;
  u.full = pos + BLOCKS * kBlock <= len;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int p = pos + kBlock * b, q = p < len ? p : pos;
    const int page = __builtin_amdgcn_readlane(pages, (BLOCKS * step + b) & 63);
    u.ok[b] = page >= 0 && page < a.pool.n_pages;
    u.full = u.full && u.ok[b];
    const size_t safe = u.ok[b] ? page : 0;
    const size_t place = ((size_t)head << a.pool.page_log2) + (q & ((1 << a.pool.page_log2) - 1));
    u.at[b] = safe * a.pool.page_bytes + place * ROW_BYTES;
    u.scale[b] = (safe * a.Hkv << a.pool.page_log2) + place;
  }
  return u;
}

// ---- both products on the matrix unit -------------------------------------------------------------------------------
//
// Lane (c, g) = (l % 16, l / 16).  logits D[key][col] = sum_d K[key][d] Q[col][d], blocks of 16 keys: the lane holds elements
// of key c, the same ones of query head c % GP, and receives the logits of that head for the keys 4 g + i of every block.
// The second product O[row][col] += sum_key P[row][key] V[key][col] contracts over the keys in an order in which its
// weights are what the lane has.
//   bf16 and 8 bits (16x16x32): a weight enters as the sum of two bf16 numbers, rows c / GP = 0 and 1 of the product (what the
// first leaves is exact and not zero; the second is that to nearest even, which is off by 2^-16 of the weight at most, either
// way: a 128th of the output's own rounding), so that groups of up to 8 heads need one instruction per 16 columns; groups of 9
// to 16 take two, one per part.  The values are 8 keys at d / 16 columns, transposed in registers.  8-bit rows: codes become
// bf16 exactly, the key's scale multiplies the logit and the value's scale the weight.
//   fp32 (16x16x4): products and sums in fp32.  Four instructions use up the 16 bytes that a lane loads of a key or of a value;
// the values' column is 4 c + e of 64.  (On the vector unit, with the dot products summed over lanes, groups of 8 and
// 16 heads were bound by its instructions: 3.9 and 2.0 TB/s.)
template <typename T, int D, int GP, bool FP8>
struct Attend {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int kEl = F32 ? 4 : (FP8 ? 1 : 2), kRowBytes = D * kEl;
  static constexpr int BLOCKS = unit_positions(sizeof(T)) / kBlock, kUnit = BLOCKS * kBlock, kKeys = 4 * BLOCKS;
  static constexpr int KL = kRowBytes / 64;          // 16-byte loads per key and lane
  static constexpr int VW = D / 16 * kEl / 4;        // dwords of a value piece
  static constexpr int PE = D / 16;                  // 16-column accumulators
  static constexpr int QV = F32 ? D / 16 : D / 32;   // 16-byte pieces of a query

  struct Unit {
    uint4 k[BLOCKS][KL];
    uint32_t v[kKeys][VW];
    float scale;
  };
  float m, z;           // of head c % GP; m is the same in the four lane groups
  f32x4_t acc[PE];      // acc[j][r]: output column column(j), product row 4 g + r
  uint4 q[QV];

  static __device__ __forceinline__ int column(int c, int j) { return F32 ? 64 * (j / 4) + 4 * c + j % 4 : PE * c + j; }

  __device__ __forceinline__ void begin(const PagedArgs& a, int r, int head) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    m = kLeast;
    z = 0.f;
#pragma unroll
    for (int j = 0; j < PE; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const char* src = a.q + r * a.q_stride + (size_t)(head * a.G + c % GP) * (D * sizeof(T));
#pragma unroll
    for (int k = 0; k < QV; ++k) {
      // the elements that the key's loads bring (16 bytes of codes are two steps of the product)
      const int e0 = F32 ? 16 * k + 4 * g : (FP8 ? 64 * (k / 2) + 16 * g + 8 * (k & 1) : 32 * k + 8 * g);
      q[k] = make_uint4(0u, 0u, 0u, 0u);
      if (c % GP < a.G) q[k] = *reinterpret_cast<const uint4*>(src + e0 * sizeof(T));
    }
  }

  // MASKED: some of the unit's positions lie behind the end or in a page that does not exist.  Positions behind the end
  // repeat the last one (their weights are zero).
  template <bool MASKED>
  __device__ __forceinline__ static void load_keys(const PagedArgs& a, Unit& t, const UnitPages<BLOCKS>& up, int pos, int len) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int last = min(len - 1 - pos - kBlock * b, 15), top = last < 0 ? min(len - 1 - pos, 15) : last;
      const char* src = a.pool.k + up.at[b] + (unsigned)((MASKED ? min(c, top) : c) * kRowBytes + 16 * g);
#pragma unroll
      for (int k = 0; k < KL; ++k) t.k[b][k] = load16_stream(src + 64 * k);
    }
  }
  template <bool MASKED>
  __device__ __forceinline__ static void load_values(const PagedArgs& a, Unit& t, const UnitPages<BLOCKS>& up, int pos, int len) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int last = min(len - 1 - pos - kBlock * b, 15), top = last < 0 ? min(len - 1 - pos, 15) : last;
      const char* src = a.pool.v + up.at[b];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char* row = src + (unsigned)((MASKED ? min(4 * g + i, top) : 4 * g + i) * kRowBytes);
        if constexpr (F32) {
#pragma unroll
          for (int x = 0; x < VW / 4; ++x) {
            const uint4 y = load16_stream(row + 256 * x + 16 * c);
            uint32_t* to = &t.v[4 * b + i][4 * x];
            to[0] = y.x; to[1] = y.y; to[2] = y.z; to[3] = y.w;
          }
        } else {
          load_piece<VW * 4>(row + c * (VW * 4), t.v[4 * b + i]);
        }
      }
      // the scales of the 8 keys that this row of 16 lanes has logits for: lanes 0..7 the keys', 8..15 the values'
      if constexpr (FP8) {
        const int row = 4 * g + (c & 3);
        if (((c >> 2) & 1) == b) t.scale = (c < 8 ? a.pool.ks : a.pool.vs)[up.scale[b] + (MASKED ? min(row, top) : row)];
      }
    }
  }

  __device__ __forceinline__ void logits(const Unit& rows, float (&t)[kKeys]) const {
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      f32x4_t s4 = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (F32) {
        // four sums of d / 4 products instead of one of d: half the rounding error
        f32x4_t x4 = s4, y4 = s4, z4 = s4, w4 = s4;
#pragma unroll
        for (int k = 0; k < QV; ++k) {
          const uint4 x = rows.k[b][k], y = q[k];
          x4 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.x), __uint_as_float(y.x), x4, 0, 0, 0);
          y4 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.y), __uint_as_float(y.y), y4, 0, 0, 0);
          z4 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.z), __uint_as_float(y.z), z4, 0, 0, 0);
          w4 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.w), __uint_as_float(y.w), w4, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s4[i] = (x4[i] + y4[i]) + (z4[i] + w4[i]);
      } else {
#pragma unroll
        for (int k = 0; k < QV; ++k) {
          uint4 x;
          if constexpr (FP8) x = e4m3x8_to_bf16x8((k & 1) ? make_uint2(rows.k[b][k / 2].z, rows.k[b][k / 2].w) : make_uint2(rows.k[b][k / 2].x, rows.k[b][k / 2].y));
          else x = rows.k[b][k];
          s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, q[k]), s4, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) t[4 * b + i] = s4[i];
    }
  }

  template <bool MASKED>
  __device__ __forceinline__ void finish(const PagedArgs& a, Unit& rows, const UnitPages<BLOCKS>& up, int pos, int len, float (&t)[kKeys]) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, part = (c / GP) & 1;
    float sk[8], sv[8];
    bool in[kKeys];
    if constexpr (FP8) {
      row_broadcast<0>(rows.scale, sk);
      row_broadcast<8>(rows.scale, sv);
    }
    float bm = kLeast;
#pragma unroll
    for (int e = 0; e < kKeys; ++e) {
      if constexpr (FP8) t[e] *= sk[e];
      if constexpr (MASKED) {
        in[e] = up.ok[e >> 2] && pos + kBlock * (e >> 2) + 4 * g + (e & 3) < len;
        t[e] = in[e] ? t[e] : -INFINITY;
#pragma unroll
        for (uint32_t& x : rows.v[e]) x = in[e] ? x : 0u;   // what is read in its place may hold an infinity
      }
      bm = fmaxf(bm, t[e]);
    }
    bm = group_max(bm);
    if (__ballot(bm > m) != 0ull) {  // a new maximum of some head: rescale what that head has so far (rare)
      const float mn = fmaxf(m, bm);
      const float c1 = weight_under(m, mn, a.scale_log2);
      z *= c1;
      m = mn;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float cr = __shfl(c1, 4 * g + r, kWave);  // product row 4 g + r belongs to the head of lane column 4 g + r
#pragma unroll
        for (int j = 0; j < PE; ++j) acc[j][r] *= cr;
      }
    }
    float w[kKeys];
#pragma unroll
    for (int e = 0; e < kKeys; ++e) {
      float p = weight_under(t[e], m, a.scale_log2);
      w[e] = FP8 ? fmaf(p, sv[e], 0.f) : p;  // the sum takes the sign of a zero
      if constexpr (MASKED) {
        p = in[e] ? p : 0.f;
        w[e] = in[e] ? w[e] : 0.f;
      }
      z += p;
    }
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < kKeys; ++e)
#pragma unroll
        for (int j = 0; j < PE; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], __uint_as_float(rows.v[e][j]), acc[j], 0, 0, 0);
    } else {
      uint32_t pa[4], pb[4];
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float x[2], y[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float hi = weight_part(w[e + u]);
          y[u] = w[e + u] - hi;
          x[u] = GP == 16 || part == 0 ? hi : y[u];
        }
        pa[e / 2] = floats_to_bf16x2(x[0], x[1]);   // (the upper part is a bf16 number: it stays as it is)
        pb[e / 2] = floats_to_bf16x2(y[0], y[1]);
      }
      const bf16x8_t wa = __builtin_bit_cast(bf16x8_t, make_uint4(pa[0], pa[1], pa[2], pa[3]));
      const bf16x8_t wb = __builtin_bit_cast(bf16x8_t, make_uint4(pb[0], pb[1], pb[2], pb[3]));
#pragma unroll
      for (int j2 = 0; j2 < PE / 2; ++j2) {  // two columns at a time: one dword of every row
        uint32_t d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (FP8) d[e] = e4m3x2_to_bf16x2(rows.v[e][j2 / 2], (j2 & 1) != 0);
          else d[e] = rows.v[e][j2];
        }
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          lo[u] = __builtin_amdgcn_perm(d[2 * u + 1], d[2 * u], 0x05040100u);
          hi[u] = __builtin_amdgcn_perm(d[2 * u + 1], d[2 * u], 0x07060302u);
        }
        const bf16x8_t v0 = __builtin_bit_cast(bf16x8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
        const bf16x8_t v1 = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        acc[2 * j2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, v0, acc[2 * j2], 0, 0, 0);
        acc[2 * j2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, v1, acc[2 * j2 + 1], 0, 0, 0);
        if constexpr (GP == 16) {
          acc[2 * j2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, v0, acc[2 * j2], 0, 0, 0);
          acc[2 * j2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, v1, acc[2 * j2 + 1], 0, 0, 0);
        }
      }
    }
  }

  // Units [u0, u1) of a (row, kv head) with `len` positions.
  __device__ __forceinline__ void units(const PagedArgs& a, const int32_t* table, int head, int u0, int u1, int len) {
    constexpr int kAhead = 64 / BLOCKS;   // units whose pages one load brings
    int pages = load_pages<BLOCKS>(a, table, u0, u1, len), pages_behind = pages, step = 0, u = u0;
    UnitPages<BLOCKS> up = unit_pages<kRowBytes, BLOCKS>(a, pages, 0, head, u * kUnit, len);
    Unit rows;
    float t[kKeys];
    bool fast = up.full;
    if (fast) load_keys<false>(a, rows, up, 0, 0);
    while (fast) {
      load_values<false>(a, rows, up, 0, 0);
      const UnitPages<BLOCKS> cur = up;
      ++u;
      ++step;
      fast = u < u1;
      if (step % kAhead == kAhead / 2) pages_behind = load_pages<BLOCKS>(a, table, u + kAhead / 2, u1, len);
      if (step % kAhead == 0) pages = pages_behind;
      if (fast) {
        up = unit_pages<kRowBytes, BLOCKS>(a, pages, step, head, u * kUnit, len);
        fast = up.full;
      }
      logits(rows, t);
      if (fast) load_keys<false>(a, rows, up, 0, 0);  // in flight while this unit is finished
      finish<false>(a, rows, cur, 0, 0, t);
    }
    for (; u < u1; ++u) {   // the last unit of a row; units behind a missing page
      const int pos = u * kUnit;
      up = unit_pages<kRowBytes, BLOCKS>(a, load_pages<BLOCKS>(a, table, u, u1, len), 0, head, pos, len);
      load_keys<true>(a, rows, up, pos, len);
      load_values<true>(a, rows, up, pos, len);
      logits(rows, t);
      finish<true>(a, rows, up, pos, len, t);
    }
  }

  // The wave's sums of a piece: o[h][column], maximum and normaliser of the GP heads.  Product row 4 g + r is part
  // (4 g + r) / GP of head (4 g + r) % GP: the two parts are summed (fp32: one part, the rows past it repeat it).
  __device__ __forceinline__ void put(float (&o)[GP][D], float (&om)[GP], float (&oz)[GP]) const {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const float zs = group_sum(z);  // the four lane groups saw different keys of the same head
    if (lane < GP) {
      om[lane] = m;
      oz[lane] = zs;
    }
#pragma unroll
    for (int j = 0; j < PE; ++j) {
      float* dst = &o[0][column(c, j)];
      if constexpr (GP == 16 || F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * g + i < GP) dst[(4 * g + i) * D] = acc[j][i];
      } else if constexpr (GP == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[j][i]), __float_as_uint(acc[j][i]), false, false);
          if (g < 2) dst[(4 * g + i) * D] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
        }
      } else if constexpr (GP == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[j][i]), __float_as_uint(acc[j][i]), false, false);
          if (g == 0) dst[i * D] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < GP; ++i)
          if (g == 0) dst[i * D] = acc[j][i] + acc[j][GP + i];
      }
    }
  }
};

// ---- shares ---------------------------------------------------------------------------------------------------------
//
// The units of all (row, kv head) pairs are numbered one pair after the other.  A workgroup takes a contiguous share of
// them, each of its waves a contiguous quarter of the share: a wave that comes to the end of a pair goes on with the next
// by itself, without a barrier (where pairs are a few units long, waves that worked on one pair together spent most of
// their time on its beginning and its end: 256 requests of 40 to 600 positions, 222 MB, 68 us, 2000 rows of 10 to 300, 96 MB,
// 53 us).  A pair that lies in one wave's quarter is written out by it.  The others leave pieces in LDS: a wave has at most
// one that goes on from the wave before (slot 0) and one that begins in it and goes on (slot 1).  After one barrier the
// workgroup adds up the pieces of every pair, and writes it out, or, where the pair goes on in other shares, as a piece of
// the share: slot 0 and 1 again, in memory, for the join.
//
// What the join finds: where there are no more pairs than workgroups, for every pair (the share that it begins in, shares
// behind that it reaches into), and for every share the pair that begins in it and goes on behind it (row * Hkv + head,
// shares behind) otherwise; (.., 0): nothing to join.  The join then has a workgroup for the smaller number of the two: those
// that find nothing cost more than the others' work (32 pairs in 440 shares, eight query heads: 16.9 us with a workgroup
// for every share, 15.1 with one for every pair; 6 pairs of long fp32 requests 40.5 and 39.5; 272 pairs 21.5 and 20.3).
struct WavePiece {
  int pair;     // row * Hkv + head
  int shares;   // slot 1: shares behind this one that the pair reaches into
  bool there;
  bool ends;    // slot 0: the pair ends in this wave
};

// Workgroups per CU, and waves per SIMD.  All workgroups of a launch are at work at once, each on one share: two per CU have
// enough bytes on their way, with fewer pieces to join than three and no register spilled (40 fp32 requests of 150 to 12000
// positions 87 us with two, 98 with three; 64 requests, 435 MB 85.2 and 85.9; one of 30000 positions, whose waves then take two
// steps each instead of one or two, 20.5 and 24.9; 2000 of 10 to 2000 87.7 and 89.9), except for 8-bit rows of 64 elements, of
// which a step is 4 KB (112 MB: 37.6 us with two, 35.6 with three).  Several rounds of shorter shares cost more in searches
// and joins than the evener end gains.
constexpr int groups_per_cu(int d, bool fp8) { return fp8 && d == 64 ? 3 : 2; }
constexpr int kCus = 256, kFewPairs = 64;

// Four columns of a row of out; a sum of weights of zero (every page is missing) gives zeros.
__device__ __forceinline__ void store4(char* dst, const float (&x)[4], float) {
  *reinterpret_cast<float4*>(dst) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store4(char* dst, const float (&x)[4], bf16_t) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(float_to_bf16_rne(x[0]) | (float_to_bf16_rne(x[1]) << 16),
                                              float_to_bf16_rne(x[2]) | (float_to_bf16_rne(x[3]) << 16));
}
template <typename T>
__device__ __forceinline__ void write_out(const PagedArgs& a, int pair, int h, int column, int D, const float4& o, float z) {
  const int r = pair / a.Hkv, head = pair - r * a.Hkv;
  const float x[4] = {z == 0.f ? 0.f : o.x / z, z == 0.f ? 0.f : o.y / z, z == 0.f ? 0.f : o.z / z, z == 0.f ? 0.f : o.w / z};
  store4(a.out + r * a.out_stride + ((size_t)(head * a.G + h) * D + column) * sizeof(T), x, T{});
}
__device__ __forceinline__ float4 scaled(const float4& x, float c) { return make_float4(x.x * c, x.y * c, x.z * c, x.w * c); }
__device__ __forceinline__ float4 add_scaled(const float4& sum, const float4& x, float c) {
  return make_float4(fmaf(x.x, c, sum.x), fmaf(x.y, c, sum.y), fmaf(x.z, c, sum.z), fmaf(x.w, c, sum.w));
}
__device__ __forceinline__ float4 either(bool first, const float4& x, const float4& y) {
  return make_float4(first ? x.x : y.x, first ? x.y : y.y, first ? x.z : y.z, first ? x.w : y.w);
}

// grid: groups_per_cu workgroups for every CU, or fewer (a share of kMinUnits units for each of the most that there can be).
template <typename T, int D, int GP, bool FP8>
__global__ void __launch_bounds__(kAttThreads, (groups_per_cu(D, FP8))) paged_attention_kernel(PagedArgs a) {
  using At = Attend<T, D, GP, FP8>;
  __shared__ __align__(16) float red_o[kAttWaves][2][GP][D];
  __shared__ float red_m[kAttWaves][2][GP], red_z[kAttWaves][2][GP];
  __shared__ WavePiece pieces[kAttWaves][2];
  const int id = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto units = [&](int r) { return (row_len(a, r) + At::kUnit - 1) / At::kUnit; };
  Shares cut_in(1, 1);
  unsigned share = 0, size = 0;   // its first unit, its units
  auto part = [&](int w) { return share + (unsigned)((unsigned long long)size * w / kAttWaves); };
  const RowOfUnit at = locate_row(
      a.R, a.Hkv, units,
      [&](unsigned total) {
        const unsigned shares = min((total + kMinUnits - 1) / kMinUnits, gridDim.x);
        if (id >= (int)shares) return;
        cut_in = Shares(total, shares);
        share = cut_in.first(id);
        size = cut_in.first(id + 1) - share;
      },
      [&](int w) { return part(w) < part(w + 1) ? part(w) : ~0u; });
  unsigned beg = part(wave);
  const unsigned end = part(wave + 1);
  if ((threadIdx.x & 63) < 2) pieces[wave][threadIdx.x & 63].there = false;
  if (at.row >= 0) {
    int r = at.row, n = at.size;
    int head = (int)((beg - at.first) / (unsigned)n), u = (int)(beg - at.first) - head * n;
    while (true) {
      const int take = min(n - u, (int)(end - beg));
      At st;
      st.begin(a, r, head);
      st.units(a, a.table + r * a.table_stride, head, u, u + take, row_len(a, r));
      beg += take;
      const int pair = r * a.Hkv + head, slot = u == 0 ? 1 : 0;
      st.put(red_o[wave][slot], red_m[wave][slot], red_z[wave][slot]);
      if (take == n) {
        // (the wave's own LDS: its writes are seen by itself in order; slot 1 is not in use before the last piece)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        for (int i = threadIdx.x & 63; i < a.G * (D / 4); i += 64) {
          const int h = i / (D / 4), j = 4 * (i - h * (D / 4));
          write_out<T>(a, pair, h, j, D, *reinterpret_cast<const float4*>(&red_o[wave][1][h][j]), red_z[wave][1][h]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if (a.cut_by_pair && (threadIdx.x & 63) == 0) a.cut[pair] = make_int2(0, 0);
      } else if ((threadIdx.x & 63) == 0) {
        pieces[wave][slot] = WavePiece{pair, (int)cut_in.share_of(beg + (n - u - take) - 1) - id, true, u + take == n};
      }
      if (beg >= end) break;
      u = 0;
      if (++head == a.Hkv) {
        head = 0;
        // (beg < end: there is another row with positions.)  One length after the other, each waited for: two rows of 50000
        // positions take 41 us next to each other, 46 with 62 empty rows between them, 61 with 254 and 197 with 2046 (70 and 271 where
        // the lengths lie 128 bytes apart); where the border of the rows is that of two waves, nothing.
        do n = units(++r); while (n == 0);
      }
    }
  }
  __syncthreads();
  // The pieces of one pair after the other: a slot 0 that no slot 1 precedes goes on from the share before; every slot 1
  // begins a pair; the slots 0 of the waves behind go on with it until it ends.
  int2 cut = make_int2(0, 0);
  unsigned there0 = 0, there1 = 0, ends0 = 0;   // bit w: wave w
#pragma unroll
  for (int w = 0; w < kAttWaves; ++w) {
    there0 |= pieces[w][0].there ? 1u << w : 0u;
    there1 |= pieces[w][1].there ? 1u << w : 0u;
    ends0 |= pieces[w][0].there && pieces[w][0].ends ? 1u << w : 0u;
  }
  there0 = __builtin_amdgcn_readfirstlane(there0);
  there1 = __builtin_amdgcn_readfirstlane(there1);
  ends0 = __builtin_amdgcn_readfirstlane(ends0);
  unsigned todo = there1;                       // pairs that begin here ...
  int slot = 1, w0 = there0 ? __builtin_ctz(there0) : 0;
  if (there0 && (there1 & ((1u << w0) - 1u)) == 0u) slot = 0;   // ... after the one that goes on from before
  while (slot == 0 || todo != 0u) {
    if (slot == 1) w0 = __builtin_ctz(todo);
    // the waves behind that have a piece of the same pair
    unsigned more = there0 & ~((2u << w0) - 1u);
    const unsigned last = ends0 & more;
    bool ends = slot == 0 && ((ends0 >> w0) & 1u) != 0u;
    if (ends) {
      more = 0u;
    } else if (last != 0u) {
      ends = true;
      more &= (2u << __builtin_ctz(last)) - 1u;
    }
    const WavePiece first = pieces[w0][slot];
    for (int i = threadIdx.x; i < a.G * (D / 4); i += kAttThreads) {   // (four columns: one round for groups of up to 8 heads)
      const int h = i / (D / 4), j = 4 * (i - h * (D / 4));
      float m[kAttWaves], mn = red_m[w0][slot][h];
      const float m0 = mn;
#pragma unroll
      for (int w = 1; w < kAttWaves; ++w) {
        m[w] = red_m[w][0][h];
        mn = (more >> w) & 1u ? fmaxf(mn, m[w]) : mn;
      }
      float c = weight_under(m0, mn, a.scale_log2);
      float zs = red_z[w0][slot][h] * c;
      float4 os = scaled(*reinterpret_cast<const float4*>(&red_o[w0][slot][h][j]), c);
#pragma unroll
      for (int w = 1; w < kAttWaves; ++w) {
        c = weight_under(m[w], mn, a.scale_log2);
        const bool in = ((more >> w) & 1u) != 0u;
        zs = in ? fmaf(red_z[w][0][h], c, zs) : zs;
        os = either(in, add_scaled(os, *reinterpret_cast<const float4*>(&red_o[w][0][h][j]), c), os);
      }
      if (slot == 1 && ends) {
        write_out<T>(a, first.pair, h, j, D, os, zs);
      } else {
        const size_t to = (size_t)(2 * id + slot) * a.G + h;
        *reinterpret_cast<float4*>(a.part + to * D + j) = os;
        if (j == 0) a.part_mz[to] = make_float2(mn, zs);
      }
    }
    if (slot == 1) {
      if (a.cut_by_pair) {
        if (threadIdx.x == 0) a.cut[first.pair] = make_int2(id, ends ? 0 : first.shares);
      } else if (!ends) {
        cut = make_int2(first.pair, first.shares);
      }
      todo &= todo - 1u;
    }
    slot = 1;
  }
  if (!a.cut_by_pair && threadIdx.x == 0) a.cut[id] = cut;
  // rows without positions, dealt to all workgroups
  for (int r = id; r < a.R; r += gridDim.x)
    if (row_len(a, r) == 0) {
      for (int i = threadIdx.x; i < a.Hq * D; i += kAttThreads) store_elem(a.out + r * a.out_stride + (size_t)i * sizeof(T), 0.f, T{});
      if (a.cut_by_pair)
        for (int i = threadIdx.x; i < a.Hkv; i += kAttThreads) a.cut[r * a.Hkv + i] = make_int2(0, 0);
    }
}

// ---- short tables -----------------------------------------------------------------------------------------------------
//
// Where no row can be long, a workgroup per (row, kv head) is enough: no search, no pieces in memory, no second launch.
// WAVES contiguous parts of the pair's units, added up in LDS.  grid (Hkv, R).
//
// How short, by the bytes of keys and values that the table can hold per pair: up to kPairBytes with enough pairs to keep the
// chip busy (pairs against shares, us: 2000 rows of up to 300 positions 28.9 and 36.7, 512 pairs of up to 600 20.2 and 23.3,
// 256 pairs of up to 1000 8-bit positions 14.8 and 20.3, 160 of 300 to 600 15.3 and 17.3), up to kFewPairBytes with half as many
// pairs as CUs or fewer, where the CU with the longest row is waited for (128 pairs of up to 384 10.6 and 11.9, of up to 600 13.9
// and 11.9; 96 of up to 300 fp32 positions 14.5 and 12.3), and with a handful up to kPairPositions, as the waves of one CU walk
// over them (8 pairs of 100 6.1 and 8.9, of 400 9.1 and 10.3, of 1000 8-bit positions 13.9 and 10.2).  Eight waves where every
// workgroup has a CU to itself, four otherwise (256 pairs of up to 1000 8-bit positions 14.8 and 16.9 us with eight and four,
// 2000 pairs of up to 300 43.5 and 28.9).
constexpr int kPairBytes = 320 << 10, kFewPairBytes = 208 << 10, kPairPositions = 512;
template <typename T, int D, int GP, bool FP8, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, (WAVES == 4 ? groups_per_cu(D, FP8) : 2)) paged_pair_kernel(PagedArgs a) {
  using At = Attend<T, D, GP, FP8>;
  __shared__ __align__(16) float red_o[WAVES][GP][D];
  __shared__ float red_m[WAVES][GP], red_z[WAVES][GP];
  const int head = blockIdx.x, r = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int len = __builtin_amdgcn_readfirstlane(row_len(a, r)), n = (len + At::kUnit - 1) / At::kUnit;
  const int each = (n + WAVES - 1) / WAVES, active = each > 0 ? (n + each - 1) / each : 0;   // waves 0 .. active - 1 have units
  if (wave < active) {
    At st;
    st.begin(a, r, head);
    st.units(a, a.table + r * a.table_stride, head, wave * each, min((wave + 1) * each, n), len);
    st.put(red_o[wave], red_m[wave], red_z[wave]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.G * (D / 4); i += 64 * WAVES) {
    const int h = i / (D / 4), j = 4 * (i - h * (D / 4));
    float mn = kLeast, zs = 0.f;
    float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mn = w < active ? fmaxf(mn, red_m[w][h]) : mn;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float c = weight_under(red_m[w][h], mn, a.scale_log2);
      zs = w < active ? fmaf(red_z[w][h], c, zs) : zs;
      os = either(w < active, add_scaled(os, *reinterpret_cast<const float4*>(&red_o[w][h][j]), c), os);
    }
    write_out<T>(a, r * a.Hkv + head, h, j, D, os, zs);
  }
}

// grid (pairs or shares, G): joins the pieces of the (row, kv head) that blockIdx.x names, one query head each.  Four columns per
// thread, kJoinLanes pieces side by side and eight of each on their way together: 128 pieces take two rounds with 256 threads
// and one with 512, which pairs of that many pieces get (a step over one pair of 30000 positions in 234 pieces 15.0 us with 256
// and 13.8 with 512 threads, four pairs in 128 each 20.9 and 20.3; eight in 96 11.5 and 12.1; 256 pairs cut in two or three 80
// and 82).  One column per thread, two pieces side by side: twice as long.
constexpr int kJoinPieces = 128;
template <typename T, int D, int kJoinThreads>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(PagedArgs a) {
  constexpr int Q = D / 4, kJoinLanes = kJoinThreads / Q, U = 8;
  __shared__ float4 lds_o[kJoinLanes][Q];
  __shared__ float lds_m[kJoinLanes], lds_z[kJoinLanes];
  const int h = blockIdx.y, j = threadIdx.x % Q, lane = threadIdx.x / Q;
  const int2 cut = a.cut[blockIdx.x];
  if (cut.y == 0) return;
  const int id = a.cut_by_pair ? cut.x : (int)blockIdx.x, pair = a.cut_by_pair ? (int)blockIdx.x : cut.x;
  const int n = cut.y + 1;   // pieces: slot 1 of share id, slot 0 of the shares behind it
  float mn = kLeast, zs = 0.f;
  float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
  auto round = [&](int s0, auto count) {
    constexpr int N = decltype(count)::value;
    float2 mz[N];
    float4 o[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int s = min(s0 + u * kJoinLanes, n - 1);
      const size_t at = (size_t)(2 * (id + s) + (s == 0 ? 1 : 0)) * a.G + h;
      mz[u] = a.part_mz[at];
      o[u] = *reinterpret_cast<const float4*>(a.part + at * D + 4 * j);
    }
    // (all of them are asked for before any is used: under the conditions below each load would wait for itself)
#pragma unroll
    for (int u = 0; u < N; ++u) asm volatile("" : "+v"(o[u].x), "+v"(o[u].y), "+v"(o[u].z), "+v"(o[u].w), "+v"(mz[u].x), "+v"(mz[u].y));
    float top = mn;
#pragma unroll
    for (int u = 0; u < N; ++u) top = fmaxf(top, mz[u].x);   // (a piece that is repeated changes no maximum)
    const float c0 = weight_under(mn, top, a.scale_log2);
    zs *= c0;
    os = scaled(os, c0);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const bool in = s0 + u * kJoinLanes < n;
      const float c = in ? weight_under(mz[u].x, top, a.scale_log2) : 0.f;
      zs = fmaf(in ? mz[u].y : 0.f, c, zs);
      os = add_scaled(os, either(in, o[u], make_float4(0.f, 0.f, 0.f, 0.f)), c);
    }
    mn = top;
  };
  int s0 = lane;
  for (; s0 + U / 4 * kJoinLanes < n; s0 += U * kJoinLanes) round(s0, std::integral_constant<int, U>());
  if (s0 < n) round(s0, std::integral_constant<int, U / 4>());
  lds_o[lane][j] = os;
  if (j == 0) {
    lds_m[lane] = mn;
    lds_z[lane] = zs;
  }
  __syncthreads();
  if (lane != 0) return;
  mn = lds_m[0];
#pragma unroll
  for (int w = 1; w < kJoinLanes; ++w) mn = fmaxf(mn, lds_m[w]);
  zs = 0.f;
  os = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kJoinLanes; ++w) {
    const float c = weight_under(lds_m[w], mn, a.scale_log2);
    zs = fmaf(lds_z[w], c, zs);
    os = add_scaled(os, lds_o[w][j], c);
  }
  write_out<T>(a, pair, h, 4 * j, D, os, zs);
}

struct PagedPlan {
  int groups, GP;
  int pair_waves;   // waves of a workgroup per (row, kv head); 0: shares
  size_t part_bytes, mz_bytes, ws_bytes;
};

constexpr double kLog2E = 1.4426950408889634074;

static meda_status make_paged_plan(const meda_page_pool* pool, const meda_paged_params* p, PagedPlan* pl) {
  if (!p) return MEDA_ERR_INVALID_ARG;
  meda_status st = check_pool_sizes(pool);
  if (st != MEDA_OK) return st;
  if (p->n_rows < 1 || p->n_q_heads < 1 || p->max_blocks < 1) return MEDA_ERR_INVALID_ARG;
  if (p->q_stride < 0 || p->out_stride < 0 || p->table_stride < 0 || p->len_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (p->n_q_heads % pool->n_kv_heads != 0) return MEDA_ERR_INVALID_ARG;
  // (as the kernels use it, times log2(e), it has to be finite too: 0 times infinity is the weight of no maximum)
  if (!(p->softmax_scale >= 0.0f) || !((double)p->softmax_scale * kLog2E <= (double)__FLT_MAX__)) return MEDA_ERR_INVALID_ARG;
  st = check_types(p->dtype, pool->dtype);
  if (st != MEDA_OK) return st;
  const int G = p->n_q_heads / pool->n_kv_heads;
  const int64_t most = (int64_t)p->max_blocks * pool->page_size;
  const int elt = dtype_bytes(p->dtype);
  if (G > kMaxGroup || p->n_rows > 65536 || most > (1 << 29)) return MEDA_ERR_UNSUPPORTED;
  if (!few_units(p->n_rows, most, pool->n_kv_heads, unit_positions(elt))) return MEDA_ERR_UNSUPPORTED;
  if ((int64_t)p->n_rows * pool->n_kv_heads > INT32_MAX) return MEDA_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)p->n_q_heads * pool->head_dim, far = 1ll << 40;
  if ((p->q_stride && p->q_stride < row) || (p->out_stride && p->out_stride < row) || (p->table_stride && p->table_stride < p->max_blocks))
    return MEDA_ERR_INVALID_ARG;
  if (p->q_stride > far || p->out_stride > far || p->table_stride > far || p->len_stride > far) return MEDA_ERR_UNSUPPORTED;
  if (p->q_stride * elt % 16 || p->out_stride * elt % 16) return MEDA_ERR_INVALID_ARG;
  const int64_t unit = unit_positions(elt), units = (most + unit - 1) / unit * pool->n_kv_heads;   // of one row, at most
  pl->GP = G <= 1 ? 1 : (G <= 2 ? 2 : (G <= 4 ? 4 : (G <= 8 ? 8 : 16)));
  const int64_t most_groups = kCus * groups_per_cu(pool->head_dim, pool->dtype == MEDA_E4M3);
  const int64_t shares = units > most_groups * kMinUnits ? most_groups : (units * p->n_rows + kMinUnits - 1) / kMinUnits;
  pl->groups = (int)(shares < most_groups ? shares : most_groups);
  pl->pair_waves = 0;
  const int64_t pairs = (int64_t)p->n_rows * pool->n_kv_heads;
  const int64_t bytes = most * 2 * pool->head_dim * dtype_bytes(pool->dtype);
  if (bytes <= (pairs > kCus / 2 ? kPairBytes : kFewPairBytes) && (pairs > kFewPairs || most <= kPairPositions) && p->n_rows <= 65535)
    pl->pair_waves = pairs <= kCus ? 8 : 4;
  pl->part_bytes = ((size_t)2 * pl->groups * G * pool->head_dim * sizeof(float) + 255) / 256 * 256;
  pl->mz_bytes = ((size_t)2 * pl->groups * G * sizeof(float2) + 255) / 256 * 256;
  pl->ws_bytes = pl->part_bytes + pl->mz_bytes + ((size_t)pl->groups * sizeof(int2) + 255) / 256 * 256;
  return MEDA_OK;
}

template <typename T, int D, int GP, bool FP8>
static hipError_t launch_paged(const PagedPlan& pl, const PagedArgs& a, hipStream_t s) {
  if (pl.pair_waves == 8) {
    hipLaunchKernelGGL((paged_pair_kernel<T, D, GP, FP8, 8>), dim3(a.Hkv, a.R), dim3(512), 0, s, a);
    return hipGetLastError();
  }
  if (pl.pair_waves == 4) {
    hipLaunchKernelGGL((paged_pair_kernel<T, D, GP, FP8, 4>), dim3(a.Hkv, a.R), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((paged_attention_kernel<T, D, GP, FP8>), dim3(pl.groups), dim3(kAttThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int joins = a.cut_by_pair ? a.R * a.Hkv : pl.groups;
  if (pl.groups >= kJoinPieces * joins) hipLaunchKernelGGL((paged_join_kernel<T, D, 512>), dim3(joins, a.G), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((paged_join_kernel<T, D, 256>), dim3(joins, a.G), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T, int D, bool FP8>
static hipError_t launch_paged_g(const PagedPlan& pl, const PagedArgs& a, hipStream_t s) {
  switch (pl.GP) {
    case 1: return launch_paged<T, D, 1, FP8>(pl, a, s);
    case 2: return launch_paged<T, D, 2, FP8>(pl, a, s);
    case 4: return launch_paged<T, D, 4, FP8>(pl, a, s);
    case 8: return launch_paged<T, D, 8, FP8>(pl, a, s);
    default: return launch_paged<T, D, 16, FP8>(pl, a, s);
  }
}

}  // namespace meda

extern "C" {

size_t meda_paged_workspace_bytes(const meda_page_pool* pool, const meda_paged_params* params) {
  meda::PagedPlan pl;
  return meda::make_paged_plan(pool, params, &pl) == MEDA_OK ? pl.ws_bytes : 0;
}

meda_status meda_paged_attention(const meda_page_pool* pool, const meda_paged_params* params, const void* q,
                                 const int32_t* table, const int32_t* lens, void* out, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  using namespace meda;
  PagedPlan pl;
  meda_status st = make_paged_plan(pool, params, &pl);
  if (st != MEDA_OK) return st;
  const meda_paged_params& p = *params;
  PagedArgs a;
  st = read_pool(pool, &a.pool);
  if (st != MEDA_OK) return st;
  if (!q || !table || !lens || !out) return MEDA_ERR_INVALID_ARG;
  if ((((uintptr_t)q | (uintptr_t)out) & 15u) || (((uintptr_t)table | (uintptr_t)lens) & 3u)) return MEDA_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < pl.ws_bytes) return MEDA_ERR_WORKSPACE;
  const int64_t row = (int64_t)p.n_q_heads * pool->head_dim, elt = dtype_bytes(p.dtype);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.table = table; a.lens = lens;
  a.part = static_cast<float*>(workspace);
  a.part_mz = reinterpret_cast<float2*>(static_cast<char*>(workspace) + pl.part_bytes);
  a.cut = reinterpret_cast<int2*>(static_cast<char*>(workspace) + pl.part_bytes + pl.mz_bytes);
  a.q_stride = (p.q_stride ? p.q_stride : row) * elt;
  a.out_stride = (p.out_stride ? p.out_stride : row) * elt;
  a.table_stride = p.table_stride ? p.table_stride : p.max_blocks;
  a.len_stride = p.len_stride ? p.len_stride : 1;
  a.R = p.n_rows; a.Hq = p.n_q_heads; a.Hkv = pool->n_kv_heads; a.G = a.Hq / a.Hkv; a.max_blocks = p.max_blocks;
  a.cut_by_pair = (int64_t)p.n_rows * pool->n_kv_heads <= pl.groups;
  const double scale = p.softmax_scale > 0.0f ? (double)p.softmax_scale : 1.0 / sqrt((double)pool->head_dim);
  a.scale_log2 = (float)(scale * kLog2E);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool wide = pool->head_dim == 128;
  hipError_t e;
  if (pool->dtype == MEDA_F32) e = wide ? launch_paged_g<float, 128, false>(pl, a, s) : launch_paged_g<float, 64, false>(pl, a, s);
  else if (pool->dtype == MEDA_BF16) e = wide ? launch_paged_g<bf16_t, 128, false>(pl, a, s) : launch_paged_g<bf16_t, 64, false>(pl, a, s);
  else e = wide ? launch_paged_g<bf16_t, 128, true>(pl, a, s) : launch_paged_g<bf16_t, 64, true>(pl, a, s);
  return e == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

}  // extern "C"
