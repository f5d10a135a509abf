// Attention of one new token per row over its pages: out = Softmax(q K^T / sqrt(d)) V.
//
// Every cached key and value is read once and takes 4 * G * d flops per pair (G query heads share a kv head), so the step
// is bound by HBM where it is long and by latency where it is short.  The work is numbered in units of 32 positions, row
// after row and kv head after kv head, and cut into contiguous shares of equal size, one per workgroup, on the device:
// lengths that differ by a factor of a thousand, empty rows and a single long request all fill the chip.  A
// (row, kv head) that lies in one share is finished by its workgroup; one that is cut leaves, per share, a running maximum,
// a normaliser and a weighted value sum, which a second kernel joins.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/meda.h"
#include "fp8.hpp"
#include "paged.hpp"

namespace meda {

constexpr int kAttThreads = kLocateThreads, kAttWaves = kAttThreads / 64;
constexpr int kUnit = 32;         // positions: a step of one wave
constexpr int kMinUnits = 4;      // a workgroup's share, at least: a step per wave
constexpr int kMaxGroup = 16;     // query heads per kv head
// Workgroups per CU, and waves per SIMD, as many as the registers allow.  All workgroups of a launch are at work at once,
// each on one share, and every CU has equally many of them: 512 workgroups of which three fit a CU were spread unevenly
// (64 requests, 435 MB: 95 us against 86 with 768), and with two or three rounds of shorter shares the workgroups' searches
// and the joins cost more than the evener end gained (104 and 111 us against 99, before the pages of 32 steps were loaded
// at once).
constexpr int groups_per_cu(int q_bytes, int d, int gp) {
  return q_bytes == 4 ? (gp <= 2 ? 4 : (gp <= 8 ? 3 : 2)) : (d == 64 ? 4 : 3);
}
constexpr int kCus = 256;

struct PagedArgs {
  Pool pool;
  const char* q;
  char* out;
  const int32_t* table;
  const int32_t* lens;
  float* part;             // [2 * groups][G][d]: value sums of the pieces
  float2* part_mz;         // [2 * groups][G]: their maximum (base-2 logits) and normaliser
  int2* cut;               // [groups]: the (row, kv head) that begins in the share and goes on behind it, as
                           // (row * Hkv + head, shares it reaches into); (0, 0): none
  long long q_stride, out_stride;   // bytes
  long long table_stride, len_stride;
  int R, Hq, Hkv, G, max_blocks;
  float scale_log2;
};

__device__ __forceinline__ int row_len(const PagedArgs& a, int r) {
  return min(max(a.lens[r * a.len_stride], 0), a.max_blocks << a.pool.page_log2);
}

// The pages of the units u, u + kAttWaves, .. of a wave (32 of them, two blocks of 16 positions each): lane 2 i + b holds
// that of block b of the i-th.  One load for 32 steps: a load of its own in every step would have to be waited for, and with
// it, as loads come back in order, for all rows that are on their way (64 requests, 435 MB: 95 us against 81).
__device__ __forceinline__ int load_pages(const PagedArgs& a, const int32_t* table, int u, int u1, int len) {
  const int lane = threadIdx.x & 63;
  const int pos = min(u + kAttWaves * (lane >> 1), u1 - 1) * kUnit;     // (units past the share repeat its last one)
  const int p = pos + 16 * (lane & 1);
  return table[(p < len ? p : pos) >> a.pool.page_log2];                // a block behind the end repeats the first one
}

// Where a unit's two blocks of 16 positions lie, as byte offsets of (page, head, place) and scale indexes.
struct UnitPages {
  size_t at[2];
  size_t scale[2];
  bool ok[2];      // the page exists
};
template <int ROW_BYTES>
__device__ __forceinline__ UnitPages unit_pages(const PagedArgs& a, int pages, int step, int head, int pos, int len) {
  UnitPages u;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int p = pos + 16 * b, q = p < len ? p : pos;
    const int page = __builtin_amdgcn_readlane(pages, 2 * (step & 31) + b);
    u.ok[b] = page >= 0 && page < a.pool.n_pages;
    const size_t safe = u.ok[b] ? page : 0;
    const size_t place = ((size_t)head << a.pool.page_log2) + (q & ((1 << a.pool.page_log2) - 1));
    u.at[b] = safe * a.pool.page_bytes + place * ROW_BYTES;
    u.scale[b] = (safe * a.Hkv << a.pool.page_log2) + place;
  }
  return u;
}

// A maximum starts at the least finite number, not at -infinity: every finite logit replaces or equals it, a logit of
// -infinity has the weight exp2(-inf) = 0 under it, and differences of maxima are never inf - inf.
constexpr float kLeast = -__FLT_MAX__;

// ---- bf16 and 8-bit pages: both products on the matrix unit ---------------------------------------------------------
//
// Lane (c, g) = (l % 16, l / 16).  logits D[key][col] = sum_d K[key][d] Q[col][d]: the lane holds 8 elements of key c per
// k-step and block of 16 keys, and receives the logits of head c % GP for the keys 4 g + i of every block.  The second
// product O[row][col] += sum_key P[row][key] V[key][col] contracts over the keys in the order (lane group, register), so
// its weights are what the lane has; its values are the same 8 keys at d / 16 columns, transposed in registers.
// A weight enters as the sum of two bf16 numbers, rows c / GP = 0 and 1 of the product (what the first leaves is exact and
// not zero, and 2^-16 of the weight is lost at most: a 128th of the output's own rounding), so that groups of up to 8
// heads need one instruction per 16 columns; groups of 9 to 16 take two, one per part.  8-bit rows: codes become bf16
// exactly, the key's scale multiplies the logit and the value's scale the weight.
template <int D>
struct AttState {
  float m, z;           // of head c % GP; m is the same in the four lane groups
  f32x4_t acc[D / 16];  // acc[j][r]: output column (d/16) c + j, product row 4 g + r
};

template <int D, int GP, bool FP8>
__device__ __forceinline__ void attend_units(AttState<D>& st, const uint4 (&qp)[D / 32], const PagedArgs& a,
                                             const int32_t* table, int head, int u0, int u1, int len) {
  constexpr int KS = D / 32, PE = D / 16, kEl = FP8 ? 1 : 2, kRowBytes = D * kEl;
  constexpr int KL = D * kEl / 64;            // 16-byte loads per key and lane
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = (c / GP) & 1;
  struct Unit {
    uint32_t k[2][KL][4], v[8][PE * kEl / 4];
    float scale;
  };
  // MASKED: some of the unit's positions lie behind the end or in a page that does not exist.  Positions behind the end
  // repeat the last one (their weights are zero).
  auto load_keys = [&](Unit& t, const UnitPages& up, int pos, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int last = min(len - 1 - pos - 16 * b, 15), top = last < 0 ? min(len - 1 - pos, 15) : last;
      const char* src = a.pool.k + up.at[b] + (unsigned)((MASKED ? min(c, top) : c) * kRowBytes + 16 * g);
#pragma unroll
      for (int k = 0; k < KL; ++k) {
        const uint4 x = load16_stream(src + 64 * k);
        t.k[b][k][0] = x.x; t.k[b][k][1] = x.y; t.k[b][k][2] = x.z; t.k[b][k][3] = x.w;
      }
    }
  };
  auto load_values = [&](Unit& t, const UnitPages& up, int pos, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int last = min(len - 1 - pos - 16 * b, 15), top = last < 0 ? min(len - 1 - pos, 15) : last;
      const char* src = a.pool.v + up.at[b];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        load_piece<PE * kEl>(src + (unsigned)((MASKED ? min(4 * g + i, top) : 4 * g + i) * kRowBytes + c * PE * kEl), t.v[4 * b + i]);
      // the scales of the 8 keys that this row of 16 lanes has logits for: lanes 0..7 the keys', 8..15 the values'
      if constexpr (FP8) {
        const int row = 4 * g + (c & 3);
        if (((c >> 2) & 1) == b) t.scale = (c < 8 ? a.pool.ks : a.pool.vs)[up.scale[b] + (MASKED ? min(row, top) : row)];
      }
    }
  };
  auto logits = [&](const Unit& rows, float (&t)[8]) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x4_t s4 = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint4 kp;
        if constexpr (FP8) kp = e4m3x8_to_bf16x8(make_uint2(rows.k[b][k / 2][2 * (k & 1)], rows.k[b][k / 2][2 * (k & 1) + 1]));
        else kp = make_uint4(rows.k[b][k][0], rows.k[b][k][1], rows.k[b][k][2], rows.k[b][k][3]);
        s4 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kp), __builtin_bit_cast(bf16x8_t, qp[k]), s4, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) t[4 * b + i] = s4[i];
    }
  };
  auto finish = [&](Unit& rows, const UnitPages& up, int pos, float (&t)[8], auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    float sk[8], sv[8];
    bool in[8];
    if constexpr (FP8) {
      row_broadcast<0>(rows.scale * a.scale_log2, sk);
      row_broadcast<8>(rows.scale, sv);
    }
    float bm = kLeast;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t[e] *= FP8 ? sk[e] : a.scale_log2;
      if constexpr (MASKED) {
        in[e] = up.ok[e >> 2] && pos + 16 * (e >> 2) + 4 * g + (e & 3) < len;
        t[e] = in[e] ? t[e] : -INFINITY;
#pragma unroll
        for (uint32_t& x : rows.v[e]) x = in[e] ? x : 0u;   // what is read in its place may hold an infinity
      }
      bm = fmaxf(bm, t[e]);
    }
    bm = group_max(bm);
    if (__ballot(bm > st.m) != 0ull) {  // a new maximum of some head: rescale what that head has so far (rare)
      const float mn = fmaxf(st.m, bm);
      const float c1 = __builtin_amdgcn_exp2f(st.m - mn);
      st.z *= c1;
      st.m = mn;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float cr = __shfl(c1, 4 * g + r, kWave);  // product row 4 g + r belongs to the head of lane column 4 g + r
#pragma unroll
        for (int j = 0; j < PE; ++j) st.acc[j][r] *= cr;
      }
    }
    uint32_t pa[4], pb[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      uint32_t x[2], y[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float p = __builtin_amdgcn_exp2f(t[e + u] - st.m);
        float w = FP8 ? fmaf(p, sv[e + u], 0.f) : p;  // the sum takes the sign of a zero
        if constexpr (MASKED) {
          p = in[e + u] ? p : 0.f;
          w = in[e + u] ? w : 0.f;
        }
        st.z += p;
        const float hi = weight_part(w), lo = w - hi;
        x[u] = __float_as_uint(GP == 16 || part == 0 ? hi : lo);
        y[u] = __float_as_uint(lo);
      }
      pa[e / 2] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
      pb[e / 2] = __builtin_amdgcn_perm(y[1], y[0], 0x07060302u);
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
      st.acc[2 * j2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, v0, st.acc[2 * j2], 0, 0, 0);
      st.acc[2 * j2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa, v1, st.acc[2 * j2 + 1], 0, 0, 0);
      if constexpr (GP == 16) {
        st.acc[2 * j2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, v0, st.acc[2 * j2], 0, 0, 0);
        st.acc[2 * j2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, v1, st.acc[2 * j2 + 1], 0, 0, 0);
      }
    }
  };

  int u = u0 + wave, step = 0;
  if (u >= u1) return;
  auto full = [&](const UnitPages& up, int pos) { return pos + kUnit <= len && up.ok[0] && up.ok[1]; };
  int pages = load_pages(a, table, u, u1, len), pages_behind = pages;
  UnitPages up = unit_pages<kRowBytes>(a, pages, step, head, u * kUnit, len);
  bool fast = full(up, u * kUnit);
  Unit rows;
  float t[8];
  if (fast) load_keys(rows, up, 0, std::false_type());
  while (fast) {
    load_values(rows, up, 0, std::false_type());
    const UnitPages cur = up;
    u += kAttWaves;
    ++step;
    fast = u < u1;
    if ((step & 31) == 16) pages_behind = load_pages(a, table, u + 16 * kAttWaves, u1, len);
    if ((step & 31) == 0) pages = pages_behind;
    if (fast) {
      up = unit_pages<kRowBytes>(a, pages, step, head, u * kUnit, len);
      fast = full(up, u * kUnit);
    }
    logits(rows, t);
    if (fast) load_keys(rows, up, 0, std::false_type());  // in flight while this unit is finished
    finish(rows, cur, 0, t, std::false_type());
  }
  for (; u < u1; u += kAttWaves) {   // the last unit of a row; units behind a missing page
    up = unit_pages<kRowBytes>(a, load_pages(a, table, u, u1, len), 0, head, u * kUnit, len);
    load_keys(rows, up, u * kUnit, std::true_type());
    logits(rows, t);
    load_values(rows, up, u * kUnit, std::true_type());
    finish(rows, up, u * kUnit, t, std::true_type());
  }
}

// ---- what a workgroup's waves have, merged: a finished output or a partial ------------------------------------------

template <typename T, int H, int D>
__device__ __forceinline__ void write_piece(const PagedArgs& a, bool whole, int slot, int r, int head,
                                            const float (&red_o)[kAttWaves][H][D], const float (&red_m)[kAttWaves][H],
                                            const float (&red_z)[kAttWaves][H]) {
  for (int i = threadIdx.x; i < a.G * D; i += kAttThreads) {
    const int h = i / D, j = i - h * D;
    float mn = red_m[0][h];
#pragma unroll
    for (int w = 1; w < kAttWaves; ++w) mn = fmaxf(mn, red_m[w][h]);
    float zs = 0.f, os = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) {
      const float c = __builtin_amdgcn_exp2f(red_m[w][h] - mn);
      zs = fmaf(red_z[w][h], c, zs);
      os = fmaf(red_o[w][h][j], c, os);
    }
    if (whole) {
      // (no weight at all, as where every page is missing: zeros)
      store_elem(a.out + r * a.out_stride + ((size_t)(head * a.G + h) * D + j) * sizeof(T), zs == 0.f ? 0.f : os / zs, T{});
    } else {
      const size_t at = (size_t)slot * a.G + h;
      a.part[at * D + j] = os;
      if (j == 0) a.part_mz[at] = make_float2(mn, zs);
    }
  }
}

// ---- fp32 pages: the vector unit ------------------------------------------------------------------------------------
//
// A row is read by LPR = row bytes / 16 lanes, a wave takes 64 / LPR rows per step; every lane group keeps, per query head,
// the running maximum, the normaliser and its piece of the weighted value sum over the rows it has seen.
template <int D, int GP>
__device__ __forceinline__ void attend_f32(const PagedArgs& a, int r, int head, const int32_t* table, int u0, int u1, int len,
                                           float (&red_o)[GP][D], float (&red_m)[GP], float (&red_z)[GP]) {
  // U steps' rows are on their way while U others are worked on (fewer where the heads need the registers)
  constexpr int LPR = D / 4, MS = 64 / LPR, E = 4, U = GP <= 4 ? 4 : 2, kRowBytes = D * 4;
  constexpr int kRows = U * MS, kParts = kUnit / kRows;   // positions of one part of a unit; a part lies in one block
  static_assert(kRows <= 16, "a part lies in one page");
  const int lane = threadIdx.x & 63, sub = lane / LPR, cc = lane - sub * LPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint4 qp[GP];
#pragma unroll
  for (int h = 0; h < GP; ++h)
    qp[h] = *reinterpret_cast<const uint4*>(a.q + r * a.q_stride + (size_t)(head * a.G + (h < a.G ? h : 0)) * kRowBytes + cc * 16);
  // running maximum and normaliser of the ONE head this lane evaluates (row_head), weighted value sums of all
  float m1 = kLeast, z1 = 0.f, o[GP][E];
#pragma unroll
  for (int h = 0; h < GP; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) o[h][e] = 0.f;

  struct Part {
    uint4 k[U], v[U];
    int n;           // its positions: fewer than kRows at the end, none in a page that does not exist
  };
  auto load = [&](Part& t, int pages, int step, int u, int part) {
    const int pos = u * kUnit + part * kRows;
    const int page = __builtin_amdgcn_readlane(pages, 2 * (step & 31) + part * kRows / 16);
    const bool ok = page >= 0 && page < a.pool.n_pages;
    t.n = ok ? min(max(len - pos, 0), kRows) : 0;
    const size_t place = ((size_t)head << a.pool.page_log2) + (pos & ((1 << a.pool.page_log2) - 1));
    const size_t at = (size_t)(ok ? page : 0) * a.pool.page_bytes + place * kRowBytes;
#pragma unroll
    for (int w = 0; w < U; ++w) {
      const unsigned ro = (unsigned)(min(w * MS + sub, max(t.n - 1, 0)) * kRowBytes + cc * 16);
      t.k[w] = load16_stream(a.pool.k + at + ro);
      t.v[w] = load16_stream(a.pool.v + at + ro);
    }
  };
  auto compute = [&](const Part& t) {
#pragma unroll
    for (int w = 0; w < U; ++w) {
      const bool ok = w * MS + sub < t.n;
      float s[GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) s[h] = dot4(qp[h], t.k[w]);
      row_reduce_scatter<GP, LPR>(s, cc);
      const float s1 = ok ? s[0] * a.scale_log2 : -INFINITY;
      if (__ballot(s1 > m1) != 0ull) {  // a new maximum of some head in some lane group (rare after the first rows)
        const float mn = fmaxf(m1, s1);
        const float c1 = __builtin_amdgcn_exp2f(m1 - mn);
        z1 *= c1;
        m1 = mn;
        float c[GP];
        row_all_gather<GP, LPR>(c1, c, cc);
#pragma unroll
        for (int h = 0; h < GP; ++h)
#pragma unroll
          for (int e = 0; e < E; ++e) o[h][e] *= c[h];
      }
      const float p1 = ok ? __builtin_amdgcn_exp2f(s1 - m1) : 0.f;
      z1 += p1;
      float p[GP], vf[E];
      row_all_gather<GP, LPR>(p1, p, cc);
      unpack4(t.v[w], vf);
#pragma unroll
      for (int e = 0; e < E; ++e) vf[e] = ok ? vf[e] : 0.f;   // (what is read in its place may hold an infinity)
#pragma unroll
      for (int h = 0; h < GP; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] = fmaf(p[h], vf[e], o[h][e]);
    }
  };
  int u = u0 + wave, step = 0, part = 0;
  if (u < u1) {
    int pages = load_pages(a, table, u, u1, len), pages_behind = pages;
    Part even, odd;
    bool more = true;
    load(even, pages, step, u, part);
    auto turn = [&](const Part& now, Part& next) {
      if (++part == kParts) {
        part = 0;
        u += kAttWaves;
        ++step;
        more = u < u1;
        if ((step & 31) == 16) pages_behind = load_pages(a, table, u + 16 * kAttWaves, u1, len);
        if ((step & 31) == 0) pages = pages_behind;
      }
      if (more) load(next, pages, step, u, part);
      compute(now);
    };
    while (more) {
      turn(even, odd);
      if (!more) break;
      turn(odd, even);
    }
  }
  // merge the lane groups of the wave, which saw different rows
  float m[GP], z[GP];
  row_all_gather<GP, LPR>(m1, m, cc);
  row_all_gather<GP, LPR>(z1, z, cc);
#pragma unroll
  for (int x = LPR; x < 64; x <<= 1) {
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      const float mo = __shfl_xor(m[h], x, kWave), zo = __shfl_xor(z[h], x, kWave);
      const float mn = fmaxf(m[h], mo);
      const float c0 = __builtin_amdgcn_exp2f(m[h] - mn), c1 = __builtin_amdgcn_exp2f(mo - mn);
      z[h] = z[h] * c0 + zo * c1;
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] = o[h][e] * c0 + __shfl_xor(o[h][e], x, kWave) * c1;
      m[h] = mn;
    }
  }
  if (sub == 0) {
#pragma unroll
    for (int h = 0; h < GP; ++h) {
#pragma unroll
      for (int e = 0; e < E; ++e) red_o[h][cc * E + e] = o[h][e];
      if (cc == 0) {
        red_m[h] = m[h];
        red_z[h] = z[h];
      }
    }
  }
}

template <int D, int GP, bool FP8>
__device__ __forceinline__ void attend_matrix(const PagedArgs& a, int r, int head, const int32_t* table, int u0, int u1, int len,
                                              float (&red_o)[GP][D], float (&red_m)[GP], float (&red_z)[GP]) {
  constexpr int PE = D / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, grp = lane >> 4;
  uint4 qp[D / 32];
#pragma unroll
  for (int k = 0; k < D / 32; ++k) {
    qp[k] = make_uint4(0u, 0u, 0u, 0u);
    // the elements that the key's loads bring (16 bytes of codes are two k-steps)
    const int e0 = FP8 ? 64 * (k / 2) + 16 * grp + 8 * (k & 1) : 32 * k + 8 * grp;
    if (c % GP < a.G) qp[k] = *reinterpret_cast<const uint4*>(a.q + r * a.q_stride + ((size_t)(head * a.G + c % GP) * D + e0) * 2);
  }
  AttState<D> st;
  st.m = kLeast;
  st.z = 0.f;
#pragma unroll
  for (int j = 0; j < PE; ++j) st.acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  attend_units<D, GP, FP8>(st, qp, a, table, head, u0, u1, len);

  const float z = group_sum(st.z);  // the four lane groups saw different keys of the same head
  if (lane < GP) {
    red_m[lane] = st.m;
    red_z[lane] = z;
  }
  // product row R = 4 grp + r is part R / GP of head R % GP (parts past the second repeat): the two parts are summed
#pragma unroll
  for (int j = 0; j < PE; ++j) {
    float* dst = &red_o[0][PE * c + j];
    if constexpr (GP == 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) dst[(4 * grp + i) * D] = st.acc[j][i];
    } else if constexpr (GP == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.acc[j][i]), __float_as_uint(st.acc[j][i]), false, false);
        if (grp < 2) dst[(4 * grp + i) * D] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
      }
    } else if constexpr (GP == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(st.acc[j][i]), __float_as_uint(st.acc[j][i]), false, false);
        if (grp == 0) dst[i * D] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < GP; ++i)
        if (grp == 0) dst[i * D] = st.acc[j][i] + st.acc[j][GP + i];
    }
  }
}

// grid: groups_per_cu workgroups for every CU, or fewer (a share of kMinUnits units for each of the most that there can be).
template <typename T, int D, int GP, bool FP8>
__global__ void __launch_bounds__(kAttThreads, (groups_per_cu(sizeof(T), D, GP))) paged_attention_kernel(PagedArgs a) {
  __shared__ float red_o[kAttWaves][GP][D];
  __shared__ float red_m[kAttWaves][GP], red_z[kAttWaves][GP];
  const int id = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto units = [&](int r) { return (row_len(a, r) + kUnit - 1) / kUnit; };
  long long all = 0, shares = 0, beg = 0, end = 0;
  const RowOfUnit at = locate_row(a.R, a.Hkv, units, [&](long long total) {
    all = total;
    shares = min((total + kMinUnits - 1) / kMinUnits, (long long)gridDim.x);
    if (id < shares) {
      beg = total * id / shares;
      end = total * (id + 1) / shares;
    }
    return beg < end ? beg : -1ll;
  });
  int2 cut = make_int2(0, 0);
  if (at.row >= 0) {
    int r = at.row, len = row_len(a, r), n = at.size;
    int head = (int)((beg - at.first) / n), u = (int)((beg - at.first) - (long long)head * n);
    while (true) {
      const int take = (int)min((long long)(n - u), end - beg);
      const bool whole = take == n;
      const int32_t* table = a.table + r * a.table_stride;
      if constexpr (sizeof(T) == 4) attend_f32<D, GP>(a, r, head, table, u, u + take, len, red_o[wave], red_m[wave], red_z[wave]);
      else attend_matrix<D, GP, FP8>(a, r, head, table, u, u + take, len, red_o[wave], red_m[wave], red_z[wave]);
      __syncthreads();
      // a share has at most one piece that goes on from the share before (slot 0) and one that begins here and goes on (1)
      write_piece<T, GP, D>(a, whole, 2 * id + (u == 0 ? 1 : 0), r, head, red_o, red_m, red_z);
      beg += take;
      if (!whole && u == 0) {
        // the last unit's share is the largest s with all * s / shares <= its number
        const long long last = beg + (n - take) - 1;
        cut = make_int2(r * a.Hkv + head, (int)(((last + 1) * shares - 1) / all) - id);
      }
      if (beg >= end) break;
      __syncthreads();
      u = 0;
      if (++head == a.Hkv) {
        head = 0;
        do len = row_len(a, ++r); while (len == 0);   // (beg < end: there is another row with positions)
        n = (len + kUnit - 1) / kUnit;
      }
    }
  }
  if (threadIdx.x == 0) a.cut[id] = cut;
  // rows without positions, dealt to all workgroups
  for (int r = id; r < a.R; r += gridDim.x)
    if (row_len(a, r) == 0)
      for (int i = threadIdx.x; i < a.Hq * D; i += kAttThreads) store_elem(a.out + r * a.out_stride + (size_t)i * sizeof(T), 0.f, T{});
}

// grid (workgroups of the first kernel, G): joins the pieces of the (row, kv head) that share blockIdx.x cuts, one query
// head each.  Four columns per thread, kJoinLanes pieces side by side and eight of each on their way together: a request cut
// into 128 pieces takes two rounds.  768 shares of seven heads, most of them cut in two or three: 4.3 us; three long fp32
// requests cut into 128 pieces per head: 6.7 us (half as many pieces side by side 5.5 and 9.5; one column per thread, two
// pieces side by side 5 and 10).
constexpr int kJoinLanes = 8;
template <typename T, int D>
__global__ void __launch_bounds__(kJoinLanes * D / 4) paged_join_kernel(PagedArgs a) {
  constexpr int Q = D / 4, U = 8;
  __shared__ float4 lds_o[kJoinLanes][Q];
  __shared__ float lds_m[kJoinLanes], lds_z[kJoinLanes];
  const int id = blockIdx.x, h = blockIdx.y, j = threadIdx.x % Q, lane = threadIdx.x / Q;
  const int2 cut = a.cut[id];
  if (cut.y == 0) return;
  const int n = cut.y + 1;   // pieces: slot 1 of share id, slot 0 of the shares behind it
  float mn = kLeast, zs = 0.f;
  float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float4& acc, const float4& x, float c) {
    acc.x = fmaf(x.x, c, acc.x); acc.y = fmaf(x.y, c, acc.y); acc.z = fmaf(x.z, c, acc.z); acc.w = fmaf(x.w, c, acc.w);
  };
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
    const float c0 = __builtin_amdgcn_exp2f(mn - top);
    zs *= c0;
    os.x *= c0; os.y *= c0; os.z *= c0; os.w *= c0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const bool in = s0 + u * kJoinLanes < n;
      const float c = in ? __builtin_amdgcn_exp2f(mz[u].x - top) : 0.f;
      zs = fmaf(in ? mz[u].y : 0.f, c, zs);
      add(os, make_float4(in ? o[u].x : 0.f, in ? o[u].y : 0.f, in ? o[u].z : 0.f, in ? o[u].w : 0.f), c);
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
    const float c = __builtin_amdgcn_exp2f(lds_m[w] - mn);
    zs = fmaf(lds_z[w], c, zs);
    add(os, lds_o[w][j], c);
  }
  const int r = cut.x / a.Hkv, head = cut.x - r * a.Hkv;
  char* dst = a.out + r * a.out_stride + ((size_t)(head * a.G + h) * D + 4 * j) * sizeof(T);
  const float x[4] = {os.x, os.y, os.z, os.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) store_elem(dst + i * sizeof(T), zs == 0.f ? 0.f : x[i] / zs, T{});
}

struct PagedPlan {
  int groups, GP;
  size_t part_bytes, mz_bytes, ws_bytes;
};

static meda_status make_paged_plan(const meda_page_pool* pool, const meda_paged_params* p, PagedPlan* pl) {
  if (!p) return MEDA_ERR_INVALID_ARG;
  meda_status st = check_pool_sizes(pool);
  if (st != MEDA_OK) return st;
  if (p->n_rows < 1 || p->n_q_heads < 1 || p->max_blocks < 1) return MEDA_ERR_INVALID_ARG;
  if (p->q_stride < 0 || p->out_stride < 0 || p->table_stride < 0 || p->len_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (p->n_q_heads % pool->n_kv_heads != 0) return MEDA_ERR_INVALID_ARG;
  if (!(p->softmax_scale >= 0.0f) || !isfinite(p->softmax_scale)) return MEDA_ERR_INVALID_ARG;
  st = check_types(p->dtype, pool->dtype);
  if (st != MEDA_OK) return st;
  const int G = p->n_q_heads / pool->n_kv_heads;
  const int64_t most = (int64_t)p->max_blocks * pool->page_size;
  if (G > kMaxGroup || p->n_rows > 65536 || most > (1 << 29) || most * pool->n_kv_heads > (1ll << 34)) return MEDA_ERR_UNSUPPORTED;
  if ((int64_t)p->n_rows * pool->n_kv_heads > INT32_MAX) return MEDA_ERR_UNSUPPORTED;
  const int elt = dtype_bytes(p->dtype);
  const int64_t row = (int64_t)p->n_q_heads * pool->head_dim, far = 1ll << 40;
  if ((p->q_stride && p->q_stride < row) || (p->out_stride && p->out_stride < row) || (p->table_stride && p->table_stride < p->max_blocks))
    return MEDA_ERR_INVALID_ARG;
  if (p->q_stride * elt % 16 || p->out_stride * elt % 16) return MEDA_ERR_INVALID_ARG;
  if (p->q_stride > far || p->out_stride > far || p->table_stride > far || p->len_stride > far) return MEDA_ERR_UNSUPPORTED;
  const int64_t units = (most + kUnit - 1) / kUnit * pool->n_kv_heads;     // of one row, at most
  pl->GP = G <= 1 ? 1 : (G <= 2 ? 2 : (G <= 4 ? 4 : (G <= 8 ? 8 : 16)));
  const int64_t most_groups = kCus * groups_per_cu(elt, pool->head_dim, pl->GP);
  const int64_t shares = units > most_groups * kMinUnits ? most_groups : (units * p->n_rows + kMinUnits - 1) / kMinUnits;
  pl->groups = (int)(shares < most_groups ? shares : most_groups);
  pl->part_bytes = ((size_t)2 * pl->groups * G * pool->head_dim * sizeof(float) + 255) / 256 * 256;
  pl->mz_bytes = ((size_t)2 * pl->groups * G * sizeof(float2) + 255) / 256 * 256;
  pl->ws_bytes = pl->part_bytes + pl->mz_bytes + ((size_t)pl->groups * sizeof(int2) + 255) / 256 * 256;
  return MEDA_OK;
}

template <typename T, int D, int GP, bool FP8>
static hipError_t launch_paged(const PagedPlan& pl, const PagedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((paged_attention_kernel<T, D, GP, FP8>), dim3(pl.groups), dim3(kAttThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(pl.groups, a.G), dim3(kJoinLanes * D / 4), 0, s, a);
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
  const double scale = p.softmax_scale > 0.0f ? (double)p.softmax_scale : 1.0 / sqrt((double)pool->head_dim);
  a.scale_log2 = (float)(scale * 1.4426950408889634074);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool wide = pool->head_dim == 128;
  hipError_t e;
  if (pool->dtype == MEDA_F32) e = wide ? launch_paged_g<float, 128, false>(pl, a, s) : launch_paged_g<float, 64, false>(pl, a, s);
  else if (pool->dtype == MEDA_BF16) e = wide ? launch_paged_g<bf16_t, 128, false>(pl, a, s) : launch_paged_g<bf16_t, 64, false>(pl, a, s);
  else e = wide ? launch_paged_g<bf16_t, 128, true>(pl, a, s) : launch_paged_g<bf16_t, 64, true>(pl, a, s);
  return e == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

}  // extern "C"
