// What the kernels over a paged cache share: the pool as kernels see it, its checks on the host, and the search for the
// row that a unit of work belongs to.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/meda.h"
#include "decode_common.hpp"

namespace meda {

struct Pool {
  char* k;
  char* v;
  float* ks;            // scales of 8-bit rows, [n_pages][Hkv][page_size]
  float* vs;
  size_t page_bytes;    // from one page to the next
  int n_pages, Hkv;
  int page_log2;        // page_size = 1 << page_log2 >= 16: a block of 16 positions lies in one page
};

static inline bool valid_page_size(int p) { return p == 16 || p == 32 || p == 64 || p == 128 || p == 256; }

static inline int dtype_bytes(int dtype) { return dtype == MEDA_F32 ? 4 : (dtype == MEDA_BF16 ? 2 : 1); }

// The sizes of a pool (its pointers are looked at by read_pool).
static inline meda_status check_pool_sizes(const meda_page_pool* p) {
  if (!p || p->n_pages < 1 || p->n_kv_heads < 1 || p->page_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (p->n_pages > INT32_MAX || p->n_kv_heads > 65535) return MEDA_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return MEDA_ERR_UNSUPPORTED;
  if (!valid_page_size(p->page_size)) return MEDA_ERR_UNSUPPORTED;
  if (p->dtype != MEDA_F32 && p->dtype != MEDA_BF16 && p->dtype != MEDA_E4M3) return MEDA_ERR_UNSUPPORTED;
  const int64_t page = (int64_t)p->n_kv_heads * p->page_size * p->head_dim;
  if (p->page_stride != 0) {
    if (p->page_stride < page || p->page_stride % (16 / dtype_bytes(p->dtype)) != 0) return MEDA_ERR_INVALID_ARG;
    if (p->page_stride > (1ll << 40)) return MEDA_ERR_UNSUPPORTED;
  }
  return MEDA_OK;
}

static inline meda_status read_pool(const meda_page_pool* p, Pool* out) {
  const meda_status st = check_pool_sizes(p);
  if (st != MEDA_OK) return st;
  if (!p->k_pages || !p->v_pages || (((uintptr_t)p->k_pages | (uintptr_t)p->v_pages) & 15u)) return MEDA_ERR_INVALID_ARG;
  const bool codes = p->dtype == MEDA_E4M3;
  if (codes && (!p->k_scales || !p->v_scales || (((uintptr_t)p->k_scales | (uintptr_t)p->v_scales) & 3u)))
    return MEDA_ERR_INVALID_ARG;
  out->k = static_cast<char*>(p->k_pages);
  out->v = static_cast<char*>(p->v_pages);
  out->ks = codes ? p->k_scales : nullptr;
  out->vs = codes ? p->v_scales : nullptr;
  const int64_t page = (int64_t)p->n_kv_heads * p->page_size * p->head_dim;
  out->page_bytes = (size_t)(p->page_stride ? p->page_stride : page) * dtype_bytes(p->dtype);
  out->n_pages = (int)p->n_pages;
  out->Hkv = p->n_kv_heads;
  out->page_log2 = __builtin_ctz((unsigned)p->page_size);
  return MEDA_OK;
}

// q, k, v of `dtype` beside pages of pool type: fp32 with fp32, bf16 with bf16 and 8 bits.
static inline meda_status check_types(int dtype, int pool_dtype) {
  if (dtype != MEDA_F32 && dtype != MEDA_BF16) return MEDA_ERR_UNSUPPORTED;
  return (dtype == MEDA_F32) == (pool_dtype == MEDA_F32) ? MEDA_OK : MEDA_ERR_UNSUPPORTED;
}

// ---- which row a unit of work belongs to ---------------------------------------------------------------------------

constexpr int kLocateThreads = 256;

// `total` units in `shares` contiguous shares of total / shares or one more: the first unit of share `id`, and the share of a
// unit.  (Numbers of units are 32-bit: the host refuses sizes that could have 2^31 of them.)
struct Shares {
  unsigned each, more;   // units of a share; the number of shares, the first ones, that have one more
  __device__ __forceinline__ Shares(unsigned total, unsigned shares) {
    each = total / shares;
    more = total - each * shares;
  }
  __device__ __forceinline__ unsigned first(unsigned id) const { return each * id + min(id, more); }
  __device__ __forceinline__ unsigned share_of(unsigned unit) const {   // (each >= 1)
    const unsigned border = (each + 1) * more;
    const bool low = unit < border;
    return (low ? unit : unit - border) / (low ? each + 1 : each) + (low ? 0u : more);
  }
};
// Rows of at most `positions` positions in units of `unit` of them: whether all units together have 32-bit numbers.
static inline bool few_units(int64_t rows, int64_t positions, int64_t heads, int64_t unit) {
  const int64_t each = (positions + unit - 1) / unit * heads;
  return each <= INT32_MAX && rows * each <= INT32_MAX;
}

struct RowOfUnit {
  int row;          // -1: no unit at all
  int size;         // units of the row, per head
  unsigned first;   // number of the row's first unit
};

// Rows 0 .. R-1 of units(r) >= 0 units in each of Hkv heads, numbered row after row and head after head: finds for every
// wave of a workgroup of kLocateThreads the row of unit number pick(wave), as the same value in all its lanes.  begin(total)
// is called once before; a number that is no unit's is that of nothing.
//
// Up to 64 rows: every wave searches on its own, a lane per row (all workgroups of a launch begin with this, and the data's
// latency is all it should cost).  More: every thread adds up the same number of consecutive rows, with two barriers.
template <typename Units, typename Begin, typename Pick>
__device__ __forceinline__ RowOfUnit locate_row(int R, unsigned Hkv, Units units, Begin begin, Pick pick) {
  constexpr int kWaves = kLocateThreads / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (R <= 64) {
    const unsigned mine = lane < R ? (unsigned)units(lane) : 0u;
    const unsigned end = (unsigned)wave_inclusive_sum((int)mine);
    begin((unsigned)__builtin_amdgcn_readlane((int)end, 63) * Hkv);
    const unsigned unit = pick(wave);
    const unsigned long long b = __ballot(unit >= (end - mine) * Hkv && unit < end * Hkv);
    RowOfUnit out{-1, 0, 0};
    if (b != 0ull) {
      out.row = __ffsll(b) - 1;
      out.size = __builtin_amdgcn_readlane((int)mine, out.row);
      out.first = (unsigned)__builtin_amdgcn_readlane((int)(end - mine), out.row) * Hkv;
    }
    return out;
  }
  __shared__ unsigned sums[kWaves];
  __shared__ RowOfUnit found[kWaves];
  constexpr int kKept = 8;   // rows of a thread that are kept in registers: loaded together, and once
  const int per = (R + kLocateThreads - 1) / kLocateThreads;
  const int r0 = min((int)threadIdx.x * per, R), r1 = min(r0 + per, R);
  unsigned mine = 0;
  int kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) {
    kept[i] = r0 + i < r1 ? units(r0 + i) : 0;
    mine += (unsigned)kept[i];
  }
#pragma unroll 4
  for (int r = r0 + kKept; r < r1; ++r) mine += (unsigned)units(r);
  unsigned end = (unsigned)wave_inclusive_sum((int)mine);
  if (lane == 63) sums[wave] = end;
  if (threadIdx.x < kWaves) found[threadIdx.x] = RowOfUnit{-1, 0, 0};
  __syncthreads();
  unsigned total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    end += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  begin((unsigned)__builtin_amdgcn_readfirstlane((int)total) * Hkv);
#pragma unroll 1
  for (int w = 0; w < kWaves; ++w) {
    const unsigned unit = pick(w);
    if (unit >= (end - mine) * Hkv && unit < end * Hkv) {
      unsigned at = end - mine;
      RowOfUnit hit{-1, 0, 0};
#pragma unroll
      for (int i = 0; i < kKept; ++i) {
        if (hit.row < 0 && unit < (at + kept[i]) * Hkv) hit = RowOfUnit{r0 + i, kept[i], at * Hkv};
        at += kept[i];
      }
#pragma unroll 1
      for (int r = r0 + kKept; r < r1 && hit.row < 0; ++r) {
        const int n = units(r);
        if (unit < (at + n) * Hkv) hit = RowOfUnit{r, n, at * Hkv};
        at += n;
      }
      found[w] = hit;
    }
  }
  __syncthreads();
  RowOfUnit out;
  out.row = __builtin_amdgcn_readfirstlane(found[wave].row);
  out.size = __builtin_amdgcn_readfirstlane(found[wave].size);
  out.first = (unsigned)__builtin_amdgcn_readfirstlane((int)found[wave].first);
  return out;
}

}  // namespace meda
