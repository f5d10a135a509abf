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

// A number that is the same in every lane, as a value the compiler knows to be uniform.
__device__ __forceinline__ long long uniform(long long v) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
  return (long long)(((unsigned long long)hi << 32) | lo);
}

struct RowOfUnit {
  int row;          // -1: no unit at all
  int size;         // units of the row, per head
  long long first;  // number of the row's first unit
};

// Rows 0 .. R-1 of units(r) >= 0 units in each of Hkv heads, numbered row after row and head after head: finds the row of
// unit number pick(total), as the same value in every thread of a workgroup of kLocateThreads.  pick sees the total and must
// give a number below it, or a negative one for nothing.
//
// Up to 64 rows: every wave searches on its own, a lane per row (all workgroups of a launch begin with this, and the data's
// latency is all it should cost).  More: every thread adds up the same number of consecutive rows, with two barriers.
template <typename Units, typename Pick>
__device__ __forceinline__ RowOfUnit locate_row(int R, int Hkv, Units units, Pick pick) {
  const int lane = threadIdx.x & 63;
  if (R <= 64) {
    const int mine = lane < R ? units(lane) : 0;
    // (64 rows of at most 2^25 units each: the sum fits 32 bits)
    const unsigned end = (unsigned)wave_inclusive_sum(mine);
    const long long total = (long long)(unsigned)__builtin_amdgcn_readlane((int)end, 63) * Hkv;
    const long long unit = pick(total);
    RowOfUnit out{-1, 0, 0};
    const unsigned long long b = __ballot(unit >= (long long)(end - (unsigned)mine) * Hkv && unit < (long long)end * Hkv);
    if (unit >= 0 && b != 0ull) {
      out.row = __ffsll(b) - 1;
      out.size = __builtin_amdgcn_readlane(mine, out.row);
      out.first = (long long)(unsigned)__builtin_amdgcn_readlane((int)(end - (unsigned)mine), out.row) * Hkv;
    }
    return out;
  }
  __shared__ long long sums[kLocateThreads / 64];
  __shared__ RowOfUnit found;
  const int wave = threadIdx.x >> 6;
  const int per = (R + kLocateThreads - 1) / kLocateThreads;
  const int r0 = min((int)threadIdx.x * per, R), r1 = min(r0 + per, R);
  long long mine = 0;
  for (int r = r0; r < r1; ++r) mine += units(r);
  long long end = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long up = __shfl_up(end, o, kWave);
    if (lane >= o) end += up;
  }
  if (lane == 63) sums[wave] = end;
  if (threadIdx.x == 0) found = RowOfUnit{-1, 0, 0};
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < kLocateThreads / 64; ++w) {
    end += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  const long long unit = pick(uniform(total) * Hkv);
  if (unit >= (end - mine) * Hkv && unit < end * Hkv) {
    long long at = end - mine;
    for (int r = r0; r < r1; ++r) {
      const int n = units(r);
      if (unit < (at + n) * Hkv) {
        found = RowOfUnit{r, n, at * Hkv};
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  RowOfUnit out;
  out.row = __builtin_amdgcn_readfirstlane(found.row);
  out.size = __builtin_amdgcn_readfirstlane(found.size);
  out.first = uniform(found.first);
  return out;
}

}  // namespace meda
