// The ragged compressed caches of a call move to the pages of a pool, as they are or in 8 bits.
//
// A (row, kv head) of the ragged cache and one of its pages are both contiguous, so the move is a copy of runs of up to
// page_size rows.  The work is numbered in pieces of 16 rows, row after row and head after head, and cut evenly over the
// workgroups: a piece lies in one page whatever the page size, and the budgets of the layers, which differ by more than a
// factor of ten, do not matter.  Bound by HBM: every row is read once and written once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/meda.h"
#include "paged.hpp"
#include "row_codec.hpp"

namespace meda {

struct StoreArgs {
  Pool pool;
  const char* k;                // ragged rows
  const char* v;
  const int32_t* layer_len;     // [N*L]
  const int64_t* layer_off;     // [N][L+1]
  const int32_t* lens;
  const int32_t* table;
  long long n_src_rows, table_stride, len_stride;
  int R, L, max_blocks;
};

constexpr int kPiece = 16;      // rows

__device__ __forceinline__ void store8_stream(void* p, const uint2& v) {  // see store16_stream
  typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
  const u32x2_t t = {v.x, v.y};
  __builtin_nontemporal_store(t, reinterpret_cast<u32x2_t*>(p));
}

// rows of row r that are stored, per kv head
__device__ __forceinline__ int stored_rows(const StoreArgs& a, int r) {
  const int most = a.max_blocks << a.pool.page_log2;
  return max(0, min(min(a.layer_len[r], a.lens[r * a.len_stride]), most));
}

// grid: any number of workgroups of 256 threads; each takes a contiguous share of the pieces, its waves every fourth one.
template <typename T, int D, bool CODES>
__global__ void __launch_bounds__(kLocateThreads) paged_store_kernel(StoreArgs a) {
  using RP = RowPiece<T>;
  constexpr int E = RP::kElems, LPR = D / E, RPW = 64 / LPR, U = kPiece / RPW;   // rows per load, loads per piece
  constexpr int kOut = CODES ? 1 : (int)sizeof(T);
  const int lane = threadIdx.x & 63, sub = lane / LPR, cc = lane - sub * LPR;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto pieces = [&](int r) { return (stored_rows(a, r) + kPiece - 1) / kPiece; };
  unsigned beg = 0, end = 0;
  const RowOfUnit at = locate_row(
      a.R, a.pool.Hkv, pieces,
      [&](unsigned total) {
        const Shares shares(total, gridDim.x);
        beg = shares.first(blockIdx.x);
        end = shares.first(blockIdx.x + 1);
      },
      [&](int w) { return beg + w < end ? beg + w : ~0u; });
  if (at.row < 0) return;
  int r = at.row;
  unsigned first = at.first;                  // number of row r's first piece
  int rows = stored_rows(a, r), per_head = at.size;
  for (unsigned u = beg + wave; u < end; u += kLocateThreads / 64) {
    while (u >= first + (unsigned)per_head * a.pool.Hkv) {   // (u < end: there is such a row)
      first += (unsigned)per_head * a.pool.Hkv;
      ++r;
      rows = stored_rows(a, r);
      per_head = (rows + kPiece - 1) / kPiece;
    }
    const int local = (int)(u - first), g = local / per_head, i0 = (local - g * per_head) * kPiece;
    const int page = a.table[r * a.table_stride + (i0 >> a.pool.page_log2)];
    if (page < 0 || page >= a.pool.n_pages) continue;
    const int seq = r / a.L;
    const long long off = a.layer_off[(long long)seq * (a.L + 1) + (r - seq * a.L)];
    const long long src0 = off * a.pool.Hkv + (long long)g * a.layer_len[r] + i0;
    const long long left = a.n_src_rows - src0;
    const int n = (int)(off < 0 || off > a.n_src_rows ? 0 : min((long long)min(rows - i0, kPiece), left));   // rows of this piece
    if (n <= 0) continue;
    const size_t in_page = ((size_t)g << a.pool.page_log2) + (i0 & ((1 << a.pool.page_log2) - 1));
    const size_t dst0 = (size_t)page * a.pool.page_bytes + in_page * (D * kOut);
    const size_t scale0 = ((size_t)page * a.pool.Hkv << a.pool.page_log2) + in_page;
    uint4 x[2][U];
#pragma unroll
    for (int w = 0; w < U; ++w) {
      const size_t o = ((size_t)src0 + min(w * RPW + sub, n - 1)) * (D * sizeof(T)) + cc * 16;
      x[0][w] = load16_stream(a.k + o);
      x[1][w] = load16_stream(a.v + o);
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      char* dst = (kv ? a.pool.v : a.pool.k) + dst0;
#pragma unroll
      for (int w = 0; w < U; ++w) {
        const int i = w * RPW + sub;
        if constexpr (!CODES) {
          if (i < n) store16_stream(dst + (size_t)i * (D * kOut) + cc * 16, x[kv][w]);
        } else {
          float f[E];
          uint32_t c[E / 4];
          RP::unpack(x[kv][w], f);
          const float scale = quantize_row<E, LPR>(f, c);
          if (i < n) {
            if constexpr (E == 8) store8_stream(dst + (size_t)i * D + cc * 8, make_uint2(c[0], c[1]));
            else *reinterpret_cast<uint32_t*>(dst + (size_t)i * D + cc * 4) = c[0];
            if (cc == 0) (kv ? a.pool.vs : a.pool.ks)[scale0 + i] = scale;
          }
        }
      }
    }
  }
}

template <typename T, int D, bool CODES>
static hipError_t launch_store(const StoreArgs& a, hipStream_t s) {
  // A workgroup for every four pieces that the source rows can make, whole ones and a last one of every (row, head): a piece per
  // wave.  (Few workgroups that walk over many pieces wait for page numbers and offsets in every step: 57 MB of 32 short layers
  // 23 us with 16 pieces per workgroup, 13.6 with four; 596 MB 124 and 111, 1968 MB to 8 bits 399 with at most 4096 workgroups
  // and 362 with all of them.  90 layers of one or two positions in 16 heads 25 us without the last pieces counted, 9 with them.)
  long long groups = (a.n_src_rows / kPiece + (long long)a.R * a.pool.Hkv + 3) / 4;
  if (groups > 1 << 22) groups = 1 << 22;   // (every workgroup then takes several)
  hipLaunchKernelGGL((paged_store_kernel<T, D, CODES>), dim3((unsigned)groups), dim3(kLocateThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace meda

extern "C" {

meda_status meda_paged_store(const meda_page_pool* pool, const meda_store_params* params, const void* k_rows,
                             const void* v_rows, const int32_t* layer_len, const int64_t* layer_off, const int32_t* lens,
                             const int32_t* table, void* hip_stream) {
  using namespace meda;
  if (!params) return MEDA_ERR_INVALID_ARG;
  const meda_store_params& p = *params;
  StoreArgs a;
  meda_status st = read_pool(pool, &a.pool);
  if (st != MEDA_OK) return st;
  if (p.n_src_rows < 0 || p.table_stride < 0 || p.len_stride < 0 || p.n_seqs < 1 || p.n_layers < 1 || p.max_blocks < 1) return MEDA_ERR_INVALID_ARG;
  st = check_types(p.dtype, pool->dtype);
  if (st != MEDA_OK) return st;
  if ((int64_t)p.n_seqs * p.n_layers > 65536 || (int64_t)p.max_blocks * pool->page_size > (1 << 29)) return MEDA_ERR_UNSUPPORTED;
  if (!few_units((int64_t)p.n_seqs * p.n_layers, (int64_t)p.max_blocks * pool->page_size, pool->n_kv_heads, kPiece) || p.n_src_rows > (1ll << 40)) return MEDA_ERR_UNSUPPORTED;
  if (p.table_stride && p.table_stride < p.max_blocks) return MEDA_ERR_INVALID_ARG;
  if (p.table_stride > (1ll << 40) || p.len_stride > (1ll << 40)) return MEDA_ERR_UNSUPPORTED;
  if (!k_rows || !v_rows || !layer_len || !layer_off || !lens || !table) return MEDA_ERR_INVALID_ARG;
  if (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15u) return MEDA_ERR_INVALID_ARG;
  if ((((uintptr_t)layer_len | (uintptr_t)lens | (uintptr_t)table) & 3u) || ((uintptr_t)layer_off & 7u)) return MEDA_ERR_INVALID_ARG;
  a.k = static_cast<const char*>(k_rows);
  a.v = static_cast<const char*>(v_rows);
  a.layer_len = layer_len; a.layer_off = layer_off; a.lens = lens; a.table = table;
  a.n_src_rows = p.n_src_rows;
  a.table_stride = p.table_stride ? p.table_stride : p.max_blocks;
  a.len_stride = p.len_stride ? p.len_stride : 1;
  a.R = p.n_seqs * p.n_layers; a.L = p.n_layers; a.max_blocks = p.max_blocks;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (pool->dtype == MEDA_F32) e = pool->head_dim == 128 ? launch_store<float, 128, false>(a, s) : launch_store<float, 64, false>(a, s);
  else if (pool->dtype == MEDA_BF16) e = pool->head_dim == 128 ? launch_store<bf16_t, 128, false>(a, s) : launch_store<bf16_t, 64, false>(a, s);
  else e = pool->head_dim == 128 ? launch_store<bf16_t, 128, true>(a, s) : launch_store<bf16_t, 64, true>(a, s);
  return e == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

}  // extern "C"
