// Rotary positions of queries and keys, and the step that writes new tokens into the pages of a cache.
//
// Both stream rows once: a row is held by LPR = row bytes / 16 lanes, which exchange the halves of the pairs among
// themselves, so that an output may be its own input.  The angles depend on the token alone: a workgroup takes
// 4 * 64 / LPR tokens, its threads compute the sines of their pairs once, into LDS, and every wave walks over heads with the
// factors of its tokens in registers, kAhead rows per lane on their way together.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/meda.h"
#include "paged.hpp"
#include "rotary.hpp"

namespace meda {

struct Rows {
  const char* in;
  char* out;
  long long in_token, in_head, out_token, out_head;   // bytes
  int heads;
};

struct RotaryArgs {
  RotaryPlan plan;
  Rows q, k;
  const char* v;                 // append: [tokens][Hkv]
  long long v_token, v_head;
  const int64_t* slots;
  long long slot_stride;
  Pool pool;
  long long tokens;
  int heads_per_part;
};

enum RotaryTo { kToRows, kToPages, kToCodes };   // k: strided rows, pages of the same type, 8-bit pages (k and v)

constexpr int kAhead = 4;

// grid (token groups, parts of the heads), 256 threads: 4 * 64 / LPR tokens, heads_per_part of the Hq + Hk (+ Hkv) heads.
// STREAM: rows are written past the caches.
template <typename T, int D, RotaryTo TO, bool STREAM>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a) {
  using RP = RowPiece<T>;
  constexpr int E = RP::kElems, LPR = D / E, TPW = 64 / LPR;
  __shared__ float exchange[4][TPW][D];            // first the pairs of the workgroup's tokens, as float2 [4 * TPW][D / 2]
  float2* pairs = reinterpret_cast<float2*>(&exchange[0][0][0]);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / LPR, cc = lane - sub * LPR;
  const long long token0 = (long long)blockIdx.x * (4 * TPW), token = token0 + wave * TPW + sub;
  const bool live = token < a.tokens;
  const long long t = live ? token : a.tokens - 1;   // lanes past the end repeat the last token and store nothing

  const int nq = a.q.heads, nk = a.k.heads, nv = TO == kToRows ? 0 : a.pool.Hkv;
  const int h0 = blockIdx.y * a.heads_per_part, h1 = min(h0 + a.heads_per_part, nq + nk + nv);
  auto fetch = [&](uint4 (&raw)[kAhead], int h) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int x = min(h + u, h1 - 1);
      const char* src = x < nq ? a.q.in + t * a.q.in_token + x * a.q.in_head
                               : (x < nq + nk ? a.k.in + t * a.k.in_token + (x - nq) * a.k.in_head
                                              : a.v + t * a.v_token + (x - nq - nk) * a.v_head);
      raw[u] = load16_stream(src + cc * 16);
    }
  };
  uint4 raw[kAhead];
  fetch(raw, h0);

  float c[E], s[E];
  if (a.plan.half > 0) {
    for (int i = threadIdx.x; i < 4 * TPW * a.plan.half; i += 256) {
      const int x = i / a.plan.half, pair = i - x * a.plan.half;
      pairs[x * (D / 2) + pair] = rotary_pair(a.plan, min(token0 + x, a.tokens - 1), pair);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < E; ++i) rotary_factors(a.plan, pairs + (wave * TPW + sub) * (D / 2), cc * E + i, c[i], s[i]);
    __syncthreads();   // the exchange below uses the same memory
  }

  // where the token's rows go in the pages
  size_t place = 0, scale_place = 0;
  bool slot_ok = false;
  constexpr int kOut = TO == kToCodes ? 1 : (int)sizeof(T);
  if constexpr (TO != kToRows) {
    const long long slot = a.slots[t * a.slot_stride], page = slot >> a.pool.page_log2;
    slot_ok = live && slot >= 0 && page < a.pool.n_pages;
    const long long at = slot & ((1ll << a.pool.page_log2) - 1);
    if (slot_ok) {
      place = (size_t)page * a.pool.page_bytes + (size_t)at * D * kOut;
      scale_place = ((size_t)page * a.pool.Hkv << a.pool.page_log2) + (size_t)at;
    }
  }

  auto finish = [&](const uint4& x, int h) {
    const bool is_q = h < nq, is_v = h >= nq + nk;
    const int g = is_q ? h : (is_v ? h - nq - nk : h - nq);
    const bool turned = !is_v && a.plan.half > 0;
    float f[E];
    uint4 y = x;
    if (turned) {
      rotary_turn<T, LPR>(a.plan, cc, x, c, s, f, exchange[wave][sub]);
      if (TO != kToCodes || is_q) y = pack_row(f);
    }
    if (TO == kToRows || is_q) {
      const Rows& to = is_q ? a.q : a.k;
      char* dst = to.out + t * to.out_token + g * to.out_head + cc * 16;
      if (live) {
        if constexpr (STREAM) store16_stream(dst, y);
        else *reinterpret_cast<uint4*>(dst) = y;
      }
    } else {
      char* pages = is_v ? a.pool.v : a.pool.k;
      const size_t row = place + ((size_t)g << a.pool.page_log2) * (D * kOut);
      if constexpr (TO == kToPages) {
        if (slot_ok) *reinterpret_cast<uint4*>(pages + row + cc * 16) = y;
      } else {
        uint32_t w[E / 4];
        if (!turned) RP::unpack(x, f);
        const float scale = quantize_row<E, LPR>(f, w);
        if (slot_ok) {
          if constexpr (E == 8) *reinterpret_cast<uint2*>(pages + row + cc * 8) = make_uint2(w[0], w[1]);
          else *reinterpret_cast<uint32_t*>(pages + row + cc * 4) = w[0];
          if (cc == 0) (is_v ? a.pool.vs : a.pool.ks)[scale_place + ((size_t)g << a.pool.page_log2)] = scale;
        }
      }
    }
  };
  for (int h = h0; h < h1; h += kAhead) {
    uint4 now[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) now[u] = raw[u];
    if (h + kAhead < h1) fetch(raw, h + kAhead);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (h + u < h1) finish(now[u], h + u);
  }
}

template <typename T, int D, RotaryTo TO>
static hipError_t launch_rotary(RotaryArgs a, hipStream_t s) {
  constexpr int TPB = 4 * 64 / (D / RowPiece<T>::kElems);
  const int heads = a.q.heads + a.k.heads + (TO == kToRows ? 0 : a.pool.Hkv);
  const long long groups = (a.tokens + TPB - 1) / TPB;
  // The heads are dealt to several workgroups where there are few, but every part computes the sines of its tokens again: parts
  // of 12 heads or more, and of fewer only where CUs would have nothing to do.  (4001 tokens, 48 heads to 8 bits: 36, 29, 27 us
  // with parts of 3, 6 and 12 heads; 4095 tokens, 40 fp32 heads: 34, 31, 32 with 5, 10 and 20; 37376 tokens, 32 heads: 123 and
  // 128 with 16 and 32.)
  const long long many = (4096 + groups - 1) / groups, some = (heads + 11) / 12, least = (512 + groups - 1) / groups;
  long long parts = some > least ? some : least;
  if (parts > many) parts = many;
  if (parts > heads) parts = heads;
  a.heads_per_part = (int)((heads + parts - 1) / parts);
  const unsigned n_parts = (unsigned)((heads + a.heads_per_part - 1) / a.heads_per_part);
  const dim3 grid((unsigned)groups, n_parts), block(256);
  // Rows that fit the 256 MB of the last-level cache stay there for whoever reads them next; others are gone before that, and go
  // past the caches.  (Bytes written, us with ordinary stores and past the caches, bf16 / fp32: 64 MB 29 and 30 / 27 and 28, 128 MB
  // 59 and 56 / 57 and 53, 256 MB 111 and 101 / 113 and 106, 320 MB 137 and 125 / 137 and 127, 640 MB 271 and 253 / 271 and 254,
  // 1600 MB 654 and 602 / 671 and 631.)
  if constexpr (TO == kToRows) {
    if (a.tokens * heads * D * (long long)sizeof(T) >= (256ll << 20)) {
      hipLaunchKernelGGL((rotary_kernel<T, D, TO, true>), grid, block, 0, s, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((rotary_kernel<T, D, TO, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

static meda_status check_rotation(int rot_dim, int d, int n_axes, int flags, int allowed) {
  if (rot_dim < 0 || rot_dim > d || (rot_dim & 1) || (flags & ~allowed)) return MEDA_ERR_INVALID_ARG;
  if (rot_dim > 0 && (n_axes < 1 || n_axes > 4)) return MEDA_ERR_INVALID_ARG;
  return MEDA_OK;
}

static meda_status make_rotation(RotaryPlan* out, const int32_t* positions, const double* inv_freq, const uint8_t* axis,
                                 int rot_dim, int n_axes, int64_t pos_stride, int64_t n_tokens, int flags) {
  *out = RotaryPlan{positions, inv_freq, axis, pos_stride ? pos_stride : n_tokens, rot_dim / 2, n_axes,
                    (flags & MEDA_ROTARY_INTERLEAVED) ? 1 : 0, (flags & MEDA_ROTARY_INVERSE) ? -1.f : 1.f};
  if (rot_dim == 0) return MEDA_OK;
  if (!positions || !inv_freq || (!axis && n_axes > 1) || pos_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (pos_stride > (1ll << 40)) return MEDA_ERR_UNSUPPORTED;
  if (((uintptr_t)positions & 3u) || ((uintptr_t)inv_freq & 7u)) return MEDA_ERR_INVALID_ARG;
  return MEDA_OK;
}

// Rows of d elements by strides, in elements; false where they cannot be moved in 16-byte pieces or where rows that are
// written share memory.
static bool make_rows(Rows* r, const void* in, void* out, const int64_t* in_stride, const int64_t* out_stride, int64_t tokens, int heads,
                      int d, int elt) {
  const int64_t most = 1ll << 40;
  for (int i = 0; i < 2; ++i) {
    if (in_stride[i] < 0 || in_stride[i] > most || (in_stride[i] * elt) % 16) return false;
    if (out && (out_stride[i] < 0 || out_stride[i] > most || (out_stride[i] * elt) % 16)) return false;
  }
  if (out) {
    // the dimension with the shorter stride lies inside a step of the other one
    const int in_dim = heads > 1 && (tokens <= 1 || out_stride[1] < out_stride[0]) ? 1 : 0;
    const int64_t n[2] = {tokens, heads}, inner = n[in_dim] > 1 ? out_stride[in_dim] : d, outer = n[1 - in_dim] > 1 ? out_stride[1 - in_dim] : most;
    if (inner < d || (double)(n[in_dim] - 1) * (double)inner + d > (double)outer) return false;
  }
  *r = Rows{static_cast<const char*>(in), static_cast<char*>(out), in_stride[0] * elt, in_stride[1] * elt,
            out ? out_stride[0] * elt : 0, out ? out_stride[1] * elt : 0, heads};
  return in && !((uintptr_t)in & 15u) && !((uintptr_t)out & 15u);
}

template <RotaryTo TO>
static hipError_t launch_rotary_of(int dtype, int d, const RotaryArgs& a, hipStream_t s) {
  if constexpr (TO != kToCodes) {
    if (dtype == MEDA_F32) return d == 128 ? launch_rotary<float, 128, TO>(a, s) : launch_rotary<float, 64, TO>(a, s);
  }
  return d == 128 ? launch_rotary<bf16_t, 128, TO>(a, s) : launch_rotary<bf16_t, 64, TO>(a, s);
}

}  // namespace meda

extern "C" {

meda_status meda_rotary(const meda_rotary_params* params, const void* q, const void* k, const int32_t* positions,
                        const double* inv_freq, const uint8_t* axis, void* q_out, void* k_out, void* hip_stream) {
  using namespace meda;
  if (!params) return MEDA_ERR_INVALID_ARG;
  const meda_rotary_params& p = *params;
  if (p.n_tokens < 0 || p.n_q_heads < 0 || p.n_k_heads < 0) return MEDA_ERR_INVALID_ARG;
  if (p.dtype != MEDA_F32 && p.dtype != MEDA_BF16) return MEDA_ERR_UNSUPPORTED;
  if (p.head_dim != 64 && p.head_dim != 128) return MEDA_ERR_UNSUPPORTED;
  if ((int64_t)p.n_q_heads + p.n_k_heads > 65535 || p.n_tokens > (1ll << 26)) return MEDA_ERR_UNSUPPORTED;
  const meda_status st = check_rotation(p.rot_dim, p.head_dim, p.n_axes, p.flags, MEDA_ROTARY_INTERLEAVED | MEDA_ROTARY_INVERSE);
  if (st != MEDA_OK) return st;
  if (p.rot_dim == 0) return MEDA_ERR_INVALID_ARG;
  if (p.n_tokens == 0 || p.n_q_heads + p.n_k_heads == 0) return MEDA_OK;
  RotaryArgs a{};
  const meda_status sr = make_rotation(&a.plan, positions, inv_freq, axis, p.rot_dim, p.n_axes, p.pos_stride, p.n_tokens, p.flags);
  if (sr != MEDA_OK) return sr;
  const int elt = dtype_bytes(p.dtype), d = p.head_dim;
  if (p.n_q_heads > 0 && (!q_out || !make_rows(&a.q, q, q_out, p.q_stride, p.q_out_stride, p.n_tokens, p.n_q_heads, d, elt))) return MEDA_ERR_INVALID_ARG;
  if (p.n_k_heads > 0 && (!k_out || !make_rows(&a.k, k, k_out, p.k_stride, p.k_out_stride, p.n_tokens, p.n_k_heads, d, elt))) return MEDA_ERR_INVALID_ARG;
  a.tokens = p.n_tokens;
  const hipError_t e = launch_rotary_of<kToRows>(p.dtype, p.head_dim, a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

meda_status meda_paged_append(const meda_page_pool* pool, const meda_append_params* params, const void* q, const void* k,
                              const void* v, const int32_t* positions, const double* inv_freq, const uint8_t* axis,
                              const int64_t* slots, void* q_out, void* hip_stream) {
  using namespace meda;
  if (!params) return MEDA_ERR_INVALID_ARG;
  const meda_append_params& p = *params;
  RotaryArgs a{};
  const meda_status sp = read_pool(pool, &a.pool);
  if (sp != MEDA_OK) return sp;
  if (p.n_tokens < 0 || p.n_q_heads < 0 || p.slot_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (p.slot_stride > (1ll << 40)) return MEDA_ERR_UNSUPPORTED;
  meda_status st = check_types(p.dtype, pool->dtype);
  if (st != MEDA_OK) return st;
  if ((int64_t)p.n_q_heads + 2ll * pool->n_kv_heads > 131070 || p.n_q_heads > 65535 || p.n_tokens > (1ll << 26)) return MEDA_ERR_UNSUPPORTED;
  st = check_rotation(p.rot_dim, pool->head_dim, p.n_axes, p.flags, MEDA_ROTARY_INTERLEAVED);
  if (st != MEDA_OK) return st;
  if (p.n_tokens == 0) return MEDA_OK;
  st = make_rotation(&a.plan, positions, inv_freq, axis, p.rot_dim, p.n_axes, p.pos_stride, p.n_tokens, p.flags);
  if (st != MEDA_OK) return st;
  const int elt = dtype_bytes(p.dtype), d = pool->head_dim;
  Rows v_rows{};
  const int64_t none[2] = {0, 0};
  if (p.n_q_heads > 0 && (!q_out || !make_rows(&a.q, q, q_out, p.q_stride, p.q_out_stride, p.n_tokens, p.n_q_heads, d, elt))) return MEDA_ERR_INVALID_ARG;
  if (!make_rows(&a.k, k, nullptr, p.k_stride, none, p.n_tokens, pool->n_kv_heads, d, elt)) return MEDA_ERR_INVALID_ARG;
  if (!make_rows(&v_rows, v, nullptr, p.v_stride, none, p.n_tokens, pool->n_kv_heads, d, elt)) return MEDA_ERR_INVALID_ARG;
  if (!slots || ((uintptr_t)slots & 7u)) return MEDA_ERR_INVALID_ARG;
  a.v = v_rows.in; a.v_token = v_rows.in_token; a.v_head = v_rows.in_head;
  a.slots = slots;
  a.slot_stride = p.slot_stride ? p.slot_stride : 1;
  a.tokens = p.n_tokens;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = pool->dtype == MEDA_E4M3 ? launch_rotary_of<kToCodes>(p.dtype, pool->head_dim, a, s)
                                               : launch_rotary_of<kToPages>(p.dtype, pool->head_dim, a, s);
  return e == hipSuccess ? MEDA_OK : MEDA_ERR_HIP;
}

}  // extern "C"
