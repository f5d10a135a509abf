// Host-side check of the paged cache's argument validation under sanitizers: random pools and parameters, valid and
// invalid, extreme sizes included.  Nothing is launched: the calls compute sizes only, or lack a pointer.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../include/meda.h"

static uint64_t rng_state = 0x9e3779b97f4a7c15ull;
static uint32_t rnd() { rng_state = rng_state * 6364136223846793005ull + 1442695040888963407ull; return (uint32_t)(rng_state >> 33); }
static int failures = 0;
#define EXPECT(cond) do { if (!(cond)) { fprintf(stderr, "line %d: %s\n", __LINE__, #cond); ++failures; } } while (0)

static bool wild;   // half of the parameter sets: any number; the others: plausible ones
static int32_t pick32(int32_t a, int32_t b, int32_t c) {
  if (!wild) return c;
  switch (rnd() % 8) {
    case 0: return a;
    case 1: return b;
    case 2: return INT32_MAX;
    case 3: return INT32_MIN;
    case 4: return 0;
    default: return c;
  }
}
static int64_t pick64(int64_t c) {
  if (!wild) return c;
  switch (rnd() % 8) {
    case 0: return INT64_MAX;
    case 1: return INT64_MIN;
    case 2: return 1ll << 40;
    case 3: return -1;
    default: return c;
  }
}

int main() {
  int sized = 0;
  void* const p = (void*)0x100000;
  for (int it = 0; it < 300000; ++it) {
    wild = rnd() % 2 != 0;
    meda_page_pool pool;
    memset(&pool, 0, sizeof pool);
    pool.n_pages = pick64(1 + rnd() % 1000000);
    pool.page_stride = rnd() % 2 ? 0 : pick64((int64_t)(rnd() % 64) * 16384);
    pool.n_kv_heads = pick32(65535, 65536, 1 + rnd() % 16);
    pool.head_dim = rnd() % 8 ? 64 + 64 * (rnd() % 2) : (int32_t)rnd();
    pool.page_size = rnd() % 8 ? 16 << (rnd() % 5) : (int32_t)rnd();
    pool.dtype = (int32_t)(rnd() % 4);
    pool.k_pages = p; pool.v_pages = p; pool.k_scales = (float*)p; pool.v_scales = (float*)p;
    meda_paged_params a;
    memset(&a, 0, sizeof a);
    a.n_rows = pick32(65536, 65537, 1 + rnd() % 300);
    a.n_q_heads = pool.n_kv_heads > 0 && pool.n_kv_heads < 70000 ? pool.n_kv_heads * (int32_t)(1 + rnd() % 18) : (int32_t)rnd();
    a.max_blocks = pick32(1 << 20, 1 << 29, 1 + rnd() % 5000);
    a.dtype = wild ? (int32_t)(rnd() % 3) : (pool.dtype == MEDA_F32 ? MEDA_F32 : MEDA_BF16);
    a.q_stride = rnd() % 2 ? 0 : pick64((int64_t)rnd() % 100000);
    a.table_stride = rnd() % 2 ? 0 : pick64((int64_t)rnd() % 100000);
    const size_t need = meda_paged_workspace_bytes(&pool, &a);
    EXPECT(need % 256 == 0 && need < ((size_t)64 << 20));
    sized += need != 0;
    EXPECT(meda_paged_attention(&pool, &a, nullptr, (int32_t*)p, (int32_t*)p, p, p, need, nullptr) != MEDA_OK);
    meda_store_params s;
    memset(&s, 0, sizeof s);
    s.n_src_rows = pick64(rnd()); s.table_stride = a.table_stride; s.n_seqs = a.n_rows; s.n_layers = pick32(1, 65536, 1 + rnd() % 40);
    s.max_blocks = a.max_blocks; s.dtype = a.dtype;
    EXPECT(meda_paged_store(&pool, &s, nullptr, p, (int32_t*)p, (int64_t*)p, (int32_t*)p, (int32_t*)p, nullptr) != MEDA_OK);
    meda_append_params e;
    memset(&e, 0, sizeof e);
    e.n_tokens = pick64(1 + rnd() % 1000); e.n_q_heads = a.n_q_heads; e.dtype = a.dtype; e.rot_dim = (int32_t)(rnd() % 140) - 2; e.n_axes = (int32_t)(rnd() % 6);
    for (int i = 0; i < 2; ++i) {
      e.q_stride[i] = pick64(1024); e.q_out_stride[i] = pick64(1 << (rnd() % 20)); e.k_stride[i] = pick64(128); e.v_stride[i] = pick64(128);
    }
    if (e.n_tokens != 0)
      EXPECT(meda_paged_append(&pool, &e, p, p, p, (int32_t*)p, (double*)p, (uint8_t*)p, nullptr, p, nullptr) != MEDA_OK);
    meda_rotary_params r;
    memset(&r, 0, sizeof r);
    r.n_tokens = e.n_tokens; r.n_q_heads = 1 + (int32_t)(rnd() % 64); r.n_k_heads = pick32(0, 65535, 2); r.head_dim = pool.head_dim; r.rot_dim = e.rot_dim;
    r.n_axes = e.n_axes; r.dtype = a.dtype; r.pos_stride = pick64(0);
    for (int i = 0; i < 2; ++i) { r.q_stride[i] = e.q_stride[i]; r.q_out_stride[i] = e.q_out_stride[i]; }
    if (r.n_tokens != 0) EXPECT(meda_rotary(&r, p, p, (int32_t*)p, nullptr, (uint8_t*)p, p, p, nullptr) != MEDA_OK);
    meda_page_params g;
    memset(&g, 0, sizeof g);
    g.n_pages = pool.n_pages; g.n_rows = a.n_rows; g.max_blocks = a.max_blocks; g.page_size = pool.page_size; g.max_new = pick32(0, 100, 1); g.rows_per_seq = pick32(0, 100, 1);
    EXPECT(meda_page_update(&g, nullptr, (int32_t*)p, (int32_t*)p, (int32_t*)p, (int64_t*)p, (int32_t*)p, (int64_t*)p, (int64_t*)p, nullptr, p, 1 << 24, nullptr) != MEDA_OK);
    EXPECT(meda_page_update_workspace_bytes(g.n_rows) % 256 == 0);
  }
  EXPECT(sized > 1000);
  if (failures) return 1;
  printf("paged sanitizer check ok (%d sizes)\n", sized);
  return 0;
}
