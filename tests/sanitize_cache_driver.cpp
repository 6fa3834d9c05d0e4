// Drives the argument checks of the norm, cache and cached-attention entry points (host code, no GPU work) against a copy of
// the library whose HOST code is compiled with -fsanitize=address,undefined.  Prints "ok" at the end.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "asa.h"

#define EXPECT(c)                                       \
  do {                                                  \
    if (!(c)) {                                         \
      printf("line %d: %s\n", __LINE__, #c);            \
      return 1;                                         \
    }                                                   \
  } while (0)

static asa_params shape(int B, int H, int L, int d, int block) {
  asa_params p;
  memset(&p, 0, sizeof(p));
  p.B = B; p.H = H; p.L = L; p.d = d; p.block = block;
  return p;
}

int main() {
  const int ints[] = {INT_MIN, -1, 0, 1, 2, 63, 64, 128, 65536, 131072, 1 << 30, INT_MAX};
  void *x = reinterpret_cast<void *>(0x10000);      // never dereferenced
  float *f = reinterpret_cast<float *>(0x10000);
  const int32_t *i32 = reinterpret_cast<int32_t *>(0x10000);
  asa_qk_norm n;
  memset(&n, 0, sizeof(n));
  asa_kv_cache c;
  memset(&c, 0, sizeof(c));
  // sizes of every kind: the workspace functions go through all checks and plans
  for (int B : ints)
    for (int H : ints)
      for (int L : ints)
        for (int m : ints) {
          asa_params p = shape(B, H, L, m % 2 ? 64 : 128, m % 3 ? 64 : 128);
          n.H_kv = m;
          c.H_kv = m > 0 && H > 0 && H % m == 0 ? m : H;
          c.max_blocks = m;
          (void)asa_qk_norm_rope_bwd_workspace_bytes(&p, &n);
          (void)asa_attn_cache_workspace_bytes(&p, &c);
          p.d = m;
          EXPECT(m == 64 || m == 128 || asa_attn_cache_workspace_bytes(&p, &c) == 0);
        }
  // strides of every kind
  const int64_t strides[] = {INT64_MIN, -8, 0, 4, 8, 64, 6400, (int64_t)1 << 23, (int64_t)1 << 24, (int64_t)1 << 62, INT64_MAX - 7};
  n.H_kv = 2;
  c.H_kv = 2;
  c.max_blocks = 4;
  for (int64_t a : strides)
    for (int64_t b : strides)
      for (int64_t l : strides) {
        asa_params p = shape(2, 2, 100, 64, 64);
        const int64_t s[3] = {a, b, l};
        memcpy(p.q_stride, s, sizeof(s));
        memcpy(p.k_stride, s, sizeof(s));
        memcpy(p.o_stride, s, sizeof(s));
        (void)asa_qk_norm_rope_bwd_workspace_bytes(&p, &n);
        (void)asa_attn_cache_workspace_bytes(&p, &c);
        EXPECT(asa_qk_norm_rope(&p, &n, nullptr, x, x, x, nullptr) == ASA_ERR_INVALID_ARG);
        EXPECT(asa_cache_read(&p, &c, nullptr, nullptr, nullptr, nullptr, nullptr) == ASA_ERR_INVALID_ARG);
      }
  // refusals
  asa_params p = shape(1, 1, INT_MAX, 64, 64);
  p.k_samples = 16;
  p.tau = 0.5f;
  p.r_max = 1.f;
  EXPECT(asa_attn_fwd(&p, x, x, x, nullptr, nullptr, x, nullptr, f, x, SIZE_MAX, nullptr) == ASA_ERR_UNSUPPORTED);
  EXPECT(asa_fwd_workspace_bytes(&p) == 0);
  p = shape(2, 2, 100, 64, 64);
  EXPECT(asa_qk_norm_rope(nullptr, &n, x, x, x, x, nullptr) == ASA_ERR_INVALID_ARG);
  EXPECT(asa_qk_norm_rope(&p, nullptr, x, x, x, x, nullptr) == ASA_ERR_INVALID_ARG);
  n.eps = NAN;
  EXPECT(asa_qk_norm_rope(&p, &n, x, x, x, x, nullptr) == ASA_ERR_INVALID_ARG);
  n.eps = 0.f;
  n.rot_dim = 64;
  n.table_rows = INT_MAX;
  n.first_row = INT_MIN;
  EXPECT(asa_qk_norm_rope(&p, &n, x, x, x, x, nullptr) == ASA_ERR_INVALID_ARG);      // no tables
  n.cos_table = n.sin_table = f;
  EXPECT(asa_qk_norm_rope(&p, &n, x, x, x, nullptr, nullptr) == ASA_ERR_INVALID_ARG);
  EXPECT(asa_qk_norm_rope_bwd(&p, &n, x, x, x, x, x, x, f, f, nullptr, nullptr, nullptr, 0, nullptr) == ASA_ERR_WORKSPACE);
  EXPECT(asa_qk_norm_rope_bwd(&p, &n, x, x, x, x, x, x, f, f, f, nullptr, x, 1 << 30, nullptr) == ASA_ERR_INVALID_ARG);
  EXPECT(asa_cache_write(&p, &c, x, x, nullptr, nullptr, nullptr) == ASA_ERR_INVALID_ARG);   // no cache memory
  c.k = c.v = x;
  c.k_scale = c.v_scale = f;
  c.max_blocks = 65537;
  EXPECT(asa_cache_write(&p, &c, x, x, nullptr, nullptr, nullptr) == ASA_ERR_UNSUPPORTED);
  c.max_blocks = 1000;
  p.L = 1;
  const size_t need = asa_attn_cache_workspace_bytes(&p, &c);
  EXPECT(need > 0);
  EXPECT(asa_attn_cache(&p, &c, i32, x, nullptr, nullptr, x, f, x, need - 1, nullptr) == ASA_ERR_WORKSPACE);
  EXPECT(asa_attn_cache(&p, &c, i32, x, i32, nullptr, x, f, x, need, nullptr) == ASA_ERR_INVALID_ARG);
  EXPECT(asa_attn_cache(&p, &c, nullptr, x, nullptr, nullptr, x, f, x, need, nullptr) == ASA_ERR_INVALID_ARG);
  p.scale = -INFINITY;
  EXPECT(asa_attn_cache_workspace_bytes(&p, &c) == 0);
  printf("ok\n");
  return 0;
}
