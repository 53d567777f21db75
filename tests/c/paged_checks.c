/* Host-side argument checks and launch shapes of the head norm and rotation and of the paged 8-bit cache, driven
 * from plain C for the sanitizers.  Every call is answered before anything is launched; pointers are never followed. */
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "decoquant.h"

#define CHECK(cond)                                                   \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "failed at line %d: %s\n", __LINE__, #cond);    \
      return 1;                                                       \
    }                                                                 \
  } while (0)

static _Alignas(16) char fake[256];

static dq_heads heads_of(int32_t n) {
  dq_heads h = {(uint16_t*)fake, 0, 1024, 128, n};
  return h;
}

int main(void) {
  dq_heads h = heads_of(8), q = heads_of(32), many = heads_of(INT_MAX), none = heads_of(0), odd = heads_of(8);
  dq_head_norm norm = {(const uint16_t*)fake, (const uint16_t*)fake, 1e-6f}, bad_norm = {(const uint16_t*)fake, NULL, -1.f};
  dq_rotary rot = {(const double*)fake, (const int32_t*)fake, NULL, 4, 1, 128, 0}, bad_rot = rot;
  dq_paged_cache c = {(uint8_t*)fake, (float*)fake, (uint8_t*)fake, (float*)fake, (uint16_t*)fake, (uint16_t*)fake, 10, 8, 128, 64, 4, DQ_F16, DQ_CODES_INT8}, x;
  dq_paged_batch b = {(const int32_t*)fake, (const int32_t*)fake, (const int32_t*)fake, NULL, 4, 0, 5, 5}, y;
  const int32_t* w = (const int32_t*)fake;
  int32_t big[] = {0, 1, 2, 3, 16, 17, 63, 64, 65, 1000, 1 << 20, INT_MAX / 2, INT_MAX}, i, j, k, l;
  const int n_big = (int)(sizeof big / sizeof big[0]);
  size_t need;

  odd.head_stride = 4;
  /* rotation */
  CHECK(dq_rotate_heads(&h, &h, &q, &q, 1, 0, 128, DQ_F16, &norm, &rot, NULL) == DQ_OK);
  CHECK(dq_rotate_heads(NULL, NULL, NULL, NULL, 1, 1, 128, DQ_F16, &norm, &rot, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&h, NULL, NULL, NULL, 1, 1, 128, DQ_F16, &norm, &rot, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&h, &h, NULL, NULL, 1, 1, 128, DQ_F16, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&h, &none, NULL, NULL, 1, 1, 128, DQ_F16, &norm, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&odd, &odd, NULL, NULL, 1, 1, 128, DQ_F16, &norm, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&h, &h, NULL, NULL, 1, 1, 128, DQ_F16, &bad_norm, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&h, &h, NULL, NULL, INT_MAX, INT_MAX, 128, DQ_F16, &norm, &rot, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&many, &many, &many, &many, 1, 1, 128, DQ_F16, &norm, &rot, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&many, &many, NULL, NULL, 1, INT_MAX, 256, DQ_BF16, &norm, &rot, NULL) == DQ_EINVAL);
  CHECK(dq_rotate_heads(&many, &many, &h, &h, 1, 7, 32, DQ_BF16, &norm, NULL, NULL) == DQ_EINVAL);
  for (i = 0; i < 9; ++i) {
    bad_rot = rot;
    if (i == 0) bad_rot.inv_freq = NULL;
    if (i == 1) bad_rot.rot_dim = 0;
    if (i == 2) bad_rot.rot_dim = 120;
    if (i == 3) bad_rot.rot_dim = 144;
    if (i == 4) bad_rot.axes = 0;
    if (i == 5) bad_rot.axes = INT_MAX;
    if (i == 6) bad_rot.axes = 2;
    if (i == 7) bad_rot.interleaved = -1;
    if (i == 8) bad_rot.positions = NULL;
    CHECK(dq_rotate_heads(&h, &h, NULL, NULL, 1, 1, 128, DQ_F16, NULL, &bad_rot, NULL) == DQ_EINVAL);
    if (i < 8) CHECK(dq_paged_append(&c, &b, &h, &h, NULL, NULL, NULL, &bad_rot, NULL) == DQ_EINVAL);
  }

  /* the cache's and the batch's own checks, through every entry point */
  need = dq_paged_workspace_bytes(&c, 4, 4, 32, 1, 20000);
  CHECK(need > 0);
  for (i = 0; i < 16; ++i) {
    x = c;
    if (i == 0) x.k_codes = NULL;
    if (i == 1) x.v_scales = NULL;
    if (i == 2) x.k_tail = (uint16_t*)(fake + 8);
    if (i == 3) x.k_scales = (float*)(fake + 2);
    if (i == 4) x.pages = 0;
    if (i == 5) x.pages = INT_MAX;
    if (i == 6) x.kv_heads = -8;
    if (i == 7) x.kv_heads = INT_MAX;
    if (i == 8) x.head_dim = 96;
    if (i == 9) x.page_tokens = 0;
    if (i == 10) x.page_tokens = INT_MIN;
    if (i == 11) x.slots = 0;
    if (i == 12) x.slots = INT_MAX;
    if (i == 13) x.dtype = 2;
    if (i == 14) x.codes = -1;
    CHECK(dq_paged_append(i < 15 ? &x : NULL, &b, &h, &h, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
    CHECK(dq_paged_read(i < 15 ? &x : NULL, &b, NULL, w, &h, &h, NULL) == DQ_EINVAL);
    CHECK(dq_paged_attention(i < 15 ? &x : NULL, &b, &q, &q, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
    CHECK(dq_paged_workspace_bytes(i < 15 ? &x : NULL, 4, 4, 32, 1, 20000) == 0);
  }
  for (i = 0; i < 9; ++i) {
    y = b;
    if (i == 0) y.seq_lens = NULL;
    if (i == 1) y.page_table = NULL;
    if (i == 2) y.batch = 0;
    if (i == 3) y.batch = INT_MAX;                        /* more than the slots */
    if (i == 4) y.rows = -1;
    if (i == 5) y.table_width = 0;
    if (i == 6) y.table_stride = 4;
    if (i == 7) y.table_width = y.table_stride = INT_MAX;
    CHECK(dq_paged_append(&c, i < 8 ? &y : NULL, &h, &h, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
    CHECK(dq_paged_read(&c, i < 8 ? &y : NULL, NULL, w, &h, &h, NULL) == DQ_EINVAL);
    CHECK(dq_paged_attention(&c, i < 8 ? &y : NULL, &q, &q, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  }
  y = b;
  y.starts = NULL;
  y.rows = 3;                                             /* one row per sequence */
  CHECK(dq_paged_append(&c, &y, &h, &h, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &y, &q, &q, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);

  /* append, read */
  CHECK(dq_paged_append(&c, &b, &h, &h, &q, &q, &norm, &rot, NULL) == DQ_OK);                 /* no rows */
  CHECK(dq_paged_append(&c, &b, &h, &q, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_append(&c, &b, NULL, &h, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_append(&c, &b, &h, &h, &q, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_append(&c, &b, &h, &h, &q, &h, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_append(&c, &b, &h, &h, NULL, NULL, &bad_norm, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_read(&c, &b, NULL, w, &h, &h, NULL) == DQ_OK);                               /* no rows */
  CHECK(dq_paged_read(&c, &b, NULL, NULL, &h, &h, NULL) == DQ_EINVAL);
  CHECK(dq_paged_read(&c, &b, w, w, &h, NULL, NULL) == DQ_EINVAL);
  /* launches of more threads than one takes */
  x = c; y = b;
  x.pages = x.slots = 1; x.kv_heads = INT_MAX; x.page_tokens = 64;
  y.rows = 1; y.batch = 1;
  h.heads = INT_MAX;
  CHECK(dq_paged_append(&x, &y, &h, &h, NULL, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_append(&x, &y, &h, &h, &many, &many, &norm, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_read(&x, &y, NULL, w, &h, &h, NULL) == DQ_EINVAL);
  h.heads = 8;
  y = b; y.rows = INT_MAX; y.tail_slots = w; y.batch = INT_MAX;
  CHECK(dq_paged_append(&c, &y, &h, &h, &many, &many, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_read(&c, &y, NULL, w, &h, &h, NULL) == DQ_EINVAL);

  /* attention: arguments */
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_OK);   /* no rows */
  CHECK(dq_paged_attention(&c, &b, &q, &h, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, NULL, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, fake + 8, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, -1, 20000, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, -1, 0.f, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 7, fake, need, 0, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, -7, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, NAN, 0, fake, need, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, fake, need, 2u, NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, fake, need, DQ_PAGED_SPLITS(65), NULL) == DQ_EINVAL);
  CHECK(dq_paged_attention(&c, &b, &q, &q, 1, 20000, 0.f, 0, fake, 16, DQ_PAGED_CAUSAL, NULL) == DQ_ENOSPACE);
  /* launch shapes of every size, as far as the workspace check */
  for (i = 0; i < n_big; ++i)
    for (j = 0; j < n_big; ++j)
      for (k = 0; k < n_big; ++k)
        for (l = 0; l < n_big; ++l) {
          const int32_t batch = big[i] ? big[i] : 1;
          int32_t st;
          y = b;
          y.tail_slots = w; y.batch = batch; y.rows = big[j];
          q.heads = l % 2 ? 8 : l % 3 ? 32 : 1 << 20;
          st = dq_paged_attention(&c, &y, &q, &q, big[k], big[l], 0.f, big[l], fake, 16, DQ_PAGED_CAUSAL | (l % 4 ? 0u : DQ_PAGED_SPLITS(64)), NULL);
          CHECK(st == DQ_ENOSPACE || st == DQ_EINVAL);
          need = dq_paged_workspace_bytes(&c, batch, big[j], q.heads, big[k], big[l]);
          CHECK(need < ((size_t)1 << 40));
        }
  printf("paged checks ok\n");
  return 0;
}
