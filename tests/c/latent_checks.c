/* Host-side argument checks and launch shapes of drafted trees, latents and expanded attention, driven from plain C for the
 * sanitizers.  No call gets as far as a launch: they are refused, have no rows, or ask for more workspace than they are given.  Pointers are
 * never followed. */
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "decoquant.h"

#define CHECK(cond)                                                   \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "failed at line %d: %s\n", __LINE__, #cond);    \
      return 1;                                                       \
    }                                                                 \
  } while (0)

static _Alignas(16) char fake[256];
static const int32_t big[] = {0, 1, 2, 3, 16, 17, 63, 64, 65, 129, 1000, 1 << 20, INT_MAX / 2, INT_MAX};
enum { N = sizeof big / sizeof big[0] };

static dq_heads heads_of(int32_t n) {
  dq_heads h = {(uint16_t*)fake, 0, 1024, 128, n};
  return h;
}

int main(void) {
  dq_heads h = heads_of(8), q = heads_of(32), many = heads_of(INT_MAX), out = heads_of(32), many_out = heads_of(INT_MAX);
  dq_paged_cache c = {(uint8_t*)fake, (float*)fake, (uint8_t*)fake, (float*)fake, (uint16_t*)fake, (uint16_t*)fake, 10, 8, 128, 64, 4, DQ_F16, DQ_CODES_INT8};
  dq_latent_cache l = {(uint16_t*)fake, 10, 64, 512, 64, DQ_BF16};
  dq_paged_batch b = {(const int32_t*)fake, (const int32_t*)fake, (const int32_t*)fake, (const int32_t*)fake, 4, 4, 5, 5}, none = b, y;
  dq_expanded e = {q, q, q, q, (const uint16_t*)fake, 64, (const int32_t*)fake, (const int32_t*)fake, 4, 4, 300, 128, 64, DQ_F16};
  dq_rotary rot = {(const double*)fake, NULL, NULL, 0, 1, 64, 0};
  const uint64_t* seen = (const uint64_t*)fake;
  const int32_t* w = (const int32_t*)fake;
  uint16_t* rows = (uint16_t*)fake;
  int i, j, k, m;
  none.rows = 0;
  out.data = many_out.data = (uint16_t*)(uintptr_t)(1ull << 60);   /* far from all inputs */
  e.out = out;

  /* sizes of all magnitudes: a size or a refusal, never an overflow, and never less than a smaller call's */
  for (i = 0; i < N; ++i)
    for (j = 0; j < N; ++j)
      for (k = 0; k < N; ++k)
        for (m = 0; m < N; ++m) {
          size_t n, less;
          n = dq_latent_workspace_bytes(&l, big[i], big[j], 16, big[k], big[m]);
          less = dq_latent_workspace_bytes(&l, big[i] / 2, big[j] / 3, 16, big[k] / 2, big[m] / 3);
          CHECK(n == 0 || less <= n);
          CHECK(n == 0 || big[i] > 0);
          dq_latent_workspace_bytes(&l, big[i], big[j], big[k], big[m], 1000);
          n = dq_paged_tree_workspace_bytes(&c, big[i], big[j], 32, big[k], big[m]);
          less = dq_paged_tree_workspace_bytes(&c, big[i] / 2, big[j] / 3, 32, big[k] / 2, big[m] / 3);
          CHECK(n == 0 || less <= n);
          CHECK(n == 0 || big[k] <= 64);
          dq_paged_tree_workspace_bytes(&c, big[i], big[j], big[k], 64, big[m]);
          n = dq_expanded_workspace_bytes(big[i], big[j], 16, 128, big[k], big[m]);
          less = dq_expanded_workspace_bytes(big[i] / 2, big[j] / 3, 16, 128, big[k] / 2, big[m] / 3);
          CHECK(n == 0 || less <= n);
          dq_expanded_workspace_bytes(big[i], big[j], big[k], 64, big[m], 1000);
          /* the calls themselves: what a size was given for fits, and nothing else than a refusal comes of the others */
          y = none;
          y.batch = big[i];
          y.rows = big[j];
          if (y.rows) {
            int32_t s = dq_latent_attention(&l, &y, &q, &out, NULL, big[k], big[m], 0.1f, fake, 0, DQ_PAGED_CAUSAL, NULL);
            CHECK(s == DQ_EINVAL || s == DQ_ENOSPACE);
            CHECK(s == DQ_EINVAL || dq_latent_workspace_bytes(&l, big[i], big[j], 32, big[k], big[m]) > 0);
            s = dq_paged_tree_attention(&c, &y, &q, &h, &h, &q, seen, big[k], big[m], 0.f, 0, fake, 0, 0, NULL);
            CHECK(s == DQ_EINVAL || s == DQ_ENOSPACE);
            CHECK(s == DQ_EINVAL || dq_paged_tree_workspace_bytes(&c, big[i], big[j], 32, big[k], big[m]) > 0);
            e.batch = big[i];
            e.rows = big[j];
            s = dq_expanded_attention(&e, big[k], big[m], 0.f, fake, 0, DQ_PAGED_CAUSAL, NULL);
            CHECK(s == DQ_EINVAL || s == DQ_ENOSPACE);
          }
        }
  e.batch = e.rows = 4;

  /* launches of more threads than one takes; heads without end */
  y = b;
  y.batch = 1;
  y.rows = INT_MAX;
  CHECK(dq_latent_attention(&l, &y, &many, &many_out, NULL, INT_MAX, INT_MAX, 1.f, fake, SIZE_MAX, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_paged_tree_attention(&c, &y, &many, &h, &h, &many, seen, 64, 1000, 0.f, 0, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  e.q = e.k = e.v = many;
  e.out = many_out;
  e.rows = INT_MAX;
  CHECK(dq_expanded_attention(&e, INT_MAX, INT_MAX, 0.f, fake, SIZE_MAX, DQ_PAGED_CAUSAL, NULL) == DQ_EINVAL);
  CHECK(dq_latent_append(&l, &y, rows, 576, rows, 576, NULL, 0.f, &many, &many, &rot, NULL) == DQ_EINVAL);
  e.q = e.k = e.v = q;
  e.out = out;
  e.rows = 4;

  /* no rows: nothing is launched, whatever the rest holds */
  CHECK(dq_latent_append(&l, &none, rows, 576, rows, 576, rows, 1e-6f, &q, &q, &rot, NULL) == DQ_OK);
  CHECK(dq_latent_read(&l, &none, NULL, w, rows, 576, NULL) == DQ_OK);
  CHECK(dq_latent_attention(&l, &none, &q, &out, seen, 64, 0, 1.f, fake, dq_latent_workspace_bytes(&l, 4, 0, 32, 64, 0), DQ_PAGED_CAUSAL, NULL) == DQ_OK);
  CHECK(dq_paged_tree_attention(&c, &none, &q, &h, &h, &q, seen, 64, 0, 0.f, 64, fake, dq_paged_tree_workspace_bytes(&c, 4, 0, 32, 64, 0), 0, NULL) == DQ_OK);
  e.rows = 0;
  CHECK(dq_expanded_attention(&e, 64, 300, 0.f, fake, dq_expanded_workspace_bytes(4, 0, 32, 128, 64, 300), 0, NULL) == DQ_OK);
  e.rows = 4;
  /* rows, but none that the bound counts */
  CHECK(dq_latent_attention(&l, &b, &q, &out, NULL, 0, 300, 1.f, fake, SIZE_MAX, 0, NULL) == DQ_OK);
  CHECK(dq_paged_tree_attention(&c, &b, &q, &h, &h, &q, seen, 0, 300, 0.f, 0, fake, SIZE_MAX, 0, NULL) == DQ_OK);
  CHECK(dq_expanded_attention(&e, 0, 300, 0.f, fake, SIZE_MAX, 0, NULL) == DQ_OK);

  /* pointers that are not there, through every entry point */
  CHECK(dq_latent_append(NULL, &b, rows, 576, rows, 576, NULL, 0.f, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_latent_append(&l, NULL, rows, 576, rows, 576, NULL, 0.f, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_latent_append(&l, &b, rows, INT64_MAX, rows, 576, NULL, 0.f, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_latent_append(&l, &b, rows, INT64_MIN, rows, 576, NULL, 0.f, NULL, NULL, NULL, NULL) == DQ_EINVAL);
  CHECK(dq_latent_read(NULL, &b, NULL, w, rows, 576, NULL) == DQ_EINVAL);
  CHECK(dq_latent_read(&l, NULL, NULL, w, rows, 576, NULL) == DQ_EINVAL);
  CHECK(dq_latent_attention(NULL, &b, &q, &out, NULL, 1, 300, 1.f, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_latent_attention(&l, NULL, &q, &out, NULL, 1, 300, 1.f, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_latent_attention(&l, &b, &q, &out, NULL, 1, 300, FLT_MAX, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_paged_tree_attention(NULL, &b, &q, &h, &h, &q, seen, 1, 300, 0.f, 0, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_paged_tree_attention(&c, NULL, &q, &h, &h, &q, seen, 1, 300, 0.f, 0, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_paged_tree_attention(&c, &b, &q, &h, &h, &q, seen, 1, 300, NAN, 0, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_expanded_attention(NULL, 1, 300, 0.f, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  CHECK(dq_expanded_attention(&e, 1, 300, INFINITY, fake, SIZE_MAX, 0, NULL) == DQ_EINVAL);
  puts("latent checks ok");
  return 0;
}
