/* Sizes and offsets of the key holder's argument structs, and kv_append's refusals (nothing is launched). */
#include "fiona.h"

#include <stdio.h>
#include <string.h>

#define SHOW(type, field) printf(#type " " #field " %zu\n", offsetof(type, field))
#define EXPECT(want, call)                                                    \
  do {                                                                        \
    int got = (call);                                                         \
    if (got != (want)) {                                                      \
      printf("line %d: %s, not %s\n", __LINE__, fiona_status_string(got), fiona_status_string(want)); \
      return 1;                                                               \
    }                                                                         \
  } while (0)

/* Addresses far apart that no call may reach. */
static char *at(unsigned i) { return (char *)((size_t)(i + 1) << 32); }

static fiona_kv_cache cache(void) {
  fiona_kv_cache c;
  memset(&c, 0, sizeof c);
  c.type = FIONA_BF16;
  c.n_pages = 4, c.page_size = 16, c.n_kv = 2, c.head_dim = 64;
  c.k = at(0), c.v = at(1);
  c.k_page = c.v_page = 16 * 2 * 64, c.k_token = c.v_token = 2 * 64, c.k_head = c.v_head = 64;
  return c;
}

static fiona_append_args append(void) {
  fiona_append_args a;
  memset(&a, 0, sizeof a);
  a.n_tok = 3, a.n_head = 4, a.rows_type = FIONA_BF16, a.rot_dim = 64, a.n_pos = 100;
  a.q = at(2), a.k = at(3), a.v = at(4), a.q_out = at(5);
  a.slots = (const int64_t *)(void *)at(6), a.positions = (const int32_t *)(void *)at(7);
  a.cos = (const float *)(void *)at(8), a.sin = (const float *)(void *)at(9);
  a.q_tok = a.q_out_tok = 4 * 64, a.k_tok = a.v_tok = 2 * 64;
  a.q_head = a.q_out_head = a.k_head = a.v_head = 64;
  return a;
}

int main(void) {
  fiona_kv_cache c = cache();
  fiona_append_args a = append();
  fiona_attention *att = (fiona_attention *)1;
  fiona_adapters *ad = (fiona_adapters *)1;
  fiona_attention_desc d = {FIONA_BF16, 6, 4, 64, 16, 1, 8};
  fiona_adapters_desc e = {FIONA_BF16, 1, 129, 64, 64, 1, 0};
  printf("sizes %zu %zu %zu %zu %zu %zu\n", sizeof(fiona_kv_cache), sizeof(fiona_append_args), sizeof(fiona_attention_desc),
         sizeof(fiona_attention_args), sizeof(fiona_adapters_desc), sizeof(fiona_adapter_args));
  SHOW(fiona_kv_cache, v_head);
  SHOW(fiona_append_args, sin);
  SHOW(fiona_attention_args, q);
  SHOW(fiona_attention_args, lengths);
  SHOW(fiona_adapter_args, base);
  SHOW(fiona_adapter_args, dx_row);

  EXPECT(FIONA_ERR_ARG, fiona_kv_append(NULL, &a, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, NULL, NULL));
  c.type = 3;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.head_dim = 257;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.n_pages = 1u << 28;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.page_size = 0;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.v = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.k = at(0) + 1;
  EXPECT(FIONA_ERR_ALIGN, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.v = c.k;
  EXPECT(FIONA_ERR_ALIAS, fiona_kv_append(&c, &a, NULL));
  c = cache(), c.k_token = 64;   /* heads of one token over the next token's */
  EXPECT(FIONA_ERR_ALIAS, fiona_kv_append(&c, &a, NULL));
  c = cache();
  a.rot_dim = 63;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  a.rot_dim = 66;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  a = append(), a.positions = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  a = append(), a.q_out = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  a = append(), a.slots = (const int64_t *)(void *)(at(6) + 4);
  EXPECT(FIONA_ERR_ALIGN, fiona_kv_append(&c, &a, NULL));
  a = append(), a.k = c.k;
  EXPECT(FIONA_ERR_ALIAS, fiona_kv_append(&c, &a, NULL));
  a = append(), a.q_out = (void *)a.q, a.q_out_tok = 8 * 64;   /* in place, but with other strides */
  EXPECT(FIONA_ERR_ALIAS, fiona_kv_append(&c, &a, NULL));
  a = append(), a.q_tok = (uint64_t)1 << 62;
  EXPECT(FIONA_ERR_ARG, fiona_kv_append(&c, &a, NULL));
  a = append(), a.n_tok = 0;
  EXPECT(FIONA_OK, fiona_kv_append(&c, &a, NULL));

  EXPECT(FIONA_ERR_ARG, fiona_attention_create(&d, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_attention_create(&d, &att));
  if (att) return 1;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_adapters_create(&e, &ad));
  if (ad) return 1;
  EXPECT(FIONA_ERR_ARG, fiona_paged_attention(NULL, &c, NULL, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_adapter_linear(NULL, NULL, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_adapter_backward(NULL, NULL, NULL));
  fiona_attention_destroy(NULL);
  fiona_adapters_destroy(NULL);
  puts("ok");
  return 0;
}
