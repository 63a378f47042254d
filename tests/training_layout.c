/* Sizes and offsets of the training step's argument structs, and refusals (nothing is launched, nothing allocated). */
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

static fiona_norm_args norm(void) {
  fiona_norm_args a;
  memset(&a, 0, sizeof a);
  a.n = 5, a.width = 64, a.type = FIONA_BF16, a.weight_type = FIONA_F32, a.eps = 1e-5f;
  a.x = at(0), a.residual = at(1), a.weight = at(2), a.bias = at(3), a.y = at(4), a.total = at(5);
  a.mean = (float *)(void *)at(6), a.rstd = (float *)(void *)at(7);
  a.x_row = a.residual_row = a.y_row = a.total_row = 64;
  return a;
}

static fiona_adamw_tensor tensor(unsigned i, uint64_t n) {
  fiona_adamw_tensor t;
  memset(&t, 0, sizeof t);
  t.param = at(8 * i), t.grad = at(8 * i + 1), t.m = at(8 * i + 2), t.v = at(8 * i + 3);
  t.n = n, t.weight_decay = 0.1;
  return t;
}

int main(void) {
  fiona_norm_args a = norm();
  fiona_norm *norm_handle = (fiona_norm *)1;
  fiona_token_loss *loss = (fiona_token_loss *)1;
  fiona_adamw *opt = (fiona_adamw *)1;
  fiona_norm_desc nd = {FIONA_BF16, FIONA_F16, 64, 4};
  fiona_token_loss_desc ld = {FIONA_BF16, 64, 0, 0};
  fiona_adamw_tensor t[2] = {tensor(0, 300), tensor(1, 300)};
  fiona_adamw_desc ad = {FIONA_F32, 32, 2, 0, 0.9, 0.999, 1e-8, t};
  float one = 1;
  int32_t step = 1;
  printf("sizes %zu %zu %zu %zu %zu %zu %zu %zu\n", sizeof(fiona_norm_args), sizeof(fiona_norm_desc),
         sizeof(fiona_norm_backward_args), sizeof(fiona_token_loss_desc), sizeof(fiona_preference_args),
         sizeof(fiona_policy_args), sizeof(fiona_adamw_tensor), sizeof(fiona_adamw_desc));
  SHOW(fiona_norm_args, x);
  SHOW(fiona_norm_args, total_row);
  SHOW(fiona_norm_backward_args, dx);
  SHOW(fiona_norm_backward_args, dx_row);
  SHOW(fiona_preference_args, targets);
  SHOW(fiona_preference_args, logps);
  SHOW(fiona_policy_args, logits);
  SHOW(fiona_policy_args, logps);
  SHOW(fiona_adamw_tensor, n);
  SHOW(fiona_adamw_desc, tensors);

  EXPECT(FIONA_ERR_ARG, fiona_layer_norm(NULL, NULL));
  a.type = 3;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_layer_norm(&a, NULL));
  a = norm(), a.weight_type = FIONA_F16;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_layer_norm(&a, NULL));
  a = norm(), a.width = 0;
  EXPECT(FIONA_ERR_ARG, fiona_layer_norm(&a, NULL));
  a = norm(), a.width = FIONA_MAX_NORM_WIDTH + 1;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_layer_norm(&a, NULL));
  a = norm(), a.n = FIONA_MAX_NORM_ROWS + 1;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_layer_norm(&a, NULL));
  a = norm(), a.eps = 0;
  EXPECT(FIONA_ERR_ARG, fiona_layer_norm(&a, NULL));
  a = norm(), a.y = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_layer_norm(&a, NULL));
  a = norm(), a.total = at(5) + 1;
  EXPECT(FIONA_ERR_ALIGN, fiona_layer_norm(&a, NULL));
  a = norm(), a.weight = at(2) + 2;
  EXPECT(FIONA_ERR_ALIGN, fiona_layer_norm(&a, NULL));
  a = norm(), a.total = a.y;
  EXPECT(FIONA_ERR_ALIAS, fiona_layer_norm(&a, NULL));
  a = norm(), a.y = (void *)a.x, a.y_row = 128;             /* in place, but with other strides */
  EXPECT(FIONA_ERR_ALIAS, fiona_layer_norm(&a, NULL));
  a = norm(), a.y_row = 63;                                 /* rows over each other */
  EXPECT(FIONA_ERR_ALIAS, fiona_layer_norm(&a, NULL));
  a = norm(), a.y = (void *)a.weight;
  EXPECT(FIONA_ERR_ALIAS, fiona_layer_norm(&a, NULL));
  a = norm(), a.mean = (float *)(void *)at(4);
  EXPECT(FIONA_ERR_ALIAS, fiona_layer_norm(&a, NULL));
  a = norm(), a.x_row = (uint64_t)1 << 62;
  EXPECT(FIONA_ERR_ARG, fiona_layer_norm(&a, NULL));
  a = norm(), a.n = 0;
  EXPECT(FIONA_OK, fiona_layer_norm(&a, NULL));

  EXPECT(FIONA_ERR_ARG, fiona_norm_create(&nd, NULL));
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_norm_create(&nd, &norm_handle));
  if (norm_handle) return 1;
  EXPECT(FIONA_ERR_ARG, fiona_layer_norm_backward(NULL, NULL, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_token_loss_create(&ld, &loss));
  if (loss) return 1;
  ld.max_tokens = (1u << 21) + 1;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_token_loss_create(&ld, &loss));
  EXPECT(FIONA_ERR_ARG, fiona_preference_loss(NULL, NULL, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_policy_loss(NULL, NULL, NULL));

  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, NULL));
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(NULL, &opt));
  if (opt) return 1;
  ad.state_bits = 16;
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_adamw_create(&ad, &opt));
  ad.state_bits = 32, ad.beta2 = 1;
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  ad.beta2 = 0.999, ad.eps = 1e-60;                          /* zero in 32 bits */
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  ad.eps = 1e-8, ad.tensors = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  ad.tensors = t, t[1].grad = NULL;
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].m_scale = (float *)(void *)at(20);
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].v = at(11) + 2;
  EXPECT(FIONA_ERR_ALIGN, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].m = t[0].v;
  EXPECT(FIONA_ERR_ALIAS, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].param = (char *)t[0].grad + 299 * 4;
  EXPECT(FIONA_ERR_ALIAS, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].weight_decay = -1;
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300), t[1].weight_decay = 1e300;          /* infinite in 32 bits */
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, (uint64_t)1 << 50);
  EXPECT(FIONA_ERR_UNSUPPORTED, fiona_adamw_create(&ad, &opt));
  t[1] = tensor(1, 300);
  ad.state_bits = 8;                                         /* without scales */
  EXPECT(FIONA_ERR_ARG, fiona_adamw_create(&ad, &opt));
  if (opt) return 1;
  EXPECT(FIONA_ERR_ARG, fiona_adamw_step(NULL, &one, &step, NULL, NULL));
  fiona_norm_destroy(NULL);
  fiona_token_loss_destroy(NULL);
  fiona_adamw_destroy(NULL);
  puts("ok");
  return 0;
}
