// fiona_preference_loss and fiona_policy_loss (include/fiona.h): losses on tokens'
// logits and their gradients.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>

#include "fiona.h"
#include "rows.hpp"
#include "token_loss_kernel.hpp"

using namespace fiona_host;

struct fiona_token_loss {
  fiona_token_loss_desc desc{};
  int device = -1;
  float *ws = nullptr;     // [3][max_tokens]: log sums, log-probabilities, derivatives
};

namespace {

constexpr uint32_t kMost = 1u << 22;   // vocab, tokens, pairs

// Checks what both calls share.
int check_logits(const fiona_token_loss *H, uint32_t n, const void *logits, const void *dlogits, const int32_t *targets,
                 uint64_t logits_row, uint64_t dlogits_row, Rows &in, Rows &out) {
  const fiona_token_loss_desc &D = H->desc;
  if (n > D.max_tokens || (n && (!logits || !targets))) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type);
  if (misaligned(logits, e) || misaligned(dlogits, e) || misaligned(targets, 4)) return FIONA_ERR_ALIGN;
  in = matrix(logits, e, n, D.vocab, logits_row), out = matrix(dlogits, e, n, D.vocab, dlogits_row);
  return FIONA_OK;
}

fiona::TokenParams params(const fiona_token_loss *H, uint32_t n, const void *logits, void *dlogits, const int32_t *targets,
                          uint64_t logits_row, uint64_t dlogits_row) {
  fiona::TokenParams P{};
  P.z = logits, P.dz = dlogits, P.targets = targets, P.z_row = logits_row, P.dz_row = dlogits_row;
  P.n_tok = n, P.vocab = H->desc.vocab;
  P.lse = H->ws, P.logp = H->ws + H->desc.max_tokens, P.coef = P.logp + H->desc.max_tokens;
  return P;
}

}  // namespace

extern "C" {

int fiona_token_loss_create(const fiona_token_loss_desc *desc, fiona_token_loss **out) {
  if (!out) return FIONA_ERR_ARG;
  *out = nullptr;
  if (!desc) return FIONA_ERR_ARG;
  const fiona_token_loss_desc &D = *desc;
  if (!known_type(D.type)) return FIONA_ERR_UNSUPPORTED;
  if (!D.vocab || !D.max_tokens) return FIONA_ERR_ARG;
  if (D.vocab > kMost || D.max_tokens > kMost || D.max_pairs > kMost) return FIONA_ERR_UNSUPPORTED;
  fiona_token_loss *H = new (std::nothrow) fiona_token_loss;
  if (!H) return FIONA_ERR_NOMEM;
  H->desc = D;
  if (hipGetDevice(&H->device) != hipSuccess) {
    delete H;
    return FIONA_ERR_HIP;
  }
  if (hipMalloc((void **)&H->ws, (uint64_t)D.max_tokens * 3 * sizeof(float)) != hipSuccess) {
    (void)hipGetLastError();
    delete H;
    return FIONA_ERR_NOMEM;
  }
  *out = H;
  return FIONA_OK;
}

void fiona_token_loss_destroy(fiona_token_loss *H) {
  if (!H) return;
  if (H->ws) (void)hipFree(H->ws);
  delete H;
}

int fiona_preference_loss(const fiona_token_loss *H, const fiona_preference_args *args, hipStream_t stream) {
  if (!H || !args) return FIONA_ERR_ARG;
  const fiona_preference_args &A = *args;
  if (A.n_pair > H->desc.max_pairs) return FIONA_ERR_ARG;
  if (!(A.beta > 0) || !std::isfinite(A.beta) || !(A.label_smoothing >= 0) || !(A.label_smoothing < 1)) return FIONA_ERR_ARG;
  Rows z, dz;
  int rc = check_logits(H, A.n_tok, A.logits, A.dlogits, A.targets, A.logits_row, A.dlogits_row, z, dz);
  if (rc != FIONA_OK) return rc;
  if (A.n_pair && (!A.offsets || !A.reference || !A.loss || !A.logps)) return FIONA_ERR_ARG;
  if (misaligned(A.offsets, 4) || misaligned(A.reference, 4) || misaligned(A.weights, 4) || misaligned(A.loss, 4) ||
      misaligned(A.logps, 4))
    return FIONA_ERR_ALIGN;
  const uint64_t p = A.n_pair;
  const Rows in[] = {z, matrix(A.targets, 4, 1, A.n_tok, 0), matrix(A.offsets, 4, 1, 2 * p + 1, 0), matrix(A.reference, 4, 1, 2 * p, 0),
                     matrix(A.weights, 4, 1, p, 0)};
  const Rows out[] = {dz, matrix(A.loss, 4, 1, p, 0), matrix(A.logps, 4, 1, 2 * p, 0)};
  const uint32_t own[] = {1, 0, 0};
  if ((rc = check_alias(in, 5, out, 3, own)) != FIONA_OK) return rc;
  if (!on_device(H->device)) return FIONA_ERR_ARG;
  const fiona::TokenParams P = params(H, A.n_tok, A.logits, A.dlogits, A.targets, A.logits_row, A.dlogits_row);
  const fiona::PairParams Q{A.offsets, A.reference, A.weights, A.loss, A.logps, A.beta, A.label_smoothing, A.n_pair};
  with_type(H->desc.type, [&](auto t) {
    using T = decltype(t);
    if (A.n_tok) hipLaunchKernelGGL((fiona::token_stats_kernel<T, false>), dim3(A.n_tok), dim3(256), 0, stream, P, fiona::PolicyParams{});
    if (A.n_pair) hipLaunchKernelGGL(fiona::pair_kernel, dim3(A.n_pair), dim3(256), 0, stream, P, Q);
    if (A.n_tok && A.dlogits) hipLaunchKernelGGL(fiona::token_grad_kernel<T>, dim3(A.n_tok), dim3(256), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

int fiona_policy_loss(const fiona_token_loss *H, const fiona_policy_args *args, hipStream_t stream) {
  if (!H || !args) return FIONA_ERR_ARG;
  const fiona_policy_args &A = *args;
  if (!(A.clip_low >= 0) || !(A.clip_low <= 1) || !(A.clip_high >= 0) || !std::isfinite(A.clip_high) || !(A.kl >= 0) ||
      !std::isfinite(A.kl))
    return FIONA_ERR_ARG;
  Rows z, dz;
  int rc = check_logits(H, A.n_tok, A.logits, A.dlogits, A.targets, A.logits_row, A.dlogits_row, z, dz);
  if (rc != FIONA_OK) return rc;
  if (!A.n_tok) return FIONA_OK;
  if (!A.old || !A.advantages || !A.loss || !A.logps || (A.kl > 0 && !A.reference)) return FIONA_ERR_ARG;
  if (misaligned(A.old, 4) || misaligned(A.advantages, 4) || misaligned(A.reference, 4) || misaligned(A.weights, 4) ||
      misaligned(A.loss, 4) || misaligned(A.logps, 4))
    return FIONA_ERR_ALIGN;
  const uint64_t n = A.n_tok;
  const Rows in[] = {z, matrix(A.targets, 4, 1, n, 0), matrix(A.old, 4, 1, n, 0), matrix(A.advantages, 4, 1, n, 0),
                     matrix(A.reference, 4, 1, n, 0), matrix(A.weights, 4, 1, n, 0)};
  const Rows out[] = {dz, matrix(A.loss, 4, 1, n, 0), matrix(A.logps, 4, 1, n, 0)};
  const uint32_t own[] = {1, 0, 0};
  if ((rc = check_alias(in, 6, out, 3, own)) != FIONA_OK) return rc;
  if (!on_device(H->device)) return FIONA_ERR_ARG;
  const fiona::TokenParams P = params(H, A.n_tok, A.logits, A.dlogits, A.targets, A.logits_row, A.dlogits_row);
  const fiona::PolicyParams Q{A.old, A.advantages, A.kl > 0 ? A.reference : nullptr, A.weights, A.loss, A.logps,
                              A.clip_low, A.clip_high, A.kl};
  with_type(H->desc.type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((fiona::token_stats_kernel<T, true>), dim3(A.n_tok), dim3(256), 0, stream, P, Q);
    if (A.dlogits) hipLaunchKernelGGL(fiona::token_grad_kernel<T>, dim3(A.n_tok), dim3(256), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
