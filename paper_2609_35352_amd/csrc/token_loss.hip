// fiona_preference_loss and fiona_policy_loss (include/fiona.h): losses on tokens'
// logits and their gradients.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>

#include "fiona.h"
#include "rows.hpp"
#include "token_loss_kernel.hpp"

using namespace fiona_host;

struct fiona_token_loss {
  fiona_token_loss_desc desc{};
  int device = -1;
  char *ws = nullptr;      // parts of rows, then [4][max_tokens]: log sums (2), logits, derivatives
  uint64_t part_cap = 0;   // parts that fit
};

namespace {

constexpr uint32_t kMost = 1u << 21;   // vocab, tokens, pairs (times 1024 threads: below 2^32)

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

// Parts of each of n rows of `pieces` pieces: enough workgroups to fill the GPU, none
// below 256 pieces (one for each of its threads).  1024 / 2048 / 4096 / 8192 workgroups,
// parts and gradient, us: 1392 tokens of 50021 in binary16 80 / 74 / 73 / 87, 885 of
// 32768 in bfloat16 28 / 30 / 32 / 44, 7955 of 32768 225 / 226 / 224 / 235.
constexpr uint32_t kWorkgroups = 2048;
uint32_t splits_of(uint32_t n, uint32_t pieces) {
  n = std::max(1u, n);
  return std::max(1u, std::min({(kWorkgroups + n - 1) / n, (pieces + 255) / 256, fiona::kLossSplits}));
}

// Elements of a line of memory less one where some row of logits starts off the 16 bytes,
// rows are long and there are many, so that it counts (us, gradients and their parts or
// whole rows, from the rows' first elements / from their lines: 6300 rows of 30011 in bfloat16 380 /
// 322, of 9001 in binary16 111 / 101, of 4001 43.0 / 42.0 (in 32 bits 86 / 80), of 2003 31.8 / 35.7; 3000 whole rows of
// 50016 in binary16 124 / 129, 8000 of 4001 in bfloat16 32.5 / 35.2, 1500 of 125001 178 / 155,
// 2000 of 50021 in 32 bits 159 / 148, 24 of them 8.5 / 9.2, 300 of 50001 in bfloat16 19.7 / 19.6).
constexpr uint64_t kLine = 128, kSkewedRow = 12288, kSkewedRows = 32 << 20;
uint32_t skew_of(const fiona_token_loss_desc &D, const void *logits, uint64_t logits_row, uint32_t n) {
  const uint64_t e = type_size(D.type), off = (uint64_t)logits | (n > 1 ? logits_row * e : 0), row = D.vocab * e;
  return off % 16 && row >= kSkewedRow && n * row >= kSkewedRows ? kLine / e - 1 : 0;
}
uint32_t pieces_of(const fiona_token_loss_desc &D, uint32_t skew) {
  const uint32_t e = 16 / type_size(D.type);
  return (D.vocab + skew + e - 1) / e;
}

fiona::TokenParams params(const fiona_token_loss *H, uint32_t n, const void *logits, void *dlogits, const int32_t *targets,
                          uint64_t logits_row, uint64_t dlogits_row) {
  fiona::TokenParams P{};
  P.z = logits, P.dz = dlogits, P.targets = targets, P.z_row = logits_row, P.dz_row = dlogits_row;
  P.n_tok = n, P.vocab = H->desc.vocab;
  P.part = (float2 *)H->ws, P.lse = P.part + H->part_cap;
  P.at_target = (float *)(P.lse + H->desc.max_tokens), P.coef = P.at_target + H->desc.max_tokens;
  P.skew = skew_of(H->desc, logits, logits_row, n);
  const uint32_t pieces = pieces_of(H->desc, P.skew);
  P.slice = (pieces + splits_of(n, pieces) - 1) / splits_of(n, pieces);
  P.splits = (pieces + P.slice - 1) / P.slice;
  return P;
}

// Calls f with whether rows are shorter than a piece, and whether they are skewed.
template <typename T, typename F>
void with_rows(const fiona::TokenParams &P, F f) {
  if (P.vocab < fiona::kLaneElems<T>) f(std::true_type{}, std::false_type{});
  else if (P.skew) f(std::false_type{}, std::true_type{});
  else f(std::false_type{}, std::false_type{});
}

template <typename T>
void launch_stats(const fiona::TokenParams &P, hipStream_t stream) {
  with_rows<T>(P, [&](auto narrow, auto skewed) {
    hipLaunchKernelGGL((fiona::token_stats_kernel<T, decltype(narrow)::value, decltype(skewed)::value>), dim3(P.n_tok, P.splits), dim3(256),
                       0, stream, P);
  });
}

template <typename T, bool POLICY>
void launch_grad(const fiona::TokenParams &P, const fiona::PolicyParams &Q, hipStream_t stream) {
  with_rows<T>(P, [&](auto narrow, auto skewed) {
    hipLaunchKernelGGL((fiona::token_grad_kernel<T, decltype(narrow)::value, decltype(skewed)::value, POLICY>),
                       dim3(P.n_tok, P.dz ? P.splits : 1), dim3(256), 0, stream, P, Q);
  });
}

// Whether each row's policy loss is one workgroup's: rows of up to 64 KiB, or enough
// of the longer ones (one workgroup reads and writes 256 KiB in 17 us), up to what the registers and
// LDS of a compute unit hold.  us of two launches, parts and gradient, without the gap
// between them / of whole rows, in bfloat16: 2 x 16000 7.2 / 4.9, 64 x 32768 8.9 / 7.6, 16 x
// 64000 7.6 / 10.4, 64 x 64000 11.8 / 11.1, 64 x 131072 12.8 / 18.2, 100 x 131072 22.8 / 19.4,
// 3000 x 131072 411 / 290, 100 x 151936 21.6 / 21.1, 2000 x 151936 352 / 237, and 1500 x 100000
// in 32 bits 348 / 220.
constexpr uint32_t kRowPieces = 1024 * 25;
bool whole_rows(uint32_t n, uint32_t pieces) { return pieces <= 4096 || (pieces <= kRowPieces && n >= pieces / 192); }

// The policy loss with whole rows.  Where there are more rows than compute units, shapes of
// which two or more workgroups share a unit, so that one reads while another writes, and in
// 16 bits even where that takes reading a quarter again (us of 1024 threads with the row in
// registers / so: 8000 rows of 32000 in bfloat16, 512 threads, 182 / 171; in LDS as well 5000 of 50000
// 205 / 177, 3000 of 70000 178 / 155, of 98000 238 / 229; reading again 2500 of 110000 in binary16 225 / 212,
// 1500 of 125001 154 / 141, 3000 of 131072 285 / 284, but 1500 of 64000 in 32 bits 135 / 141).  256 rows
// of 50000 take 13.5 / 14.2, and 300 21.3 / 19.6.  Threads as a row needs, not in whole shapes:
// 8000 rows of 2000 22.9 / 15.6, 3000 of 20000 56 / 48.
template <typename T, int NV, int NL, int NR, bool SKEWED>
void launch_row(const fiona::TokenParams &P, const fiona::PolicyParams &Q, uint32_t threads, hipStream_t stream) {
  hipLaunchKernelGGL((fiona::policy_row_kernel<T, NV, NL, NR, SKEWED>), dim3(P.n_tok), dim3(threads), 0, stream, P, Q, threads);
}
template <typename T, bool SKEWED>
void launch_shape(const fiona::TokenParams &P, const fiona::PolicyParams &Q, uint32_t pieces, hipStream_t stream) {
  const bool many = P.n_tok > 256;
  auto threads = [&](uint32_t nv) { return (pieces + 64 * nv - 1) / (64 * nv) * 64; };
  if (pieces <= 4 * 512) launch_row<T, 4, 0, 0, SKEWED>(P, Q, threads(many ? 4 : 2), stream);
  else if (many && pieces <= 8 * 512) launch_row<T, 8, 0, 0, SKEWED>(P, Q, threads(8), stream);
  else if (many && pieces <= 8 * 1024) launch_row<T, 4, 4, 0, SKEWED>(P, Q, 1024, stream);
  else if (many && pieces <= 12 * 1024) launch_row<T, 8, 4, 0, SKEWED>(P, Q, 1024, stream);
  else if (pieces <= 4 * 1024) launch_row<T, 4, 0, 0, SKEWED>(P, Q, 1024, stream);
  else if (pieces <= 8 * 1024) launch_row<T, 8, 0, 0, SKEWED>(P, Q, 1024, stream);
  else if (pieces <= 16 * 1024) {
    if constexpr (sizeof(T) == 2) {
      if (many) return launch_row<T, 8, 4, 4, SKEWED>(P, Q, 1024, stream);
    }
    launch_row<T, 16, 0, 0, SKEWED>(P, Q, 1024, stream);
  } else {
    launch_row<T, 16, 9, 0, SKEWED>(P, Q, 1024, stream);
  }
}
template <typename T>
void launch_rows(const fiona::TokenParams &P, const fiona::PolicyParams &Q, uint32_t pieces, hipStream_t stream) {
  if (P.skew) launch_shape<T, true>(P, Q, pieces, stream);
  else launch_shape<T, false>(P, Q, pieces, stream);
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
  H->part_cap = (uint64_t)D.max_tokens + kWorkgroups;     // (n rounded-up quotients of kWorkgroups / n, or 64 of few rows)
  if (hipMalloc((void **)&H->ws, H->part_cap * sizeof(float2) + (uint64_t)D.max_tokens * 4 * sizeof(float)) != hipSuccess) {
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
    if (A.n_tok) launch_stats<T>(P, stream);
    uint32_t lanes = 1;
    while (lanes < P.splits) lanes *= 2;
    if (A.n_pair) hipLaunchKernelGGL(fiona::pair_kernel, dim3(A.n_pair), dim3(1024), 0, stream, P, Q, lanes);
    if (A.n_tok && A.dlogits) launch_grad<T, false>(P, fiona::PolicyParams{}, stream);
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
  fiona::TokenParams P = params(H, A.n_tok, A.logits, A.dlogits, A.targets, A.logits_row, A.dlogits_row);
  const fiona::PolicyParams Q{A.old, A.advantages, A.kl > 0 ? A.reference : nullptr, A.weights, A.loss, A.logps,
                              A.clip_low, A.clip_high, A.kl};
  with_type(H->desc.type, [&](auto t) {
    using T = decltype(t);
    uint32_t pieces = pieces_of(H->desc, P.skew);
    if (pieces > kRowPieces && pieces_of(H->desc, 0) <= kRowPieces) {     // (rows that just fit: by less than lines)
      while (pieces > kRowPieces) P.skew /= 2, pieces = pieces_of(H->desc, P.skew);
    }
    if (A.dlogits && whole_rows(A.n_tok, pieces) && P.vocab >= fiona::kLaneElems<T>) {
      launch_rows<T>(P, Q, pieces, stream);
      return;
    }
    launch_stats<T>(P, stream);
    launch_grad<T, true>(P, Q, stream);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
