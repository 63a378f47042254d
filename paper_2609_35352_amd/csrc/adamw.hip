// fiona_adamw_step (include/fiona.h): one optimiser step over many tensors.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "adamw_kernel.hpp"
#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_adamw {
  int device = -1;
  uint32_t type = 0, bits = 32;
  fiona::AdamwParams P{};
};

namespace {

struct Piece {
  uint64_t at, end;
  bool written;
};

// Whether what is written overlaps anything else.
bool pieces_overlap(std::vector<Piece> &pieces) {
  std::sort(pieces.begin(), pieces.end(), [](const Piece &a, const Piece &b) { return a.at < b.at; });
  uint64_t end = 0, written = 0;   // of the pieces so far, and of those written
  for (const Piece &p : pieces) {
    if (p.at < (p.written ? end : written)) return true;
    end = std::max(end, p.end);
    if (p.written) written = std::max(written, p.end);
  }
  return false;
}

int check_tensors(const fiona_adamw_desc &D, uint64_t &chunks) {
  const uint64_t e = type_size(D.type);
  const bool small = D.state_bits == 8;
  std::vector<Piece> pieces;
  chunks = 0;
  for (uint32_t i = 0; i < D.n_tensor; ++i) {
    const fiona_adamw_tensor &T = D.tensors[i];
    if (!(T.weight_decay >= 0) || !std::isfinite((float)T.weight_decay)) return FIONA_ERR_ARG;
    if (!T.n) continue;
    if (T.n >= (uint64_t)1 << 40) return FIONA_ERR_UNSUPPORTED;
    if (!T.param || !T.grad || !T.m || !T.v || (T.m_scale != nullptr) != small || (T.v_scale != nullptr) != small)
      return FIONA_ERR_ARG;
    if (T.master && D.type == FIONA_F32) return FIONA_ERR_ARG;
    const uint64_t s = small ? 1 : 4, blocks = (T.n + FIONA_ADAMW_BLOCK - 1) / FIONA_ADAMW_BLOCK;
    if (misaligned(T.param, e) || misaligned(T.grad, e) || misaligned(T.master, 4) || misaligned(T.m, s) || misaligned(T.v, s) ||
        misaligned(T.m_scale, 4) || misaligned(T.v_scale, 4))
      return FIONA_ERR_ALIGN;
    auto add = [&](const void *p, uint64_t bytes, bool written) {
      if (p) pieces.push_back({(uint64_t)p, (uint64_t)p + bytes, written});
    };
    add(T.param, T.n * e, true), add(T.grad, T.n * e, false), add(T.master, T.n * 4, true);
    add(T.m, T.n * s, true), add(T.v, T.n * s, true), add(T.m_scale, blocks * 4, true), add(T.v_scale, blocks * 4, true);
    chunks += (T.n + fiona::kChunk - 1) / fiona::kChunk;
  }
  if (chunks >= 1u << 24) return FIONA_ERR_UNSUPPORTED;   // (times 256 threads: below 2^32)
  return pieces_overlap(pieces) ? FIONA_ERR_ALIAS : FIONA_OK;
}

int make(const fiona_adamw_desc &D, fiona_adamw *H) {
  uint64_t n_chunk = 0;
  const int rc = check_tensors(D, n_chunk);
  if (rc != FIONA_OK) return rc;
  std::vector<fiona::AdamwChunk> chunks;
  chunks.reserve(n_chunk);
  const uint64_t e = type_size(D.type), s = D.state_bits == 8 ? 1 : 4, step = fiona::kChunk;
  uint64_t first = 0;
  for (uint32_t i = 0; i < D.n_tensor; ++i) {
    const fiona_adamw_tensor &T = D.tensors[i];
    auto at = [](const void *p, uint64_t bytes) { return p ? (char *)p + bytes : nullptr; };
    for (uint64_t k = 0; k < T.n; k += step) {
      const uint64_t b = k / FIONA_ADAMW_BLOCK * 4;
      chunks.push_back({at(T.param, k * e), at(T.grad, k * e), (float *)at(T.master, k * 4), at(T.m, k * s), at(T.v, k * s),
                        (float *)at(T.m_scale, b), (float *)at(T.v_scale, b), (uint32_t)std::min(step, T.n - k),
                        (uint32_t)(first + k), (float)T.weight_decay});
    }
    first += (T.n + FIONA_ADAMW_BLOCK - 1) / FIONA_ADAMW_BLOCK * FIONA_ADAMW_BLOCK;
  }
  if (hipGetDevice(&H->device) != hipSuccess) return FIONA_ERR_HIP;
  H->type = D.type, H->bits = D.state_bits;
  fiona::AdamwParams &P = H->P;
  P.n_chunk = (uint32_t)n_chunk, P.seed = D.seed;
  P.b1 = (float)D.beta1, P.a1 = (float)(1 - D.beta1), P.b2 = (float)D.beta2, P.a2 = (float)(1 - D.beta2), P.eps = (float)D.eps;
  P.log_b1 = (float)std::log(D.beta1), P.log_b2 = (float)std::log(D.beta2);
  if (!n_chunk) return FIONA_OK;
  void *table = nullptr;
  if (hipMalloc(&table, n_chunk * sizeof(fiona::AdamwChunk)) != hipSuccess) {
    (void)hipGetLastError();
    return FIONA_ERR_NOMEM;
  }
  P.chunks = (fiona::AdamwChunk *)table;
  return hipMemcpy(table, chunks.data(), n_chunk * sizeof(fiona::AdamwChunk), hipMemcpyHostToDevice) == hipSuccess ? FIONA_OK
                                                                                                                   : FIONA_ERR_HIP;
}

}  // namespace

extern "C" {

int fiona_adamw_create(const fiona_adamw_desc *desc, fiona_adamw **out) {
  if (!out) return FIONA_ERR_ARG;
  *out = nullptr;
  if (!desc) return FIONA_ERR_ARG;
  const fiona_adamw_desc &D = *desc;
  if (!known_type(D.type) || (D.state_bits != 8 && D.state_bits != 32)) return FIONA_ERR_UNSUPPORTED;
  if (!(D.beta1 >= 0) || !(D.beta1 < 1) || !(D.beta2 >= 0) || !(D.beta2 < 1) || !((float)D.eps >= FLT_MIN) || !std::isfinite((float)D.eps) ||
      (D.n_tensor && !D.tensors))
    return FIONA_ERR_ARG;
  fiona_adamw *H = new (std::nothrow) fiona_adamw;
  if (!H) return FIONA_ERR_NOMEM;
  int rc;
  try {
    rc = make(D, H);
  } catch (const std::bad_alloc &) {
    rc = FIONA_ERR_NOMEM;
  }
  if (rc != FIONA_OK) {
    fiona_adamw_destroy(H);
    return rc;
  }
  *out = H;
  return FIONA_OK;
}

void fiona_adamw_destroy(fiona_adamw *H) {
  if (!H) return;
  if (H->P.chunks) (void)hipFree((void *)H->P.chunks);
  delete H;
}

int fiona_adamw_step(const fiona_adamw *H, const float *lr, const int32_t *step, const float *grad_scale, hipStream_t stream) {
  if (!H || !lr || !step) return FIONA_ERR_ARG;
  if (misaligned(lr, 4) || misaligned(step, 4) || misaligned(grad_scale, 4)) return FIONA_ERR_ALIGN;
  if (!H->P.n_chunk) return FIONA_OK;
  if (!on_device(H->device)) return FIONA_ERR_ARG;
  fiona::AdamwParams P = H->P;
  P.lr = lr, P.step = step, P.grad_scale = grad_scale;
  with_type(H->type, [&](auto t) {
    using T = decltype(t);
    if (H->bits == 8) hipLaunchKernelGGL((fiona::adamw_kernel<T, true>), dim3(P.n_chunk), dim3(256), 0, stream, P);
    else hipLaunchKernelGGL((fiona::adamw_kernel<T, false>), dim3(P.n_chunk), dim3(256), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
