// fiona_adapter_linear and fiona_adapter_backward (include/fiona.h): low-rank
// adapters of many requests beside a shared projection.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>

#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_adapters {
  fiona_adapters_desc desc{};
  int device = -1;
  float *h = nullptr, *g = nullptr;   // [max_tokens][max_rank] each
};

namespace fiona {

struct AdapterParams {
  const void *x, *A, *B, *base, *dy, *dx_base;
  void *y, *dx, *dA, *dB;
  float *h, *g;
  const int32_t *ids, *ranks;
  const float *scaling;
  uint64_t x_row, base_row, y_row, dy_row, dx_base_row, dx_row;
  uint32_t n_tok, n_adapter, R, d_in, d_out;
};

__device__ __forceinline__ uint32_t rank_of(const AdapterParams &P, int32_t a) {
  if (a < 0 || (uint32_t)a >= P.n_adapter) return 0;
  if (!P.ranks) return P.R;
  const int32_t r = P.ranks[a];
  return r < 0 ? 0 : (uint32_t)r > P.R ? P.R : (uint32_t)r;
}

// h[t][r] = A_a[r] . x_t and, in the backward pass, g[t][r] = c (B_a^T dy_t)[r]:
// one wavefront per value.
template <typename T>
__global__ void __launch_bounds__(64) adapter_inner_kernel(AdapterParams P) {
  const uint32_t t = blockIdx.x, r = blockIdx.y, lane = threadIdx.x;
  const int32_t a = P.ids[t];
  if (r >= rank_of(P, a)) return;
  float s = 0;
  if (blockIdx.z == 0) {
    for (uint32_t i = lane; i < P.d_in; i += 64)
      s += (float)((const T *)P.x)[t * P.x_row + i] * (float)((const T *)P.A)[((uint64_t)a * P.R + r) * P.d_in + i];
  } else {
    for (uint32_t i = lane; i < P.d_out; i += 64)
      s += (float)((const T *)P.dy)[t * P.dy_row + i] * (float)((const T *)P.B)[((uint64_t)a * P.d_out + i) * P.R + r];
    if (P.scaling) s *= P.scaling[a];
  }
  for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
  if (lane == 0) (blockIdx.z ? P.g : P.h)[(uint64_t)t * P.R + r] = s;
}

// y_t = base_t + c B_a h_t, or (backward) dx_t = dx_base_t + A_a^T g_t.
template <typename T>
__global__ void __launch_bounds__(256) adapter_outer_kernel(AdapterParams P, bool backward) {
  const uint32_t t = blockIdx.x, i = blockIdx.y * 256 + threadIdx.x, n = backward ? P.d_in : P.d_out;
  if (i >= n) return;
  const int32_t a = P.ids[t];
  const uint32_t rank = rank_of(P, a);
  float s = 0;
  for (uint32_t r = 0; r < rank; ++r)
    s += backward ? P.g[(uint64_t)t * P.R + r] * (float)((const T *)P.A)[((uint64_t)a * P.R + r) * P.d_in + i]
                  : P.h[(uint64_t)t * P.R + r] * (float)((const T *)P.B)[((uint64_t)a * P.d_out + i) * P.R + r];
  if (!backward && rank && P.scaling) s *= P.scaling[a];
  const T *base = (const T *)(backward ? P.dx_base : P.base);
  const uint64_t base_row = backward ? P.dx_base_row : P.base_row;
  if (base) s += (float)base[t * base_row + i];
  (backward ? (T *)P.dx + t * P.dx_row : (T *)P.y + t * P.y_row)[i] = (T)s;
}

// dA_a[r] = sum g_t[r] x_t, or dB_a[.][r] = c sum dy_t h_t[r].
template <typename T>
__global__ void __launch_bounds__(256) adapter_grad_kernel(AdapterParams P, bool of_b) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x, r = blockIdx.y, a = blockIdx.z, n = of_b ? P.d_out : P.d_in;
  if (i >= n) return;
  float s = 0;
  if (r < rank_of(P, (int32_t)a))
    for (uint32_t t = 0; t < P.n_tok; ++t) {
      if (P.ids[t] != (int32_t)a) continue;
      s += of_b ? P.h[(uint64_t)t * P.R + r] * (float)((const T *)P.dy)[t * P.dy_row + i]
                : P.g[(uint64_t)t * P.R + r] * (float)((const T *)P.x)[t * P.x_row + i];
    }
  if (of_b) {
    if (P.scaling) s *= P.scaling[a];
    ((T *)P.dB)[((uint64_t)a * P.d_out + i) * P.R + r] = (T)s;
  } else {
    ((T *)P.dA)[((uint64_t)a * P.R + r) * P.d_in + i] = (T)s;
  }
}

}  // namespace fiona

namespace {

// Checks what both calls share and fills the parameters.
int check_common(const fiona_adapters *H, const fiona_adapter_args *args, fiona::AdapterParams &P) {
  if (!H || !args) return FIONA_ERR_ARG;
  const fiona_adapters_desc &D = H->desc;
  const fiona_adapter_args &A = *args;
  if (A.n_tok > D.max_tokens) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type);
  if (A.n_tok && (!A.x || !A.ids)) return FIONA_ERR_ARG;
  if (D.n_adapter && D.max_rank && (!A.A || !A.B)) return FIONA_ERR_ARG;
  if (misaligned(A.x, e) || misaligned(A.A, e) || misaligned(A.B, e) || misaligned(A.ids, 4) ||
      misaligned(A.ranks, 4) || misaligned(A.scaling, 4))
    return FIONA_ERR_ALIGN;
  P.x = A.x, P.A = A.A, P.B = A.B, P.ids = A.ids, P.ranks = A.ranks, P.scaling = A.scaling;
  P.x_row = A.x_row;
  P.n_tok = A.n_tok, P.n_adapter = D.n_adapter, P.R = D.max_rank, P.d_in = D.d_in, P.d_out = D.d_out;
  P.h = H->h, P.g = H->g;
  return FIONA_OK;
}

Rows matrix(const void *p, uint64_t e, uint64_t n, uint64_t width, uint64_t row) {
  return Rows{p, e, width, {n, 1, 1}, {row, 0, 0}};
}

// FIONA_ERR_ALIAS where an output's rows overlap each other, another output
// or an input; `own` pairs (an output that may be its base itself) are passed
// over where pointer and row stride agree.
int check_alias(const Rows *in, int n_in, const Rows *out, int n_out, const int *own) {
  uint64_t elems;
  for (int i = 0; i < n_in; ++i)
    if (!empty(in[i]) && !span(in[i], elems)) return FIONA_ERR_ARG;
  for (int o = 0; o < n_out; ++o) {
    if (empty(out[o])) continue;
    if (!span(out[o], elems) || !rows_distinct(out[o])) return FIONA_ERR_ALIAS;
    for (int p = o + 1; p < n_out; ++p)
      if (may_overlap(out[o], out[p])) return FIONA_ERR_ALIAS;
    for (int i = 0; i < n_in; ++i) {
      if (own[o] == i && in[i].base == out[o].base && (in[i].stride[0] == out[o].stride[0] || in[i].n[0] == 1)) continue;
      if (may_overlap(out[o], in[i])) return FIONA_ERR_ALIAS;
    }
  }
  return FIONA_OK;
}

bool on_device(const fiona_adapters *H) {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && dev == H->device;
}

}  // namespace

extern "C" {

int fiona_adapters_create(const fiona_adapters_desc *desc, fiona_adapters **out) {
  if (!out) return FIONA_ERR_ARG;
  *out = nullptr;
  if (!desc) return FIONA_ERR_ARG;
  const fiona_adapters_desc &D = *desc;
  if (!known_type(D.type)) return FIONA_ERR_UNSUPPORTED;
  if (!D.n_adapter || !D.max_rank || !D.d_in || !D.d_out || !D.max_tokens) return FIONA_ERR_ARG;
  if (D.max_rank > FIONA_MAX_RANK || D.n_adapter > 65535 || D.d_in > (1u << 20) || D.d_out > (1u << 20) ||
      D.max_tokens > (1u << 22))
    return FIONA_ERR_UNSUPPORTED;
  fiona_adapters *H = new (std::nothrow) fiona_adapters;
  if (!H) return FIONA_ERR_NOMEM;
  H->desc = D;
  if (hipGetDevice(&H->device) != hipSuccess) {
    delete H;
    return FIONA_ERR_HIP;
  }
  const size_t words = (size_t)D.max_tokens * D.max_rank;
  if (hipMalloc((void **)&H->h, 2 * words * sizeof(float)) != hipSuccess) {
    (void)hipGetLastError();
    delete H;
    return FIONA_ERR_NOMEM;
  }
  H->g = H->h + words;
  *out = H;
  return FIONA_OK;
}

void fiona_adapters_destroy(fiona_adapters *H) {
  if (!H) return;
  if (H->h) (void)hipFree(H->h);
  delete H;
}

int fiona_adapter_linear(const fiona_adapters *H, const fiona_adapter_args *args, hipStream_t stream) {
  fiona::AdapterParams P{};
  int rc = check_common(H, args, P);
  if (rc != FIONA_OK) return rc;
  const fiona_adapter_args &A = *args;
  const fiona_adapters_desc &D = H->desc;
  if (A.n_tok == 0) return FIONA_OK;
  if (!A.y) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type), n = A.n_tok;
  if (misaligned(A.base, e) || misaligned(A.y, e)) return FIONA_ERR_ALIGN;
  const Rows in[] = {matrix(A.x, e, n, D.d_in, A.x_row), matrix(A.A, e, 1, (uint64_t)D.n_adapter * D.max_rank * D.d_in, 0),
                     matrix(A.B, e, 1, (uint64_t)D.n_adapter * D.max_rank * D.d_out, 0), matrix(A.ids, 4, 1, n, 0),
                     matrix(A.ranks, 4, 1, D.n_adapter, 0), matrix(A.scaling, 4, 1, D.n_adapter, 0),
                     matrix(A.base, e, n, D.d_out, A.base_row)};
  const Rows out[] = {matrix(A.y, e, n, D.d_out, A.y_row)};
  const int own[] = {6};
  if ((rc = check_alias(in, 7, out, 1, own)) != FIONA_OK) return rc;
  if (!on_device(H)) return FIONA_ERR_ARG;
  P.base = A.base, P.y = A.y, P.base_row = A.base_row, P.y_row = A.y_row;
  with_type(D.type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(fiona::adapter_inner_kernel<T>, dim3(A.n_tok, D.max_rank, 1), dim3(64), 0, stream, P);
    hipLaunchKernelGGL(fiona::adapter_outer_kernel<T>, dim3(A.n_tok, (D.d_out + 255) / 256), dim3(256), 0, stream, P, false);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

int fiona_adapter_backward(const fiona_adapters *H, const fiona_adapter_args *args, hipStream_t stream) {
  fiona::AdapterParams P{};
  int rc = check_common(H, args, P);
  if (rc != FIONA_OK) return rc;
  const fiona_adapter_args &A = *args;
  const fiona_adapters_desc &D = H->desc;
  if (!A.dA || !A.dB || (A.n_tok && (!A.dy || !A.dx))) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type), n = A.n_tok;
  if (misaligned(A.dy, e) || misaligned(A.dx_base, e) || misaligned(A.dx, e) || misaligned(A.dA, e) || misaligned(A.dB, e))
    return FIONA_ERR_ALIGN;
  const uint64_t wa = (uint64_t)D.n_adapter * D.max_rank * D.d_in, wb = (uint64_t)D.n_adapter * D.max_rank * D.d_out;
  const Rows in[] = {matrix(A.x, e, n, D.d_in, A.x_row), matrix(A.A, e, 1, wa, 0), matrix(A.B, e, 1, wb, 0),
                     matrix(A.ids, 4, 1, n, 0), matrix(A.ranks, 4, 1, D.n_adapter, 0),
                     matrix(A.scaling, 4, 1, D.n_adapter, 0), matrix(A.dy, e, n, D.d_out, A.dy_row),
                     matrix(A.dx_base, e, n, D.d_in, A.dx_base_row)};
  const Rows out[] = {matrix(A.dx, e, n, D.d_in, A.dx_row), matrix(A.dA, e, 1, wa, 0), matrix(A.dB, e, 1, wb, 0)};
  const int own[] = {7, -1, -1};
  if ((rc = check_alias(in, 8, out, 3, own)) != FIONA_OK) return rc;
  if (!on_device(H)) return FIONA_ERR_ARG;
  P.dy = A.dy, P.dx_base = A.dx_base, P.dx = A.dx, P.dA = A.dA, P.dB = A.dB;
  P.dy_row = A.dy_row, P.dx_base_row = A.dx_base_row, P.dx_row = A.dx_row;
  with_type(D.type, [&](auto t) {
    using T = decltype(t);
    if (A.n_tok) {
      hipLaunchKernelGGL(fiona::adapter_inner_kernel<T>, dim3(A.n_tok, D.max_rank, 2), dim3(64), 0, stream, P);
      hipLaunchKernelGGL(fiona::adapter_outer_kernel<T>, dim3(A.n_tok, (D.d_in + 255) / 256), dim3(256), 0, stream, P, true);
    }
    hipLaunchKernelGGL(fiona::adapter_grad_kernel<T>, dim3((D.d_in + 255) / 256, D.max_rank, D.n_adapter), dim3(256), 0,
                       stream, P, false);
    hipLaunchKernelGGL(fiona::adapter_grad_kernel<T>, dim3((D.d_out + 255) / 256, D.max_rank, D.n_adapter), dim3(256), 0,
                       stream, P, true);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
