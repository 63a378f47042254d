// fiona_adapter_linear and fiona_adapter_backward (include/fiona.h): low-rank
// adapters of many requests beside a shared projection.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <type_traits>

#include "adapter_kernel.hpp"
#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_adapters {
  fiona_adapters_desc desc{};
  int device = -1;
  uint32_t RP = 0;                       // ranks in whole tiles
  uint64_t part_cap = 0, grad_splits = 1;
  char *ws = nullptr;
  // Into ws.  part: sums of h and g; g: whole g; column: h and g by rank; AT, BT:
  // the factors transposed; grad: a split's gradients; ids: whole steps of them.
  float *part[2] = {}, *g = nullptr, *grad[2] = {};
  void *column[2] = {}, *AT = nullptr, *BT = nullptr;
  int32_t *ids = nullptr;
};

// Rows below kMinWidth elements can be shorter than a lane's 16 bytes, which the
// tiled kernels may always read: one value per wavefront or thread.  Right, and slow
// where the other side is wide or the tokens are many: a gradient's thread goes
// through all of them (bfloat16, rank 16: 8192 tokens of 4096 x 4 325 us, a training
// step of them 3.3 ms, of 512 182 us).
constexpr uint32_t kMinWidth = 8;

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
  if (A.n_tok > 1 && A.x_row > fiona::kMaxStride) return FIONA_ERR_UNSUPPORTED;
  if (D.n_adapter && D.max_rank && (!A.A || !A.B)) return FIONA_ERR_ARG;
  if (misaligned(A.x, e) || misaligned(A.A, e) || misaligned(A.B, e) || misaligned(A.ids, 4) ||
      misaligned(A.ranks, 4) || misaligned(A.scaling, 4))
    return FIONA_ERR_ALIGN;
  P.x = A.x, P.A = A.A, P.B = A.B, P.ids = A.ids, P.ranks = A.ranks, P.scaling = A.scaling;
  P.x_row = A.x_row;
  P.n_tok = A.n_tok, P.n_adapter = D.n_adapter, P.R = D.max_rank, P.d_in = D.d_in, P.d_out = D.d_out;
  P.h = H->part[0], P.g = H->part[1];
  return FIONA_OK;
}

bool narrow(const fiona_adapters_desc &D) { return D.d_in < kMinWidth || D.d_out < kMinWidth; }

uint32_t blocks_of(uint64_t n) { return (uint32_t)((n + fiona::kRows - 1) / fiona::kRows); }

// Workgroups that share the adapters among 64 tokens: 256 over the blocks, as
// with few tokens each may have its own; two at least, for the blocks in which
// one request ends and the next begins.  Calls of 4096 x 4096 at rank 16, us, with
// 128 / 256 / 512 over the blocks: 1024 tokens of 64 requests 20.6 / 20.5 / 20.7; 4096
// of 200 44.2 / 51.3 / 54.1; 8192 of 12 46.9 / 46.9 / 59.3, of 400 81 / 81 / 99; 16384
// of 30 131 with one at least, 118 with two.
uint32_t slots_of(uint32_t n, uint32_t adapters) {
  const uint32_t want = std::max(2u, 256 / blocks_of(n));
  return std::min({want, adapters, std::min(n, fiona::kRows)});
}

// Parts of a row's contraction: enough workgroups to fill the GPU, and not so
// many that adding them up costs more (us with 256 / 512 / 1024 workgroups: 8192
// tokens of 4096, rank 16, 49.2 / 47.1 / 50.1; 613 of 1000, 20, 23.4 / 22.1 / 22.3;
// a training step of 8192 of 4096, 64, 156.0 / 151.0 / 161.9; with at most 1 / 2 /
// 4 / 8 parts: 16 of 4096, rank 16, 21.0 / 15.3 / 12.3 / 11.3).
constexpr uint32_t kMaxSplits = 8, kWorkgroups = 512;
uint32_t splits_of(uint32_t n, uint32_t adapters) {
  const uint32_t slots = slots_of(n, adapters), wgs = blocks_of(n) * (slots > 2 ? slots : 1);
  return std::max(1u, std::min(kMaxSplits, (kWorkgroups + wgs - 1) / wgs));
}

uint32_t grad_slices(uint32_t n, uint32_t type, uint32_t RP) {
  const uint32_t cols = 16 * (type == FIONA_F32 ? fiona::grad_width<float>(RP) : fiona::grad_width<__bf16>(RP));
  return (n + cols - 1) / cols;
}

// Parts of the tokens in the gradients' sums, where their columns alone do not
// fill the GPU (us with 256 / 512 / 1024 workgroups: 2048 tokens of 768, rank 8,
// 34.9 / 34.7 / 35.7; 8192 of 4096, 64, 150.7 / 151.0 / 177.2).
constexpr uint32_t kGradWorkgroups = 512;
uint32_t grad_splits_of(const fiona_adapters_desc &D, uint32_t RP, uint32_t n) {
  const uint64_t wgs = (uint64_t)(grad_slices(D.d_in, D.type, RP) + grad_slices(D.d_out, D.type, RP)) * D.n_adapter * ((RP + 63) / 64);
  const uint64_t want = (kGradWorkgroups + wgs - 1) / wgs;
  return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(want, (n + 255) / 256));
}

template <typename F>
void with_tiles(uint32_t RP, F f) {
  if (RP == 16) f(std::integral_constant<int, 1>{});
  else if (RP == 32) f(std::integral_constant<int, 2>{});
  else if (RP == 64) f(std::integral_constant<int, 4>{});
  else f(std::integral_constant<int, 8>{});
}

template <typename T>
void launch_shrink(const fiona_adapters *H, const fiona::AdapterIds &I, const fiona::ShrinkSide *sides, uint32_t n_sides,
                   uint32_t splits, hipStream_t stream) {
  fiona::ShrinkParams P{};
  P.I = I, P.splits = splits, P.slots = slots_of(I.n_tok, I.n_adapter);
  for (uint32_t i = 0; i < n_sides; ++i) P.side[i] = sides[i];
  with_tiles(H->RP, [&](auto rt) {
    constexpr int RT = decltype(rt)::value;
    const dim3 grid(blocks_of(I.n_tok), splits, P.slots * n_sides);
    if (n_sides == 1) hipLaunchKernelGGL((fiona::shrink_kernel<T, RT, true>), grid, dim3(256), 0, stream, P);
    else hipLaunchKernelGGL((fiona::shrink_kernel<T, RT, false>), grid, dim3(256), 0, stream, P);
  });
}

// Whether the sums of h and g share a launch with expand, which then adds up g's
// parts by itself in every slice of columns: for small ranks, where those are few.
// A training step apart / together, us: rank 8 of 768, 13 tokens 25.1 / 19.7, 2048
// 38.5 / 34.6; of 4096, rank 16, 8192 tokens 122.8 / 118.4; rank 32, 1024 tokens 48.1 /
// 43.6, 8192 125.1 / 125.0; rank 64, 64 tokens 37.5 / 36.7, 512 46.9 / 46.5, 1024 59.7 /
// 62.8, 8192 150.7 / 158.1; rank 128, 64 tokens 53.7 / 56.8, 512 75.8 / 88.5.
constexpr bool together(uint32_t RP) { return RP <= 32; }

template <typename T, bool INNER>
void launch_expand(const fiona_adapters *H, fiona::ExpandParams P, hipStream_t stream) {
  const uint32_t n = P.I.n_tok, steps = (P.O + 255) / 256;
  P.slots = slots_of(n, P.I.n_adapter + 1);
  // (512 / 1024 / 2048 workgroups, us of the whole call: 8192 tokens of 4096, rank 16, 47.1 / 47.7 / 51.4;
  // a training step at rank 64 151.0 / 150.4 / 156.0)
  const uint32_t wgs = blocks_of(n), slices = std::max(1u, std::min(steps, (kWorkgroups + wgs - 1) / wgs));
  P.slice = (steps + slices - 1) / slices * 256;
  const dim3 grid((P.O + P.slice - 1) / P.slice, blocks_of(n), P.slots);
  if (INNER) P.inner_z = (2 * ((P.inner.RP + 31) / 32) + grid.x - 1) / grid.x;
  with_tiles(H->RP, [&](auto rt) {
    constexpr int RT = decltype(rt)::value;
    if constexpr (!INNER || together(16 * RT))
      hipLaunchKernelGGL((fiona::expand_kernel<T, RT, INNER>), dim3(grid.x, grid.y, grid.z + P.inner_z), dim3(256), 0, stream, P);
  });
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
  if (D.max_rank > FIONA_MAX_RANK || D.n_adapter > 32767 || D.d_in > (1u << 20) || D.d_out > (1u << 20) ||
      D.max_tokens > (1u << 21))
    return FIONA_ERR_UNSUPPORTED;
  fiona_adapters *H = new (std::nothrow) fiona_adapters;
  if (!H) return FIONA_ERR_NOMEM;
  H->desc = D;
  if (hipGetDevice(&H->device) != hipSuccess) {
    delete H;
    return FIONA_ERR_HIP;
  }
  H->RP = D.max_rank <= 16 ? 16 : D.max_rank <= 32 ? 32 : D.max_rank <= 64 ? 64 : 128;
  const bool both = !(D.flags & FIONA_ADAPTERS_FORWARD_ONLY);
  const uint64_t e = type_size(D.type), n_pad = (uint64_t)blocks_of(D.max_tokens) * 64, RP = H->RP;
  for (uint32_t n = std::min(64u, D.max_tokens);; n = std::min(n + 64, D.max_tokens)) {
    H->part_cap = std::max<uint64_t>(H->part_cap, (uint64_t)n * splits_of(n, D.n_adapter));
    if (n == D.max_tokens) break;
  }
  H->part_cap = std::max<uint64_t>(H->part_cap, 64 * kMaxSplits);   // (fewer than 64 tokens)
  H->grad_splits = grad_splits_of(D, H->RP, D.max_tokens);
  // Sizes in order; every part starts at a multiple of 256 bytes.
  const uint64_t grads = (uint64_t)D.n_adapter * D.max_rank * 4 * (H->grad_splits > 1 ? H->grad_splits : 0);
  const uint64_t size[] = {H->part_cap * RP * 4, both ? H->part_cap * RP * 4 : 0,
                           both && !together(H->RP) ? D.max_tokens * RP * 4 : 0,
                           both ? n_pad * RP * 4 : 0, both ? n_pad * RP * 4 : 0,
                           both ? RP * D.n_adapter * D.d_in * e : 0, both ? RP * D.n_adapter * D.d_out * e : 0,
                           both ? grads * D.d_in : 0, both ? grads * D.d_out : 0, both ? n_pad * 4 : 0};
  uint64_t at[11] = {0};
  for (int i = 0; i < 10; ++i) at[i + 1] = at[i] + (size[i] + 255) / 256 * 256;
  if (hipMalloc((void **)&H->ws, at[10]) != hipSuccess) {
    (void)hipGetLastError();
    delete H;
    return FIONA_ERR_NOMEM;
  }
  H->part[0] = (float *)(H->ws + at[0]), H->part[1] = (float *)(H->ws + at[1]), H->g = (float *)(H->ws + at[2]);
  H->column[0] = H->ws + at[3], H->column[1] = H->ws + at[4], H->AT = H->ws + at[5], H->BT = H->ws + at[6];
  H->grad[0] = (float *)(H->ws + at[7]), H->grad[1] = (float *)(H->ws + at[8]), H->ids = (int32_t *)(H->ws + at[9]);
  *out = H;
  return FIONA_OK;
}

void fiona_adapters_destroy(fiona_adapters *H) {
  if (!H) return;
  if (H->ws) (void)hipFree(H->ws);
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
  if (n > 1 && (A.base_row > fiona::kMaxStride || A.y_row > fiona::kMaxStride)) return FIONA_ERR_UNSUPPORTED;
  const Rows in[] = {matrix(A.x, e, n, D.d_in, A.x_row), matrix(A.A, e, 1, (uint64_t)D.n_adapter * D.max_rank * D.d_in, 0),
                     matrix(A.B, e, 1, (uint64_t)D.n_adapter * D.max_rank * D.d_out, 0), matrix(A.ids, 4, 1, n, 0),
                     matrix(A.ranks, 4, 1, D.n_adapter, 0), matrix(A.scaling, 4, 1, D.n_adapter, 0),
                     matrix(A.base, e, n, D.d_out, A.base_row)};
  const Rows out[] = {matrix(A.y, e, n, D.d_out, A.y_row)};
  const uint32_t own[] = {1u << 6};
  if ((rc = check_alias(in, 7, out, 1, own)) != FIONA_OK) return rc;
  if (!on_device(H->device)) return FIONA_ERR_ARG;
  P.base = A.base, P.y = A.y, P.base_row = A.base_row, P.y_row = A.y_row;
  with_type(D.type, [&](auto t) {
    using T = decltype(t);
    if (!narrow(D)) {
      const uint32_t splits = splits_of(A.n_tok, D.n_adapter);
      const fiona::AdapterIds I{A.ids, A.ranks, A.n_tok, D.n_adapter, D.max_rank};
      const fiona::ShrinkSide side{A.x, A.A, H->part[0], A.x_row, D.d_in, D.max_rank};
      launch_shrink<T>(H, I, &side, 1, splits, stream);
      launch_expand<T, false>(H, fiona::ExpandParams{I, H->part[0], A.scaling, A.B, A.base, A.y, A.base_row, A.y_row, D.d_out,
                                              D.max_rank, splits}, stream);
      return;
    }
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
  if (D.flags & FIONA_ADAPTERS_FORWARD_ONLY) return FIONA_ERR_ARG;
  if (!A.dA || !A.dB || (A.n_tok && (!A.dy || !A.dx))) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type), n = A.n_tok;
  if (misaligned(A.dy, e) || misaligned(A.dx_base, e) || misaligned(A.dx, e) || misaligned(A.dA, e) || misaligned(A.dB, e))
    return FIONA_ERR_ALIGN;
  if (n > 1 && (A.dy_row > fiona::kMaxStride || A.dx_base_row > fiona::kMaxStride || A.dx_row > fiona::kMaxStride))
    return FIONA_ERR_UNSUPPORTED;
  const uint64_t wa = (uint64_t)D.n_adapter * D.max_rank * D.d_in, wb = (uint64_t)D.n_adapter * D.max_rank * D.d_out;
  const Rows in[] = {matrix(A.x, e, n, D.d_in, A.x_row), matrix(A.A, e, 1, wa, 0), matrix(A.B, e, 1, wb, 0),
                     matrix(A.ids, 4, 1, n, 0), matrix(A.ranks, 4, 1, D.n_adapter, 0),
                     matrix(A.scaling, 4, 1, D.n_adapter, 0), matrix(A.dy, e, n, D.d_out, A.dy_row),
                     matrix(A.dx_base, e, n, D.d_in, A.dx_base_row)};
  const Rows out[] = {matrix(A.dx, e, n, D.d_in, A.dx_row), matrix(A.dA, e, 1, wa, 0), matrix(A.dB, e, 1, wb, 0)};
  const uint32_t own[] = {1u << 7, 0, 0};
  if ((rc = check_alias(in, 8, out, 3, own)) != FIONA_OK) return rc;
  if (!on_device(H->device)) return FIONA_ERR_ARG;
  P.dy = A.dy, P.dx_base = A.dx_base, P.dx = A.dx, P.dA = A.dA, P.dB = A.dB;
  P.dy_row = A.dy_row, P.dx_base_row = A.dx_base_row, P.dx_row = A.dx_row;
  with_type(D.type, [&](auto t) {
    using T = decltype(t);
    if (!narrow(D)) {
      const uint32_t splits = splits_of(std::max(1u, A.n_tok), D.n_adapter), blocks = blocks_of(A.n_tok);
      const fiona::AdapterIds I{A.ids, A.ranks, A.n_tok, D.n_adapter, D.max_rank};
      if (A.n_tok) {
        hipLaunchKernelGGL(fiona::transpose_kernel<T>, dim3((D.d_in + 63) / 64 + (D.d_out + 63) / 64, D.n_adapter), dim3(256), 0,
                           stream, fiona::TransposeParams{I, A.A, A.B, H->AT, H->BT, D.d_in, D.d_out, H->RP});
        const fiona::ShrinkSide sides[2] = {{A.x, A.A, H->part[0], A.x_row, D.d_in, D.max_rank},
                                            {A.dy, H->BT, H->part[1], A.dy_row, D.d_out, H->RP}};
        launch_shrink<T>(H, I, sides, 2, splits, stream);
        fiona::InnerParams inner{I, {H->part[0], H->part[1]}, A.scaling, nullptr, H->ids, {H->column[0], H->column[1]},
                                 H->RP, blocks * 64, splits};
        fiona::ExpandParams E{I, H->part[1], A.scaling, H->AT, A.dx_base, A.dx, A.dx_base_row, A.dx_row, D.d_in, H->RP, splits};
        if (together(H->RP)) {
          E.inner = inner;
          launch_expand<T, true>(H, E, stream);
        } else {
          inner.g = H->g;
          hipLaunchKernelGGL(fiona::inner_kernel<T>, dim3(blocks, (H->RP + 31) / 32, 2), dim3(256), 0, stream, inner);
          E.part = H->g, E.scaling = nullptr, E.splits = 1;
          launch_expand<T, false>(H, E, stream);
        }
      }
      const uint32_t RP = H->RP;
      fiona::GradParams G{};
      G.I = I, G.ids = H->ids, G.RP = H->RP, G.n_pad = blocks * 64, G.r_chunks = (H->RP + 63) / 64;
      G.splits = (uint32_t)std::min<uint64_t>(H->grad_splits, grad_splits_of(D, H->RP, A.n_tok));
      G.per_split = (std::max(1u, A.n_tok) + G.splits * 64 - 1) / (G.splits * 64) * 64;
      G.side[0] = {A.x, H->column[1], A.dA, H->grad[0], A.x_row, D.d_in, grad_slices(D.d_in, D.type, RP)};
      G.side[1] = {A.dy, H->column[0], A.dB, H->grad[1], A.dy_row, D.d_out, grad_slices(D.d_out, D.type, RP)};
      const dim3 grid(G.side[0].slices + G.side[1].slices, D.n_adapter * G.r_chunks, G.splits);
      if (H->RP == 16) hipLaunchKernelGGL((fiona::grad_kernel<T, 1>), grid, dim3(256), 0, stream, G);
      else if (H->RP == 32) hipLaunchKernelGGL((fiona::grad_kernel<T, 2>), grid, dim3(256), 0, stream, G);
      else hipLaunchKernelGGL((fiona::grad_kernel<T, 4>), grid, dim3(256), 0, stream, G);
      if (G.splits > 1)
        hipLaunchKernelGGL(fiona::grad_sum_kernel<T>, dim3((uint32_t)((wa + wb + 255) / 256)), dim3(256), 0, stream,
                           fiona::GradSumParams{{H->grad[0], H->grad[1]}, {A.dA, A.dB}, {wa, wb}, G.splits});
      return;
    }
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
