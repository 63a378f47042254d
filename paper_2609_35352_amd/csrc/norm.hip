// fiona_layer_norm and fiona_layer_norm_backward (include/fiona.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>

#include "fiona.h"
#include "norm_kernel.hpp"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_norm {
  fiona_norm_desc desc{};
  int device = -1;
  float *part = nullptr;     // parts of dweight and dbias
};

namespace {

// Calls f with values of the rows' type and of the weights'.
template <typename F>
void with_types(uint32_t type, uint32_t weight_type, F f) {
  with_type(type, [&](auto t) {
    if (weight_type == type) f(t, t);
    else f(t, float{});
  });
}

int check_types(uint32_t type, uint32_t weight_type, uint32_t width) {
  if (!known_type(type) || (weight_type != type && weight_type != FIONA_F32)) return FIONA_ERR_UNSUPPORTED;
  if (!width) return FIONA_ERR_ARG;
  return width > FIONA_MAX_NORM_WIDTH ? FIONA_ERR_UNSUPPORTED : FIONA_OK;
}

// The wavefronts and pieces that hold rows of q pieces: f(waves, pieces a lane).  (Three
// quarters of a shape where they hold the row, us: 16384 rows of 1280 in bfloat16 33.2 / 30.6, 8192
// of 5120 64.3 / 58.2, 2048 of 20480 79 / 73.)  The widest shape of 32 bits spills 5 registers
// forwards; for dx see norm_grad_kernel.
template <int W, int NV>
struct Shape {
  static constexpr int kWaves = W, kPieces = NV;
};
template <typename T, typename F>
void with_shape(uint32_t q, F f) {
  if (q <= 64) f(Shape<1, 1>{});
  else if (q <= 128) f(Shape<1, 2>{});
  else if (q <= 192) f(Shape<1, 3>{});
  else if (q <= 256) f(Shape<1, 4>{});
  else if (q <= 512) f(Shape<4, 2>{});
  else if (q <= 768) f(Shape<4, 3>{});
  else if (q <= 1024) f(Shape<4, 4>{});
  else if (q <= 2048) f(Shape<16, 2>{});
  else if (q <= 3 * 1024) f(Shape<16, 3>{});
  else if (q <= 4096) f(Shape<16, 4>{});
  else if constexpr (sizeof(T) == 4) f(Shape<16, 8>{});
}

// The same in the backward pass with the weights' gradients, where a lane holds at most
// 16 elements: with their sums, weights and the next row that is a hundred registers
// (32 elements, rows of 16384, spilled: 413 us for 2048 of them in bfloat16, 353 in 32
// bits; a pass over columns takes 29 and 48 beside 55 and 92 for dx).  (Three quarters of
// a shape, us without the parts' sum: 16384 rows of 1280 in bfloat16 38.4 / 33.5, of 2560 72 / 58, 8192 of 5120
// 63.3 / 59.5, 2048 of 768 in 32 bits 9.3 / 8.5.)
constexpr uint32_t kMostSums = 8192;
template <typename T, typename F>
void with_grad_shape(uint32_t q, F f) {
  constexpr bool wide = sizeof(T) == 4;
  if (q <= 64) f(Shape<1, 1>{});
  else if (q <= 128) f(Shape<1, 2>{});
  else if (q <= 192) f(std::conditional_t<wide, Shape<1, 3>, Shape<3, 1>>{});
  else if (q <= 256) f(std::conditional_t<wide, Shape<1, 4>, Shape<4, 1>>{});
  else if (q <= 384) f(Shape<3, 2>{});
  else if (q <= 512) f(Shape<4, 2>{});
  else if (q <= 768) f(std::conditional_t<wide, Shape<4, 3>, Shape<6, 2>>{});
  else if (q <= 1024) f(std::conditional_t<wide, Shape<4, 4>, Shape<8, 2>>{});
  else if constexpr (wide) f(Shape<8, 4>{});
}

// Parts of the rows' sums: a workgroup's each, as many as are resident at once (rows of
// several wavefronts take all registers of a compute unit with eight; 512 / 1024 parts of one
// wavefront's rows, us with their sum: 2048 of 768 in 32 bits 13.2 / 17.7; 256 / 512 parts of the
// others': 8192 rows of 4096 in bfloat16 50.6 / 53.9, 4096 of 8192 50.9 / 57.7, 600 of 8192
// in binary16 16.4 / 23.2).
constexpr uint32_t kMostParts = 512;
uint32_t most_parts(uint32_t waves) { return waves == 1 ? kMostParts : 256; }
// Where a lane holds one piece of a row, many rows go two at a time, for the bytes in
// flight (one / two at a time, us without the parts' sum: 16384 of 1376 in bfloat16 47.6 / 39.9,
// 8192 of 2048 25.8 / 26.0, 1531 of 1373 8.4 / 9.3, 1000 of 2048 7.7 / 8.1).
constexpr uint32_t kTwoRows = 4096;
// The wavefronts of a row's group there, and the groups of a workgroup.
void grad_groups(uint32_t type, uint32_t d, uint32_t &waves, uint32_t &groups) {
  with_type(type, [&](auto t) {
    constexpr uint32_t E = fiona::kLaneElems<decltype(t)>;
    with_grad_shape<decltype(t)>((d + E - 1) / E, [&](auto s) {
      waves = decltype(s)::kWaves, groups = fiona::kGradGroups<decltype(s)::kWaves>;
    });
  });
}
constexpr uint32_t pitch_of(uint32_t d) { return (d + 3) / 4 * 4; }
bool by_columns(uint32_t type, uint32_t d) { return d < 16 / type_size(type) || d > kMostSums; }
// Rows that one workgroup goes through, so that no parts are left to add up: four for each
// of four groups (us on the GPU, one launch / two without the gap between them, which takes
// the host 2 us more: 5 rows of 768 in bfloat16 4.4 / 6.4, 16 6.2 / 6.4, 32 9.9 / 7.2).
// Of other rows one to a group.
uint32_t few_rows(uint32_t waves) { return waves == 1 ? 16 : 1; }
uint32_t parts_of(uint32_t type, uint32_t d, uint32_t n) {
  if (by_columns(type, d)) return std::max(1u, std::min(d > kMostSums ? 64 : kMostParts, (n + 15) / 16));
  uint32_t waves = 1, groups = 1;
  grad_groups(type, d, waves, groups);
  return n <= few_rows(waves) ? 1 : std::min(most_parts(waves), (n + groups - 1) / groups);
}

}  // namespace

extern "C" {

int fiona_layer_norm(const fiona_norm_args *args, hipStream_t stream) {
  if (!args) return FIONA_ERR_ARG;
  const fiona_norm_args &A = *args;
  int rc = check_types(A.type, A.weight_type, A.width);
  if (rc != FIONA_OK) return rc;
  if (!(A.eps > 0) || !std::isfinite(A.eps)) return FIONA_ERR_ARG;
  if (!A.n) return FIONA_OK;
  if (A.n > FIONA_MAX_NORM_ROWS) return FIONA_ERR_UNSUPPORTED;
  if (!A.x || !A.y) return FIONA_ERR_ARG;
  const uint64_t e = type_size(A.type), w = type_size(A.weight_type), n = A.n, d = A.width;
  if (misaligned(A.x, e) || misaligned(A.residual, e) || misaligned(A.y, e) || misaligned(A.total, e) ||
      misaligned(A.weight, w) || misaligned(A.bias, w) || misaligned(A.mean, 4) || misaligned(A.rstd, 4))
    return FIONA_ERR_ALIGN;
  const Rows in[] = {matrix(A.x, e, n, d, A.x_row), matrix(A.residual, e, n, d, A.residual_row), matrix(A.weight, w, 1, d, 0),
                     matrix(A.bias, w, 1, d, 0)};
  const Rows out[] = {matrix(A.y, e, n, d, A.y_row), matrix(A.total, e, n, d, A.total_row), matrix(A.mean, 4, 1, n, 0),
                      matrix(A.rstd, 4, 1, n, 0)};
  const uint32_t own[] = {3, 3, 0, 0};
  if ((rc = check_alias(in, 4, out, 4, own)) != FIONA_OK) return rc;
  const fiona::NormParams P{A.x, A.residual, A.weight, A.bias, A.y, A.total, A.mean, A.rstd,
                            A.x_row, A.residual_row, A.y_row, A.total_row, A.n, A.width, A.eps};
  with_types(A.type, A.weight_type, [&](auto t, auto v) {
    using T = decltype(t);
    using W = decltype(v);
    constexpr uint32_t E = fiona::kLaneElems<T>;
    if (A.width < E) {
      hipLaunchKernelGGL((fiona::norm_narrow_kernel<T, W>), dim3((A.n + 255) / 256), dim3(256), 0, stream, P);
      return;
    }
    with_shape<T>((A.width + E - 1) / E, [&](auto s) {
      constexpr int WAVES = decltype(s)::kWaves, NV = decltype(s)::kPieces, threads = fiona::kNormThreads<WAVES>;
      constexpr uint32_t rows = threads / 64 / WAVES;
      hipLaunchKernelGGL((fiona::norm_kernel<T, W, WAVES, NV>), dim3((A.n + rows - 1) / rows), dim3(threads), 0, stream, P);
    });
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

int fiona_norm_create(const fiona_norm_desc *desc, fiona_norm **out) {
  if (!out) return FIONA_ERR_ARG;
  *out = nullptr;
  if (!desc) return FIONA_ERR_ARG;
  const int rc = check_types(desc->type, desc->weight_type, desc->width);
  if (rc != FIONA_OK) return rc;
  if (!desc->max_rows) return FIONA_ERR_ARG;
  if (desc->max_rows > FIONA_MAX_NORM_ROWS) return FIONA_ERR_UNSUPPORTED;
  fiona_norm *H = new (std::nothrow) fiona_norm;
  if (!H) return FIONA_ERR_NOMEM;
  H->desc = *desc;
  if (hipGetDevice(&H->device) != hipSuccess) {
    delete H;
    return FIONA_ERR_HIP;
  }
  const uint64_t bytes = (uint64_t)parts_of(desc->type, desc->width, desc->max_rows) * 2 * pitch_of(desc->width) * sizeof(float);
  if (hipMalloc((void **)&H->part, bytes) != hipSuccess) {
    (void)hipGetLastError();
    delete H;
    return FIONA_ERR_NOMEM;
  }
  *out = H;
  return FIONA_OK;
}

void fiona_norm_destroy(fiona_norm *norm) {
  if (!norm) return;
  if (norm->part) (void)hipFree(norm->part);
  delete norm;
}

int fiona_layer_norm_backward(const fiona_norm *norm, const fiona_norm_backward_args *args, hipStream_t stream) {
  if (!norm || !args) return FIONA_ERR_ARG;
  const fiona_norm_desc &D = norm->desc;
  const fiona_norm_backward_args &A = *args;
  if (A.n > D.max_rows) return FIONA_ERR_ARG;
  if (A.n && (!A.dy || !A.x || !A.mean || !A.rstd || !A.dx)) return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type), w = type_size(D.weight_type), n = A.n, d = D.width;
  if (misaligned(A.dy, e) || misaligned(A.x, e) || misaligned(A.weight, w) || misaligned(A.mean, 4) || misaligned(A.rstd, 4) ||
      misaligned(A.dx_base, e) || misaligned(A.dx, e) || misaligned(A.dweight, w) || misaligned(A.dbias, w))
    return FIONA_ERR_ALIGN;
  const Rows in[] = {matrix(A.dy, e, n, d, A.dy_row), matrix(A.x, e, n, d, A.x_row), matrix(A.dx_base, e, n, d, A.dx_base_row),
                     matrix(A.weight, w, 1, d, 0), matrix(A.mean, 4, 1, n, 0), matrix(A.rstd, 4, 1, n, 0)};
  const Rows out[] = {matrix(A.dx, e, n, d, A.dx_row), matrix(A.dweight, w, 1, d, 0), matrix(A.dbias, w, 1, d, 0)};
  const uint32_t own[] = {7, 0, 0};
  const int rc = check_alias(in, 6, out, 3, own);
  if (rc != FIONA_OK) return rc;
  if (!on_device(norm->device)) return FIONA_ERR_ARG;
  const uint32_t parts = parts_of(D.type, D.width, A.n);
  const fiona::NormGradParams P{A.dy, A.x, A.weight, A.dx_base, A.mean, A.rstd, A.dx, A.dweight, A.dbias, norm->part,
                                A.dy_row, A.x_row, A.dx_base_row, A.dx_row, A.n, D.width, parts, pitch_of(D.width)};
  const bool sums = A.dweight || A.dbias, columns = by_columns(D.type, D.width);
  with_types(D.type, D.weight_type, [&](auto t, auto v) {
    using T = decltype(t);
    using W = decltype(v);
    constexpr uint32_t E = fiona::kLaneElems<T>;
    const uint32_t q = (D.width + E - 1) / E;
    if (sums && D.width < E)    // (before dx, which may be dy or x)
      hipLaunchKernelGGL(fiona::norm_narrow_column_kernel<T>, dim3(parts), dim3(64), 0, stream, P);
    else if (sums && columns)
      hipLaunchKernelGGL(fiona::norm_column_kernel<T>, dim3((q + 255) / 256, parts), dim3(256), 0, stream, P);
    if (D.width < E) {
      if (A.n) hipLaunchKernelGGL((fiona::norm_narrow_grad_kernel<T, W>), dim3((A.n + 255) / 256), dim3(256), 0, stream, P);
    } else if (sums && !columns) {
      with_grad_shape<T>(q, [&](auto s) {
        constexpr int WAVES = decltype(s)::kWaves, NV = decltype(s)::kPieces;
        const dim3 grid(parts), threads(64 * WAVES * fiona::kGradGroups<WAVES>);
        if constexpr (NV == 1) {
          if (A.n >= kTwoRows) {
            hipLaunchKernelGGL((fiona::norm_grads_kernel<T, W, WAVES, NV, 2>), grid, threads, 0, stream, P);
            return;
          }
        }
        hipLaunchKernelGGL((fiona::norm_grads_kernel<T, W, WAVES, NV, 1>), grid, threads, 0, stream, P);
      });
    } else if (A.n) {
      with_shape<T>(q, [&](auto s) {
        constexpr int WAVES = decltype(s)::kWaves, NV = decltype(s)::kPieces, threads = fiona::kNormThreads<WAVES>;
        constexpr uint32_t rows = threads / 64 / WAVES;
        hipLaunchKernelGGL((fiona::norm_grad_kernel<T, W, WAVES, NV>), dim3((A.n + rows - 1) / rows), dim3(threads), 0, stream, P);
      });
    }
    if (sums && (parts > 1 || columns)) hipLaunchKernelGGL(fiona::norm_sum_kernel<W>, dim3((2 * P.pitch + 63) / 64), dim3(1024), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
