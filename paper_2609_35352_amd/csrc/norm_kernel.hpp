// Kernels of fiona_layer_norm and fiona_layer_norm_backward.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fiona {

struct NormParams {
  const void *x, *residual, *weight, *bias;
  void *y, *total;
  float *mean, *rstd;
  uint64_t x_row, residual_row, y_row, total_row;
  uint32_t n, d;
  float eps;
};

struct NormGradParams {
  const void *dy, *x, *weight, *dx_base;
  const float *mean, *rstd;
  void *dx, *dweight, *dbias;
  uint64_t dy_row, x_row, dx_base_row, dx_row;
  uint32_t n, d;
};

// Sums of two values over a workgroup of 256, the same in every thread.
__device__ __forceinline__ float2 sum_256(float a, float b) {
  __shared__ float2 part[4];
  for (int k = 32; k; k >>= 1) a += __shfl_xor(a, k), b += __shfl_xor(b, k);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = {a, b};
  __syncthreads();
  return {part[0].x + part[1].x + (part[2].x + part[3].x), part[0].y + part[1].y + (part[2].y + part[3].y)};
}

// A workgroup to a row, read three times.
template <typename T, typename W>
__global__ void __launch_bounds__(256) norm_kernel(NormParams P) {
  const uint64_t t = blockIdx.x;
  const T *x = (const T *)P.x + t * P.x_row, *r = P.residual ? (const T *)P.residual + t * P.residual_row : nullptr;
  auto value = [&](uint32_t i) { return r ? (float)(T)((float)x[i] + (float)r[i]) : (float)x[i]; };
  float s = 0, q = 0;
  for (uint32_t i = threadIdx.x; i < P.d; i += 256) s += value(i);
  const float mean = sum_256(s, 0).x / P.d;
  for (uint32_t i = threadIdx.x; i < P.d; i += 256) {
    const float c = value(i) - mean;
    q += c * c;
  }
  const float rstd = 1 / sqrtf(sum_256(q, 0).x / P.d + P.eps);
  for (uint32_t i = threadIdx.x; i < P.d; i += 256) {
    const float v = value(i), w = P.weight ? (float)((const W *)P.weight)[i] : 1.f, b = P.bias ? (float)((const W *)P.bias)[i] : 0.f;
    if (P.total) ((T *)P.total)[t * P.total_row + i] = (T)v;
    ((T *)P.y)[t * P.y_row + i] = (T)((v - mean) * rstd * w + b);
  }
  if (threadIdx.x == 0) {
    if (P.mean) P.mean[t] = mean;
    if (P.rstd) P.rstd[t] = rstd;
  }
}

// A workgroup to a row, read twice.
template <typename T, typename W>
__global__ void __launch_bounds__(256) norm_grad_kernel(NormGradParams P) {
  const uint64_t t = blockIdx.x;
  const T *x = (const T *)P.x + t * P.x_row, *dy = (const T *)P.dy + t * P.dy_row;
  const float mean = P.mean[t], rstd = P.rstd[t];
  float s = 0, q = 0;
  for (uint32_t i = threadIdx.x; i < P.d; i += 256) {
    const float u = (float)dy[i] * (P.weight ? (float)((const W *)P.weight)[i] : 1.f);
    s += u, q += u * (((float)x[i] - mean) * rstd);
  }
  const float2 sums = sum_256(s, q);
  for (uint32_t i = threadIdx.x; i < P.d; i += 256) {
    const float u = (float)dy[i] * (P.weight ? (float)((const W *)P.weight)[i] : 1.f), xh = ((float)x[i] - mean) * rstd;
    const float dx = rstd * (u - sums.x / P.d - xh * (sums.y / P.d));
    ((T *)P.dx)[t * P.dx_row + i] = (T)(P.dx_base ? (float)((const T *)P.dx_base)[t * P.dx_base_row + i] + dx : dx);
  }
}

// A thread to a column.
template <typename T, typename W>
__global__ void __launch_bounds__(256) norm_weight_grad_kernel(NormGradParams P) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= P.d) return;
  float dw = 0, db = 0;
  for (uint64_t t = 0; t < P.n; ++t) {
    const float dy = (float)((const T *)P.dy)[t * P.dy_row + i];
    dw += dy * (((float)((const T *)P.x)[t * P.x_row + i] - P.mean[t]) * P.rstd[t]);
    db += dy;
  }
  if (P.dweight) ((W *)P.dweight)[i] = (W)dw;
  if (P.dbias) ((W *)P.dbias)[i] = (W)db;
}

}  // namespace fiona
