// Kernels of fiona_layer_norm and fiona_layer_norm_backward.
//
// A group of WAVES wavefronts holds a row, NV pieces of 16 bytes to a lane, so that
// every row is read once: mean, deviations and the result come from registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pieces.hpp"

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
  float *part;               // [parts][2][d]: sums of dy xh and of dy
  uint64_t dy_row, x_row, dx_base_row, dx_row;
  uint32_t n, d, parts;
};

// Workgroups: four wavefronts, or the sixteen of one group.
template <int WAVES>
constexpr int kNormThreads = WAVES > 4 ? 64 * WAVES : 256;

// Sums of two values over a group; `slot` alternates from call to call, so that one
// barrier is enough.
template <int WAVES>
__device__ __forceinline__ void group_sum(float &a, float &b, uint32_t slot) {
  a = wave_sum(a), b = wave_sum(b);
  if constexpr (WAVES > 1) {
    __shared__ float2 part[2][kNormThreads<WAVES> / 64];
    const uint32_t w = wave_index();
    if (threadIdx.x % 64 == 0) part[slot][w] = {a, b};
    __syncthreads();
    const uint32_t first = w / WAVES * WAVES;
    a = b = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) a += part[slot][first + i].x, b += part[slot][first + i].y;
  }
}

// The weights at a row's elements from `at` on; `other` without weights.
template <typename T, typename W>
__device__ __forceinline__ void load_weights(const void *weight, uint32_t at, uint32_t d, float other, float (&w)[kLaneElems<T>]) {
  constexpr int E = kLaneElems<T>, EW = kLaneElems<W>;
  if (!weight) {
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = other;
    return;
  }
#pragma unroll
  for (int k = 0; k < E / EW; ++k) {
    float part[EW];
    unpack<W>(piece_fix<W>(load_shared(piece_at((const W *)weight, at + k * EW, d)), at + k * EW, d), part);
#pragma unroll
    for (int j = 0; j < EW; ++j) w[k * EW + j] = part[j];
  }
}

template <typename T, typename W, int WAVES, int NV>
__global__ void __launch_bounds__(kNormThreads<WAVES>) norm_kernel(NormParams P) {
  constexpr int E = kLaneElems<T>, GROUPS = kNormThreads<WAVES> / 64 / WAVES;
  const uint32_t lane = threadIdx.x % (64 * WAVES), d = P.d;
  uint64_t t = (uint64_t)blockIdx.x * GROUPS + wave_index() / WAVES;
  const bool live = t < P.n;
  if (WAVES == 1 && !live) return;
  if (!live) t = P.n - 1;
  const T *x = (const T *)P.x + t * P.x_row, *r = (const T *)P.residual + (P.residual ? t * P.residual_row : 0);
  u4 raw[NV], add[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) raw[k] = load_once(piece_at(x, (k * 64 * WAVES + lane) * E, d));
  if (P.residual) {
#pragma unroll
    for (int k = 0; k < NV; ++k) add[k] = load_once(piece_at(r, (k * 64 * WAVES + lane) * E, d));
  }
  float s[NV][E], sum = 0, none = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
    raw[k] = piece_fix<T>(raw[k], at, d);
    unpack<T>(raw[k], s[k]);
    if (P.residual) {
      float more[E];
      unpack<T>(piece_fix<T>(add[k], at, d), more);
#pragma unroll
      for (int j = 0; j < E; ++j) s[k][j] += more[j];
      raw[k] = pack<T>(s[k]);
      unpack<T>(raw[k], s[k]);           // (what the backward pass finds is what is normalised)
    }
#pragma unroll
    for (int j = 0; j < E; ++j) sum += s[k][j];
  }
  group_sum<WAVES>(sum, none, 0);
  const float mean = sum / d;
  float square = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      s[k][j] -= mean;
      square += at + j < d ? s[k][j] * s[k][j] : 0.f;
    }
  }
  group_sum<WAVES>(square, none, 1);
  const float rstd = 1 / sqrtf(square / d + P.eps);
  if (!live) return;
  T *y = (T *)P.y + t * P.y_row, *total = (T *)P.total + (P.total ? t * P.total_row : 0);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
    if (at >= d) continue;
    float w[E], b[E];
    load_weights<T, W>(P.weight, at, d, 1.f, w);
    load_weights<T, W>(P.bias, at, d, 0.f, b);
    if (P.total) store_piece(total, at, d, raw[k]);
#pragma unroll
    for (int j = 0; j < E; ++j) w[j] = s[k][j] * rstd * w[j] + b[j];
    store_piece(y, at, d, pack<T>(w));
  }
  if (lane == 0) {
    if (P.mean) P.mean[t] = mean;
    if (P.rstd) P.rstd[t] = rstd;
  }
}

// dx row by row, and with SUMS this workgroup's part of the weights' gradients, which
// its lanes add up in registers over the rows they take.
template <typename T, typename W, int WAVES, int NV, bool SUMS>
__global__ void __launch_bounds__(kNormThreads<WAVES>) norm_grad_kernel(NormGradParams P) {
  constexpr int E = kLaneElems<T>, GROUPS = kNormThreads<WAVES> / 64 / WAVES;
  const uint32_t lane = threadIdx.x % (64 * WAVES), group = wave_index() / WAVES, d = P.d;
  const float per = 1.f / d;
  float w[NV][E], dw[SUMS ? NV : 1][E], db[SUMS ? NV : 1][E];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    load_weights<T, W>(P.weight, (k * 64 * WAVES + lane) * E, d, 1.f, w[k]);
    if (SUMS)
#pragma unroll
      for (int j = 0; j < E; ++j) dw[k][j] = db[k][j] = 0;
  }
  const uint64_t step = (uint64_t)gridDim.x * GROUPS;
  uint32_t slot = 0;
  // (a group without a row at the end goes along with the last one, for the barriers)
  for (uint64_t first = (uint64_t)blockIdx.x * GROUPS; first < P.n; first += step, slot ^= 1) {
    const bool live = first + group < P.n;
    const uint64_t t = live ? first + group : P.n - 1;
    const T *x = (const T *)P.x + t * P.x_row, *dy = (const T *)P.dy + t * P.dy_row;
    const T *base = (const T *)P.dx_base + (P.dx_base ? t * P.dx_base_row : 0);
    u4 rx[NV], rg[NV], rb[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t at = (k * 64 * WAVES + lane) * E;
      rx[k] = load_once(piece_at(x, at, d)), rg[k] = load_once(piece_at(dy, at, d));
      if (P.dx_base) rb[k] = load_once(piece_at(base, at, d));
    }
    const float mean = P.mean[t], rstd = P.rstd[t];
    float s1 = 0, s2 = 0;
    float xh[NV][E], g[NV][E];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t at = (k * 64 * WAVES + lane) * E;
      unpack<T>(piece_fix<T>(rx[k], at, d), xh[k]);
      unpack<T>(piece_fix<T>(rg[k], at, d), g[k]);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        xh[k][j] = (xh[k][j] - mean) * rstd;
        if (SUMS && live) dw[k][j] += g[k][j] * xh[k][j], db[k][j] += g[k][j];
        g[k][j] *= w[k][j];
        s1 += g[k][j], s2 += g[k][j] * xh[k][j];
      }
    }
    group_sum<WAVES>(s1, s2, slot);
    if (!live) continue;
    s1 *= per, s2 *= per;
    T *dx = (T *)P.dx + t * P.dx_row;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const uint32_t at = (k * 64 * WAVES + lane) * E;
      if (at >= d) continue;
      float add[E];
      if (P.dx_base) unpack<T>(piece_fix<T>(rb[k], at, d), add);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float v = rstd * (g[k][j] - s1 - xh[k][j] * s2);
        g[k][j] = P.dx_base ? add[j] + v : v;
      }
      store_piece(dx, at, d, pack<T>(g[k]));
    }
  }
  if constexpr (SUMS) {
    // The groups' sums one after another through LDS, then this workgroup's part.
    float *part = P.part + (uint64_t)blockIdx.x * 2 * d;
    if constexpr (GROUPS > 1) {
      __shared__ float sh[2][64 * WAVES * NV * E];
      for (int q = 0; q < GROUPS; ++q) {
        if (group == (uint32_t)q)
#pragma unroll
          for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < E; ++j) {
              const uint32_t at = (k * 64 * WAVES + lane) * E + j;
              sh[0][at] = q ? sh[0][at] + dw[k][j] : dw[k][j];
              sh[1][at] = q ? sh[1][at] + db[k][j] : db[k][j];
            }
        __syncthreads();
      }
      for (uint32_t i = threadIdx.x; i < d; i += kNormThreads<WAVES>) part[i] = sh[0][i], part[d + i] = sh[1][i];
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const uint32_t at = (k * 64 * WAVES + lane) * E + j;
          if (at < d) part[at] = dw[k][j], part[d + at] = db[k][j];
        }
    }
  }
}

// The parts of dweight and dbias added up, 64 columns to a workgroup, its
// sixteen wavefronts a sixteenth of the parts each.
template <typename W>
__global__ void __launch_bounds__(1024) norm_sum_kernel(NormGradParams P) {
  __shared__ float sh[16][64];
  const uint32_t i = blockIdx.x * 64 + threadIdx.x % 64, w = wave_index(), columns = 2 * P.d;
  float s = 0;
  if (i < columns) {
#pragma unroll 8
    for (uint32_t p = w; p < P.parts; p += 16) s += P.part[(uint64_t)p * columns + i];
  }
  sh[w][threadIdx.x % 64] = s;
  __syncthreads();
  if (w || i >= columns) return;
  s = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += sh[k][threadIdx.x];
  W *out = (W *)(i < P.d ? P.dweight : P.dbias);
  if (out) out[i < P.d ? i : i - P.d] = (W)s;
}

// Rows shorter than a piece, or too long for their sums to stay in registers: a part of
// the weights' gradients for 256 columns, a thread to a column.
template <typename T>
__global__ void __launch_bounds__(256) norm_column_kernel(NormGradParams P) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= P.d) return;
  float dw = 0, db = 0;
  for (uint64_t t = blockIdx.y; t < P.n; t += gridDim.y) {
    const float dy = (float)((const T *)P.dy)[t * P.dy_row + i];
    dw += dy * (((float)((const T *)P.x)[t * P.x_row + i] - P.mean[t]) * P.rstd[t]);
    db += dy;
  }
  float *part = P.part + (uint64_t)blockIdx.y * 2 * P.d;
  part[i] = dw, part[P.d + i] = db;
}

// Rows shorter than a piece: a thread to a row.
template <typename T, typename W>
__global__ void __launch_bounds__(256) norm_narrow_kernel(NormParams P) {
  const uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= P.n) return;
  constexpr int E = kLaneElems<T>;
  const T *x = (const T *)P.x + t * P.x_row, *r = (const T *)P.residual + (P.residual ? t * P.residual_row : 0);
  float s[E], sum = 0, square = 0;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    s[j] = 0;
    if (j < (int)P.d) s[j] = P.residual ? (float)(T)((float)x[j] + (float)r[j]) : (float)x[j];
    sum += s[j];
  }
  const float mean = sum / P.d;
#pragma unroll
  for (int j = 0; j < E; ++j) square += j < (int)P.d ? (s[j] - mean) * (s[j] - mean) : 0.f;
  const float rstd = 1 / sqrtf(square / P.d + P.eps);
#pragma unroll
  for (int j = 0; j < E; ++j) {
    if (j >= (int)P.d) continue;
    const float w = P.weight ? (float)((const W *)P.weight)[j] : 1.f, b = P.bias ? (float)((const W *)P.bias)[j] : 0.f;
    if (P.total) ((T *)P.total)[t * P.total_row + j] = (T)s[j];
    ((T *)P.y)[t * P.y_row + j] = (T)((s[j] - mean) * rstd * w + b);
  }
  if (P.mean) P.mean[t] = mean;
  if (P.rstd) P.rstd[t] = rstd;
}

template <typename T, typename W>
__global__ void __launch_bounds__(256) norm_narrow_grad_kernel(NormGradParams P) {
  const uint64_t t = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= P.n) return;
  constexpr int E = kLaneElems<T>;
  const T *x = (const T *)P.x + t * P.x_row, *dy = (const T *)P.dy + t * P.dy_row;
  const T *base = (const T *)P.dx_base + (P.dx_base ? t * P.dx_base_row : 0);
  const float mean = P.mean[t], rstd = P.rstd[t];
  float g[E], xh[E], s1 = 0, s2 = 0;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    g[j] = xh[j] = 0;
    if (j < (int)P.d) g[j] = (float)dy[j] * (P.weight ? (float)((const W *)P.weight)[j] : 1.f), xh[j] = ((float)x[j] - mean) * rstd;
    s1 += g[j], s2 += g[j] * xh[j];
  }
  s1 /= P.d, s2 /= P.d;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    if (j >= (int)P.d) continue;
    const float v = rstd * (g[j] - s1 - xh[j] * s2);
    ((T *)P.dx)[t * P.dx_row + j] = (T)(P.dx_base ? (float)base[j] + v : v);
  }
}

}  // namespace fiona
