// Kernels of fiona_layer_norm and fiona_layer_norm_backward.
//
// A group of WAVES wavefronts holds a row, NV pieces of 16 bytes to a lane, so that
// every row is read once: the mean, the sum of the squared deviations from it (not the
// squares' mean less the mean's square, which loses what is small beside the mean) and
// the result come from registers.  In the backward pass
//     dx = rstd (u - mean u - xh mean(u xh)),  u = weight dy,  xh = (x - mean) rstd
// takes one pair of sums over the row, and dweight = sum dy xh, dbias = sum dy one pair
// over the rows for every column: each group of a workgroup goes through its share of the
// rows with its columns' sums in registers, the workgroup leaves one part of them, and a
// second launch adds the parts up, all in a fixed order.
//
// What bounds them: memory, at 10 to 15 operations for 4 to 16 bytes.  Measured: 16384
// rows of 4096 in bfloat16 with a residual (537 MB) 90 us, 6.0 TB/s where a copy reaches
// 5.2 (reads alone 7.0); its gradients for 8192 rows (269 MB, and 8 MB of parts each
// way) 46 us and 4.6 for the parts' sum, 6.0 TB/s; a step of 8 rows of 768 4.3 us, one
// launch and two dependent loads.  Rows read with the weights asked for before the sums
// instead of after them: 3.1 instead of 3.6 us for one row of 4096, 51 instead of 43 for
// 16384 of 1373 (fewer wavefronts fit).
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
  float *part;               // [parts][2][pitch]: sums of dy xh and of dy
  uint64_t dy_row, x_row, dx_base_row, dx_row;
  uint32_t n, d, parts, pitch;
};

// Workgroups: four wavefronts, or the sixteen of one group.
template <int WAVES>
constexpr int kNormThreads = WAVES > 4 ? 64 * WAVES : 256;
// With the weights' gradients: groups of a workgroup, whose sums become one part: 4 to 12
// wavefronts (groups of four wavefronts, two in 256 parts / one in 512, us with the parts' sum: 8192
// rows of 4096 in bfloat16 50.6 / 53.9, 8192 of 2048 30.4 / 33.5, 1531 of 1373 11.9 / 14.0; three spill,
// 49 and up; of three, four / three / two, without that sum: 16384 rows of 2560 58.5 / 57.5 / 70, of 1280 33.9 /
// 40 / 35; of six, two / one: 8192 of 6144 68.5 / 73).
template <int WAVES>
constexpr int kGradGroups = WAVES == 1 || WAVES == 3 ? 4 : WAVES == 4 || WAVES == 6 ? 2 : 1;

// Sums of N values over a group; `slot` alternates from call to call, so that one
// barrier is enough.
template <int WAVES, int N, int THREADS = kNormThreads<WAVES>>
__device__ __forceinline__ void group_sum(float (&x)[N], uint32_t slot) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i]);
  if constexpr (WAVES > 1) {
    __shared__ float part[2][THREADS / 64][N];
    const uint32_t w = wave_index();
    if (threadIdx.x % 64 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) part[slot][w][i] = x[i];
    __syncthreads();
    const uint32_t first = w / WAVES * WAVES;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = 0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += part[slot][first + k][i];
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
  const uint64_t t = (uint64_t)blockIdx.x * GROUPS + wave_index() / WAVES;
  if (t >= P.n) return;      // (groups of one wavefront, which meet at no barrier)
  const T *x = (const T *)P.x + t * P.x_row, *r = (const T *)P.residual + (P.residual ? t * P.residual_row : 0);
  u4 raw[NV], add[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) raw[k] = load_once(piece_at(x, (k * 64 * WAVES + lane) * E, d));
  if (P.residual) {
#pragma unroll
    for (int k = 0; k < NV; ++k) add[k] = load_once(piece_at(r, (k * 64 * WAVES + lane) * E, d));
  }
  float s[NV][E], sum[1] = {0}, square[1] = {0};
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
    for (int j = 0; j < E; ++j) sum[0] += s[k][j];
  }
  group_sum<WAVES>(sum, 0);
  const float mean = sum[0] / d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      s[k][j] -= mean;
      square[0] += at + j < d ? s[k][j] * s[k][j] : 0.f;
    }
  }
  group_sum<WAVES>(square, 1);
  const float rstd = 1 / sqrtf(square[0] / d + P.eps);
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

// A lane's elements of u = weight dy and xh.
template <typename T>
__device__ __forceinline__ void unpack_grad(u4 x, u4 dy, uint32_t at, uint32_t d, float mean, float rstd, const float (&w)[kLaneElems<T>],
                                            float (&u)[kLaneElems<T>], float (&xh)[kLaneElems<T>]) {
  unpack<T>(piece_fix<T>(x, at, d), xh);
  unpack<T>(piece_fix<T>(dy, at, d), u);
#pragma unroll
  for (int j = 0; j < (int)kLaneElems<T>; ++j) xh[j] = (xh[j] - mean) * rstd, u[j] *= w[j];
}

// A lane's piece of dx.
template <typename T>
__device__ __forceinline__ void store_grad(T *dx, uint32_t at, uint32_t d, bool based, u4 base, float rstd, float s1, float s2,
                                           const float (&u)[kLaneElems<T>], const float (&xh)[kLaneElems<T>]) {
  constexpr int E = kLaneElems<T>;
  if (at >= d) return;
  float v[E], more[E];
  if (based) unpack<T>(piece_fix<T>(base, at, d), more);
#pragma unroll
  for (int j = 0; j < E; ++j) {
    v[j] = rstd * (u[j] - s1 - xh[j] * s2);
    if (based) v[j] += more[j];
  }
  store_piece(dx, at, d, pack<T>(v));
}

// dx alone, a group to a row, read once.  (Where a lane holds 24 elements or fewer of it nothing
// spills; over 24576 elements of 16 bits 24 to 38 of a lane's registers do, over 16384 of 32 bits
// 153 of them: the elements unpacked for the sums are kept for the result.)
template <typename T, typename W, int WAVES, int NV>
__global__ void __launch_bounds__(kNormThreads<WAVES>) norm_grad_kernel(NormGradParams P) {
  constexpr int E = kLaneElems<T>, GROUPS = kNormThreads<WAVES> / 64 / WAVES;
  const uint32_t lane = threadIdx.x % (64 * WAVES), d = P.d;
  const uint64_t t = (uint64_t)blockIdx.x * GROUPS + wave_index() / WAVES;
  if (t >= P.n) return;
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
  float sum[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
    float w[E], u[E], xh[E];
    load_weights<T, W>(P.weight, at, d, 1.f, w);
    unpack_grad<T>(rx[k], rg[k], at, d, mean, rstd, w, u, xh);
#pragma unroll
    for (int j = 0; j < E; ++j) sum[0] += u[j], sum[1] += u[j] * xh[j];
  }
  group_sum<WAVES>(sum, 0);
  const float s1 = sum[0] / d, s2 = sum[1] / d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const uint32_t at = (k * 64 * WAVES + lane) * E;
    float w[E], u[E], xh[E];
    load_weights<T, W>(P.weight, at, d, 1.f, w);
    unpack_grad<T>(rx[k], rg[k], at, d, mean, rstd, w, u, xh);
    store_grad((T *)P.dx + t * P.dx_row, at, d, P.dx_base, rb[k], rstd, s1, s2, u, xh);
  }
}

// dx of R rows at a time of every gridDim-th, and this workgroup's part of the weights'
// gradients, which its lanes add up in registers over those rows.
template <typename T, typename W, int WAVES, int NV, int R>
__global__ void __launch_bounds__(64 * WAVES * kGradGroups<WAVES>) norm_grads_kernel(NormGradParams P) {
  constexpr int E = kLaneElems<T>, GROUPS = kGradGroups<WAVES>;
  const uint32_t lane = threadIdx.x % (64 * WAVES), group = wave_index() / WAVES, d = P.d;
  const float per = 1.f / d;
  const uint64_t step = (uint64_t)gridDim.x * GROUPS;
  // The next rows are on their way while these are computed (where none is left the
  // last one is taken along).
  u4 rx[R][NV], rg[R][NV], rb[R][NV];
  float mean[R], rstd[R];
  auto load = [&](uint64_t first) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint64_t t = first + i * step < P.n ? first + i * step : P.n - 1;
      const T *x = (const T *)P.x + t * P.x_row, *dy = (const T *)P.dy + t * P.dy_row;
      const T *base = (const T *)P.dx_base + (P.dx_base ? t * P.dx_base_row : 0);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const uint32_t at = (k * 64 * WAVES + lane) * E;
        rx[i][k] = load_once(piece_at(x, at, d)), rg[i][k] = load_once(piece_at(dy, at, d));
        if (P.dx_base) rb[i][k] = load_once(piece_at(base, at, d));
      }
      mean[i] = P.mean[t], rstd[i] = P.rstd[t];
    }
  };
  uint64_t first = (uint64_t)blockIdx.x * GROUPS;
  if (first < P.n) load(first + group);
  float w[NV][E], dw[NV][E], db[NV][E];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    load_weights<T, W>(P.weight, (k * 64 * WAVES + lane) * E, d, 1.f, w[k]);
#pragma unroll
    for (int j = 0; j < E; ++j) dw[k][j] = db[k][j] = 0;
  }
  for (uint32_t slot = 0; first < P.n; first += R * step, slot ^= 1) {
    const uint64_t t = first + group;
    float xh[R][NV][E], g[R][NV][E], m[R], r[R], sum[2 * R];
    u4 add[R][NV];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const uint32_t at = (k * 64 * WAVES + lane) * E;
        unpack<T>(piece_fix<T>(rx[i][k], at, d), xh[i][k]);
        unpack<T>(piece_fix<T>(rg[i][k], at, d), g[i][k]);
        add[i][k] = rb[i][k];
      }
      m[i] = mean[i], r[i] = rstd[i];
    }
    if (first + R * step < P.n) load(t + R * step);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool live = t + i * step < P.n;
      float s1 = 0, s2 = 0;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          xh[i][k][j] = (xh[i][k][j] - m[i]) * r[i];
          if (live) dw[k][j] += g[i][k][j] * xh[i][k][j], db[k][j] += g[i][k][j];
          g[i][k][j] *= w[k][j];
          s1 += g[i][k][j], s2 += g[i][k][j] * xh[i][k][j];
        }
      sum[2 * i] = s1, sum[2 * i + 1] = s2;
    }
    group_sum<WAVES, 2 * R, 64 * WAVES * GROUPS>(sum, slot);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (t + i * step >= P.n) continue;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        store_grad((T *)P.dx + (t + i * step) * P.dx_row, (k * 64 * WAVES + lane) * E, d, P.dx_base, add[i][k], r[i], sum[2 * i] * per,
                   sum[2 * i + 1] * per, g[i][k], xh[i][k]);
    }
  }
  // This workgroup's part, or with no other the gradients: its groups' sums, through LDS.
  if constexpr (GROUPS > 1) {
    __shared__ f4 sh[GROUPS - 1][2][64 * WAVES * NV * E / 4];
    if (group) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < E; j += 4) {
          const uint32_t at = (k * E + j) / 4 * 64 * WAVES + lane;
          sh[group - 1][0][at] = (f4){dw[k][j], dw[k][j + 1], dw[k][j + 2], dw[k][j + 3]};
          sh[group - 1][1][at] = (f4){db[k][j], db[k][j + 1], db[k][j + 2], db[k][j + 3]};
        }
    }
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < E; j += 4)
#pragma unroll
        for (int q = 0; q < GROUPS - 1; ++q) {
          const uint32_t at = (k * E + j) / 4 * 64 * WAVES + lane;
          const f4 a = sh[q][0][at], b = sh[q][1][at];
#pragma unroll
          for (int i = 0; i < 4; ++i) dw[k][j + i] += a[i], db[k][j + i] += b[i];
        }
  }
  float *part = P.part + (uint64_t)blockIdx.x * 2 * P.pitch;
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < E; j += 4) {
      const uint32_t at = (k * 64 * WAVES + lane) * E + j;
      if (at >= d) continue;      // (the pitch is in whole steps of 4)
      if (P.parts > 1) {
        *(f4 *)(part + at) = (f4){dw[k][j], dw[k][j + 1], dw[k][j + 2], dw[k][j + 3]};
        *(f4 *)(part + P.pitch + at) = (f4){db[k][j], db[k][j + 1], db[k][j + 2], db[k][j + 3]};
        continue;
      }
#pragma unroll
      for (int i = j; i < j + 4; ++i) {
        if (at + i - j >= d) continue;
        if (P.dweight) ((W *)P.dweight)[at + i - j] = (W)dw[k][i];
        if (P.dbias) ((W *)P.dbias)[at + i - j] = (W)db[k][i];
      }
    }
}

// The parts of dweight and dbias added up, 64 columns to a workgroup, its
// sixteen wavefronts a sixteenth of the parts each.
template <typename W>
__global__ void __launch_bounds__(1024) norm_sum_kernel(NormGradParams P) {
  __shared__ float sh[16][64];
  const uint32_t i = blockIdx.x * 64 + threadIdx.x % 64, w = wave_index(), columns = 2 * P.pitch;
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
  W *out = (W *)(i < P.pitch ? P.dweight : P.dbias);
  const uint32_t c = i < P.pitch ? i : i - P.pitch;
  if (out && c < P.d) out[c] = (W)s;
}

// Rows too long for their sums to stay in registers beside them: a part of the weights'
// gradients alone, a thread to a piece of columns, four rows of it in flight.
template <typename T>
__global__ void __launch_bounds__(256) norm_column_kernel(NormGradParams P) {
  constexpr int E = kLaneElems<T>, U = 4;
  const uint32_t at = (blockIdx.x * 256 + threadIdx.x) * E, d = P.d;
  if (at >= d) return;
  float dw[E], db[E];
#pragma unroll
  for (int j = 0; j < E; ++j) dw[j] = db[j] = 0;
  for (uint64_t first = blockIdx.y; first < P.n; first += U * gridDim.y) {
    u4 rx[U], rg[U];
    float mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint64_t t = first + u * gridDim.y < P.n ? first + u * gridDim.y : first;
      rx[u] = load_shared(piece_at((const T *)P.x + t * P.x_row, at, d)), rg[u] = load_shared(piece_at((const T *)P.dy + t * P.dy_row, at, d));
      mean[u] = P.mean[t], rstd[u] = P.rstd[t];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (first + u * gridDim.y >= P.n) continue;
      float x[E], g[E];
      unpack<T>(piece_fix<T>(rx[u], at, d), x);
      unpack<T>(piece_fix<T>(rg[u], at, d), g);
#pragma unroll
      for (int j = 0; j < E; ++j) dw[j] += g[j] * ((x[j] - mean[u]) * rstd[u]), db[j] += g[j];
    }
  }
  float *part = P.part + (uint64_t)blockIdx.y * 2 * P.pitch + at;
#pragma unroll
  for (int j = 0; j < E; j += 4) {
    if (at + j >= d) continue;      // (the pitch is in whole steps of 4)
    *(f4 *)(part + j) = (f4){dw[j], dw[j + 1], dw[j + 2], dw[j + 3]};
    *(f4 *)(part + P.pitch + j) = (f4){db[j], db[j + 1], db[j + 2], db[j + 3]};
  }
}

// Rows shorter than a piece: a thread to a column.
template <typename T>
__global__ void __launch_bounds__(64) norm_narrow_column_kernel(NormGradParams P) {
  const uint32_t i = threadIdx.x;
  if (i >= P.d) return;
  float dw = 0, db = 0;
  for (uint64_t t = blockIdx.x; t < P.n; t += gridDim.x) {
    const float dy = (float)((const T *)P.dy)[t * P.dy_row + i];
    dw += dy * (((float)((const T *)P.x)[t * P.x_row + i] - P.mean[t]) * P.rstd[t]);
    db += dy;
  }
  float *part = P.part + (uint64_t)blockIdx.x * 2 * P.pitch;
  part[i] = dw, part[P.pitch + i] = db;
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
