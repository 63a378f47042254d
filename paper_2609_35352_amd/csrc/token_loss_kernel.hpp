// Kernels of fiona_preference_loss and fiona_policy_loss.
//
// A row's log sum of exponentials in parts, as a softmax over a long axis: a part with
// elements J has m_J = max z_j and s_J = sum exp(z_j - m_J), and two parts join as
// m = max(m_1, m_2), s = sum_i s_i exp(m_i - m).  Exponentials are to base 2, of the
// difference of two logits, taken before it is scaled (a scaled maximum, rounded, would be
// off by 2^-24 of itself).
//
// The policy loss of a token depends on its own row alone: where there are enough rows, or
// short ones, a workgroup holds one in its registers, packed, and reads it once.  The
// preference loss needs every row of a pair before the first of their gradients: parts,
// then pairs, then gradients, in three launches, and rows read twice.  Long rows that are
// few are split over workgroups in either.
//
// What bounds them: memory, and the vector units close behind (an exponential takes four
// issue slots; parts of bfloat16 rows keep them 55% busy).  Measured: 2700 rows of 131072
// in bfloat16 read and written once (1.49 GB with 300 rows of zeros) 281 us, 5.3 TB/s, 8000 of
// 32000 (1.02 GB) 172, 6.0; 7955
// rows of 32768 74 us for the parts (419 MB, 5.7 TB/s), 6 for the pairs, 151 for the
// gradients (419 MB again and 521 MB written, 6.2 TB/s: the rows read last are the first
// again, some of them still in the memory-side cache; read past the caches in both passes
// 66 and 165).  24 rows of 50021 in 32 bits: 4.0 and 4.6 us, each one launch and its chain
// of loads.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pieces.hpp"

namespace fiona {

constexpr float kLossLog2e = 1.4426950408889634f, kLossLn2 = 0.6931471805599453f;
constexpr uint32_t kLossSplits = 64;   // parts of one row

struct TokenParams {
  const void *z;
  void *dz;
  const int32_t *targets;
  float2 *part;                   // [n_tok][splits]: maximum and sum of a part of a row
  float2 *lse;                    // [n_tok]: log sum of exponentials (see log_sum)
  float *at_target, *coef;        // [n_tok]: the target's logit, derivative of the loss
  uint64_t z_row, dz_row;
  uint32_t n_tok, vocab;
  uint32_t splits, slice;         // parts of a row, and their pieces
  uint32_t skew;                  // elements of a line less one (see before)
};

struct PairParams {
  const int32_t *offsets;
  const float *reference, *weights;
  float *loss, *logps;
  float beta, smoothing;
  uint32_t n_pair;
};

struct PolicyParams {
  const float *old, *advantages, *reference, *weights;
  float *loss, *logps;
  float clip_low, clip_high, kl;
};

// The policy loss of a token with log-probability l, and its derivative.
__device__ __forceinline__ float policy_of(const PolicyParams &Q, uint32_t n_tok, uint32_t t, float l, float &loss) {
  const float w = Q.weights ? Q.weights[t] : 1.f / n_tok, a = Q.advantages[t], x = l - Q.old[t], r = expf(x);
  if (w == 0) return loss = 0;
  // (a ratio beyond 2^128 is infinite here, but its product with no advantage is zero)
  const float open = a == 0 && x < INFINITY ? 0.f : r * a, held = fminf(fmaxf(r, 1 - Q.clip_low), 1 + Q.clip_high) * a;
  const bool free = !(open > held);          // (also where r is no number)
  float c = free ? -open : 0.f, s = free ? -open : -held;
  if (Q.reference) {
    const float d = Q.reference[t] - l, e = expm1f(d);
    s += Q.kl * (e - d), c -= Q.kl * e;
  }
  loss = w * s;
  return w * c;
}

__device__ __forceinline__ bool counts(int32_t target, uint32_t vocab) { return target >= 0 && (uint32_t)target < vocab; }

// Rows of SKEWED kernels start anywhere, their pieces at lines of memory: a row is worked on
// as one that begins at the line of its first element, with up to skew elements before it that
// are no part of it.  (A wavefront's 1024 bytes across the ends of lines leave two of them
// half written, and at an odd element of 16 bits take longer to read.)
template <typename T, bool SKEWED>
__device__ __forceinline__ uint32_t before(const void *row, uint32_t skew) {
  return SKEWED ? (uint32_t)((uint64_t)row / sizeof(T)) & skew : 0;
}

// A lane's piece of a row whose elements are those from `from` up to n.  NARROW: rows
// shorter than a piece, from 0.
template <typename T, bool NARROW>
__device__ __forceinline__ u4 read_piece(const T *row, uint32_t at, uint32_t from, uint32_t n) {
  if constexpr (!NARROW) {
    return load_shared(row + max(at + kLaneElems<T> <= n ? at : n - kLaneElems<T>, from));
  } else {
    uint32_t w[4];
    load_row<T, kLaneElems<T>, false>(row, at ? 0 : (int)n, w);
    return (u4){w[0], w[1], w[2], w[3]};
  }
}

// The elements of such a piece, -inf outside the row.  whole: it is known to lie inside.
template <typename T, bool NARROW>
__device__ __forceinline__ void logits_of(u4 v, uint32_t at, uint32_t from, uint32_t n, float (&x)[kLaneElems<T>], bool whole = false) {
  if (whole || (at >= from && at + kLaneElems<T> <= n)) {
    unpack<T>(v, x);
    return;
  }
  if (at < from) v = __builtin_bit_cast(u4, __builtin_bit_cast(unsigned __int128, v) << (min(from - at, kLaneElems<T> - 1) * 8 * sizeof(T)));
  unpack<T>(NARROW ? v : piece_fix<T>(v, at, n), x);
#pragma unroll
  for (int j = 0; j < (int)kLaneElems<T>; ++j)
    if (at + j < from || at + j >= n) x[j] = -INFINITY;
}

// Adds elements to a running maximum and sum of exponentials.
template <int N>
__device__ __forceinline__ void gather(const float (&x)[N], float &m, float &s) {
  float top = m;
#pragma unroll
  for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
  const float ms = top == -INFINITY ? 0.f : top;
  float more[4] = {s * __builtin_amdgcn_exp2f((m - ms) * kLossLog2e), 0, 0, 0};   // (four chains of additions)
#pragma unroll
  for (int j = 0; j < N; ++j) more[j % 4] += __builtin_amdgcn_exp2f((x[j] - ms) * kLossLog2e);
  s = more[0] + more[1] + (more[2] + more[3]);
  m = top;
}

// U pieces of a row, 256 of them apart, for a lane whose first one starts at `at`.
// Steps that lie inside the row (`whole`, the same in the wavefront) need no checks.
template <typename T, bool NARROW, int U>
__device__ __forceinline__ void read_step(const T *row, uint32_t at, uint32_t from, uint32_t n, bool whole, u4 (&v)[U]) {
  if (whole) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load_shared(row + at + u * 256 * kLaneElems<T>);
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = read_piece<T, NARROW>(row, at + u * 256 * kLaneElems<T>, from, n);
  }
}

// Parts held by the lanes of a wavefront joined, the same in each.
__device__ __forceinline__ void join_wave(float &m, float &s) {
  const float top = wave_max(m), ms = top == -INFINITY ? 0.f : top;
  s = wave_sum(s * __builtin_amdgcn_exp2f((m - ms) * kLossLog2e));
  m = top;
}
// A row's log sum of exponentials as its maximum and log2 of the sum, which are never added up: rounded to 32 bits
// their sum would be off by 2^-24 of the maximum, and so would every log-probability and every exponent.
__device__ __forceinline__ float2 log_sum(float m, float s) { return {m, __builtin_amdgcn_logf(s)}; }
__device__ __forceinline__ float log_prob(float z, float2 lse) { return (z - lse.x) - kLossLn2 * lse.y; }

// A workgroup to a part of a token's row.
template <typename T, bool NARROW, bool SKEWED>
__global__ void __launch_bounds__(256) token_stats_kernel(TokenParams P) {
  constexpr int E = kLaneElems<T>, U = 2;
  const uint32_t t = blockIdx.x, split = blockIdx.y;
  const int32_t y = P.targets[t];
  if (split == 0 && threadIdx.x == 0) P.coef[t] = 0;          // (of a token in no sequence)
  if (!counts(y, P.vocab)) return;
  const T *z = (const T *)P.z + t * P.z_row;
  const uint32_t from = before<T, SKEWED>(z, P.skew), n = P.vocab + from, w = wave_index();
  z -= from;
  constexpr uint32_t STEP = U * 256 * E;
  const uint32_t start = split * P.slice * E, end = min(start + P.slice * E, n);
  auto inside = [&](uint32_t base) { return base + STEP <= end && (!from || base || w); };
  u4 v[U];
  read_step<T, NARROW>(z, start + threadIdx.x * E, from, n, inside(start), v);
  float zt = 0;
  if (split == 0 && threadIdx.x == 0) zt = (float)z[from + y];
  float m = -INFINITY, s = 0;
  for (uint32_t base = start; base < end; base += STEP) {
    const uint32_t at = base + threadIdx.x * E;
    const bool whole = inside(base);
    float x[U * E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float e[E];
      logits_of<T, NARROW>(v[u], at + u * 256 * E, from, end, e, whole);
#pragma unroll
      for (int j = 0; j < E; ++j) x[u * E + j] = e[j];
    }
    if (base + STEP < end) read_step<T, NARROW>(z, at + STEP, from, n, inside(base + STEP), v);
    gather(x, m, s);
  }
  join_wave(m, s);
  __shared__ float2 part[4];
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = {m, s};
  __syncthreads();
  if (threadIdx.x) return;
  const float top = fmaxf(fmaxf(part[0].x, part[1].x), fmaxf(part[2].x, part[3].x)), ms = top == -INFINITY ? 0.f : top;
  s = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) s += part[i].y * __builtin_amdgcn_exp2f((part[i].x - ms) * kLossLog2e);
  P.part[(uint64_t)t * P.splits + split] = {top, s};
  if (split == 0) P.at_target[t] = zt;
}

// A workgroup to a pair: its sequences' sums, its loss, and their tokens' derivatives.
// `lanes`, a power of two, share a token's parts.
__global__ void __launch_bounds__(1024) pair_kernel(TokenParams P, PairParams Q, uint32_t lanes) {
  const uint32_t lane = threadIdx.x % lanes;
  __shared__ double sh[2][16];
  const uint32_t p = blockIdx.x;
  int32_t end[3];      // sequence k: from end[k] to end[k + 1]
#pragma unroll
  for (int k = 0; k < 3; ++k) end[k] = min(max(Q.offsets[2 * p + k], 0), (int32_t)P.n_tok);
  const int32_t from = min(end[0], end[1]), to = max(end[1], end[2]);
  auto sequence = [&](int32_t t) { return t >= end[0] && t < end[1] ? 0 : t >= end[1] && t < end[2] ? 1 : -1; };
  double sum[2] = {0, 0};
  for (int32_t t = from + (int32_t)(threadIdx.x / lanes); t < to; t += 1024 / lanes) {
    const int k = sequence(t);
    float m = -INFINITY, s = 0;
    if (lane < P.splits) {
      const float2 part = P.part[(uint64_t)t * P.splits + lane];
      m = part.x, s = part.y;
    }
    const float zt = P.at_target[t];
    const bool live = k >= 0 && counts(P.targets[t], P.vocab);     // (what the others' parts hold is not used)
    float top = m;
    for (uint32_t i = 1; i < lanes; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
    s *= __builtin_amdgcn_exp2f((m - (top == -INFINITY ? 0.f : top)) * kLossLog2e);
    for (uint32_t i = 1; i < lanes; i *= 2) s += __shfl_xor(s, i);
    const float2 lse = log_sum(top, s);
    const float l = log_prob(zt, lse);
    if (lane || !live) continue;
    P.lse[t] = lse;
    sum[0] += k ? 0. : l, sum[1] += k ? l : 0.;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    for (int i = 32; i; i >>= 1) sum[k] += __shfl_xor(sum[k], i);
    if (threadIdx.x % 64 == 0) sh[k][threadIdx.x / 64] = sum[k];
  }
  __syncthreads();
  sum[0] = sum[1] = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[0] += sh[0][i], sum[1] += sh[1][i];
  const double h = Q.beta * ((sum[0] - Q.reference[2 * p]) - (sum[1] - Q.reference[2 * p + 1]));
  const double w = Q.weights ? Q.weights[p] : 1. / Q.n_pair, e = Q.smoothing, x = exp(-fabs(h)), big = 1 / (1 + x), small = x / (1 + x);
  const double up = h >= 0 ? big : small, down = h >= 0 ? small : big;      // sigmoid(h), sigmoid(-h)
  const float g = w == 0 ? 0.f : (float)(w * Q.beta * (e * up - (1 - e) * down));
  for (int32_t t = from + (int32_t)threadIdx.x; t < to; t += 1024) {
    const int k = sequence(t);
    if (k >= 0 && counts(P.targets[t], P.vocab)) P.coef[t] = k ? -g : g;
  }
  if (threadIdx.x) return;
  // -log sigmoid(h) = log(1 + exp(-|h|)) + max(-h, 0)
  const double loss = log1p(x) + (h < 0 ? (1 - e) * -h : e > 0 && h > 0 ? e * h : 0.);
  Q.loss[p] = w == 0 ? 0.f : (float)(w * loss);
  Q.logps[2 * p] = (float)sum[0], Q.logps[2 * p + 1] = (float)sum[1];
}

// c (onehot(y) - softmax(z)) of a lane's piece.
template <typename T, bool NARROW>
__device__ __forceinline__ u4 gradient_of(u4 v, uint32_t at, uint32_t from, uint32_t n, uint32_t y, float c, float2 lse, bool whole = false) {
  constexpr int E = kLaneElems<T>;
  float x[E];
  logits_of<T, NARROW>(v, at, from, n, x, whole);
#pragma unroll
  for (int j = 0; j < E; ++j) x[j] = -c * __builtin_amdgcn_exp2f(__builtin_fmaf(x[j] - lse.x, kLossLog2e, -lse.y));
  if (y - at < (uint32_t)E) {
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (at + j == y) x[j] += c;
  }
  return pack<T>(x);
}

// A lane's piece of a row of the gradient stored.
template <typename T>
__device__ __forceinline__ void store_inside(T *row, uint32_t at, uint32_t from, uint32_t n, u4 v) {
  if (at >= from) return store_piece(row, at, n, v);
#pragma unroll
  for (int j = 0; j < (int)kLaneElems<T>; ++j)
    if (at + j >= from && at + j < n) {
      if constexpr (sizeof(T) == 4) ((uint32_t *)row)[at + j] = v[j];
      else ((uint16_t *)row)[at + j] = (uint16_t)(v[j / 2] >> (j % 2 * 16));
    }
}

// A workgroup to a part of a token's row of the gradient.  POLICY: the token's loss as
// well, from the parts of its row.
template <typename T, bool NARROW, bool SKEWED, bool POLICY>
__global__ void __launch_bounds__(256) token_grad_kernel(TokenParams P, PolicyParams Q) {
  constexpr int E = kLaneElems<T>, U = 2;
  // From the last token on: its logits were read last.
  const uint32_t t = P.n_tok - 1 - blockIdx.x, split = blockIdx.y;
  const int32_t y = P.targets[t];
  const T *z = (const T *)P.z + t * P.z_row;
  const uint32_t from = before<T, SKEWED>(z, P.skew), n = P.vocab + from, w = wave_index();
  z -= from;
  constexpr uint32_t STEP = U * 256 * E;
  const uint32_t start = split * P.slice * E, end = min(start + P.slice * E, n);
  auto inside = [&](uint32_t base) { return base + STEP <= end && (!from || base || w); };
  u4 v[U];
  auto load = [&](uint32_t base) { read_step<T, NARROW>(z, base + threadIdx.x * E, from, n, inside(base), v); };
  float c = 0;
  float2 lse = {0, 0};
  if constexpr (POLICY) {
    const bool live = counts(y, P.vocab);
    float l = 0, loss = 0;
    if (live) {
      if (P.dz) load(start);
      const uint32_t lane = threadIdx.x % 64;
      float m = -INFINITY, s = 0;
      if (lane < P.splits) m = P.part[(uint64_t)t * P.splits + lane].x, s = P.part[(uint64_t)t * P.splits + lane].y;
      join_wave(m, s);
      lse = log_sum(m, s);
      l = log_prob(P.at_target[t], lse);
      c = policy_of(Q, P.n_tok, t, l, loss);
    }
    if (split == 0 && threadIdx.x == 0) Q.loss[t] = loss, Q.logps[t] = l;
    if (!P.dz) return;
  } else {
    c = P.coef[t], lse = P.lse[t];
    if (c != 0) load(start);
  }
  T *dz = (T *)P.dz + t * P.dz_row - from;
  if (c == 0) {
    for (uint32_t at = start + threadIdx.x * E; at < end; at += 256 * E) store_inside(dz, at, from, n, (u4){0, 0, 0, 0});
    return;
  }
  for (uint32_t base = start; base < end; base += STEP) {
    u4 g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) g[u] = v[u];
    if (base + STEP < end) load(base + STEP);
    const uint32_t at = base + threadIdx.x * E;
    const bool whole = inside(base);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = at + u * 256 * E;
      if (whole) __builtin_nontemporal_store(gradient_of<T, NARROW>(g[u], i, from, n, from + y, c, lse, true), (u4_any *)(dz + i));
      else if (i < end) store_inside(dz, i, from, n, gradient_of<T, NARROW>(g[u], i, from, n, from + y, c, lse));
    }
  }
}

// The policy loss with a workgroup holding the whole row: read once.  NV pieces to a lane
// stay in registers, NL more in LDS, and NR more of the longest rows are read again, from the
// caches.  With NL, 1024 threads, and with 4 of them registers for two workgroups to a
// compute unit.  (24 in registers spill: 302 us for 1500 rows of 190000 in bfloat16, 284 in two launches.)
template <typename T, int NV, int NL, int NR, bool SKEWED>
__global__ void __launch_bounds__(1024, NL == 4 ? 8 : 4) policy_row_kernel(TokenParams P, PolicyParams Q, uint32_t threads) {
  constexpr uint32_t E = kLaneElems<T>;
  if (NL) threads = 1024;
  const uint32_t t = blockIdx.x;
  const int32_t y = P.targets[t];
  const T *z = (const T *)P.z + t * P.z_row;
  const uint32_t from = before<T, SKEWED>(z, P.skew), n = P.vocab + from, wave = wave_index();
  z -= from;
  T *dz = (T *)P.dz + t * P.dz_row - from;
  if (!counts(y, P.vocab)) {
    if (threadIdx.x == 0) Q.loss[t] = 0, Q.logps[t] = 0;
    for (uint32_t at = threadIdx.x * E; at < n; at += threads * E) store_inside(dz, at, from, n, (u4){0, 0, 0, 0});
    return;
  }
  auto place = [&](uint32_t k) {
    const uint32_t at = (k * threads + threadIdx.x) * E;
    return z + max(at + E <= n ? at : n - E, from);
  };
  auto inside = [&](uint32_t k) { return (k + 1) * threads * E <= n && (k || !from || wave); };
  // (by one thread, through LDS: where dlogits are the logits the element is overwritten after the barrier)
  __shared__ float at_target;
  if (threadIdx.x == 0) at_target = (float)z[from + y];
  float m = -INFINITY, s = 0;
  __shared__ u4 far[NL ? NL * 1024 : 1];
  constexpr int U = NL == 4 ? 4 : 3;
  if constexpr (NL > 0) {
    static_assert(NL % U == 0 && NR % U == 0);
#pragma unroll
    for (int k = 0; k < NL + NR; k += U) {
      if ((NV + k) * threads * E >= n) continue;
      u4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = k < NL ? load_once(place(NV + k + u)) : load_shared(place(NV + k + u));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k < NL) far[(k + u) * 1024 + threadIdx.x] = v[u];
        float x[E];
        logits_of<T, false>(v[u], ((NV + k + u) * threads + threadIdx.x) * E, from, n, x, inside(NV + k + u));
        gather(x, m, s);
      }
    }
  }
  u4 v[NV];
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) v[k] = load_once(place(k));
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    if (k * threads * E >= n) continue;
    float x[E];
    logits_of<T, false>(v[k], (k * threads + threadIdx.x) * E, from, n, x, inside(k));
    gather(x, m, s);
    // (only the packed row stays: its elements kept as 32-bit values for the second pass spilled, 599 us for 200)
    asm volatile("" : "+v"(v[k]));
  }
  __shared__ float2 part[16];
  join_wave(m, s);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = {m, s};
  __syncthreads();
  const uint32_t lane = threadIdx.x % 64;
  m = lane < threads / 64 ? part[lane].x : -INFINITY, s = lane < threads / 64 ? part[lane].y : 0.f;
  join_wave(m, s);
  const float2 lse = log_sum(m, s);
  const float l = log_prob(at_target, lse);
  float loss;
  const float c = policy_of(Q, P.n_tok, t, l, loss);
  if (c == 0) {
    if (threadIdx.x == 0) Q.loss[t] = loss, Q.logps[t] = l;
    for (uint32_t at = threadIdx.x * E; at < n; at += threads * E) store_inside(dz, at, from, n, (u4){0, 0, 0, 0});
    return;
  }
  if (threadIdx.x == 0) Q.loss[t] = loss, Q.logps[t] = l;
  auto store = [&](uint32_t k, u4 v) {
    const uint32_t at = (k * threads + threadIdx.x) * E;
    const bool whole = inside(k);
    const u4 g = gradient_of<T, false>(v, at, from, n, from + y, c, lse, whole);
    if (whole) __builtin_nontemporal_store(g, (u4_any *)(dz + at));
    else store_inside(dz, at, from, n, g);
  };
#pragma unroll
  for (uint32_t k = 0; k < NV; ++k) {
    if (k * threads * E >= n) continue;
    store(k, v[k]);
  }
  if constexpr (NL > 0) {
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      if ((NV + k) * threads * E >= n) continue;
      store(NV + k, far[k * 1024 + threadIdx.x]);
    }
#pragma unroll
    for (int k = NL; k < NL + NR; k += U) {
      if ((NV + k) * threads * E >= n) continue;
      u4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = load_shared(place(NV + k + u));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if ((NV + k + u) * threads * E >= n) continue;
        store(NV + k + u, v[u]);
      }
    }
  }
}

}  // namespace fiona
