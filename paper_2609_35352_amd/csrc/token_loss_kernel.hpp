// Kernels of fiona_preference_loss and fiona_policy_loss.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fiona {

struct TokenParams {
  const void *z;
  void *dz;
  const int32_t *targets;
  float *lse, *logp, *coef;       // [n_tok]: log sum of exponentials, log-probability, derivative of the loss
  uint64_t z_row, dz_row;
  uint32_t n_tok, vocab;
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

__device__ __forceinline__ float max_256(float a) {
  __shared__ float part[4];
  for (int k = 32; k; k >>= 1) a = fmaxf(a, __shfl_xor(a, k));
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = a;
  __syncthreads();
  return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}
template <typename F>
__device__ __forceinline__ F add_256(F a) {
  __shared__ F part[4];
  for (int k = 32; k; k >>= 1) a += __shfl_xor(a, k);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = a;
  __syncthreads();
  return part[0] + part[1] + (part[2] + part[3]);
}

// The policy loss of a token with log-probability l, and its derivative.
__device__ __forceinline__ float policy_of(const PolicyParams &Q, uint32_t n_tok, uint32_t t, float l, float &loss) {
  const float w = Q.weights ? Q.weights[t] : 1.f / n_tok, a = Q.advantages[t], r = expf(l - Q.old[t]);
  if (w == 0) return loss = 0;
  const float open = r * a, held = fminf(fmaxf(r, 1 - Q.clip_low), 1 + Q.clip_high) * a;
  const bool free = !(open > held);          // (also where r is no number)
  float c = free ? -open : 0.f, s = free ? -open : -held;
  if (Q.reference) {
    const float d = Q.reference[t] - l, e = expm1f(d);
    s += Q.kl * (e - d), c -= Q.kl * e;
  }
  loss = w * s;
  return w * c;
}

// A workgroup to a token: its log-probability, and with POLICY its loss.
template <typename T, bool POLICY>
__global__ void __launch_bounds__(256) token_stats_kernel(TokenParams P, PolicyParams Q) {
  const uint32_t t = blockIdx.x;
  const int32_t y = P.targets[t];
  float l = 0, lse = 0;
  const bool live = y >= 0 && (uint32_t)y < P.vocab;
  const T *z = (const T *)P.z + t * P.z_row;
  if (live) {
    float m = -INFINITY, s = 0;
    for (uint32_t i = threadIdx.x; i < P.vocab; i += 256) m = fmaxf(m, (float)z[i]);
    m = max_256(m);
    const float ms = m == -INFINITY ? 0.f : m;
    for (uint32_t i = threadIdx.x; i < P.vocab; i += 256) s += expf((float)z[i] - ms);
    lse = ms + logf(add_256(s));
    l = (float)z[y] - lse;
  }
  if (threadIdx.x) return;
  P.lse[t] = lse, P.logp[t] = l;
  if (POLICY) {
    float loss = 0;
    P.coef[t] = live ? policy_of(Q, P.n_tok, t, l, loss) : 0.f;
    Q.loss[t] = loss, Q.logps[t] = l;
  } else {
    P.coef[t] = 0;          // (of a token in no sequence)
  }
}

// A workgroup to a pair: its sequences' sums, its loss, and their tokens' derivatives.
__global__ void __launch_bounds__(256) pair_kernel(TokenParams P, PairParams Q) {
  const uint32_t p = blockIdx.x;
  double sum[2];
  int32_t first[2], last[2];
  for (int k = 0; k < 2; ++k) {
    first[k] = min(max(Q.offsets[2 * p + k], 0), (int32_t)P.n_tok);
    last[k] = min(max(Q.offsets[2 * p + k + 1], 0), (int32_t)P.n_tok);
    double s = 0;
    for (int32_t t = first[k] + (int32_t)threadIdx.x; t < last[k]; t += 256) s += P.logp[t];
    sum[k] = add_256(s);
  }
  const double h = Q.beta * ((sum[0] - Q.reference[2 * p]) - (sum[1] - Q.reference[2 * p + 1]));
  const double w = Q.weights ? Q.weights[p] : 1. / Q.n_pair, e = Q.smoothing, x = exp(-fabs(h)), big = 1 / (1 + x), small = x / (1 + x);
  const double up = h >= 0 ? big : small, down = h >= 0 ? small : big;      // sigmoid(h), sigmoid(-h)
  const float g = w == 0 ? 0.f : (float)(w * Q.beta * (e * up - (1 - e) * down));
  for (int k = 0; k < 2; ++k)
    for (int32_t t = first[k] + (int32_t)threadIdx.x; t < last[k]; t += 256) {
      const int32_t y = P.targets[t];
      P.coef[t] = y >= 0 && (uint32_t)y < P.vocab ? (k ? -g : g) : 0.f;
    }
  if (threadIdx.x) return;
  // -log sigmoid(h) = log(1 + exp(-|h|)) + max(-h, 0)
  const double loss = log1p(x) + (h < 0 ? (1 - e) * -h : e > 0 && h > 0 ? e * h : 0.);
  Q.loss[p] = w == 0 ? 0.f : (float)(w * loss);
  Q.logps[2 * p] = (float)sum[0], Q.logps[2 * p + 1] = (float)sum[1];
}

// A workgroup to a token: its row of the gradient.
template <typename T>
__global__ void __launch_bounds__(256) token_grad_kernel(TokenParams P) {
  const uint32_t t = blockIdx.x;
  const float c = P.coef[t], lse = P.lse[t];
  const int32_t y = P.targets[t];
  const T *z = (const T *)P.z + t * P.z_row;
  T *dz = (T *)P.dz + t * P.dz_row;
  for (uint32_t i = threadIdx.x; i < P.vocab; i += 256) {
    const float p = c == 0 ? 0.f : c * (expf((float)z[i] - lse));
    dz[i] = (T)(c == 0 ? 0.f : (int32_t)i == y ? c - p : -p);
  }
}

}  // namespace fiona
