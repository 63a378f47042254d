// Kernel of fiona_adamw_step.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fiona.h"

namespace fiona {

constexpr uint32_t kChunkBlocks = 4;   // blocks of a workgroup

// What a workgroup works on: part of one tensor, from a block's first element on.
struct AdamwChunk {
  void *param, *grad;
  float *master;
  void *m, *v;
  float *m_scale, *v_scale;
  uint32_t n, first;       // elements, and the first one's number for the dither
  float decay;
};

struct AdamwParams {
  const AdamwChunk *chunks;
  const float *lr, *grad_scale;
  const int32_t *step;
  float b1, a1, b2, a2, eps, log_b1, log_b2;     // betas, one minus them, their logarithms
  uint32_t n_chunk, seed;
};

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16, x *= 0xA3D8B167u;
  x ^= x >> 15, x *= 0xC94F6E2Bu;
  return x ^ x >> 16;
}

// y in [0, 448], times its neighbouring e4m3 values' spacing: rounded up or down by
// the dither, in (0, 1).  With LEAST never down to zero.
template <bool LEAST>
__device__ __forceinline__ float to_code(float y, float dither) {
  const uint32_t e = __builtin_bit_cast(uint32_t, y) >> 23, u = (e > 121 ? e : 121) - 3;   // 2^-6: the smallest normal value
  const float unit = __builtin_bit_cast(float, u << 23), per = __builtin_bit_cast(float, (254 - u) << 23);
  float k = __builtin_floorf(y * per + dither);
  if (LEAST) k = fmaxf(k, 1.f);
  return k * unit;
}

template <typename T, bool SMALL>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwParams P) {
  // Each operation rounded by itself: a state is the same wherever the same operations are done.
#pragma clang fp contract(off)
  const AdamwChunk C = P.chunks[blockIdx.x];
  const int32_t step = *P.step < 1 ? 1 : *P.step;
  // 1 - beta^t without the difference of two near numbers.
  const float c1 = -expm1f(step * P.log_b1), c2 = sqrtf(-expm1f(step * P.log_b2)), lr = *P.lr;
  const float gs = P.grad_scale ? *P.grad_scale : 1.f;
  const uint32_t key = mix((uint32_t)step * 0x9E3779B1u + P.seed);
  __shared__ float top[2][4];
  for (uint32_t b = 0; b < kChunkBlocks && b * FIONA_ADAMW_BLOCK < C.n; ++b) {
    const uint32_t i = b * FIONA_ADAMW_BLOCK + threadIdx.x;
    const bool in = i < C.n;
    float m = 0, v = 0, r = 0;
    if (in) {
      const float g = (float)((const T *)C.grad)[i] * gs;
      if (SMALL) {
        m = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)C.m)[i], 0) * C.m_scale[b];
        v = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)C.v)[i], 0) * C.v_scale[b];
        v = v * v;
      } else {
        m = ((const float *)C.m)[i], v = ((const float *)C.v)[i];
      }
      m = P.b1 * m + P.a1 * g;
      v = P.b2 * v + P.a2 * (g * g);
      r = __builtin_sqrtf(v);   // (rounded once; the library function may be off by a unit)
      float p = C.master ? C.master[i] : (float)((const T *)C.param)[i];
      p = p - lr * C.decay * p - lr * (m / c1) / (r / c2 + P.eps);
      if (C.master) C.master[i] = p;
      ((T *)C.param)[i] = (T)p;
      if (!SMALL) ((float *)C.m)[i] = m, ((float *)C.v)[i] = v;
    }
    if constexpr (SMALL) {
      // The block's largest magnitudes, as bits: a NaN is above all numbers.
      uint32_t tm = __builtin_bit_cast(uint32_t, m) & 0x7FFFFFFFu, tv = __builtin_bit_cast(uint32_t, r) & 0x7FFFFFFFu;
      for (int k = 32; k; k >>= 1) tm = max(tm, (uint32_t)__shfl_xor((int)tm, k)), tv = max(tv, (uint32_t)__shfl_xor((int)tv, k));
      __syncthreads();
      if (threadIdx.x % 64 == 0)
        top[0][threadIdx.x / 64] = __builtin_bit_cast(float, tm), top[1][threadIdx.x / 64] = __builtin_bit_cast(float, tv);
      __syncthreads();
      for (int k = 0; k < 4; ++k)
        tm = max(tm, __builtin_bit_cast(uint32_t, top[0][k])), tv = max(tv, __builtin_bit_cast(uint32_t, top[1][k]));
      const float xm = __builtin_bit_cast(float, tm) < 0x1p-100f ? 0.f : __builtin_bit_cast(float, tm);
      const float xv = __builtin_bit_cast(float, tv) < 0x1p-100f ? 0.f : __builtin_bit_cast(float, tv);
      const uint32_t h = mix((C.first + i) ^ key);
      const float um = ((float)(h & 0xFFFFu) + 0.5f) / 65536.f, uv = ((float)(h >> 16) + 0.5f) / 65536.f;
      const float ym = xm > 0 ? fminf(fabsf(m) * (448.f / xm), 448.f) : 0.f, yv = xv > 0 ? fminf(r * (448.f / xv), 448.f) : 0.f;
      const float km = xm > 0 ? __builtin_copysignf(to_code<false>(ym, um), m) : 0.f;
      const float kv = xv > 0 && r > 0 ? to_code<true>(yv, uv) : 0.f;
      const uint32_t codes = __builtin_amdgcn_cvt_pk_fp8_f32(km, kv, 0, false);
      if (in) ((uint8_t *)C.m)[i] = (uint8_t)codes, ((uint8_t *)C.v)[i] = (uint8_t)(codes >> 8);
      if (threadIdx.x == 0) C.m_scale[b] = xm / 448.f, C.v_scale[b] = xv / 448.f;
    }
  }
}

}  // namespace fiona
