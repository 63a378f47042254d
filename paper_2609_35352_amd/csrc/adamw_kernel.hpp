// Kernel of fiona_adamw_step: all tensors in one launch, a workgroup to a chunk of one.
//
// A chunk's record holds its addresses, so that a workgroup's first load is all it waits for
// before its data.  With 8-bit states a block of 256 is a wavefront's, four elements to a
// lane: its scales need one maximum over the lanes.  A value y in units of its scale lies
// between two e4m3 values that are 2^(e - 3) apart, e its exponent, and goes to the upper one
// with the probability of what it is above the lower, which keeps its mean.
//
// What bounds it: memory, 28 bytes an element with 32-bit states, 16 with 8-bit ones beside
// masters (38 million elements: 171 us, 6.3 TB/s, and 107 us, 5.7; a copy reaches 5.2);
// with 8-bit states and neither masters nor 32-bit parameters (10 bytes, 101 us) the vector
// units: about 90 instructions an element, two 32-bit products of the dither's among them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fiona.h"
#include "pieces.hpp"

namespace fiona {

constexpr uint32_t kChunk = 4 * FIONA_ADAMW_BLOCK;   // elements of a workgroup: a block to a wavefront

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

// y in [0, 448] to one of the two neighbouring e4m3 values: up where what it is above
// the lower one, in steps between them, and a dither in (0, 1) make one together.
// one_and: the dither and one, as 24 bits hold it.  Exponents stay those of the value's
// binade, from 2^-6 (the smallest normal value) on.
__device__ __forceinline__ float to_code(float y, float one_and) {
  const uint32_t e = __builtin_bit_cast(uint32_t, y) & 0x7F800000u, u = e > (121u << 23) ? e : 121u << 23;
  const float step = __builtin_bit_cast(float, u - (3u << 23)), per = __builtin_bit_cast(float, (257u << 23) - u);
  return __builtin_fmaf(__builtin_floorf(__builtin_fmaf(y, per, one_and)), step, -step);
}

// Four consecutive elements of T, at any address that they may stand at.
typedef uint32_t u1_any __attribute__((aligned(1)));
template <typename T>
struct Four {
  u2 v;
};
template <>
struct Four<float> {
  u4 v;
};
template <>
struct Four<uint8_t> {
  uint32_t v;
};

// `valid` of them, in whole pieces where `whole` says so; the rest zero.
template <typename T>
__device__ __forceinline__ void load_four(const void *base, uint64_t at, bool whole, int valid, Four<T> &f) {
  const T *p = (const T *)base + at;
  if constexpr (sizeof(T) == 4) {
    if (whole) f.v = __builtin_nontemporal_load((const u4_any *)p);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = j < valid ? ((const uint32_t *)p)[j] : 0;
  } else if constexpr (sizeof(T) == 2) {
    if (whole) f.v = __builtin_nontemporal_load((const u2_any *)p);
    else
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t lo = 2 * j < valid ? ((const uint16_t *)p)[2 * j] : 0, hi = 2 * j + 1 < valid ? ((const uint16_t *)p)[2 * j + 1] : 0;
        f.v[j] = lo | hi << 16;
      }
  } else {
    if (whole) f.v = __builtin_nontemporal_load((const u1_any *)p);
    else {
      f.v = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v |= j < valid ? (uint32_t)((const uint8_t *)p)[j] << 8 * j : 0;
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_four(void *base, uint64_t at, bool whole, int valid, Four<T> f) {
  T *p = (T *)base + at;
  if constexpr (sizeof(T) == 4) {
    if (whole) __builtin_nontemporal_store(f.v, (u4_any *)p);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < valid) ((uint32_t *)p)[j] = f.v[j];
  } else if constexpr (sizeof(T) == 2) {
    if (whole) __builtin_nontemporal_store(f.v, (u2_any *)p);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < valid) ((uint16_t *)p)[j] = (uint16_t)(f.v[j / 2] >> 16 * (j % 2));
  } else {
    if (whole) __builtin_nontemporal_store(f.v, (u1_any *)p);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < valid) ((uint8_t *)p)[j] = (uint8_t)(f.v >> 8 * j);
  }
}

template <typename T>
__device__ __forceinline__ void floats_of(Four<T> f, float (&x)[4]) {
  if constexpr (sizeof(T) == 4) {
    const f4 y = __builtin_bit_cast(f4, f.v);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = y[j];
  } else if constexpr (__is_same(T, _Float16)) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    const h4 y = __builtin_bit_cast(h4, f.v);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (float)y[j];
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t word = j < 2 ? f.v[0] : f.v[1];
      x[j] = __builtin_bit_cast(float, j % 2 ? word & 0xFFFF0000u : word << 16);
    }
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)f.v, 0), x[1] = __builtin_amdgcn_cvt_f32_fp8((int)f.v, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)f.v, 2), x[3] = __builtin_amdgcn_cvt_f32_fp8((int)f.v, 3);
  }
}
template <typename T>
__device__ __forceinline__ Four<T> four_of(const float (&x)[4]) {
  Four<T> f;
  if constexpr (sizeof(T) == 4) f.v = __builtin_bit_cast(u4, (f4){x[0], x[1], x[2], x[3]});
  else if constexpr (sizeof(T) == 2) f.v = (u2){pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
  else f.v = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), true);
  return f;
}

// A block's values as codes, and its scale.  A value that is no number gets the code
// for that; an infinity makes the scale one, and with it the block.
template <bool ROOTS>
__device__ __forceinline__ float block_codes(float (&x)[4], const float (&one_and)[4]) {
  const float t = wave_max(fmaxf(fmaxf(__builtin_fabsf(x[0]), __builtin_fabsf(x[1])), fmaxf(__builtin_fabsf(x[2]), __builtin_fabsf(x[3]))));
  const float most = t < 0x1p-100f ? 0.f : t, per = most > 0 ? 448.f * __builtin_amdgcn_rcpf(most) : 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float y = __builtin_fabsf(x[j]) * per, c = to_code(y > 448.f ? 448.f : y, one_and[j]);
    x[j] = ROOTS ? x[j] > 0 && most > 0 ? fmaxf(c, 0x1p-9f) : c : __builtin_copysignf(c, x[j]);
  }
  return most * (1 / 448.f);
}

// A workgroup to a chunk, a wavefront to a block, four elements to a lane.  (Four blocks
// to a wavefront, all their loads first: 117 us instead of 107 for the 38 million elements
// above, 190 instead of 171 with 32-bit states.)
template <typename T, bool SMALL>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwParams P) {
  using S = std::conditional_t<SMALL, uint8_t, float>;
  const AdamwChunk C = P.chunks[blockIdx.x];
  const uint32_t b = wave_index(), lane = threadIdx.x % 64, i = b * FIONA_ADAMW_BLOCK + 4 * lane;
  if (b * FIONA_ADAMW_BLOCK >= C.n) return;
  const bool whole = (b + 1) * FIONA_ADAMW_BLOCK <= C.n;
  const int valid = (int)C.n - (int)i;
  Four<T> rp, rg;
  Four<float> rx;
  Four<S> rm, rv;
  float sm = 1, sv = 1;
  load_four<T>(C.grad, i, whole, valid, rg);
  load_four<S>(C.m, i, whole, valid, rm);
  load_four<S>(C.v, i, whole, valid, rv);
  if (C.master) load_four<float>(C.master, i, whole, valid, rx);
  else load_four<T>(C.param, i, whole, valid, rp);
  if (SMALL) sm = C.m_scale[b], sv = C.v_scale[b];
  __builtin_amdgcn_sched_barrier(0);
  const int32_t step = *P.step < 1 ? 1 : *P.step;
  // 1 - beta^t without the difference of two near numbers.
  const float c1 = 1.f / -expm1f(step * P.log_b1), c2 = 1.f / sqrtf(-expm1f(step * P.log_b2)), lr = *P.lr;
  const float gs = P.grad_scale ? *P.grad_scale : 1.f, keep = 1.f - lr * C.decay;
  const uint32_t key = mix((uint32_t)step * 0x9E3779B1u + P.seed);
  float g[4], m[4], v[4], x[4], um[4], uv[4];
  floats_of(rg, g), floats_of(rm, m), floats_of(rv, v);
  if (C.master) floats_of(rx, x);
  else floats_of(rp, x);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float gj = g[j] * gs;
    if (SMALL) m[j] *= sm, v[j] *= sv, v[j] *= v[j];
    m[j] = __builtin_fmaf(P.b1, m[j], P.a1 * gj);
    v[j] = __builtin_fmaf(P.a2 * gj, gj, P.b2 * v[j]);
    const float r = __builtin_amdgcn_sqrtf(v[j]);
    x[j] = x[j] * keep - lr * (m[j] * c1 * __builtin_amdgcn_rcpf(r * c2 + P.eps));
    if (sizeof(T) == 2) asm volatile("" : "+v"(x[j]));   // (param is this value rounded, not its last product's binary16 form)
    if (SMALL) {
      v[j] = r;
      const uint32_t h = mix((C.first + i + j) ^ key);
      // one + (16 bits + 1/2) / 2^16, the bits below the leading one's seven places up
      um[j] = __builtin_bit_cast(float, (h & 0xFFFFu) << 7 | 0x3F800040u);
      uv[j] = __builtin_bit_cast(float, (h >> 9 & 0x7FFF80u) | 0x3F800040u);
    }
  }
  if (C.master) store_four(C.master, i, whole, valid, four_of<float>(x));
  store_four(C.param, i, whole, valid, four_of<T>(x));
  if constexpr (SMALL) {
    const float tm = block_codes<false>(m, um), tv = block_codes<true>(v, uv);
    if (lane == 0) C.m_scale[b] = tm, C.v_scale[b] = tv;
  }
  store_four(C.m, i, whole, valid, four_of<S>(m));
  store_four(C.v, i, whole, valid, four_of<S>(v));
}

}  // namespace fiona
