// Kernel of fiona_adamw_step: all tensors in one launch, a workgroup to a chunk of one.
//
// A chunk's record holds its addresses, so that a workgroup's first load is all it waits for
// before its data.  With 8-bit states a block of 256 is a wavefront's, four elements to a
// lane: its scales need one maximum over the lanes.  A value y in units of its scale lies
// between two e4m3 values that are 2^(e - 3) apart, e its exponent, and goes to the upper one
// with the probability of what it is above the lower, which keeps its mean.
//
// What bounds it: memory, 28 bytes an element with 32-bit states, 16 with 8-bit ones beside
// masters (38 million elements: 175 us, 6.1 TB/s, and 103 us, 6.0; a copy reaches 5.2);
// with 8-bit states and neither masters nor 32-bit parameters (10 bytes, 97 us) the vector
// units: nearly 100 instructions an element, two 32-bit products of the dither's among them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cfloat>
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
// Exponents stay those of the value's binade, from 2^-6 (the smallest normal value) on.
__device__ __forceinline__ float to_code(float y, float dither) {
  const uint32_t e = __builtin_bit_cast(uint32_t, y) & 0x7F800000u, u = e > (121u << 23) ? e : 121u << 23;
  const float step = __builtin_bit_cast(float, u - (3u << 23)), per = __builtin_bit_cast(float, (257u << 23) - u);
  return __builtin_floorf(__builtin_fmaf(y, per, dither)) * step;      // (both products are exact)
}

// x^1/2 as rounded, from the hardware's x^-1/2 (a unit off at most) and one correction;
// half the instructions of the compiler's.  Below 2^-126 less than the root, but above zero.
__device__ __forceinline__ float root_of(float x) {
  const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-126f)), r = x * y;
  return __builtin_fmaf(__builtin_fmaf(-r, r, x), 0.5f * y, r);
}

// x^1/2, a unit off at most, subnormal x included (the hardware's root takes those as zero).
__device__ __forceinline__ float wide_root(float x) {
  const bool low = x < 0x1p-100f;
  return __builtin_amdgcn_sqrtf(low ? x * 0x1p32f : x) * (low ? 0x1p-16f : 1.f);
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

__device__ __forceinline__ float lane_value(float x, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// The largest magnitudes of a block's m, in lanes 0 to 31, and of its roots, in lanes 32
// to 63: from the 16 lanes of a row on one register carries both.
__device__ __forceinline__ float block_tops(const float (&m)[4], const float (&r)[4]) {
  auto row = [](float x) {
    x = fmaxf(x, dpp<0xB1>(x));
    x = fmaxf(x, dpp<0x4E>(x));
    x = fmaxf(x, dpp<0x141>(x));
    return fmaxf(x, dpp<0x140>(x));
  };
  const float a = row(fmaxf(fmaxf(__builtin_fabsf(m[0]), __builtin_fabsf(m[1])), fmaxf(__builtin_fabsf(m[2]), __builtin_fabsf(m[3]))));
  const float b = row(fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3])));
  const auto h = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const float x = fmaxf(__builtin_bit_cast(float, (uint32_t)h[0]), __builtin_bit_cast(float, (uint32_t)h[1]));
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto q = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}

// Values as codes, per: 448 over the block's largest magnitude (zero where there is none).
// A value that is no number gets the code for that; an infinity makes per no number and
// the scale infinite, and every code of the block the one for no number.
template <bool ROOTS>
__device__ __forceinline__ void codes_of(float (&x)[4], const float (&dither)[4], float per) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float y = __builtin_fabsf(x[j]) * per, c = to_code(__builtin_elementwise_minimum(y, 448.f), dither[j]);
    x[j] = ROOTS ? x[j] * per > 0 ? fmaxf(c, 0x1p-9f) : c : __builtin_copysignf(c, x[j]);
  }
}

// A workgroup to a chunk, a wavefront to a block, four elements to a lane.  (Four blocks
// to a wavefront, all their loads first: 10 us more for the 38 million elements above, 19
// more with 32-bit states.)
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
  // 1 / (1 - beta1^t) in the lower lanes, 1 / (1 - beta2^t)^1/2 in the upper ones, without
  // the difference of two near numbers (both in every lane: a tenth more instructions).
  const bool low = lane < 32;
  const float left = -expm1f(step * (low ? P.log_b1 : P.log_b2)), c = low ? __builtin_amdgcn_rcpf(left) : __builtin_amdgcn_rsqf(left);
  const float c1 = lane_value(c, 0), c2 = lane_value(c, 32), lr = *P.lr;
  const float gs = P.grad_scale ? *P.grad_scale : 1.f, decay = lr * C.decay, rate = lr * c1;
  const uint32_t key = mix((uint32_t)step * 0x9E3779B1u + P.seed);
  float g[4], m[4], v[4], x[4], um[4], uv[4];
  floats_of(rg, g), floats_of(rm, m), floats_of(rv, v);
  if (C.master) floats_of(rx, x);
  else floats_of(rp, x);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float gj = g[j] * gs;
    if (SMALL) m[j] *= sm, v[j] *= sv, v[j] *= v[j];
    // Each of the states' operations is rounded by itself, so that they are the same wherever
    // the same operations are done in 32 bits.
    float r;
    {
#pragma clang fp contract(off)
      m[j] = P.b1 * m[j] + P.a1 * gj;
      v[j] = P.b2 * v[j] + P.a2 * (gj * gj);
      r = SMALL ? root_of(v[j]) : wide_root(v[j]);
    }
    // Decay and update are rounded into x together: 1 - lr decay by itself is a multiple of 2^-24, none of the decay at
    // lr 2e-6 and decay 0.01.  (An infinite x stays: its decay is that of the largest number.)
    const float u = m[j] * __builtin_amdgcn_rcpf(r * c2 + P.eps);
    x[j] -= __builtin_fmaf(rate, u, decay * __builtin_amdgcn_fmed3f(x[j], -FLT_MAX, FLT_MAX));
    if (sizeof(T) == 2) asm volatile("" : "+v"(x[j]));   // (param is this value rounded, not its last product's binary16 form)
    if (SMALL) {
      v[j] = r;
      const uint32_t h = mix((C.first + i + j) ^ key);
      // (16 bits + 1/2) / 2^16: one and that, the bits below the leading one's seven places up, less one
      um[j] = __builtin_bit_cast(float, (h & 0xFFFFu) << 7 | 0x3F800040u) - 1.f;
      uv[j] = __builtin_bit_cast(float, (h >> 9 & 0x7FFF80u) | 0x3F800040u) - 1.f;
    }
  }
  if (C.master) store_four(C.master, i, whole, valid, four_of<float>(x));
  store_four(C.param, i, whole, valid, four_of<T>(x));
  if constexpr (SMALL) {
    const float t = block_tops(m, v), most = t < 0x1p-100f ? 0.f : t, rcp = __builtin_amdgcn_rcpf(most);
    const float per = most > 0 ? 448.f * __builtin_fmaf(__builtin_fmaf(-most, rcp, 1.f), rcp, rcp) : 0.f;
    if (lane % 32 == 0) (lane ? C.v_scale : C.m_scale)[b] = most * (1 / 448.f);
    codes_of<false>(m, um, lane_value(per, 0));
    codes_of<true>(v, uv, lane_value(per, 32));
  }
  store_four(C.m, i, whole, valid, four_of<S>(m));
  store_four(C.v, i, whole, valid, four_of<S>(v));
}

}  // namespace fiona
