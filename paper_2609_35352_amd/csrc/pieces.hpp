// Rows held in registers, 16 bytes of a row per lane and piece, and sums over
// wavefronts: what the norm's and the losses' kernels share.
//
// Rows start at any element (the memory system takes 16-byte accesses at any
// address), and hold at least one piece: a lane whose piece passes the row's end loads
// the row's last 16 bytes and moves them (mma.hpp's piece_at and piece_fix), so that
// loads need no branch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mma.hpp"

namespace fiona {

template <typename T>
__device__ __forceinline__ void unpack(u4 v, float (&x)[kLaneElems<T>]) {
  if constexpr (sizeof(T) == 4) {
    const f4 f = __builtin_bit_cast(f4, v);   // (a bit cast of one element of a vector takes its first)
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f[j];
  } else if constexpr (__is_same(T, _Float16)) {
    const h8 h = __builtin_bit_cast(h8, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)h[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __builtin_bit_cast(float, v[j] << 16);
      x[2 * j + 1] = __builtin_bit_cast(float, v[j] & 0xFFFF0000u);
    }
  }
}

template <typename T>
__device__ __forceinline__ u4 pack(const float (&x)[kLaneElems<T>]) {
  u4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) v[j] = __builtin_bit_cast(uint32_t, x[j]);
    else v[j] = pack2<T>(x[2 * j], x[2 * j + 1]);
  }
  return v;
}

// A lane's piece of a row of n elements, from element `at`: nothing from n on.
template <typename T>
__device__ __forceinline__ void store_piece(T *row, uint32_t at, uint32_t n, u4 v) {
  if (at + kLaneElems<T> <= n) {
    __builtin_nontemporal_store(v, (u4_any *)(row + at));
  } else {
#pragma unroll
    for (int j = 0; j < (int)kLaneElems<T>; ++j)
      if (at + j < n) {
        if constexpr (sizeof(T) == 4) ((uint32_t *)row)[at + j] = v[j];
        else ((uint16_t *)row)[at + j] = (uint16_t)(v[j / 2] >> (j % 2 * 16));
      }
  }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  const int v = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, true));
}

// Over the 64 lanes, the same in each: steps within 16 lanes by DPP (neighbours,
// pairs, mirrored halves, mirrored rows), then the four rows of 16.
__device__ __forceinline__ float wave_sum(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  x += dpp<0x141>(x);
  x += dpp<0x140>(x);
  return column_sum(x);
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  x = fmaxf(x, dpp<0x141>(x));
  x = fmaxf(x, dpp<0x140>(x));
  return column_max(x);
}

}  // namespace fiona
