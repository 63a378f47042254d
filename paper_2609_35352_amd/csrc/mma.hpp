// Matrix-core tiles of the key holder's operators: 16 x 16 products of rows
// held 16 bytes per lane.
//
// A fragment is 16 bytes of one row: lane l holds row l % 16, and the four
// lanes of a row (l / 16) hold consecutive 16-byte pieces.  The contraction
// takes the pieces in any order as long as both operands use the same one, so
// rows that are contiguous in memory need no shuffle.  In the result lane l
// holds column l % 16, rows 4 (l / 16) + i, i < 4.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fiona {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// Elements in a lane's 16 bytes, and of a row in one fragment.
template <typename T>
constexpr uint32_t kLaneElems = 16 / sizeof(T);
template <typename T>
constexpr uint32_t kFragElems = 4 * kLaneElems<T>;

template <typename T>
__device__ __forceinline__ f4 mma(u4 a, u4 b, f4 c) {
  if constexpr (sizeof(T) == 4) {
    const f4 x = __builtin_bit_cast(f4, a), y = __builtin_bit_cast(f4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  } else if constexpr (__is_same(T, _Float16)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  }
}

// Words of W elements of T from p of which the first `valid` may be read, the
// rest zero.  VEC: p is aligned to the W elements and valid is 0 or >= W.
// Nontemporal: what these operators read once per call passes the caches by.
template <typename T, int W, bool VEC>
__device__ __forceinline__ void load_row(const T *p, int valid, uint32_t (&w)[W * sizeof(T) / 4]) {
  constexpr int N = W * sizeof(T) / 4;
  if constexpr (VEC) {
    if constexpr (N == 4) {
      const u4 v = valid > 0 ? __builtin_nontemporal_load((const u4 *)p) : (u4){0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else {
      static_assert(N == 2, "8 or 16 bytes per lane");
      const u2 v = valid > 0 ? __builtin_nontemporal_load((const u2 *)p) : (u2){0, 0};
      w[0] = v[0], w[1] = v[1];
    }
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = i < valid ? ((const uint32_t *)p)[i] : 0;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t lo = 2 * i < valid ? ((const uint16_t *)p)[2 * i] : 0;
      const uint32_t hi = 2 * i + 1 < valid ? ((const uint16_t *)p)[2 * i + 1] : 0;
      w[i] = lo | hi << 16;
    }
  }
}

// A lane's 16 bytes of a row of n >= kLaneElems elements, from element `at`.
// piece_at gives an address inside the row whatever `at` is (the row's last 16
// bytes where fewer follow), so that loads need no branch; piece_fix then
// moves what was loaded to its place, zero from n on.  Rows start at any
// element: the memory system takes 16-byte accesses at any address.
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));
template <typename T>
__device__ __forceinline__ const T *piece_at(const T *row, uint32_t at, uint32_t n) {
  return row + (at + kLaneElems<T> <= n ? at : n - kLaneElems<T>);
}
template <typename T>
__device__ __forceinline__ u4 piece_fix(u4 v, uint32_t at, uint32_t n) {
  if (at + kLaneElems<T> <= n) return v;
  if (at >= n) return (u4){0, 0, 0, 0};
  const uint32_t bits = (at + kLaneElems<T> - n) * 8 * sizeof(T);
  return __builtin_bit_cast(u4, __builtin_bit_cast(unsigned __int128, v) >> bits);
}
// Read once per call (past the caches), or by many workgroups.
template <typename T>
__device__ __forceinline__ u4 load_once(const T *p) {
  return __builtin_nontemporal_load((const u4_any *)p);
}
template <typename T>
__device__ __forceinline__ u4 load_shared(const T *p) {
  return *(const u4_any *)p;
}

// The first `valid` elements of a lane's 16 bytes as a mask.
template <typename T>
__device__ __forceinline__ u4 first_mask(int valid) {
  u4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) m[i] = i < valid ? ~0u : 0;
    else m[i] = 2 * i + 1 < valid ? ~0u : 2 * i < valid ? 0xFFFFu : 0;
  }
  return m;
}

// 32-bit values for a contraction with rows of T: in 16 bits as the sum of two
// bfloat16 parts (an error of 2^-16 of the value, and its whole range; one part
// would lose 2^-8, binary16 its range as well).
__device__ __forceinline__ uint32_t split_pair(float a, float b, uint32_t &lo) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  const bf2 h = {(__bf16)a, (__bf16)b};
  const bf2 l = {(__bf16)(a - (float)h[0]), (__bf16)(b - (float)h[1])};
  lo = __builtin_bit_cast(uint32_t, l);
  return __builtin_bit_cast(uint32_t, h);
}

// c += a * w, a a fragment of T, w one of 32-bit values in two parts.  binary16
// rows are split the same way, exactly (11 bits).
template <typename T>
__device__ __forceinline__ f4 mma_wide(u4 a, u4 hi, u4 lo, f4 c) {
  if constexpr (sizeof(T) == 4) {
    return mma<T>(a, hi, c);
  } else if constexpr (__is_same(T, _Float16)) {
    const h8 x = __builtin_bit_cast(h8, a);
    u4 ah, al;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t l;
      ah[i] = split_pair((float)x[2 * i], (float)x[2 * i + 1], l);
      al[i] = l;
    }
    return mma<__bf16>(ah, hi, mma<__bf16>(ah, lo, mma<__bf16>(al, hi, c)));
  } else {
    return mma<T>(a, hi, mma<T>(a, lo, c));
  }
}

// Two values rounded to 16 bits, the first in the low half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  static_assert(sizeof(T) == 2, "16-bit types");
  typedef T t2 __attribute__((ext_vector_type(2)));
  const t2 v = {(T)a, (T)b};
  return __builtin_bit_cast(uint32_t, v);
}

// The halves of two rows' words side by side: (low a, low b) or (high a, high b).
__device__ __forceinline__ uint32_t pair_low(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t pair_high(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// This wavefront's number in its workgroup, in a scalar register: branches and
// addresses that depend on it need no lane masks.  grad_kernel's results need it too:
// with the number in a vector register its loop over steps counts as divergent, and
// the two sets of operands that take turns in it came out overwritten.
__device__ __forceinline__ uint32_t wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// What one lane of a wavefront wrote to LDS another reads next.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Sum and maximum over the four lanes of one column (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float column_max(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float y = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const uint32_t v = __builtin_bit_cast(uint32_t, y);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float y = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
  const uint32_t v = __builtin_bit_cast(uint32_t, y);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}

}  // namespace fiona
