// fiona_kv_append (include/fiona.h): new keys and values into a paged cache,
// rotated by position on the way, the queries rotated in the same launch.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

namespace fiona {

struct AppendParams {
  const void *q, *k, *v;
  void *q_out, *kc, *vc;
  const int64_t *slots;
  const int32_t *positions;
  const float *cos, *sin;
  uint64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, qo_tok, qo_head;
  uint64_t kc_page, kc_token, kc_head, vc_page, vc_token, vc_head;
  uint32_t n_tok, n_head, n_kv, d, half, n_pos, interleaved, page_size;
  uint32_t page_mul, page_shift;   // slot / page_size (see page_divisor)
  uint32_t tokens;                 // of a workgroup
  int64_t n_slot;
};

// The page and place of a token's slot; false where it is not in the cache.
__device__ __forceinline__ bool place_of(const AppendParams &P, uint32_t t, uint64_t &page, uint64_t &at) {
  const int64_t slot = P.slots[t];
  if (slot < 0 || slot >= P.n_slot) return false;
  page = P.page_mul ? __umulhi((uint32_t)slot, P.page_mul) >> P.page_shift : (uint32_t)slot;
  at = (uint32_t)slot - (uint32_t)page * P.page_size;
  return true;
}

// A row's source and destination by its number in the token: query heads, key
// heads, value heads; false where it is not written.
template <typename T, typename C>
__device__ __forceinline__ bool row_of(const AppendParams &P, uint32_t t, uint32_t h, const T *&in, C *&out, bool &turn) {
  turn = true;
  if (h < P.n_head) {
    in = (const T *)P.q + t * P.q_tok + h * P.q_head;
    out = (C *)P.q_out + t * P.qo_tok + h * P.qo_head;
    return true;
  }
  uint64_t page, at;
  if (!place_of(P, t, page, at)) return false;
  h -= P.n_head;
  if (h < P.n_kv) {
    in = (const T *)P.k + t * P.k_tok + h * P.k_head;
    out = (C *)P.kc + page * P.kc_page + at * P.kc_token + h * P.kc_head;
  } else {
    h -= P.n_kv;
    in = (const T *)P.v + t * P.v_tok + h * P.v_head;
    out = (C *)P.vc + page * P.vc_page + at * P.vc_token + h * P.vc_head;
    turn = false;
  }
  return true;
}

// Eight elements from and to 16-byte aligned rows, through 32 bits.
template <typename T>
struct alignas(16) Eight {
  T x[8];
};
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
  const Eight<T> v = *(const Eight<T> *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v.x[i];
}
template <typename C>
__device__ __forceinline__ void store8(C *p, const float (&x)[8]) {
  Eight<C> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v.x[i] = (C)x[i];
  typedef uint32_t w4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (uint32_t i = 0; i < sizeof(v) / 16; ++i) __builtin_nontemporal_store(((const w4 *)&v)[i], (w4 *)p + i);
}

// Whole pieces: a thread takes 16 elements of a row (eight pairs, or up to two
// runs of eight copied ones), consecutive threads consecutive pieces of a row,
// then rows, then tokens; workgroups hold whole tokens where more than one fits.
// Two loads and two stores of 16 bytes a thread (four of each in 32 bits) are all
// that is in flight, and the rotation is 3 operations a byte.  Everything is read
// and written once: what bounds it is memory (16384 tokens of 32 + 8 + 8 heads of
// 128 in bfloat16, 411 MB: 69 us, 6.0 TB/s; stores that pass the caches by reach
// more than a plain copy's 5.1), or for a few tokens the launch (8 of 12 + 12 + 12
// heads of 64: 3.4 us on the GPU, 10.2 a call from Python).
template <typename T, typename C>
__global__ void __launch_bounds__(256) append_kernel(AppendParams P) {
  const uint32_t units = (P.d + 15) / 16, items = (P.n_head + 2 * P.n_kv) * units;
  const uint32_t i = blockIdx.y * 256 + threadIdx.x;
  const uint32_t t = blockIdx.x * P.tokens + i / items, h = i % items / units, u = i % units;
  if (i >= P.tokens * items || t >= P.n_tok) return;
  const T *in;
  C *out;
  bool turn;
  if (!row_of(P, t, h, in, out, turn)) return;
  float a[8], b[8], x[8], y[8];
  if (turn && 8 * u < P.half) {
    const uint32_t ia = P.interleaved ? 16 * u : 8 * u, ib = P.interleaved ? 16 * u + 8 : 8 * u + P.half;
    const int32_t pos = P.positions[t];
    const bool known = pos >= 0 && (uint32_t)pos < P.n_pos;
    const uint64_t at = (uint64_t)(known ? pos : 0) * P.half + 8 * u;
    load8(in + ia, a);
    load8(in + ib, b);
    load8(P.cos + at, x);
    load8(P.sin + at, y);
    if (!known)
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __builtin_nanf("");
    if (P.interleaved) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {   // pairs 0..3 in the first run, 4..7 in the second
        float(&r)[8] = k < 4 ? a : b;
        const float p = r[2 * k % 8], q = r[2 * k % 8 + 1];
        r[2 * k % 8] = p * x[k] - q * y[k];
        r[2 * k % 8 + 1] = p * y[k] + q * x[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float p = a[k], q = b[k];
        a[k] = p * x[k] - q * y[k];
        b[k] = p * y[k] + q * x[k];
      }
    }
    store8(out + ia, a);
    store8(out + ib, b);
    return;
  }
  const uint32_t e = 16 * u;
  const bool two = e + 8 < P.d;
  load8(in + e, a);
  load8(in + (two ? e + 8 : e), b);
  store8(out + e, a);
  if (two) store8(out + e + 8, b);
}

// Rows of any size and alignment: one workgroup per token, one pair or copied
// element per thread and turn; bound by the instructions to do so (16384 tokens
// of 48 heads of 65 in bfloat16, 210 MB: 109 us, 1.9 TB/s).
template <typename T, typename C>
__global__ void __launch_bounds__(256) append_any_kernel(AppendParams P) {
  const uint32_t t = blockIdx.x, rot = 2 * P.half, units = P.d - P.half;   // pairs, then copied elements
  const int32_t pos = P.half ? P.positions[t] : 0;
  const bool known = pos >= 0 && (uint32_t)pos < P.n_pos;
  for (uint32_t i = threadIdx.x; i < (P.n_head + 2 * P.n_kv) * units; i += 256) {
    const uint32_t u = i % units;
    const T *in;
    C *out;
    bool turn;
    if (!row_of(P, t, i / units, in, out, turn)) continue;
    if (u >= P.half) {
      out[rot + (u - P.half)] = (C)(float)in[rot + (u - P.half)];
      continue;
    }
    const uint32_t ia = P.interleaved ? 2 * u : u, ib = P.interleaved ? 2 * u + 1 : u + P.half;
    const float a = (float)in[ia], b = (float)in[ib];
    const float c = !turn ? 1.f : known ? P.cos[(uint64_t)pos * P.half + u] : __builtin_nanf("");
    const float s = !turn ? 0.f : known ? P.sin[(uint64_t)pos * P.half + u] : 0.f;
    out[ia] = (C)(turn ? a * c - b * s : a);
    out[ib] = (C)(turn ? a * s + b * c : b);
  }
}

}  // namespace fiona

extern "C" int fiona_kv_append(const fiona_kv_cache *cache, const fiona_append_args *args, hipStream_t stream) {
  if (!cache || !args) return FIONA_ERR_ARG;
  const fiona_kv_cache &K = *cache;
  const fiona_append_args &A = *args;
  if (!known_type(K.type) || !known_type(A.rows_type)) return FIONA_ERR_UNSUPPORTED;
  if (K.n_kv == 0 || K.head_dim == 0 || K.page_size == 0) return FIONA_ERR_ARG;
  if (K.head_dim > FIONA_MAX_HEAD_DIM || (uint64_t)K.n_pages * K.page_size >= (1u << 31) ||
      (uint64_t)A.n_head + 2ull * K.n_kv > 65535 || A.n_tok >= (1u << 24))
    return FIONA_ERR_UNSUPPORTED;
  if (A.rot_dim % 2 != 0 || A.rot_dim > K.head_dim) return FIONA_ERR_ARG;
  if (A.n_tok == 0) return FIONA_OK;
  if (!A.k || !A.v || !A.slots || (K.n_pages && (!K.k || !K.v))) return FIONA_ERR_ARG;
  if (A.n_head && (!A.q || !A.q_out)) return FIONA_ERR_ARG;
  if (A.rot_dim && (!A.positions || (A.n_pos && (!A.cos || !A.sin)))) return FIONA_ERR_ARG;
  const uint64_t es = type_size(A.rows_type), ec = type_size(K.type), d = K.head_dim;
  if (misaligned(A.k, es) || misaligned(A.v, es) || misaligned(K.k, ec) || misaligned(K.v, ec) ||
      misaligned(A.slots, 8) || (A.n_head && (misaligned(A.q, es) || misaligned(A.q_out, ec))) ||
      (A.rot_dim && (misaligned(A.positions, 4) || misaligned(A.cos, 4) || misaligned(A.sin, 4))))
    return FIONA_ERR_ALIGN;
  const uint64_t n = A.n_tok;
  const Rows in[] = {{A.k, es, d, {n, K.n_kv, 1}, {A.k_tok, A.k_head, 0}},
                     {A.v, es, d, {n, K.n_kv, 1}, {A.v_tok, A.v_head, 0}},
                     {A.n_head ? A.q : nullptr, es, d, {n, A.n_head, 1}, {A.q_tok, A.q_head, 0}},
                     {A.slots, 8, n, {1, 1, 1}, {0, 0, 0}},
                     {A.rot_dim ? A.positions : nullptr, 4, n, {1, 1, 1}, {0, 0, 0}},
                     {A.rot_dim ? A.cos : nullptr, 4, A.rot_dim / 2, {A.n_pos, 1, 1}, {A.rot_dim / 2, 0, 0}},
                     {A.rot_dim ? A.sin : nullptr, 4, A.rot_dim / 2, {A.n_pos, 1, 1}, {A.rot_dim / 2, 0, 0}}};
  const Rows out[] = {{K.k, ec, d, {K.n_pages, K.page_size, K.n_kv}, {K.k_page, K.k_token, K.k_head}},
                      {K.v, ec, d, {K.n_pages, K.page_size, K.n_kv}, {K.v_page, K.v_token, K.v_head}},
                      {A.n_head ? A.q_out : nullptr, ec, d, {n, A.n_head, 1}, {A.q_out_tok, A.q_out_head, 0}}};
  uint64_t elems;
  for (const Rows &r : in)
    if (!empty(r) && !span(r, elems)) return FIONA_ERR_ARG;
  for (const Rows &r : out)
    if (!empty(r) && (!span(r, elems) || !rows_distinct(r))) return FIONA_ERR_ALIAS;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (may_overlap(out[i], out[j])) return FIONA_ERR_ALIAS;
  const bool in_place = A.n_head && A.q == A.q_out && A.rows_type == K.type && A.q_tok == A.q_out_tok &&
                        A.q_head == A.q_out_head;
  for (const Rows &o : out)
    for (const Rows &r : in)
      if (!(in_place && &o == &out[2] && &r == &in[2]) && may_overlap(o, r)) return FIONA_ERR_ALIAS;

  fiona::AppendParams P{};
  P.q = A.q, P.k = A.k, P.v = A.v, P.q_out = A.q_out, P.kc = K.k, P.vc = K.v;
  P.slots = A.slots, P.positions = A.positions, P.cos = A.cos, P.sin = A.sin;
  P.q_tok = A.q_tok, P.q_head = A.q_head, P.k_tok = A.k_tok, P.k_head = A.k_head, P.v_tok = A.v_tok, P.v_head = A.v_head;
  P.qo_tok = A.q_out_tok, P.qo_head = A.q_out_head;
  P.kc_page = K.k_page, P.kc_token = K.k_token, P.kc_head = K.k_head;
  P.vc_page = K.v_page, P.vc_token = K.v_token, P.vc_head = K.v_head;
  P.n_tok = A.n_tok, P.n_head = A.n_head, P.n_kv = K.n_kv, P.d = K.head_dim, P.half = A.rot_dim / 2, P.n_pos = A.n_pos;
  P.interleaved = A.interleaved != 0, P.page_size = K.page_size;
  P.n_slot = (int64_t)K.n_pages * K.page_size;
  page_divisor(K.page_size, P.page_mul, P.page_shift);
  // 16-byte pieces where every row and its halves hold whole ones (16384 tokens of 48
  // heads 5.9 TB/s, by elements 1.9; 1531 of 25, 80 and 81 elements long, the same),
  // and the tables have a row, as a position outside them reads the first, unused.
  const bool pieces = d % 8 == 0 && P.half % 8 == 0 && rows_aligned16(in[0]) && rows_aligned16(in[1]) &&
                      rows_aligned16(out[0]) && rows_aligned16(out[1]) &&
                      (!A.n_head || (rows_aligned16(in[2]) && rows_aligned16(out[2]))) &&
                      (!A.rot_dim || (A.n_pos && rows_aligned16(in[5]) && rows_aligned16(in[6])));
  const uint32_t items = (A.n_head + 2 * K.n_kv) * ((uint32_t)(d + 15) / 16);
  P.tokens = std::max(1u, 256 / items);
  const dim3 grid = pieces ? dim3((A.n_tok + P.tokens - 1) / P.tokens, (P.tokens * items + 255) / 256) : dim3(A.n_tok);
  with_type(A.rows_type, [&](auto t) {
    with_type(K.type, [&](auto c) {
      using T = decltype(t);
      using C = decltype(c);
      if (pieces) hipLaunchKernelGGL((fiona::append_kernel<T, C>), grid, dim3(256), 0, stream, P);
      else hipLaunchKernelGGL((fiona::append_any_kernel<T, C>), grid, dim3(256), 0, stream, P);
    });
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}
