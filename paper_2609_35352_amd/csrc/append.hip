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
  int64_t n_slot;
};

// One workgroup per token, one pair or copied element per thread and turn.
template <typename T, typename C>
__global__ void __launch_bounds__(256) append_kernel(AppendParams P) {
  const uint32_t t = blockIdx.x, rot = 2 * P.half, units = P.d - P.half;   // pairs, then copied elements
  const int64_t slot = P.slots[t];
  const bool keep = slot >= 0 && slot < P.n_slot;
  const uint64_t page = keep ? (uint64_t)slot / P.page_size : 0, at = keep ? (uint64_t)slot % P.page_size : 0;
  const int32_t pos = P.half ? P.positions[t] : 0;
  const bool known = pos >= 0 && (uint32_t)pos < P.n_pos;
  const uint32_t heads = P.n_head + 2 * P.n_kv;
  for (uint32_t i = threadIdx.x; i < heads * units; i += 256) {
    uint32_t h = i / units, u = i % units;
    const T *in;
    C *out;
    bool turn = true;
    if (h < P.n_head) {
      in = (const T *)P.q + t * P.q_tok + h * P.q_head;
      out = (C *)P.q_out + t * P.qo_tok + h * P.qo_head;
    } else {
      if (!keep) continue;
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
    }
    if (u >= P.half) {
      out[rot + (u - P.half)] = (C)(float)in[rot + (u - P.half)];
      continue;
    }
    const uint32_t ia = P.interleaved ? 2 * u : u, ib = P.interleaved ? 2 * u + 1 : u + P.half;
    const float a = (float)in[ia], b = (float)in[ib];
    if (!turn) {
      out[ia] = (C)a;
      out[ib] = (C)b;
      continue;
    }
    const float c = known ? P.cos[(uint64_t)pos * P.half + u] : __builtin_nanf("");
    const float s = known ? P.sin[(uint64_t)pos * P.half + u] : __builtin_nanf("");
    out[ia] = (C)(a * c - b * s);
    out[ib] = (C)(a * s + b * c);
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
  if (A.rot_dim && (!A.positions || !A.cos || !A.sin)) return FIONA_ERR_ARG;
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
  with_type(A.rows_type, [&](auto t) {
    with_type(K.type, [&](auto c) {
      hipLaunchKernelGGL((fiona::append_kernel<decltype(t), decltype(c)>), dim3(A.n_tok), dim3(256), 0, stream, P);
    });
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}
