// fiona_paged_attention (include/fiona.h): one new token of each sequence over
// its paged cache.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>

#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_attention {
  fiona_attention_desc desc{};
  int device = -1;
};

namespace fiona {

struct AttendParams {
  const void *q, *kc, *vc;
  void *out;
  float *lse;
  const int32_t *table, *lengths;
  uint64_t q_seq, q_head, out_seq, out_head, table_stride;
  uint64_t k_page, k_token, k_head, v_page, v_token, v_head;
  uint32_t n_head, group, d, page_size, n_pages, window, max_length;
  float scale, softcap;
};

// A workgroup of four wavefronts per (sequence, query head).  Wavefront w
// takes keys w, w + 4, ... with a running maximum and sum, each lane holding
// up to four elements of the head; the four are joined at the end.
template <typename T>
__global__ void __launch_bounds__(256) attend_kernel(AttendParams P) {
  __shared__ float sm[4], sl[4], so[4][FIONA_MAX_HEAD_DIM];
  const uint32_t h = blockIdx.x, s = blockIdx.y, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int32_t n = P.lengths[s];
  n = n < 0 ? 0 : (uint32_t)n > P.max_length ? (int32_t)P.max_length : n;
  const int32_t first = P.window && (uint32_t)n > P.window ? n - (int32_t)P.window : 0;
  const T *q = (const T *)P.q + s * P.q_seq + h * P.q_head;
  float qv[4], o[4] = {0, 0, 0, 0}, m = -INFINITY, l = 0;
  for (int e = 0; e < 4; ++e) qv[e] = lane + 64 * e < P.d ? (float)q[lane + 64 * e] : 0.f;
  for (int32_t j = first + (int32_t)w; j < n; j += 4) {
    const int32_t page = P.table[s * P.table_stride + (uint32_t)j / P.page_size];
    if (page < 0 || (uint32_t)page >= P.n_pages) continue;
    const uint64_t at = (uint32_t)j % P.page_size, kh = h / P.group;
    const T *k = (const T *)P.kc + page * P.k_page + at * P.k_token + kh * P.k_head;
    const T *v = (const T *)P.vc + page * P.v_page + at * P.v_token + kh * P.v_head;
    float dot = 0, vv[4];
    for (int e = 0; e < 4; ++e) {
      const bool in = lane + 64 * e < P.d;
      dot += in ? qv[e] * (float)k[lane + 64 * e] : 0.f;
      vv[e] = in ? (float)v[lane + 64 * e] : 0.f;
    }
    for (int x = 32; x; x >>= 1) dot += __shfl_xor(dot, x);
    dot *= P.scale;
    if (P.softcap > 0) dot = P.softcap * tanhf(dot / P.softcap);
    const float mn = fmaxf(m, dot), ms = mn == -INFINITY ? 0.f : mn;
    const float keep = expf(m - ms), p = expf(dot - ms);
    l = l * keep + p;
    for (int e = 0; e < 4; ++e) o[e] = o[e] * keep + p * vv[e];
    m = mn;
  }
  if (lane == 0) sm[w] = m, sl[w] = l;
  for (int e = 0; e < 4; ++e) so[w][lane + 64 * e] = o[e];
  __syncthreads();
  const float mt = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), ms = mt == -INFINITY ? 0.f : mt;
  float lt = 0, ot = 0;
  const uint32_t e = threadIdx.x;
  for (int i = 0; i < 4; ++i) {
    const float f = expf(sm[i] - ms);
    lt += sl[i] * f;
    ot += so[i][e] * f;
  }
  if (e < P.d) ((T *)P.out)[s * P.out_seq + h * P.out_head + e] = (T)(lt == 0 ? 0.f : ot / lt);
  if (e == 0 && P.lse) P.lse[(uint64_t)s * P.n_head + h] = lt == 0 ? -INFINITY : ms + logf(lt);
}

}  // namespace fiona

extern "C" {

int fiona_attention_create(const fiona_attention_desc *desc, fiona_attention **out) {
  if (!out) return FIONA_ERR_ARG;
  *out = nullptr;
  if (!desc) return FIONA_ERR_ARG;
  const fiona_attention_desc &D = *desc;
  if (!known_type(D.type)) return FIONA_ERR_UNSUPPORTED;
  if (!D.n_head || !D.n_kv || D.n_head % D.n_kv || !D.head_dim || !D.page_size || !D.max_seq || !D.max_length)
    return FIONA_ERR_ARG;
  if (D.head_dim > FIONA_MAX_HEAD_DIM || D.n_head > 65535 || D.max_seq > 65535 || D.max_length >= (1u << 30) ||
      D.page_size >= (1u << 30))
    return FIONA_ERR_UNSUPPORTED;
  fiona_attention *H = new (std::nothrow) fiona_attention;
  if (!H) return FIONA_ERR_NOMEM;
  H->desc = D;
  if (hipGetDevice(&H->device) != hipSuccess) {
    delete H;
    return FIONA_ERR_HIP;
  }
  *out = H;
  return FIONA_OK;
}

void fiona_attention_destroy(fiona_attention *att) { delete att; }

int fiona_paged_attention(const fiona_attention *att, const fiona_kv_cache *cache, const fiona_attention_args *args,
                          hipStream_t stream) {
  if (!att || !cache || !args) return FIONA_ERR_ARG;
  const fiona_attention_desc &D = att->desc;
  const fiona_kv_cache &K = *cache;
  const fiona_attention_args &A = *args;
  if (K.type != D.type || K.n_kv != D.n_kv || K.head_dim != D.head_dim || K.page_size != D.page_size)
    return FIONA_ERR_ARG;
  if (A.n_seq > D.max_seq || !(A.scale > 0) || !std::isfinite(A.scale) || !(A.softcap >= 0) || !std::isfinite(A.softcap))
    return FIONA_ERR_ARG;
  if ((uint64_t)K.n_pages * K.page_size >= (1u << 31)) return FIONA_ERR_UNSUPPORTED;
  if (A.n_seq == 0) return FIONA_OK;
  if (!A.q || !A.out || !A.lengths || (A.table_width && !A.page_table) || A.table_stride < A.table_width ||
      (K.n_pages && (!K.k || !K.v)))
    return FIONA_ERR_ARG;
  const uint64_t e = type_size(D.type), d = D.head_dim, n = A.n_seq;
  if (misaligned(A.q, e) || misaligned(A.out, e) || misaligned(K.k, e) || misaligned(K.v, e) ||
      misaligned(A.lse, 4) || misaligned(A.page_table, 4) || misaligned(A.lengths, 4))
    return FIONA_ERR_ALIGN;
  const Rows in[] = {{A.q, e, d, {n, D.n_head, 1}, {A.q_seq, A.q_head, 0}},
                     {K.k, e, d, {K.n_pages, K.page_size, K.n_kv}, {K.k_page, K.k_token, K.k_head}},
                     {K.v, e, d, {K.n_pages, K.page_size, K.n_kv}, {K.v_page, K.v_token, K.v_head}},
                     {A.page_table, 4, A.table_width, {n, 1, 1}, {A.table_stride, 0, 0}},
                     {A.lengths, 4, n, {1, 1, 1}, {0, 0, 0}}};
  const Rows out[] = {{A.out, e, d, {n, D.n_head, 1}, {A.out_seq, A.out_head, 0}},
                      {A.lse, 4, n * D.n_head, {1, 1, 1}, {0, 0, 0}}};
  uint64_t elems;
  for (const Rows &r : in)
    if (!empty(r) && !span(r, elems)) return FIONA_ERR_ARG;
  for (const Rows &r : out)
    if (!empty(r) && (!span(r, elems) || !rows_distinct(r))) return FIONA_ERR_ALIAS;
  if (may_overlap(out[0], out[1])) return FIONA_ERR_ALIAS;
  for (const Rows &o : out)
    for (const Rows &r : in)
      if (may_overlap(o, r)) return FIONA_ERR_ALIAS;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != att->device) return FIONA_ERR_ARG;

  fiona::AttendParams P{};
  P.q = A.q, P.kc = K.k, P.vc = K.v, P.out = A.out, P.lse = A.lse, P.table = A.page_table, P.lengths = A.lengths;
  P.q_seq = A.q_seq, P.q_head = A.q_head, P.out_seq = A.out_seq, P.out_head = A.out_head, P.table_stride = A.table_stride;
  P.k_page = K.k_page, P.k_token = K.k_token, P.k_head = K.k_head;
  P.v_page = K.v_page, P.v_token = K.v_token, P.v_head = K.v_head;
  P.n_head = D.n_head, P.group = D.n_head / D.n_kv, P.d = D.head_dim, P.page_size = D.page_size, P.n_pages = K.n_pages;
  P.window = A.window, P.scale = A.scale, P.softcap = A.softcap;
  P.max_length = (uint32_t)std::min<uint64_t>(D.max_length, (uint64_t)A.table_width * D.page_size);
  with_type(D.type, [&](auto t) {
    hipLaunchKernelGGL((fiona::attend_kernel<decltype(t)>), dim3(D.n_head, A.n_seq), dim3(256), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
