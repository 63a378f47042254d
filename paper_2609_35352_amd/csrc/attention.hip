// fiona_paged_attention (include/fiona.h): one new token of each sequence over
// its paged cache.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>

#include "attention_kernel.hpp"
#include "fiona.h"
#include "rows.hpp"

using namespace fiona_host;

struct fiona_attention {
  fiona_attention_desc desc{};
  int device = -1;
  float *part = nullptr;      // the parts of split sequences
  uint64_t part_cap = 0;      // (sequence, split) pairs that fit, n_head heads each
};

namespace {

// Keys of one workgroup's chunk for calls over up to `keys` keys of `units`
// sequences times key heads: enough chunks to fill the GPU several times, but
// none below kMinChunk (a chunk's first loads wait for the length, then the
// table), none above kMaxChunk so that ragged lengths even out, at most
// kMaxSplits parts to join, and no join for what one workgroup does as fast.
// Chunks of 256 / 512 / 768 / 1024 / 2048 / 4096, us: 64 sequences of 100 to 8192
// keys, 8 key heads of 128, 106 / 101 / 95 / 111 / 142 / 143; 19 of up to 3000,
// 7 of 80, 20.2 / 24.8 / 25.5 / 27.0 / 32.0 / 38.3; 2 of 100000 and 131072, 8 of
// 128 (2048 at least for 64 parts), 159, at 4096 156; 1 of 300, 12 of 64 in 32 bits,
// 11.2 in two parts, 8.8 whole.
constexpr uint32_t kMinChunk = 256, kMaxChunk = 768, kNoSplit = 512, kWorkgroups = 2048;
using fiona::kMaxSplits;
uint32_t chunk_of(uint64_t keys, uint64_t units) {
  if (keys <= kNoSplit) return kNoSplit;
  uint64_t c = (keys * units + kWorkgroups - 1) / kWorkgroups;
  c = std::max<uint64_t>(kMinChunk, std::min<uint64_t>(c, kMaxChunk));
  c = std::max<uint64_t>(c, (keys + kMaxSplits - 1) / kMaxSplits);
  return (uint32_t)((c + 127) / 128 * 128);
}

uint32_t splits_of(uint64_t keys, uint32_t chunk) { return keys ? (uint32_t)((keys + chunk - 1) / chunk) : 1; }

uint32_t head_blocks(const fiona_attention_desc &D) { return (D.n_head / D.n_kv + 15) / 16; }

template <typename T, int HD>
void launch_split(const fiona::AttendParams &P, bool vec, bool span, dim3 grid, hipStream_t stream) {
  if (vec && span) hipLaunchKernelGGL((fiona::attend_kernel<T, HD, true, true>), grid, dim3(256), 0, stream, P);
  else if (vec) hipLaunchKernelGGL((fiona::attend_kernel<T, HD, true, false>), grid, dim3(256), 0, stream, P);
  else hipLaunchKernelGGL((fiona::attend_kernel<T, HD, false, false>), grid, dim3(256), 0, stream, P);
}

}  // namespace

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
  for (uint64_t n = 1; n <= D.max_seq; ++n) {
    const uint32_t splits = splits_of(D.max_length, chunk_of(D.max_length, n * D.n_kv * head_blocks(D)));
    if (splits > 1) H->part_cap = std::max<uint64_t>(H->part_cap, n * splits);
  }
  const uint64_t bytes = H->part_cap * D.n_head * (D.head_dim + 2) * sizeof(float);
  if (bytes && hipMalloc((void **)&H->part, bytes) != hipSuccess) {
    (void)hipGetLastError();
    delete H;
    return FIONA_ERR_NOMEM;
  }
  *out = H;
  return FIONA_OK;
}

void fiona_attention_destroy(fiona_attention *att) {
  if (!att) return;
  if (att->part) (void)hipFree(att->part);
  delete att;
}

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
  if (!A.q || !A.out || !A.lengths || (A.table_width && !A.page_table) || (K.n_pages && (!K.k || !K.v)))
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
  P.n_head = D.n_head, P.group = D.n_head / D.n_kv, P.head_blocks = head_blocks(D), P.d = D.head_dim;
  P.page_size = D.page_size, P.n_pages = K.n_pages, P.window = A.window;
  P.unit = (float)std::min<double>((double)A.scale * fiona::kLog2e, FLT_MAX);
  if (A.softcap > 0) {
    P.unit = fiona::kLog2e, P.scale = A.scale, P.cap = A.softcap;
    P.cap_in = (float)std::min<double>(2. * fiona::kLog2e * A.scale / A.softcap, FLT_MAX);
  }
  page_divisor(D.page_size, P.page_mul, P.page_shift);
  P.max_length = (uint32_t)std::min<uint64_t>(D.max_length, (uint64_t)A.table_width * D.page_size);
  if (K.n_pages == 0) P.max_length = 0;
  // A window's keys start anywhere in a tile.
  const uint64_t keys = A.window ? std::min<uint64_t>(P.max_length, (uint64_t)A.window + 32) : P.max_length;
  P.chunk = chunk_of(keys, n * D.n_kv * P.head_blocks);
  P.splits = splits_of(keys, P.chunk);
  while (P.splits > 1 && n * P.splits > att->part_cap) P.chunk *= 2, P.splits = splits_of(keys, P.chunk);
  P.part_ml = att->part, P.part = att->part + 2 * att->part_cap * D.n_head;
  const dim3 grid(D.n_kv * P.head_blocks, P.splits, A.n_seq);
  with_type(D.type, [&](auto t) {
    using T = decltype(t);
    const bool vec = D.head_dim % fiona::kLaneElems<T> == 0 && rows_aligned16(in[0]) && rows_aligned16(in[1]) && rows_aligned16(in[2]);
    const bool span = D.page_size % (uint32_t)fiona::kSpan<T> == 0;
    if (D.head_dim <= 64) launch_split<T, 64>(P, vec, span, grid, stream);
    else if (D.head_dim <= 128) launch_split<T, 128>(P, vec, span, grid, stream);
    else launch_split<T, 256>(P, vec, span, grid, stream);
    const dim3 rows(D.n_head, A.n_seq);
    if (P.splits > 16) hipLaunchKernelGGL((fiona::attend_join_kernel<T, 4>), rows, dim3(1024), 0, stream, P);
    else if (P.splits > 1) hipLaunchKernelGGL((fiona::attend_join_kernel<T, 1>), rows, dim3(256), 0, stream, P);
  });
  return hipGetLastError() == hipSuccess ? FIONA_OK : FIONA_ERR_HIP;
}

}  // extern "C"
