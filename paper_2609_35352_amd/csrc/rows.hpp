// Element types and strided rows of the key holder's operators
// (kv_append, paged attention, adapters).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <utility>

#include "fiona.h"

namespace fiona_host {

inline bool known_type(uint32_t type) { return type == FIONA_F32 || type == FIONA_F16 || type == FIONA_BF16; }
inline uint32_t type_size(uint32_t type) { return type == FIONA_F32 ? 4 : 2; }

// Calls f with a value of the element type.
template <typename F>
void with_type(uint32_t type, F f) {
  if (type == FIONA_F32) f(float{});
  else if (type == FIONA_F16) f(_Float16{});
  else f(__bf16{});
}

// Rows of `width` contiguous elements at up to three strided axes.
struct Rows {
  const void *base;
  uint64_t elem, width;
  uint64_t n[3], stride[3];
};

inline bool empty(const Rows &r) { return !r.base || !r.width || !r.n[0] || !r.n[1] || !r.n[2]; }

// Elements from the first row's start to the last row's end; false where the
// sum passes 2^62 bytes (no such buffer exists).
inline bool span(const Rows &r, uint64_t &elems) {
  unsigned __int128 e = r.width;
  for (int i = 0; i < 3; ++i) e += (unsigned __int128)(r.n[i] - 1) * r.stride[i];
  elems = (uint64_t)e;
  return e * r.elem < ((unsigned __int128)1 << 62);
}

// Whether no two rows share an element: from the smallest stride up, each
// axis steps over all that the smaller ones span.
inline bool rows_distinct(const Rows &r) {
  std::pair<uint64_t, uint64_t> ax[3];
  for (int i = 0; i < 3; ++i) ax[i] = {r.stride[i], r.n[i]};
  std::sort(ax, ax + 3);
  unsigned __int128 reach = r.width;
  for (auto &a : ax) {
    if (a.second <= 1) continue;
    if (a.first < reach) return false;
    reach += (unsigned __int128)(a.second - 1) * a.first;
  }
  return true;
}

// Whether two sets of rows may share a byte.  Where their ranges overlap they
// are still apart if both step by the same largest stride and what they hold
// of one step does not meet (queries, keys and values side by side in the
// rows of one projection; keys and values side by side in one page).
inline bool may_overlap(const Rows &a, const Rows &b) {
  if (empty(a) || empty(b)) return false;
  uint64_t ea, eb;
  if (!span(a, ea) || !span(b, eb)) return true;
  const uint64_t a0 = (uint64_t)a.base, b0 = (uint64_t)b.base;
  const uint64_t sa = ea * a.elem, sb = eb * b.elem;
  if (a0 + sa <= b0 || b0 + sb <= a0) return false;
  uint64_t step[2] = {0, 0}, window[2];
  const Rows *rs[2] = {&a, &b};
  const uint64_t bytes[2] = {sa, sb};
  for (int k = 0; k < 2; ++k) {
    uint64_t count = 1;
    for (int i = 0; i < 3; ++i)
      if (rs[k]->n[i] > 1 && rs[k]->stride[i] * rs[k]->elem > step[k]) {
        step[k] = rs[k]->stride[i] * rs[k]->elem;
        count = rs[k]->n[i];
      }
    window[k] = bytes[k] - (count - 1) * step[k];
  }
  if (step[0] != step[1] || step[0] == 0) return true;
  const uint64_t s = step[0];
  const uint64_t delta = b0 >= a0 ? (b0 - a0) % s : (s - (a0 - b0) % s) % s;
  return !(delta >= window[0] && delta + window[1] <= s);
}

// Whether every row starts at a multiple of 16 bytes.
inline bool rows_aligned16(const Rows &r) {
  if ((uint64_t)r.base & 15u) return false;
  for (int i = 0; i < 3; ++i)
    if (r.n[i] > 1 && (r.stride[i] * r.elem) % 16 != 0) return false;
  return true;
}

// Division by a page size: token / page_size = umulhi(token, mul) >> shift for
// token < 2^31, with 2^shift < page_size <= 2^(shift + 1) and
// mul = ceil(2^(32 + shift) / page_size) (whose error, below page_size, times the
// token stays below 2^(32 + shift)); mul 0 for pages of one token.
inline void page_divisor(uint32_t page_size, uint32_t &mul, uint32_t &shift) {
  mul = shift = 0;
  if (page_size <= 1) return;
  shift = 31 - __builtin_clz(page_size - 1);
  mul = (uint32_t)((((uint64_t)1 << (32 + shift)) + page_size - 1) / page_size);
}

inline bool misaligned(const void *p, uint64_t elem) { return ((uint64_t)p & (elem - 1)) != 0; }

}  // namespace fiona_host
