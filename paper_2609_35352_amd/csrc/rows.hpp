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

// Two sets of rows axis by axis, in bytes: axes from the largest step down, what a
// whole set reaches, and how far b starts after a.  At the largest step the sets
// split into copies of what is left; a copy of a and one of b whose steps differ by
// i can meet only where their reaches do, for one or two i in sets that nest.
struct Axis {
  uint64_t step, n;
};
inline bool axes_meet(const Axis *a, int na, __int128 reach_a, const Axis *b, int nb, __int128 reach_b, __int128 delta) {
  if (delta >= reach_a || -delta >= reach_b) return false;
  if (!na && !nb) return true;
  const __int128 s = std::max(na ? a->step : 0, nb ? b->step : 0);
  const bool in_a = na && a->step == (uint64_t)s, in_b = nb && b->step == (uint64_t)s;
  const __int128 most = in_a ? a->n - 1 : 0, least = in_b ? -(__int128)(b->n - 1) : 0;
  reach_a -= most * s, reach_b += least * s;
  // -reach_b < delta - i s < reach_a
  auto floor_div = [&](__int128 x) { return x >= 0 ? x / s : -((-x + s - 1) / s); };
  const __int128 first = std::max(least, floor_div(delta - reach_a) + 1), last = std::min(most, -floor_div(-delta - reach_b) - 1);
  if (last - first > 3) return true;   // (rows over each other, or no common steps: taken to meet)
  for (__int128 i = first; i <= last; ++i)
    if (axes_meet(a + in_a, na - in_a, reach_a, b + in_b, nb - in_b, reach_b, delta - i * s)) return true;
  return false;
}

// Whether two sets of rows may share a byte: exact where their steps nest (queries,
// keys and values side by side in the rows of one projection; keys and values side by
// side in a page, in a token or in a head), true in doubt.
inline bool may_overlap(const Rows &a, const Rows &b) {
  if (empty(a) || empty(b)) return false;
  uint64_t ea, eb;
  if (!span(a, ea) || !span(b, eb)) return true;
  const __int128 delta = (__int128)(uint64_t)b.base - (__int128)(uint64_t)a.base;
  const uint64_t bytes[2] = {ea * a.elem, eb * b.elem};
  if (delta >= (__int128)bytes[0] || -delta >= (__int128)bytes[1]) return false;
  Axis ax[2][3];
  int n[2] = {0, 0};
  const Rows *rs[2] = {&a, &b};
  for (int k = 0; k < 2; ++k) {
    for (int i = 0; i < 3; ++i)
      if (rs[k]->n[i] > 1 && rs[k]->stride[i]) ax[k][n[k]++] = {rs[k]->stride[i] * rs[k]->elem, rs[k]->n[i]};
    std::sort(ax[k], ax[k] + n[k], [](const Axis &x, const Axis &y) { return x.step > y.step; });
  }
  return axes_meet(ax[0], n[0], bytes[0], ax[1], n[1], bytes[1], delta);
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

inline Rows matrix(const void *p, uint64_t e, uint64_t n, uint64_t width, uint64_t row) {
  return Rows{p, e, width, {n, 1, 1}, {row, 0, 0}};
}

// FIONA_ERR_ALIAS where an output's rows overlap each other, another output
// or an input; inputs whose bit is set in own[o] may be output o itself: they are
// passed over where pointer and row stride agree.
inline int check_alias(const Rows *in, int n_in, const Rows *out, int n_out, const uint32_t *own) {
  uint64_t elems;
  for (int i = 0; i < n_in; ++i)
    if (!empty(in[i]) && !span(in[i], elems)) return FIONA_ERR_ARG;
  for (int o = 0; o < n_out; ++o) {
    if (empty(out[o])) continue;
    if (!span(out[o], elems) || !rows_distinct(out[o])) return FIONA_ERR_ALIAS;
    for (int p = o + 1; p < n_out; ++p)
      if (may_overlap(out[o], out[p])) return FIONA_ERR_ALIAS;
    for (int i = 0; i < n_in; ++i) {
      if (own[o] >> i & 1u && in[i].base == out[o].base && (in[i].stride[0] == out[o].stride[0] || in[i].n[0] == 1)) continue;
      if (may_overlap(out[o], in[i])) return FIONA_ERR_ALIAS;
    }
  }
  return FIONA_OK;
}

// Whether a handle's device is the current one, to which every launch goes.
inline bool on_device(int device) {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && dev == device;
}

}  // namespace fiona_host
