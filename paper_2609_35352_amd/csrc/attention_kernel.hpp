// Kernels of fiona_paged_attention.
//
// Softmax over a long axis in parts: a part with keys J has
//     m_J = max s_j,  l_J = sum exp(s_j - m_J),  o_J = sum exp(s_j - m_J) v_j,
// and two parts join as m = max(m_1, m_2), l = sum_i l_i exp(m_i - m), o alike;
// so every key and value is read once, by whichever wavefront holds its part.
// Exponentials are to base 2, with log2(e) in the scale, and of the difference of
// two scores, taken before it is scaled: never above zero, whatever the scores' size
// (a scaled maximum of 2^33, rounded, is off by up to 2^9 powers of two).
//
// A workgroup takes one chunk of one sequence's keys for one key head and up
// to 16 of the query heads that share it; its four wavefronts take tiles of
// the chunk in turn.  Per tile of 32 keys (16 in 32 bits) a wavefront computes
//     S^T = K Q^T     keys x heads
//     O^T += V^T P^T  dims x heads: P^T stays in the registers S^T came in
// Both caches are read whole rows at a time, 16 bytes of 16 lanes to a row.
// K's rows pass through LDS, private to the wavefront, to become fragments:
// read as fragments from memory (64 bytes of 16 rows per instruction) the same
// bytes took 168 to 184 us where rows take 139 to 158 (944 MB of pages, loads alone,
// nontemporal; a plain stream takes 135).  V^T's fragments are picked from the tokens'
// words in registers.  Key `row` of S^T's tile s stands for token (row / 4) *
// kSpan + 4 s + row % 4 of the tile, so that the kSpan tokens whose weights a
// lane ends up with are consecutive, and are the tokens whose rows it loads.
// Softmax weights are rounded to the values' type, each by at most half a unit of
// itself; their sum l uses them unrounded.  binary16, whose normal numbers end at
// 2^-14, takes them times 2^15, so that this holds down to 2^-29 of the largest, and
// below it to within 2^-40 of the largest (a key that outweighs the rest by 2^25 may
// hold no value); l and o carry that factor to the end, where it leaves with their
// quotient.
//
// What bounds it: the cache is read once, and 2 or 4 operations per byte and
// query head are far below the matrix cores' rate.  Two sequences of 100000 and
// 131072 keys, 8 key heads of 128 in bfloat16 (947 MB): 152 us and 5 for the join,
// 6.0 TB/s of the call (a plain stream reads 7.0); 64 of 100 to 8192 (492 MB) 88 and
// 5 us, 5.2 TB/s: chunks of unequal sequences end at unequal times, and each starts
// with a chain of three loads (length, page, keys).  One of 300 keys, 12 heads of 64
// in 32 bits: 8.1 us, those chains.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fiona.h"
#include "mma.hpp"

namespace fiona {

constexpr uint32_t kMaxSplits = 64;   // parts of one sequence
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendParams {
  const void *q, *kc, *vc;
  void *out;
  float *lse;
  const int32_t *table, *lengths;
  float *part, *part_ml;                        // [n_seq][n_head][splits][d]: o, and [..][2]: m and l
  uint64_t q_seq, q_head, out_seq, out_head, table_stride;
  uint64_t k_page, k_token, k_head, v_page, v_token, v_head;
  uint32_t n_head, group, head_blocks, d, page_size, n_pages, window, max_length;
  uint32_t page_mul, page_shift;                // token / page_size (see page_of)
  uint32_t chunk, splits;
  float unit;                                   // of a product q k in powers of two, scale log2(e); log2(e) with a softcap
  float scale, cap, cap_in;                     // with a softcap: scale, the cap (0 without) and 2 log2(e) scale / cap
};

// token / page_size for token < 2^31 (see page_divisor).
__device__ __forceinline__ uint32_t page_of(const AttendParams &P, uint32_t token) {
  return P.page_mul ? __umulhi(token, P.page_mul) >> P.page_shift : token;
}

// The tokens sequence s attends to, [first, n).
__device__ __forceinline__ void key_range(const AttendParams &P, uint32_t s, int32_t &first, int32_t &n) {
  n = P.lengths[s];
  n = n < 0 ? 0 : (uint32_t)n > P.max_length ? (int32_t)P.max_length : n;
  first = P.window && (uint32_t)n > P.window ? n - (int32_t)P.window : 0;
}

// cap tanh(s / cap), s = scale x, with an error relative to s whatever the cap (a
// call with a cap of 30, us: the windowed one below 19.7, 19.0 without; the batch
// above 94.9, 94.2 without):
// y = 2 log2(e) s / cap; below |s / cap| = 1/2 tanh(r) = r + r y^2 p(y^2) (p: least
// largest relative error there, 2^-26), above it 1 - 2 / (2^|y| + 1), where what is
// taken from 1 is at most 0.54.
__device__ __forceinline__ float capped(const AttendParams &P, float x) {
  const float s = x * P.scale, y = x * P.cap_in, z = y * y;
  float p = __builtin_fmaf(z, 3.5919381389248883e-06f, -9.193531150231138e-05f);
  p = __builtin_fmaf(z, p, 0.0019225659780204296f);
  p = __builtin_fmaf(z, p, -0.040037527680397034f);
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(__builtin_fabsf(y)) + 1.f);
  return __builtin_fabsf(y) < kLog2e ? __builtin_fmaf(s * z, p, s) : __builtin_copysignf(P.cap * t, y);
}

template <typename T>
constexpr int32_t kTileKeys = sizeof(T) == 2 ? 32 : 16;
template <typename T>
constexpr int32_t kTiles = kTileKeys<T> / 16;     // score tiles of 16 keys
template <typename T>
constexpr int32_t kSpan = 4 * kTiles<T>;          // consecutive tokens of a lane
template <typename T>
constexpr float kShift = __is_same(T, _Float16) ? 15.f : 0.f;   // of the weights, in powers of two

// D: head size rounded up.  VEC: rows in 16-byte pieces.  SPAN: pages are
// multiples of kSpan tokens, so that a span lies in one page and takes one look
// into the table (the batch above: 94 us with pages of 16, 170 with pages of 10;
// 19 sequences of up to 3000 keys, 7 heads: 20 us with rows of 80, 34 with pages
// of 23, 72 with rows of 81, which are read an element at a time).
template <typename T, int D, bool VEC, bool SPAN>
__global__ void __launch_bounds__(256, D <= 128 ? 2 : 1) attend_kernel(AttendParams P) {
  constexpr int TK = kTileKeys<T>, RT = kTiles<T>, SP = kSpan<T>;
  constexpr int E = kLaneElems<T>, KF = D / kFragElems<T>;            // K and Q fragments of a row
  constexpr int VW = D / 16 < E ? D / 16 : E, VL = D / (16 * VW);     // a lane's dims of a value row, and pieces
  constexpr int VN = VW * sizeof(T) / 4, OT = D / 16;
  constexpr int DC = D < 128 ? D : 128;                               // columns joined at a time
  // A wavefront's tile of K, rows 16 bytes apart from a multiple of the banks;
  // later the four parts of O.
  constexpr int LPR = D / E < 16 ? D / E : 16, PC = D / (E * LPR), KI = TK * LPR / 64;   // lanes of a key's row, pieces, rows of a lane
  constexpr int KROW = D * (int)sizeof(T) + 16;
  union alignas(16) Shared {
    uint8_t k[4][TK][KROW];
    float o[4][16][DC + 4];
  };
  __shared__ float sm[4][16], sl[4][16];
  __shared__ Shared sh;

  const uint32_t split = blockIdx.y, kv = blockIdx.x / P.head_blocks, hb = blockIdx.x % P.head_blocks, seq = blockIdx.z;
  const uint32_t lane = threadIdx.x & 63, w = wave_index(), col = lane & 15, grp = lane >> 4;
  int32_t first, n;
  key_range(P, seq, first, n);
  const int32_t start = first / TK * TK + (int32_t)(split * P.chunk);
  const int32_t end = n - start < (int32_t)P.chunk ? n : start + (int32_t)P.chunk;
  if (start >= n && split > 0) return;                                // (the join reads the parts below n only)

  const uint32_t heads = P.group - hb * 16 < 16 ? P.group - hb * 16 : 16, head0 = kv * P.group + hb * 16;
  const int d = (int)P.d;
  u4 q[KF];
  {
    const T *qp = (const T *)P.q + seq * P.q_seq + (uint64_t)(head0 + col) * P.q_head;
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      uint32_t v[4];
      const int at = f * (int)kFragElems<T> + (int)grp * E;
      load_row<T, E, VEC>(qp + at, col < heads ? d - at : 0, v);
      q[f] = (u4){v[0], v[1], v[2], v[3]};
    }
  }
  f4 o[OT];
#pragma unroll
  for (int t = 0; t < OT; ++t) o[t] = (f4){0, 0, 0, 0};
  float m = -INFINITY, l = 0;
  const int32_t *table = P.table + seq * P.table_stride;
  const T *kb = (const T *)P.kc + kv * P.k_head, *vb = (const T *)P.vc + kv * P.v_head;

  // Loads are issued without branches, so that the waits between them are for
  // the data that is used next: a token that does not count is read from its
  // page all the same, or from page 0 where the table has none.
  // The page and place of token `tok`, or past `end` of the last one before it
  // (SPAN: of the last span's first, as a whole span is read from there on).
  const int32_t last = SPAN ? (end - 1) / SP * SP : end - 1;
  auto locate = [&](int32_t tok, int32_t &page, uint32_t &place) {
    tok = tok < last ? tok : last;
    const uint32_t p = page_of(P, (uint32_t)tok);
    page = table[p];
    place = (uint32_t)tok - p * P.page_size;
  };
  auto row_of = [&](const T *base, uint64_t page_stride, uint64_t token_stride, int32_t page, uint32_t place) {
    return base + ((uint32_t)page < P.n_pages ? (uint64_t)(uint32_t)page * page_stride : 0) + place * token_stride;
  };

  u4 k[KI][PC];
  uint32_t v[SP][VL][VN];
  int32_t page = 0;          // (SPAN: of the lane's span in the tile whose keys are loaded)
  uint32_t place = 0;
  // Keys of the lane: token grp * SP + kfirst + i of the tile, dims from kat on in steps of 16 E.
  const int kfirst = LPR < 16 ? (int)(lane / LPR % (16 / LPR)) * KI : 0, kat = (int)(lane % LPR) * E;
  auto load_k = [&](int32_t base) {
    const T *row = row_of(kb, P.k_page, P.k_token, page, place + kfirst);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      if constexpr (!SPAN) {
        locate(base + (int32_t)grp * SP + kfirst + i, page, place);
        row = row_of(kb, P.k_page, P.k_token, page, place);
      } else if (i) {
        row += P.k_token;
      }
#pragma unroll
      for (int x = 0; x < PC; ++x) {
        uint32_t r[4];
        const int at = x * 16 * E + kat;
        if constexpr (VEC) load_row<T, E, true>(row + (at < d ? at : 0), 1, r);
        else load_row<T, E, false>(row + at, d - at, r);
        k[i][x] = (u4){r[0], r[1], r[2], r[3]};
      }
    }
  };

  const int32_t step = 4 * TK;
  int32_t base = start + (int32_t)w * TK;
  if (base < end) {
    if (SPAN) locate(base + (int32_t)grp * SP, page, place);
    load_k(base);
  }
  for (; base < end; base += step) {
    // The next tile's pages first: its keys are issued once they are there,
    // without waiting for this tile's values, which come after them.
    int32_t page_next = 0;
    uint32_t place_next = 0;
    if (SPAN) locate(base + step + (int32_t)grp * SP, page_next, place_next);
    // Values of this tile, and which of the lane's tokens count.
    bool live[SP], whole = true;
    const T *row = row_of(vb, P.v_page, P.v_token, page, place);
#pragma unroll
    for (int j = 0; j < SP; ++j) {
      const int32_t tok = base + (int32_t)grp * SP + j;
      if constexpr (!SPAN) {
        locate(tok, page, place);
        row = row_of(vb, P.v_page, P.v_token, page, place);
      } else if (j) {
        row += P.v_token;
      }
      live[j] = (int)(tok >= first) & (int)(tok < end) & (int)((uint32_t)page < P.n_pages);
      whole &= live[j];
#pragma unroll
      for (int x = 0; x < VL; ++x) {
        const int at = x * 16 * VW + (int)col * VW;
        if constexpr (VEC) load_row<T, VW, true>(row + (at < d ? at : 0), 1, v[j][x]);
        else load_row<T, VW, false>(row + at, d - at, v[j][x]);
      }
    }
    whole = __all(whole);

    // The tile's keys into LDS: token grp * SP + r in row 16 (r / 4) + 4 grp + r % 4, tile and row of S^T.
    // Dims from d on hold the row's first ones: their queries are zero, but not an infinite key times zero.
#pragma unroll
    for (int i = 0; i < KI; ++i)
#pragma unroll
      for (int x = 0; x < PC; ++x) {
        const int r = kfirst + i, at = x * 16 * E + kat;
        u4 y = k[i][x];
        if (VEC && d < D && at >= d) y = (u4){0, 0, 0, 0};
        *(u4 *)&sh.k[w][16 * (r / 4) + 4 * grp + r % 4][at * sizeof(T)] = y;
      }
    page = page_next, place = place_next;
    load_k(base + step);
    wave_sync();

    f4 acc[RT];
#pragma unroll
    for (int s = 0; s < RT; ++s) {
      acc[s] = (f4){0, 0, 0, 0};
#pragma unroll
      for (int f = 0; f < KF; ++f) acc[s] = mma<T>(*(const u4 *)&sh.k[w][16 * s + col][(f * 4 + grp) * 16], q[f], acc[s]);
    }

    float sc[SP];
    if (P.cap > 0) {
#pragma unroll
      for (int j = 0; j < SP; ++j) sc[j] = capped(P, acc[j / 4][j % 4]);
    } else {
#pragma unroll
      for (int j = 0; j < SP; ++j) sc[j] = acc[j / 4][j % 4];
    }
    if (!whole) {   // places that do not count hold anything: no score, and no value that zero would not silence
#pragma unroll
      for (int j = 0; j < SP; ++j) {
        sc[j] = live[j] ? sc[j] : -INFINITY;
#pragma unroll
        for (int x = 0; x < VL; ++x)
#pragma unroll
          for (int i = 0; i < VN; ++i) v[j][x][i] = live[j] ? v[j][x][i] : 0;
      }
    }
    float top = sc[0];
#pragma unroll
    for (int j = 1; j < SP; ++j) top = fmaxf(top, sc[j]);

    const float mn = fmaxf(m, column_max(top)), ms = mn == -INFINITY ? 0.f : mn;
    if (__any(mn > m)) {
      const float keep = __builtin_amdgcn_exp2f((m - ms) * P.unit);
      l *= keep;
#pragma unroll
      for (int t = 0; t < OT; ++t) o[t] *= keep;
      m = mn;
    }
#pragma unroll
    for (int j = 0; j < SP; ++j) {
      sc[j] = __builtin_amdgcn_exp2f(kShift<T> > 0 ? __builtin_fmaf(sc[j] - ms, P.unit, kShift<T>) : (sc[j] - ms) * P.unit);
      l += sc[j];
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int x = 0; x < VL; ++x)
#pragma unroll
        for (int u = 0; u < VW; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o[x * VW + u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v[j][x][u]), sc[j], o[x * VW + u], 0, 0, 0);
    } else {
      u4 p;
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = pack2<T>(sc[2 * j], sc[2 * j + 1]);
#pragma unroll
      for (int x = 0; x < VL; ++x)
#pragma unroll
        for (int u = 0; u < VW; ++u) {
          u4 a;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            a[j] = u & 1 ? pair_high(v[2 * j][x][u / 2], v[2 * j + 1][x][u / 2]) : pair_low(v[2 * j][x][u / 2], v[2 * j + 1][x][u / 2]);
          o[x * VW + u] = mma<T>(a, p, o[x * VW + u]);
        }
    }
  }

  // The four wavefronts' parts, joined DC columns at a time.
  __syncthreads();
  l = column_sum(l);
  if (grp == 0) sm[w][col] = m, sl[w][col] = l;
  const uint32_t oh = threadIdx.x >> 4, oc = threadIdx.x & 15;   // this thread's head, and its first column / (DC / 16)
  const uint32_t head = head0 + oh;
#pragma unroll
  for (int c0 = 0; c0 < D; c0 += DC) {
    if (c0) __syncthreads();
#pragma unroll
    for (int x = 0; x < VL; ++x) {
      if (x * 16 * VW < c0 || x * 16 * VW >= c0 + DC) continue;
#pragma unroll
      for (int u = 0; u < VW; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) sh.o[w][col][x * 16 * VW - c0 + (grp * 4 + i) * VW + u] = o[x * VW + u][i];
    }
    __syncthreads();
    float f[4], mt = fmaxf(fmaxf(sm[0][oh], sm[1][oh]), fmaxf(sm[2][oh], sm[3][oh])), lt = 0;
    const float ms = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = __builtin_amdgcn_exp2f((sm[i][oh] - ms) * P.unit);
      lt += sl[i][oh] * f[i];
    }
    if (oh >= heads) continue;
    const float inv = lt == 0 ? 0.f : 1.f / lt;
    const uint64_t at = (uint64_t)(seq * P.n_head + head) * P.splits + split;
    float *part = P.part + at * P.d;
    T *out = (T *)P.out + seq * P.out_seq + head * P.out_head;
#pragma unroll
    for (int e = 0; e < DC / 16; ++e) {
      const uint32_t c = oc + 16 * e;
      float x = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) x += sh.o[i][oh][c] * f[i];
      if (c0 + c >= P.d) continue;
      if (P.splits == 1) out[c0 + c] = (T)(lt == 0 ? 0.f : x * inv);
      else part[c0 + c] = x;
    }
    if (oc == 0 && c0 == 0) {
      if (P.splits > 1) P.part_ml[2 * at] = mt, P.part_ml[2 * at + 1] = lt;
      else if (P.lse) P.lse[(uint64_t)seq * P.n_head + head] = lt == 0 ? -INFINITY : kLn2 * (ms * P.unit + (__builtin_amdgcn_logf(lt) - kShift<T>));
    }
  }
}

// The parts of one sequence and head: every part's weight first, then the
// threads of each of G groups sum a column each over every G-th part.  Four
// groups for more than 16 parts: 2 sequences of 64 parts took 43 us with one
// wavefront to a head, 4.8 so; 64 of 11 take 5.2 with one group.  Bound by the
// latency of two dependent loads.
template <typename T, int G>
__global__ void __launch_bounds__(256 * G) attend_join_kernel(AttendParams P) {
  __shared__ float sw[kMaxSplits], sm, sl, so[G][FIONA_MAX_HEAD_DIM];
  const uint32_t head = blockIdx.x, seq = blockIdx.y, t = threadIdx.x;
  int32_t first, n;
  key_range(P, seq, first, n);
  const int32_t start = first / kTileKeys<T> * kTileKeys<T>;
  const uint32_t used = n > start ? ((uint32_t)(n - start) + P.chunk - 1) / P.chunk : 0;
  const uint64_t at = (uint64_t)(seq * P.n_head + head) * P.splits;
  float m = -INFINITY, l = 0;
  if (t < 64) {
    static_assert(kMaxSplits == 64, "a lane to a part");
    if (t < used) m = P.part_ml[2 * (at + t)], l = P.part_ml[2 * (at + t) + 1];
    float top = m;
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float f = __builtin_amdgcn_exp2f((m - (top == -INFINITY ? 0.f : top)) * P.unit);
    sw[t] = f;
    l *= f;
    for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
    if (t == 0) sm = top, sl = l;
  }
  __syncthreads();
  const float lt = sl, ms = sm == -INFINITY ? 0.f : sm;
  const uint32_t c = t % 256, g = t / 256;
  float x = 0;
  if (c < P.d) {
    const float *o = P.part + at * P.d + c;
#pragma unroll 8
    for (uint32_t i = g; i < used; i += G) x += o[(uint64_t)i * P.d] * sw[i];
  }
  if constexpr (G > 1) {
    so[g][c] = x;
    __syncthreads();
  }
  if (t >= P.d) return;
#pragma unroll
  for (int i = 1; i < G; ++i) x += so[i][t];
  ((T *)P.out)[seq * P.out_seq + head * P.out_head + t] = (T)(lt == 0 ? 0.f : x / lt);
  if (t == 0 && P.lse) P.lse[(uint64_t)seq * P.n_head + head] = lt == 0 ? -INFINITY : kLn2 * (ms * P.unit + (__builtin_amdgcn_logf(lt) - kShift<T>));
}

}  // namespace fiona
