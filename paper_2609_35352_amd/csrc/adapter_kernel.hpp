// Kernels of fiona_adapter_linear and fiona_adapter_backward.
//
// An adapter's product goes through its rank: h = A x is a few numbers a token,
// y = base + c B h as long as the row.  So a call is two passes, each bound by
// the rows it reads or writes: `shrink` contracts rows with A into partial sums
// of h (split over the row where there are few tokens), `expand` adds them up,
// multiplies by B and adds the base row.  The backward pass is the same two
// passes on dy with the factors transposed, and `grad`, which contracts over
// the tokens.
//
// Tokens come in any order.  A workgroup of shrink or expand takes 64 of them
// and goes through the adapters among them (a ballot per adapter): one for a
// prompt, up to 64 for single tokens, which are then spread over workgroups
// (slots).  Products run on the matrix cores with all rows of a tile; rows of
// other adapters are dropped on the way out.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mma.hpp"

namespace fiona {

constexpr uint64_t kMaxStride = 1 << 24;   // elements from one token's row to the next
constexpr uint32_t kRows = 64;        // tokens of a workgroup in shrink and expand

struct AdapterIds {
  const int32_t *ids, *ranks;
  uint32_t n_tok, n_adapter, R;
};

// The adapter of token t and its rank; rank 0 for none.
__device__ __forceinline__ uint32_t adapter_rank(const AdapterIds &I, int32_t a) {
  if ((uint32_t)a >= I.n_adapter) return 0;
  if (!I.ranks) return I.R;
  const int32_t r = I.ranks[a];
  return r < 0 ? 0 : (uint32_t)r > I.R ? I.R : (uint32_t)r;
}

// Calls f(adapter or -1, its rank, the rows that have it) for every adapter
// among the workgroup's rows whose turn it is; the same in every wavefront.
template <typename F>
__device__ __forceinline__ void for_adapters(const AdapterIds &I, uint32_t row0, uint32_t lane, uint32_t slot,
                                             uint32_t slots, bool with_none, F f) {
  const bool in = row0 + lane < I.n_tok;
  int32_t id = in ? I.ids[row0 + lane] : -1;
  const uint32_t rank = adapter_rank(I, id);
  if (rank == 0) id = -1;
  uint64_t left = __ballot(in && (with_none || rank > 0));
  for (uint32_t i = 0; left; ++i) {
    const int lead = __builtin_ctzll(left);
    const int32_t a = __builtin_amdgcn_readlane(id, lead);
    const uint64_t rows = __ballot(in && id == a) & left;
    left &= ~rows;
    if (i % slots == slot) f(a, (uint32_t)__builtin_amdgcn_readlane((int)rank, lead), rows, (uint32_t)lead);
  }
}

// ---------------------------------------------------------------------------
// shrink: part[split][t][r] = sum over the split's columns of x_t[k] w_a[r][k]
// ---------------------------------------------------------------------------
struct ShrinkSide {
  const void *x, *w;        // w [n_adapter][w_rows][K]
  float *part;              // [splits][n_tok][16 RT]
  uint64_t x_row;
  uint32_t K, w_rows;
};
struct ShrinkParams {
  AdapterIds I;
  ShrinkSide side[2];
  uint32_t splits, slots;
};

// ONCE: the rows are read by this pass alone (the forward call).
// Row pieces of 256 bytes pass through LDS to become fragments: rows are read
// whole (16 lanes to a piece) and the factor's rows are shared by the
// workgroup's four wavefronts, 16 tokens each.  8192 tokens of 4096 in bfloat16 at
// rank 16 (67 MB): 15.8 us, 4.3 TB/s; both sides of a backward pass at rank 64
// (134 MB) 37, of which 30 remain without the loads: LDS (30k of a unit's 56k busy
// cycles) and the barriers between pieces.  Operands as fragments straight from memory,
// 64 bytes of 16 rows to an instruction, without LDS or barriers: 27 and 57 us.
template <typename T, int RT, bool ONCE>
__global__ void __launch_bounds__(256) shrink_kernel(ShrinkParams P) {
  constexpr uint32_t E = kLaneElems<T>, CE = 16 * E, RP = 16 * RT;
  __shared__ alignas(16) uint8_t sx[kRows][272], sw[RP][272];
  const ShrinkSide &S = P.side[blockIdx.z / P.slots];
  const uint32_t lane = threadIdx.x & 63, wave = wave_index(), col = lane & 15, grp = lane >> 4;
  const uint32_t row0 = blockIdx.x * kRows, tr = threadIdx.x / 16, pc = threadIdx.x % 16;
  const uint32_t chunks = (S.K + CE - 1) / CE, split = blockIdx.y;
  const uint32_t c0 = chunks * split / P.splits, c1 = chunks * (split + 1) / P.splits;
  for_adapters(P.I, row0, lane, blockIdx.z % P.slots, P.slots, false,
               [&](int32_t a, uint32_t rank, uint64_t rows, uint32_t lead) {
    const T *xr[4], *wr[RT];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = tr + 16 * i;
      xr[i] = (const T *)S.x + (uint64_t)(row0 + (rows >> r & 1 ? r : lead)) * S.x_row;
    }
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const uint32_t r = tr + 16 * j;
      wr[j] = (const T *)S.w + ((uint64_t)a * S.w_rows + (r < rank ? r : rank - 1)) * S.K;
    }
    f4 acc[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[j] = (f4){0, 0, 0, 0};
    u4 xv[4], wv[RT];
    auto load = [&](uint32_t c) {
      const uint32_t at = c * CE + pc * E;
#pragma unroll
      for (int i = 0; i < 4; ++i) xv[i] = ONCE ? load_once<T>(piece_at<T>(xr[i], at, S.K)) : load_shared<T>(piece_at<T>(xr[i], at, S.K));
#pragma unroll
      for (int j = 0; j < RT; ++j) wv[j] = load_shared<T>(piece_at<T>(wr[j], at, S.K));
    };
    if (c0 < c1) load(c0);
    for (uint32_t c = c0; c < c1; ++c) {
      if ((c + 1) * CE > S.K) {
        const uint32_t at = c * CE + pc * E;
#pragma unroll
        for (int i = 0; i < 4; ++i) xv[i] = piece_fix<T>(xv[i], at, S.K);
#pragma unroll
        for (int j = 0; j < RT; ++j) wv[j] = piece_fix<T>(wv[j], at, S.K);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) *(u4 *)&sx[tr + 16 * i][pc * 16] = xv[i];
#pragma unroll
      for (int j = 0; j < RT; ++j) *(u4 *)&sw[tr + 16 * j][pc * 16] = wv[j];
      __syncthreads();
      if (c + 1 < c1) load(c + 1);
      if ((rows >> (16 * wave) & 0xFFFF) == 0) continue;
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        const u4 x = *(const u4 *)&sx[16 * wave + col][(f * 4 + grp) * 16];
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[j] = mma<T>(x, *(const u4 *)&sw[16 * j + col][(f * 4 + grp) * 16], acc[j]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = 16 * wave + 4 * grp + i;
      if (!(rows >> r & 1)) continue;
      float *out = S.part + ((uint64_t)split * P.I.n_tok + row0 + r) * RP;
#pragma unroll
      for (int j = 0; j < RT; ++j) out[16 * j + col] = 16 * j + col < rank ? acc[j][i] : 0.f;   // (rows from rank on repeat another)
    }
  });
}

// ---------------------------------------------------------------------------
// inner: parts of h and g summed and scaled, as columns of tokens for the
// gradients, in two bfloat16 parts for 16-bit types; with a launch of its own g
// whole as well, for expand.  8192 tokens of rank 64, four parts (23 MB): 7.4 us,
// latency of ids, ranks and parts in turn.
// ---------------------------------------------------------------------------
// Tokens of one step of the gradients: a fragment's.
template <typename T>
constexpr uint32_t kGradTokens = sizeof(T) == 2 ? 32 : 16;
// The lane's 16 bytes of the fragment of a step's tokens and 16 ranks: ranks by
// lane % 16, tokens by lane / 16; bfloat16 has a second fragment for the rest.
template <typename T>
__device__ __forceinline__ char *column_at(const void *column, uint32_t RP, uint64_t step, uint32_t tile, uint32_t part, uint32_t lane) {
  return (char *)column + (((step * (RP / 16) + tile) * (sizeof(T) == 2 ? 2 : 1) + part) * 64 + lane) * 16;
}

struct InnerParams {
  AdapterIds I;
  const float *part[2], *scaling;   // of h, of g
  float *g;                         // [n_tok][RP], or null
  int32_t *ids;                     // [n_pad]: the tokens' adapters, -1 for none
  void *column[2];                  // h and g as fragments of the gradients' steps (see column_at)
  uint32_t RP, n_pad, splits;
};
// 64 tokens from row0 and 32 ranks from r0 on of h (side 0) or g.
template <typename T>
__device__ __forceinline__ void inner_tile(const InnerParams &P, uint32_t side, uint32_t row0, uint32_t r0, float (*tile)[65]) {
  if (side == 0 && r0 == 0 && threadIdx.x < 64) {
    const uint32_t t = row0 + threadIdx.x;
    const int32_t a = t < P.I.n_tok ? P.I.ids[t] : -1;
    P.ids[t] = adapter_rank(P.I, a) ? a : -1;
  }
  // A thread takes one rank of eight tokens; their ids, ranks and parts are each
  // asked for together, without branches.
  constexpr uint32_t M = 8;
  const uint32_t q = threadIdx.x / 32, r = r0 + threadIdx.x % 32, rc = r < P.RP ? r : P.RP - 1;
  uint32_t a[M], at[M];
  bool live[M];
  float x[M];
#pragma unroll
  for (uint32_t i = 0; i < M; ++i) {
    const uint32_t t = row0 + q + 8 * i;
    at[i] = t < P.I.n_tok ? t : P.I.n_tok - 1;
    const int32_t id = P.I.ids[at[i]];
    live[i] = (int)(t < P.I.n_tok) & (int)((uint32_t)id < P.I.n_adapter);
    a[i] = live[i] ? (uint32_t)id : 0;
    x[i] = 0;
  }
  if (P.I.ranks) {
#pragma unroll
    for (uint32_t i = 0; i < M; ++i) live[i] &= P.I.ranks[a[i]] > 0;
  }
#pragma unroll 2
  for (uint32_t s = 0; s < P.splits; ++s)
#pragma unroll
    for (uint32_t i = 0; i < M; ++i) x[i] += P.part[side][((uint64_t)s * P.I.n_tok + at[i]) * P.RP + rc];
  if (P.scaling) {
#pragma unroll
    for (uint32_t i = 0; i < M; ++i) x[i] *= P.scaling[a[i]];
  }
#pragma unroll
  for (uint32_t i = 0; i < M; ++i) {
    if (!live[i] || r >= P.RP) x[i] = 0;   // (nothing is written there)
    if (side == 1 && P.g && r < P.RP && row0 + q + 8 * i < P.I.n_tok) P.g[(uint64_t)at[i] * P.RP + r] = x[i];
    tile[threadIdx.x % 32][q + 8 * i] = x[i];
  }
  __syncthreads();
  if constexpr (sizeof(T) == 4) {   // 4 steps of 16 tokens, 2 tiles of 16 ranks, 64 lanes of 4 tokens
    for (uint32_t e = threadIdx.x; e < 512; e += 256) {
      const uint32_t lane = e % 64, j = e / 64 % 2, step = e / 128, t = 16 * step + lane / 16 * 4;
      if (r0 + 16 * j >= P.RP) continue;
      f4 x;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = tile[16 * j + lane % 16][t + i];
      *(f4 *)column_at<T>(P.column[side], P.RP, row0 / 16 + step, r0 / 16 + j, 0, lane) = x;
    }
  } else {                          // 2 steps of 32 tokens, 2 tiles of 16 ranks, 64 lanes of 8 tokens
    const uint32_t lane = threadIdx.x % 64, j = threadIdx.x / 64 % 2, step = threadIdx.x / 128, t = 32 * step + lane / 16 * 8;
    if (r0 + 16 * j >= P.RP) return;
    u4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t l;
      hi[i] = split_pair(tile[16 * j + lane % 16][t + 2 * i], tile[16 * j + lane % 16][t + 2 * i + 1], l);
      lo[i] = l;
    }
    *(u4 *)column_at<T>(P.column[side], P.RP, row0 / 32 + step, r0 / 16 + j, 0, lane) = hi;
    *(u4 *)column_at<T>(P.column[side], P.RP, row0 / 32 + step, r0 / 16 + j, 1, lane) = lo;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) inner_kernel(InnerParams P) {
  __shared__ float tile[32][65];
  inner_tile<T>(P, blockIdx.z, blockIdx.x * 64, blockIdx.y * 32, tile);
}

// ---------------------------------------------------------------------------
// expand: out_t[o] = base_t[o] + c_a sum_r w_a[o][r] h_t[r],  h = sum of parts
// ---------------------------------------------------------------------------
struct ExpandParams {
  AdapterIds I;
  const float *part, *scaling;   // part [splits][n_tok][16 RT]; scaling may be null
  const void *w, *base;          // w [n_adapter][O][w_cols]; base may be null
  void *out;
  uint64_t base_row, out_row;
  uint32_t O, w_cols, splits, slots, slice;   // slice: columns of a workgroup, a multiple of 256
  uint32_t inner_z;              // INNER: of the grid's z, the first ones for inner
  InnerParams inner;
};

// The workgroup first adds up its tokens' parts of h and keeps them in LDS as
// fragments (two bfloat16 parts for 16-bit types).  A wavefront then takes 16
// tokens and 64 columns at a time: the factor's rows are fragments as they lie
// (contiguous, and shared through the caches), and the tile passes through LDS
// to meet the base rows 128 or 256 bytes of a row at a time.  Bound by memory:
// 8192 tokens of 4096 in bfloat16 with a base (134 MB), 31 us at rank 16 (4.3 TB/s;
// a copy takes 26), 40 at rank 64, where eight times the products pass through LDS.
// For few tokens, by its chain of loads (ids, ranks, parts, factor): 6.3 us for 16.
// INNER: the launch's first workgroups are inner's.
template <typename T, int RT, bool INNER>
__global__ void __launch_bounds__(256, sizeof(T) == 2 && RT <= 2 ? 3 : (sizeof(T) == 2 ? RT <= 4 : RT <= 2) ? 2 : 1) expand_kernel(ExpandParams P) {
  constexpr uint32_t E = kLaneElems<T>, FK = kFragElems<T>, RP = 16 * RT;
  constexpr int KF = (RP + FK - 1) / FK, PARTS = sizeof(T) == 2 ? 2 : 1;
  constexpr uint32_t LP = 64 / E, NI = 16 * LP / 64;    // lanes of a row's 64 columns, and rows of a lane in a tile of 16
  constexpr uint32_t HB = KF * 64;                      // bytes of a token's h, and of its second part
  __shared__ alignas(16) float so[4][16][68];
  __shared__ alignas(16) uint8_t sh[kRows][PARTS * HB + 16];
  const uint32_t lane = threadIdx.x & 63, wave = wave_index(), col = lane & 15, grp = lane >> 4;
  const uint32_t row0 = blockIdx.y * kRows, tr = lane / LP, pc = lane % LP;
  uint32_t slot = blockIdx.z;
  if constexpr (INNER) {
    if (slot < P.inner_z) {
      const uint32_t i = slot * gridDim.x + blockIdx.x;
      static_assert(sizeof(so) >= sizeof(float[32][65]), "inner's tile");
      if (i / 2 * 32 < P.inner.RP) inner_tile<T>(P.inner, i % 2, row0, i / 2 * 32, (float(*)[65])so);
      return;
    }
    slot -= P.inner_z;
  }
  const uint32_t end = blockIdx.x * P.slice + P.slice < P.O ? blockIdx.x * P.slice + P.slice : P.O;
  const uint32_t here = P.I.n_tok - row0 < kRows ? P.I.n_tok - row0 : kRows;   // tokens of this workgroup
  for_adapters(P.I, row0, lane, slot, P.slots, true, [&](int32_t a, uint32_t rank, uint64_t rows, uint32_t lead) {
    if (rank == 0 && P.base == P.out) return;
    u4 mask[KF];
    // The adapter's factor and the elements from there to the table's end (rows
    // without an adapter read the first one's where there is no branch, unused).
    const uint32_t fa = rank ? (uint32_t)a : 0;
    const T *wa = (const T *)P.w + (uint64_t)fa * P.O * P.w_cols;
    const uint64_t left = (uint64_t)(P.I.n_adapter - fa) * P.O * P.w_cols;
    const uint32_t wn = left < 0x7FFFFFFF ? (uint32_t)left : 0x7FFFFFFF;
    float scale = 1;
    if (rank) {
      if (P.scaling) scale = P.scaling[a];
#pragma unroll
      for (int f = 0; f < KF; ++f) mask[f] = first_mask<T>((int)rank - (int)(f * FK + grp * E));
      // h: a thread takes four ranks of RT tokens.
      f4 x[RT];
      const float *p[RT];
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const uint32_t e = threadIdx.x + 256 * j, row = e / (RP / 4);
        x[j] = (f4){0, 0, 0, 0};
        p[j] = P.part + (uint64_t)(row0 + (rows >> row & 1 ? row : lead)) * RP + e % (RP / 4) * 4;
      }
#pragma unroll 4
      for (uint32_t s = 0; s < P.splits; ++s)
#pragma unroll
        for (int j = 0; j < RT; ++j) x[j] += *(const f4 *)(p[j] + (uint64_t)s * P.I.n_tok * RP);
      __syncthreads();   // (the last adapter's fragments are read)
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const uint32_t e = threadIdx.x + 256 * j, row = e / (RP / 4), r = e % (RP / 4) * 4;
        if (!(rows >> row & 1)) x[j] = (f4){0, 0, 0, 0};
        if constexpr (sizeof(T) == 4) {
          *(f4 *)&sh[row][r * 4] = x[j];
        } else {
          u2 hi, lo;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t l;
            hi[i] = split_pair(x[j][2 * i], x[j][2 * i + 1], l);
            lo[i] = l;
          }
          *(u2 *)&sh[row][r * 2] = hi;
          *(u2 *)&sh[row][HB + r * 2] = lo;
        }
      }
      if constexpr (RP < FK * KF) {   // ranks of a fragment that no tile holds
        const uint32_t row = threadIdx.x / 4, part = threadIdx.x / 2 % 2, half = threadIdx.x % 2;
        *(u4 *)&sh[row][part * HB + 32 + 16 * half] = (u4){0, 0, 0, 0};
      }
      __syncthreads();
    }
    uint32_t start = blockIdx.x * P.slice + 64 * wave;
    if (start >= end) return;
    // A tile's base rows are asked for two tiles ahead, the next columns'
    // factor as soon as the last tile's products are done (the call with one / two
    // tiles ahead, us: 45.6 / 47.1 at rank 16, a training step at rank 64 154.2 / 151.0).
    constexpr uint32_t SETS = 2;
    u4 b[SETS][NI], w[KF][4];
    auto load_w = [&](uint32_t o0) {
#pragma unroll
      for (int f = 0; f < KF; ++f)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t o = o0 + 16 * u + col < P.O ? o0 + 16 * u + col : P.O - 1;
          w[f][u] = load_shared<T>(piece_at<T>(wa, o * P.w_cols + f * FK + grp * E, wn));
        }
    };
    // Rows are a scalar address and a 32-bit offset: 64 rows at most kMaxStride apart.
    const char *base0 = (const char *)P.base + (uint64_t)row0 * P.base_row * sizeof(T);
    char *out0 = (char *)P.out + (uint64_t)row0 * P.out_row * sizeof(T);
    const uint32_t base_bytes = (uint32_t)(P.base_row * sizeof(T)), out_bytes = (uint32_t)(P.out_row * sizeof(T));
    const uint32_t base_last = (here - 1) * base_bytes;
    auto load_base = [&](u4 (&b)[NI], uint32_t o0, uint32_t t) {
      const uint32_t at = o0 + pc * E, from = (at + E <= P.O ? at : P.O - E) * (uint32_t)sizeof(T);
#pragma unroll
      for (uint32_t i = 0; i < NI; ++i) {
        const uint32_t off = (tr + 16 * t + (64 / LP) * i) * base_bytes;
        b[i] = load_shared<T>((const T *)(base0 + ((off < base_last ? off : base_last) + from)));
      }
    };
    // Values of a lane's row piece: products from LDS and base, as they are stored.
    auto finish = [&](uint32_t i, u4 v) {
      f4 y[E / 4];
#pragma unroll
      for (uint32_t e = 0; e < E / 4; ++e)
        y[e] = rank ? *(const f4 *)&so[wave][tr + (64 / LP) * i][pc * E + 4 * e] : (f4){0, 0, 0, 0};
      u4 out;
      if constexpr (sizeof(T) == 4) {
        out = __builtin_bit_cast(u4, y[0] + __builtin_bit_cast(f4, v));
      } else {
        typedef T t8 __attribute__((ext_vector_type(8)));
        const t8 z = __builtin_bit_cast(t8, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e / 4][e % 4] += (float)z[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = pack2<T>(y[e / 2][2 * (e % 2)], y[e / 2][2 * (e % 2) + 1]);
      }
      return out;
    };
    // The products of a tile of tokens and 64 columns, into LDS.
    auto multiply = [&](uint32_t t) {
      f4 acc[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[u] = (f4){0, 0, 0, 0};
#pragma unroll
      for (int f = 0; f < KF; ++f) {
        const u4 hi = *(const u4 *)&sh[16 * t + col][f * 64 + grp * 16];
        const u4 lo = *(const u4 *)&sh[16 * t + col][(PARTS - 1) * HB + f * 64 + grp * 16];
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = mma_wide<T>(w[f][u] & mask[f], hi, lo, acc[u]);   // what the rank leaves out holds anything
      }
      wave_sync();   // (the last tile is read)
#pragma unroll
      for (int u = 0; u < 4; ++u) *(f4 *)&so[wave][col][16 * u + 4 * grp] = acc[u] * scale;
      wave_sync();
    };
    // Whole tiles of columns with a base: loads without branches, so that a wait
    // is for what is used next only (loads and stores complete in order).
    auto whole = [&](uint32_t o0) { return o0 + 64 <= end && (rank == 0 || (o0 + 63) * P.w_cols + KF * FK <= wn); };
    auto columns = [&](auto full) {   // full: all 64 tokens have the adapter
      constexpr bool FULL = decltype(full)::value;
      load_w(start);
#pragma unroll
      for (uint32_t t = 0; t < SETS; ++t) load_base(b[t], start, t);
      for (; whole(start); start += 256) {
        const uint32_t next = whole(start + 256) ? start + 256 : start;   // (the last columns' again)
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t) {
          const bool any = FULL || (rows >> (16 * t) & 0xFFFF) != 0;
          if (any && (FULL || rank)) multiply(t);
          if (t == 3) load_w(next);
          u4 out[NI];
#pragma unroll
          for (uint32_t i = 0; i < NI; ++i) out[i] = finish(i, b[t % SETS][i]);
          load_base(b[t % SETS], t + SETS < 4 ? start : next, (t + SETS) % 4);
#pragma unroll
          for (uint32_t i = 0; i < NI; ++i) {
            const uint32_t row = 16 * t + tr + (64 / LP) * i;
            if (FULL || (rows >> row & 1))
              __builtin_nontemporal_store(out[i], (u4_any *)(out0 + (row * out_bytes + (start + pc * E) * (uint32_t)sizeof(T))));
          }
        }
      }
    };
    // (the registers of 128 ranks in 32 bits leave no room for it)
    if constexpr (sizeof(T) == 2 || RT < 8) {
      if (P.base && whole(start)) {
        if (sizeof(T) == 2 && rows == ~(uint64_t)0 && rank) columns(std::true_type{});
        else columns(std::false_type{});
        if (start >= end) return;
      }
    }
    // The last columns, the table's end, and calls without a base.
    for (uint32_t t = 0; t < 4; ++t) {
      if ((rows >> (16 * t) & 0xFFFF) == 0) continue;
      if (rank) load_w(start);
      if (P.base) load_base(b[0], start, t);
      for (uint32_t o0 = start; o0 < end; o0 += 256) {
        const uint32_t at = o0 + pc * E;
        if (rank) {
          if ((o0 + 64) * P.w_cols + KF * FK > wn) {
#pragma unroll
            for (int f = 0; f < KF; ++f)
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const uint32_t o = o0 + 16 * u + col < P.O ? o0 + 16 * u + col : P.O - 1;
                w[f][u] = piece_fix<T>(w[f][u], o * P.w_cols + f * FK + grp * E, wn);
              }
          }
          multiply(t);
          if (o0 + 256 < end) load_w(o0 + 256);
        }
        u4 v[NI];
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) v[i] = P.base ? piece_fix<T>(b[0][i], at, P.O) : (u4){0, 0, 0, 0};
        if (P.base && o0 + 256 < end) load_base(b[0], o0 + 256, t);
#pragma unroll
        for (uint32_t i = 0; i < NI; ++i) {
          const uint32_t row = 16 * t + tr + (64 / LP) * i;
          const u4 out = finish(i, v[i]);
          if (!(rows >> row & 1)) continue;
          T *p = (T *)(out0 + (row * out_bytes + at * (uint32_t)sizeof(T)));
          if (at + E <= P.O) {
            __builtin_nontemporal_store(out, (u4_any *)p);
          } else {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e) {
              if (at + e >= P.O) break;
              if constexpr (sizeof(T) == 4) ((uint32_t *)p)[e] = out[e];
              else ((uint16_t *)p)[e] = (uint16_t)(out[e / 2] >> (16 * (e % 2)));
            }
          }
        }
      }
    }
  });
}

// ---------------------------------------------------------------------------
// transpose: the factors for the backward pass, rows from the rank on zero, so
// that both of its products contract over contiguous rows.  4 adapters of 4096 x
// 64 twice in bfloat16 (8 MB): 6.5 us, latency.
// ---------------------------------------------------------------------------
struct TransposeParams {
  AdapterIds I;
  const void *A, *B;
  void *AT, *BT;                 // [n_adapter][d_in][RP], [n_adapter][RP][d_out]
  uint32_t d_in, d_out, RP;
};
template <typename T>
__global__ void __launch_bounds__(256) transpose_kernel(TransposeParams P) {
  __shared__ T tile[64][65];
  const uint32_t a = blockIdx.y, nb_in = (P.d_in + 63) / 64, c = threadIdx.x % 64, q = threadIdx.x / 64;
  const uint32_t rank = adapter_rank(P.I, (int32_t)a);
  const bool of_b = blockIdx.x >= nb_in;
  const uint32_t n = of_b ? P.d_out : P.d_in, k0 = (blockIdx.x - (of_b ? nb_in : 0)) * 64;
  for (uint32_t r0 = 0; r0 < P.RP; r0 += 64) {
    if (r0) __syncthreads();
    T v[16];
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) {
      const uint32_t k = k0 + (of_b ? 4 * i + q : c), r = r0 + (of_b ? c : 4 * i + q);
      const uint32_t ki = k < n ? k : n - 1, ri = r < P.I.R ? r : P.I.R - 1;
      v[i] = of_b ? ((const T *)P.B)[((uint64_t)a * n + ki) * P.I.R + ri] : ((const T *)P.A)[((uint64_t)a * P.I.R + ri) * n + ki];
    }
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) tile[4 * i + q][c] = r0 + (of_b ? c : 4 * i + q) < rank ? v[i] : (T)0.f;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 16; ++i) {
      const uint32_t k = k0 + (of_b ? c : 4 * i + q), r = r0 + (of_b ? 4 * i + q : c);
      if (k >= n || r >= P.RP) continue;
      if (of_b) ((T *)P.BT)[((uint64_t)a * P.RP + r) * n + k] = tile[c][4 * i + q];
      else ((T *)P.AT)[((uint64_t)a * n + k) * P.RP + r] = tile[c][4 * i + q];
    }
  }
}

// ---------------------------------------------------------------------------
// grad: dA_a[r] = sum_t g_t[r] x_t and dB_a[.][r] = sum_t c h_t[r] dy_t
// ---------------------------------------------------------------------------
struct GradSide {
  const void *x, *column;
  void *out;                 // dA [n_adapter][R][n] or dB [n_adapter][n][R]
  float *part;               // the same in 32 bits, [splits] times, where the tokens are split
  uint64_t x_row;
  uint32_t n, slices;
};
struct GradParams {
  AdapterIds I;
  GradSide side[2];
  const int32_t *ids;        // [n_pad], -1 for tokens without an adapter and past the last (inner_tile)
  uint32_t RP, n_pad, splits, per_split, r_chunks;   // per_split: tokens, a multiple of 64
};
// Columns of a lane and of a workgroup: 16 bytes of 16 lanes, or 8 from 32 ranks
// of 16 bits on, whose sums of 16 bytes' columns (8 x 4 tiles) and two steps' rows
// would leave one wavefront to a SIMD.
template <typename T>
constexpr uint32_t grad_width(uint32_t RP) {
  return sizeof(T) == 2 && RP >= 32 ? 4 : kLaneElems<T>;
}
constexpr uint32_t kGradWaves = 4;

// Element u of each of a lane's tokens: the lane's part of a transposed fragment.
template <typename T, int SP, int W>
__device__ __forceinline__ u4 column_of(const uint32_t (&x)[SP][W], uint32_t u) {
  if constexpr (sizeof(T) == 4) {
    return (u4){x[0][u], x[1][u], x[2][u], x[3][u]};
  } else {
    const uint32_t i = u / 2;
    if (u & 1) return (u4){pair_high(x[0][i], x[1][i]), pair_high(x[2][i], x[3][i]), pair_high(x[4][i], x[5][i]), pair_high(x[6][i], x[7][i])};
    return (u4){pair_low(x[0][i], x[1][i]), pair_low(x[2][i], x[3][i]), pair_low(x[4][i], x[5][i]), pair_low(x[6][i], x[7][i])};
  }
}

// A workgroup takes 128 or 256 bytes of the rows' columns for one adapter and up to 64
// of its ranks; its four wavefronts take the steps that hold a token of the
// adapter in turn.  Rows are read whole pieces at a time, 16 lanes to a piece,
// eight tokens (four in 32 bits) to a lane; the transposed fragments (columns x tokens) are
// picked from the tokens' words in registers, as values are in the attention.
// 8192 tokens of 4096 + 4096 in bfloat16 at rank 64 (134 MB of rows and as much of
// columns, the latter through the caches): 47 us, 2.9 TB/s of rows.  Bound by the
// loads of both (36 us without the rows', 39 without the columns', 32 without
// either); with the tokens in two parts 61.
template <typename T, int RT>
__global__ void __launch_bounds__(256) grad_kernel(GradParams P) {
  constexpr uint32_t E = grad_width<T>(16 * RT), C = 16 * E, TB = kGradTokens<T>, SP = TB / 4, W = E * sizeof(T) / 4;
  __shared__ alignas(16) float so[kGradWaves][16][C];   // column c of rank r at c ^ 4 r, off each other's banks
  const uint32_t lane = threadIdx.x & 63, wave = wave_index(), col = lane & 15, grp = lane >> 4;
  const bool second = blockIdx.x >= P.side[0].slices;
  const GradSide &S = P.side[second];
  const uint32_t slice = blockIdx.x - (second ? P.side[0].slices : 0), c0 = slice * C;
  const uint32_t a = blockIdx.y / P.r_chunks, n0 = blockIdx.y % P.r_chunks * 64, split = blockIdx.z;
  const uint32_t rank = adapter_rank(P.I, (int32_t)a);
  const uint32_t t0 = split * P.per_split, t1 = t0 + P.per_split < P.I.n_tok ? t0 + P.per_split : P.I.n_tok;
  f4 acc[E][RT];
#pragma unroll
  for (uint32_t u = 0; u < E; ++u)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[u][j] = (f4){0, 0, 0, 0};

  // The lane's columns; at the row's end they step back to its last 16 bytes
  // (and are dropped on the way out where another lane has them).
  const uint32_t at = c0 + col * E, cat = at + E <= S.n ? at : S.n - E;
  // The next step's rows and fragments are on their way while a step is computed.
  struct Rows {
    uint32_t x[SP][W];
  } x0, x1;
  struct Columns {
    u4 hi[RT], lo[sizeof(T) == 2 ? RT : 1];
  } v0, v1;
  // A row's address is a scalar (token step + j) plus the lane's offset of its
  // own tokens and columns, below 2^32 bytes (row strides are at most kMaxStride).
  const uint32_t row_bytes = (uint32_t)(S.x_row * sizeof(T)), lane_at = grp * SP * row_bytes + cat * (uint32_t)sizeof(T);
  auto load_rows = [&](Rows &r, uint32_t step) {   // (its first token)
#pragma unroll
    for (uint32_t j = 0; j < SP; ++j) {
      const uint32_t row = step + j < P.I.n_tok ? step + j : P.I.n_tok - 1;
      const char *p = (const char *)S.x + (uint64_t)row * row_bytes +
                      (row + grp * SP < P.I.n_tok ? lane_at : cat * (uint32_t)sizeof(T));
      if constexpr (W == 4) {
        const u4 v = load_shared<T>((const T *)p);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.x[j][i] = v[i];
      } else {
        // (the rows' last reading; past the caches a training step of 8192 tokens took 150.6 us instead
        // of 154.2 at rank 64, 124.3 for 130.5 at 20; the wider pieces of small ranks gained nothing)
        const u2 v = __builtin_nontemporal_load((const u2_any *)p);
        r.x[j][0] = v[0], r.x[j][1] = v[1];
      }
    }
  };
  auto load_columns = [&](Columns &c, uint32_t step) {
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      c.hi[j] = *(const u4 *)column_at<T>(S.column, P.RP, step / TB, n0 / 16 + j, 0, lane);
      if constexpr (sizeof(T) == 2) c.lo[j] = *(const u4 *)column_at<T>(S.column, P.RP, step / TB, n0 / 16 + j, 1, lane);
    }
  };
  constexpr uint32_t kWindow = 128;   // steps looked over at a time
  __shared__ uint16_t lists[kGradWaves][kWindow / kGradWaves];
  __shared__ uint32_t any_of[kWindow / 32], all_of[kWindow / 32];   // a bit per step
  static_assert(kWindow / 32 == kGradWaves, "32 steps to a wavefront");
  for (uint32_t w0 = t0; rank > n0 && w0 < t1; w0 += kWindow * TB) {
    // The steps that hold a token of the adapter: each wavefront looks over 32,
    // 64 tokens at a time.
    uint32_t any = 0, all = 0;
#pragma unroll 8
    for (uint32_t i = 0; i < 32; i += 64 / TB) {
      const uint32_t t = w0 + (32 * wave + i) * TB + lane;
      const uint64_t is = __ballot(t < P.n_pad && P.ids[t < P.n_pad ? t : 0] == (int32_t)a);
#pragma unroll
      for (uint32_t k = 0; k < 64 / TB; ++k) {
        const uint32_t m = (uint32_t)(is >> (TB * k)) & (TB == 32 ? ~0u : 0xFFFFu);
        any |= (uint32_t)(m != 0) << (i + k);
        all |= (uint32_t)(m == (TB == 32 ? ~0u : 0xFFFFu)) << (i + k);
      }
    }
    // (a split's steps end at its last token's)
    const uint32_t left = w0 + 32 * wave * TB < t1 ? (t1 - w0 - 32 * wave * TB + TB - 1) / TB : 0;
    if (left < 32) any &= (1u << left) - 1;
    __syncthreads();   // (the last window's are read)
    if (lane == 0) any_of[wave] = any, all_of[wave] = all;
    __syncthreads();
    // This wavefront's every fourth of them: the step's number, and kWindow if
    // it holds others' tokens as well.
    uint32_t found = 0;
#pragma unroll
    for (uint32_t k = 0; k < kWindow / 64; ++k) {
      const bool any_k = any_of[2 * k + lane / 32] >> (lane % 32) & 1, all_k = all_of[2 * k + lane / 32] >> (lane % 32) & 1;
      const uint64_t have = __ballot(any_k);
      const uint32_t i = found + __builtin_popcountll(have & (((uint64_t)1 << lane) - 1));
      if (any_k && i % kGradWaves == wave) lists[wave][i / kGradWaves] = (uint16_t)(64 * k + lane + (all_k ? 0 : kWindow));
      found += __builtin_popcountll(have);
    }
    wave_sync();
    const uint32_t mine = found / kGradWaves + (wave < found % kGradWaves);
    auto step_of = [&](uint32_t i) {
      return (uint32_t)__builtin_amdgcn_readfirstlane(lists[wave][i < mine ? i : mine - 1]);
    };
    if (mine == 0) continue;
    auto first_token = [&](uint32_t i) { return w0 + step_of(i) % kWindow * TB; };
    load_rows(x0, first_token(0));
    load_columns(v0, first_token(0));
    // Step i; its operands are asked for without branches, which would make the
    // waits wait for all, and stay in the registers they come to.
    auto compute = [&](uint32_t i, Rows &x, Columns &v, Columns &v_next, Rows &x_next) {
      load_columns(v_next, first_token(i + 1));
      load_rows(x_next, first_token(i + 1));
      const uint32_t s = step_of(i);
      if (s >= kWindow) {   // rows of other adapters count nothing, whatever they hold
        const uint32_t t = w0 + s % kWindow * TB + grp * SP;
#pragma unroll
        for (uint32_t j = 0; j < SP; ++j) {
          const bool live = P.ids[t + j] == (int32_t)a;
#pragma unroll
          for (uint32_t k = 0; k < W; ++k) x.x[j][k] = live ? x.x[j][k] : 0;
          const uint32_t keep = live || sizeof(T) == 4 ? ~0u : ~(0xFFFFu << (16 * (j % 2)));
#pragma unroll
          for (int q = 0; q < RT; ++q) {
            if constexpr (sizeof(T) == 4) {
              v.hi[q][j] = live ? v.hi[q][j] : 0;
            } else {
              v.hi[q][j / 2] &= keep;
              v.lo[q][j / 2] &= keep;
            }
          }
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < E; ++u) {
        const u4 f = column_of<T>(x.x, u);
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[u][j] = mma_wide<T>(f, v.hi[j], v.lo[sizeof(T) == 2 ? j : 0], acc[u][j]);
      }
    };
    for (uint32_t i = 0;; i += 2) {
      compute(i, x0, v0, v1, x1);
      if (i + 1 >= mine) break;
      compute(i + 1, x1, v1, v0, x0);
      if (i + 2 >= mine) break;
    }
    wave_sync();   // (the list is read)
  }

  // The wavefronts' sums, 16 ranks at a time.  acc[u][j][i]: column (4 grp + i) of the
  // slice's 16 lanes, its element u; rank n0 + 16 j + col.
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    __syncthreads();
#pragma unroll
    for (uint32_t u = 0; u < E; u += 4)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f4 *)&so[wave][col][((4 * grp + i) * E + u) ^ (4 * col)] = (f4){acc[u][j][i], acc[u + 1][j][i], acc[u + 2][j][i], acc[u + 3][j][i]};
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < 4 * C; e += 256) {   // four columns of a rank
      // dA: consecutive threads along the columns; dB: along the ranks
      const uint32_t r = second ? e % 16 : e / (C / 4), c = (second ? e / 16 : e % (C / 4)) * 4;
      f4 s = (f4){0, 0, 0, 0};
#pragma unroll
      for (uint32_t w = 0; w < kGradWaves; ++w) s += *(const f4 *)&so[w][r][c ^ (4 * r)];
      // Column c of the slice is element c % E of lane c / E, whose columns may have stepped back.
      const uint32_t want = c0 + c / E * E, from = want + E <= S.n ? want : S.n - E, k = from + c % E;
      const uint32_t rr = n0 + 16 * j + r;
      if (want >= S.n || rr >= P.I.R) continue;
      if (rr >= rank) s = (f4){0, 0, 0, 0};   // (a NaN row times the zeros there)
      const uint64_t o = second ? ((uint64_t)a * S.n + k) * P.I.R + rr : ((uint64_t)a * P.I.R + rr) * S.n + k;
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        if (k + q < want) continue;
        const uint64_t at = o + (second ? q * P.I.R : q);
        if (P.splits > 1) S.part[(uint64_t)split * P.I.n_adapter * P.I.R * S.n + at] = s[q];
        else ((T *)S.out)[at] = (T)s[q];
      }
    }
  }
}

// The splits' sums of a gradient, rounded once (49152 of 6 splits: 3.8 us).
struct GradSumParams {
  const float *part[2];
  void *out[2];
  uint64_t n[2];
  uint32_t splits;
};
template <typename T>
__global__ void __launch_bounds__(256) grad_sum_kernel(GradSumParams P) {
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t side = i >= P.n[0];
  const uint64_t k = i - (side ? P.n[0] : 0);
  if (k >= P.n[side]) return;
  float s = 0;
  for (uint32_t j = 0; j < P.splits; ++j) s += P.part[side][(uint64_t)j * P.n[side] + k];
  ((T *)P.out[side])[k] = (T)s;
}

}  // namespace fiona
