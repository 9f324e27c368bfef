// What the attention operators share: element types, where queries, keys and values lie, which keys a query sees,
// and softmax row by row in fp32.
//
// Query token i of n_q, over n_k keys, stands at position p = n_k - n_q + i; it sees key j where
//   j <= p  and  (window == 0  or  p - j < window  or  j < sinks).
// The keys that a run of tokens sees are at most two ranges: the sinks, if they end before the window begins, and
// from the first token's window to the last token's position.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kp_common.h"

namespace kp {
namespace attn {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The reference that the exponentials of a row are taken against before it has seen a key: low enough that the
// first key moves it, finite so that a masked score (-inf) against it is exp2(-inf) = 0 and never inf - inf.
constexpr float kNoKey = -1e30f;

struct Bf16 {
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ float to_float(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
  // two fp32 -> packed pair (lo in bits 15:0), round to nearest even
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), x2));
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  // codes 0, 1 (HI: 2, 3) of a word of e4m3 codes, times a power of two
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
  }
};

struct Fp16 {
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ float to_float(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), x2));
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  }
  template <bool HI>
  static __device__ __forceinline__ uint32_t from_e4m3(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HI));
  }
};

// 2^(e - 127) for an exponent byte of the cache; bytes 0 and 255 (never written) read as 2^-126 and 2^127
__device__ __forceinline__ float power_of(uint32_t e) {
  const uint32_t c = e < 1u ? 1u : (e > 254u ? 254u : e);
  return __builtin_bit_cast(float, c << 23);
}

// [sequence, head, token, D] somewhere in device memory: strides in elements, D contiguous
struct Heads {
  const uint16_t* at;
  int64_t seq, head, token;
};

enum { kPlain = 0, kPaged = 1, kPagedE4m3 = 2 };  // where the keys are: one piece per sequence, pages, pages of e4m3 codes

struct Args {
  Heads q, o, k, v;          // o is written; paged: k, v .at is the cache, q and o have no sequence stride
  float* lse;                // may be NULL
  int64_t lse_seq, lse_head;
  const uint8_t *k_exp, *v_exp;  // exponent bytes of an e4m3 cache
  const int32_t *table, *lens, *starts;  // paged: block table, keys per sequence, first query token of each sequence
  uint32_t table_width, page_log2, n_pages;
  uint32_t seqs, hkv, group, n_q, n_k;  // paged: n_q = query tokens of all sequences, n_k = most keys the table can hold
  uint32_t window, sinks;
  float scale_log2;          // scale * log2(e)
  uint32_t tiles, splits;    // row tiles of one kv head over all sequences (an upper bound if paged); runs of key tiles
  float* part;               // partial results, splits > 1
  // recording
  uint32_t region_mask;
  void* trace;
  uint32_t cap_lds, cap_hbm, flush, n_wg, rec_cost, group_log2, collab, flags;
};

// One row tile: which sequence, and which of its rows.  Rows are numbered token by token, the query heads of a group
// within a token, so that the heads that share keys share a tile.
struct Tile {
  uint32_t seq, n_q, n_k, q0, first, rows;  // first: the tile's first row, rows: rows of the sequence
};

__device__ __forceinline__ uint32_t clamp_to(int32_t v, uint32_t lo, uint32_t hi) {
  return v < (int32_t)lo ? lo : ((uint32_t)v > hi ? hi : (uint32_t)v);
}

// Tile number `t` (0 .. args.tiles - 1) of ROWS rows; false: there is no such tile.  All lanes of a wave call it.
template <int ROWS, bool PAGED>
__device__ __forceinline__ bool find_tile(const Args& g, uint32_t t, Tile* out) {
  if constexpr (!PAGED) {
    const uint32_t per_seq = g.tiles / g.seqs;
    out->seq = t / per_seq;
    out->n_q = g.n_q; out->n_k = g.n_k; out->q0 = 0;
    out->first = (t - out->seq * per_seq) * ROWS;
    out->rows = g.n_q * g.group;
    return true;
  } else {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;  // tiles of the sequences ahead of this step's 64
    for (uint32_t s0 = 0; s0 < g.seqs; s0 += 64u) {
      const uint32_t s = s0 + lane;
      uint32_t a = 0, n = 0;
      if (s < g.seqs) {
        a = clamp_to(g.starts[s], 0u, g.n_q);
        n = clamp_to(g.starts[s + 1], a, g.n_q) - a;
      }
      const uint32_t mine = (n * g.group + ROWS - 1u) / ROWS;
      uint32_t sum = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(sum, d, 64);
        if (lane >= (uint32_t)d) sum += up;
      }
      const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > t);
      if (past != 0ull) {
        const int l = __builtin_ctzll(past);
        out->seq = s0 + (uint32_t)l;
        out->q0 = __builtin_amdgcn_readlane(a, l);
        out->n_q = __builtin_amdgcn_readlane(n, l);
        out->first = (t - before - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(mine, l))) * ROWS;
        out->rows = out->n_q * g.group;
        out->n_k = clamp_to(__builtin_amdgcn_readfirstlane(g.lens[out->seq]), 0u, g.n_k);
        return true;
      }
      before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
  }
}

// The keys that tokens at positions p_first .. p_last see between them: [0, sink_end) and [lo, end).
struct Span {
  uint32_t sink_end, lo, end;
};
__device__ __forceinline__ Span span_of(int32_t p_first, int32_t p_last, uint32_t window, uint32_t sinks) {
  Span s;
  s.end = p_last < 0 ? 0u : (uint32_t)p_last + 1u;
  s.lo = window != 0u && p_first >= (int32_t)window ? (uint32_t)p_first - window + 1u : 0u;
  s.sink_end = sinks < s.lo ? sinks : 0u;
  if (sinks >= s.lo) s.lo = 0u;
  return s;
}

// The same keys, 64 at a time.  The last sinks, where there are not 64 of them, and the first keys of the window are one tile,
// the first: a window of 512 with one sink takes a tile of 128 rows over 10 tiles of keys, 11 if sinks had their own.
struct KeyTiles {
  uint32_t mixed;  // sinks in the first tile: keys 0 .. mixed - 1
  uint32_t all;
  __device__ __forceinline__ KeyTiles(const Span& s) : mixed(s.sink_end & 63u) {
    const uint32_t whole = s.sink_end >> 6;  // tiles of sinks alone: keys mixed .. sink_end - 1
    all = whole + (s.end > s.lo ? (s.end - s.lo + mixed + 63u) / 64u : 0u);
    sink_end = s.sink_end; end = s.end;
    past_sinks = whole + (mixed != 0u ? 1u : 0u);
    sinks_from = mixed - (mixed != 0u ? 64u : 0u);
    window_from = s.lo - mixed - 64u * whole;
    first = past_sinks == 0u || mixed != 0u ? s.lo - mixed : 0u;
  }
  __device__ __forceinline__ bool is_mixed(uint32_t t) const { return t == 0u && mixed != 0u; }
  // Number of the first key of tile t > 0, and one past the last key that there is for it.
  __device__ __forceinline__ uint32_t start(uint32_t t, uint32_t* limit) const {
    const bool sinks = t < past_sinks;
    *limit = sinks ? sink_end : end;
    return 64u * t + (sinks ? sinks_from : window_from);
  }
  // Of any tile.  Element c of the mixed one is key start + c, but key c in front of `mixed`; there RowMask takes start +
  // mixed for the number of sinks, since its comparison is of start + c.  (Where a window hides sinks from some row of the
  // tile, they end in front of its first key.)
  __device__ __forceinline__ uint32_t start_of(uint32_t t, uint32_t* limit, uint32_t* sinks) const {
    const uint32_t from = start(t, limit);
    if (is_mixed(t)) { *limit = end; *sinks = first + mixed; }
    return t == 0u ? first : from;
  }

 private:
  uint32_t sink_end, end, past_sinks, sinks_from, window_from, first;
};

// Which of a row's scores against a run of keys are visible: element c, the key first + c, is if c - from <= count
// (unsigned) or, where the run holds sinks (mixed), if c <= sink.  One subtraction and one comparison per score.
struct RowMask {
  uint32_t from, count;
  int32_t sink;
  // the row stands at p and sees nothing from `limit` on
  __device__ __forceinline__ RowMask(int32_t p, uint32_t limit, int32_t first, uint32_t window, uint32_t sinks) {
    const int32_t hi = (p < (int32_t)limit ? p : (int32_t)limit - 1) - first, lo = (window != 0u ? p - (int32_t)window + 1 : 0) - first;
    const int32_t sk = (int32_t)sinks - 1 - first;
    from = hi < lo ? 1u << 30 : (uint32_t)lo;
    count = hi < lo ? 0u : (uint32_t)(hi - lo);
    sink = sk < hi ? sk : hi;
  }
  // For a branch of its own: the compiler would make the comparisons that two branches share in front of both, and keep the
  // results in scalar registers that the loop has none left of (chunks over an e4m3 cache of 64: 77 us, 86 that way).
  __device__ __forceinline__ void apart() { asm volatile("" : "+v"(from), "+v"(count), "+v"(sink)); }
  __device__ __forceinline__ bool sees(int c) const { return (uint32_t)c - from <= count; }
  __device__ __forceinline__ bool sees_mixed(int c) const { return ((uint32_t)c - from <= count) | (c <= sink); }
};

// Keys and values of one kv head of one sequence.
template <int D, int SRC>
struct Source {
  static constexpr uint32_t kBytes = SRC == kPagedE4m3 ? D : 2 * D;  // of a row
  const uint8_t *k, *v;
  int64_t k_step, v_step;  // bytes from key to key (kPlain)
  const uint8_t *k_exp, *v_exp;
  const int32_t* table;
  uint32_t page_log2, n_pages, hkv, head;

  __device__ __forceinline__ Source(const Args& g, uint32_t seq, uint32_t h) {
    k = reinterpret_cast<const uint8_t*>(g.k.at);
    v = reinterpret_cast<const uint8_t*>(g.v.at);
    k_step = 2 * g.k.token;
    v_step = 2 * g.v.token;
    k_exp = g.k_exp; v_exp = g.v_exp;
    page_log2 = g.page_log2; n_pages = g.n_pages; hkv = g.hkv; head = h;
    table = nullptr;
    if constexpr (SRC == kPlain) {
      k += 2 * (g.k.seq * (int64_t)seq + g.k.head * (int64_t)h);
      v += 2 * (g.v.seq * (int64_t)seq + g.v.head * (int64_t)h);
    } else {
      table = g.table + (size_t)seq * g.table_width;
    }
  }
  // Number of the cache's row that holds key j (j < n_k), all ones where the table names no page.
  __device__ __forceinline__ uint32_t row_of_page(int32_t page, uint32_t j) const {
    const uint32_t row = (((uint32_t)page * hkv + head) << page_log2) + (j & ((1u << page_log2) - 1u));
    return (uint32_t)page < n_pages ? row : ~0u;
  }
  __device__ __forceinline__ uint32_t row_of(uint32_t j) const {
    if constexpr (SRC == kPlain) return j;
    else return row_of_page(table[j >> page_log2], j);
  }
  __device__ __forceinline__ const uint8_t* k_at(uint32_t row) const {
    if constexpr (SRC == kPlain) return k + k_step * (int64_t)row; else return k + (size_t)row * kBytes;
  }
  __device__ __forceinline__ const uint8_t* v_at(uint32_t row) const {
    if constexpr (SRC == kPlain) return v + v_step * (int64_t)row; else return v + (size_t)row * kBytes;
  }
};

// Elements lane * E .. lane * E + E - 1 of a row of D = 64 E, in fp32.
template <class T, int E>
__device__ __forceinline__ void row_elements(const uint8_t* row, uint32_t lane, float (&out)[E]) {
  if constexpr (E == 1) {
    out[0] = T::to_float(reinterpret_cast<const uint16_t*>(row)[lane]);
  } else {
    const uint32_t w = reinterpret_cast<const uint32_t*>(row)[lane];
    out[0] = T::to_float(w & 0xFFFFu);
    out[1] = T::to_float(w >> 16);
  }
}
template <int E>
__device__ __forceinline__ void row_codes(const uint8_t* row, uint32_t lane, float scale, float (&out)[E]) {
  uint32_t w = 0;
  if constexpr (E == 1) w = row[lane]; else w = reinterpret_cast<const uint16_t*>(row)[lane];
  out[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale;
  if constexpr (E == 2) out[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
  return x;
}

// The rows of the softmax, one at a time and in fp32 throughout: a lane owns E elements of D.  A matrix instruction
// multiplies every value of a tile by some probability, 0 where the row does not see the key, and 0 times an infinity or
// a NaN is a NaN; a row whose sums came out not finite is taken again here, where only what it sees is touched.
template <int E>
struct Row {
  float m = kNoKey, l = 0.f, o[E] = {};
};
template <class T, int D, int SRC>
__device__ __forceinline__ void row_over_keys(Row<D / 64>& r, const float (&q)[D / 64], const Source<D, SRC>& src, int32_t p,
                                              uint32_t window, uint32_t sinks, float scale_log2, uint32_t from, uint32_t to) {
  constexpr int E = D / 64;
  const uint32_t lane = threadIdx.x & 63u;
  if (p < 0) return;
  if (to > (uint32_t)p + 1u) to = (uint32_t)p + 1u;
  for (uint32_t j = from; j < to; ++j) {
    if (window != 0u && (uint32_t)p - j >= window && j >= sinks) {
      j = (uint32_t)p - window;  // (the next key is the window's first)
      continue;
    }
    const uint32_t row = src.row_of(j);
    if (SRC != kPlain && row == ~0u) continue;
    float kk[E], vv[E], dot = 0.f;
    if constexpr (SRC == kPagedE4m3) {
      row_codes<E>(src.k_at(row), lane, power_of(src.k_exp[row]), kk);
      row_codes<E>(src.v_at(row), lane, power_of(src.v_exp[row]), vv);
    } else {
      row_elements<T, E>(src.k_at(row), lane, kk);
      row_elements<T, E>(src.v_at(row), lane, vv);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) dot = __builtin_fmaf(q[e], kk[e], dot);
    const float s = wave_sum(dot) * scale_log2;
    const float m = fmaxf(r.m, s), alpha = __builtin_amdgcn_exp2f(r.m - m), w = __builtin_amdgcn_exp2f(s - m);
    r.m = m;
    r.l = r.l * alpha + w;
#pragma unroll
    for (int e = 0; e < E; ++e) r.o[e] = __builtin_fmaf(w, vv[e], r.o[e] * alpha);
  }
}

// A row's result, by a whole wave (lane: elements lane * E ..).
template <class T, int E>
__device__ __forceinline__ void store_row(const Row<E>& r, uint16_t* o, float* lse) {
  const uint32_t lane = threadIdx.x & 63u;
  const float inv = r.l == 0.f ? 0.f : 1.0f / r.l;
  if constexpr (E == 1) o[lane] = (uint16_t)T::pack(r.o[0] * inv, 0.f);
  else reinterpret_cast<uint32_t*>(o)[lane] = T::pack(r.o[0] * inv, r.o[1] * inv);
  if (lse && lane == 0) *lse = r.l == 0.f ? -INFINITY : (r.m + __builtin_amdgcn_logf(r.l)) * kLn2;
}

}  // namespace attn
}  // namespace kp
