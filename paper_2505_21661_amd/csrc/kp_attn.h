// What the attention operators share: element types, where queries, keys and values lie, which keys a query sees,
// and rows in fp32.
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
// The reference that the exponentials of a row are taken against before it has seen a key: the lowest finite number, which any
// finite score moves, and finite so that a masked score (-inf) against it is exp2(-inf) = 0 and never inf - inf.
constexpr float kNoKey = -3.4028234663852886e38f;

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

// where the keys are: one piece per sequence, pages, pages of e4m3 codes; and pages of which drafted tokens see what their bits name
enum { kPlain = 0, kPaged = 1, kPagedE4m3 = 2, kTree = 3, kTreeE4m3 = 4 };
template <int SRC> constexpr bool kCodes = SRC == kPagedE4m3 || SRC == kTreeE4m3;
template <int SRC> constexpr bool kDrafts = SRC == kTree || SRC == kTreeE4m3;

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
  // drafted tokens: [n_q][words] bits of 64, [n_q] how deep each stands (may be NULL)
  const uint32_t* seen;
  const int32_t* depth;
  uint32_t words;
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

// Which keys a drafted token sees of its sequence's drafted ones, the last n_q of n_k: its bits, `words` of 64 of them.
// Context, the keys in front, is seen as ever, from the position of the context's end and the token's depth.
struct Drafts {
  const uint32_t* bits;
  uint32_t words, n_q;
  int32_t first;  // the key that the first drafted token is (before the first key there is where n_q > n_k)

  __device__ __forceinline__ Drafts(const Args& g, const Tile& t, uint32_t token)
      : bits(g.seen + (size_t)(t.q0 + token) * (2u * g.words)), words(2u * g.words), n_q(t.n_q), first((int32_t)t.n_k - (int32_t)t.n_q) {}
  // Keys start .. start + 31, a bit for each; context is none of them.
  __device__ __forceinline__ uint32_t of(uint32_t start) const {
    const int32_t from = (int32_t)start - first, word = from >> 5, left = (int32_t)n_q - from;
    if ((from <= -32) | (left <= 0)) return 0u;
    const uint32_t lo = word >= 0 && (uint32_t)word < words ? bits[word] : 0u, hi = (uint32_t)(word + 1) < words ? bits[word + 1] : 0u;
    const uint32_t some = (uint32_t)(((uint64_t)hi << 32 | lo) >> (from & 31));
    return left < 32 ? some & ((1u << left) - 1u) : some;
  }
  __device__ __forceinline__ bool sees(uint32_t key) const { return (of(key) & 1u) != 0u; }
};
// Where a drafted token stands: behind its context, as deep as it says (none where nothing says so).
__device__ __forceinline__ int32_t draft_position(const Args& g, const Tile& t, uint32_t token) {
  const int32_t deep = g.depth ? g.depth[t.q0 + token] : 0, most = 1 << 30;
  return (int32_t)t.n_k - (int32_t)t.n_q + (deep < 0 ? 0 : (deep < most ? deep : most - 1));
}

// Keys and values of one kv head of one sequence.
template <int D, int SRC>
struct Source {
  static constexpr uint32_t kBytes = kCodes<SRC> ? D : 2 * D;  // of a row
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

// ---- rows in fp32, one at a time by a whole wave ---------------------------------------------------------------------
// A matrix instruction multiplies every value of a tile by some probability, 0 where the row does not see the key, and 0 times
// an infinity or a NaN is a NaN; a row whose sums came out not finite is taken again in this way, where only what it sees is
// touched.  64 of the rows that it meets at a time (Rows); what is a NaN for good is left.  It is the slow way, bound by
// memory once the rows leave L2: 32/8 x 8192 x 128 without a window takes 0.5 ms forward, 33 with a NaN in one value that every
// token sees; its gradient 2.2 ms, 110 with an infinity or a NaN in one token's d_o (3 with one in a key or a value).
// (Pair by pair, with no end before the last, it was ten times that.)

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
  return x;
}

// 64 rows of D in 16 bits or e4m3 codes.  kLanes lanes have 16 bytes each of a row, and a load brings kRows of them: whole lines
// of memory.  What belongs to a row as a whole (its product with another, its weight) is in lane l for row number place(l).
template <class T, int D, bool E4M3>
struct Rows {
  static constexpr uint32_t kLanes = (E4M3 ? D : 2 * D) / 16, kRows = 64u / kLanes;
  static constexpr int kElements = E4M3 ? 16 : 8;  // of a row in a lane: those from kElements * (lane % kLanes) on
  static __device__ __forceinline__ uint32_t place(uint32_t lane) { return lane % kLanes * kRows + lane / kLanes; }

  static __device__ __forceinline__ void widen(const u32x4& raw, float (&x)[kElements]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (E4M3) {
        x[4 * w] = __builtin_amdgcn_cvt_f32_fp8((int)raw[w], 0);
        x[4 * w + 1] = __builtin_amdgcn_cvt_f32_fp8((int)raw[w], 1);
        x[4 * w + 2] = __builtin_amdgcn_cvt_f32_fp8((int)raw[w], 2);
        x[4 * w + 3] = __builtin_amdgcn_cvt_f32_fp8((int)raw[w], 3);
      } else {
        x[2 * w] = T::to_float(raw[w] & 0xFFFFu);
        x[2 * w + 1] = T::to_float(raw[w] >> 16);
      }
    }
  }
  // A single row in 16 bits, laid out as the others.
  static __device__ __forceinline__ void one(const uint16_t* row, float (&x)[kElements]) {
    const uint16_t* const at = row + kElements * ((threadIdx.x & 63u) % kLanes);
#pragma unroll
    for (int n = 0; n < kElements; n += 8) {
      const u32x4 raw = *reinterpret_cast<const u32x4*>(at + n);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        x[n + 2 * w] = T::to_float(raw[w] & 0xFFFFu);
        x[n + 2 * w + 1] = T::to_float(raw[w] >> 16);
      }
    }
  }
  // Products of row x with the rows, of which number place(l) is at at(l), for any lane l.
  template <class At>
  static __device__ __forceinline__ float products(const float (&x)[kElements], At at) {
    const uint32_t lane = threadIdx.x & 63u, c = lane % kLanes, group = lane / kLanes;
    float mine = 0.f;
#pragma unroll 4
    for (uint32_t t = 0; t < kLanes; ++t) {
      float y[kElements], s = 0.f;
      widen(*reinterpret_cast<const u32x4*>(at(t + group * kLanes) + 16u * c), y);
#pragma unroll
      for (int e = 0; e < kElements; ++e) s = __builtin_fmaf(x[e], y[e], s);
      s += moved<0xB1>(s);   // over kLanes lanes: from the next lane, the next two, the next four, the next eight
      s += moved<0x4E>(s);
      if constexpr (kLanes >= 8) s += moved<0x141>(s);
      if constexpr (kLanes >= 16) s += moved<0x140>(s);
      mine = c == t ? s : mine;
    }
    return mine;
  }
  // Adds the rows times `by`, those with `seen`; finish() adds up what the lanes have of an element.
  template <class At>
  static __device__ __forceinline__ void add(float (&sum)[kElements], float by, bool seen, At at) {
    const uint32_t lane = threadIdx.x & 63u, c = lane % kLanes, group = lane / kLanes;
    const float there = seen ? 1.f : 0.f;
#pragma unroll 4
    for (uint32_t t = 0; t < kLanes; ++t) {
      const uint32_t from = t + group * kLanes;
      u32x4 raw = *reinterpret_cast<const u32x4*>(at(from) + 16u * c);
      const float counts = __shfl(there, (int)from, 64), weight_or_nan = __shfl(by, (int)from, 64), weight = counts != 0.f ? weight_or_nan : 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) raw[w] = counts != 0.f ? raw[w] : 0u;
      float y[kElements];
      widen(raw, y);
#pragma unroll
      for (int e = 0; e < kElements; ++e) sum[e] = __builtin_fmaf(weight, y[e], sum[e]);
    }
  }
  static __device__ __forceinline__ void finish(float (&sum)[kElements]) {
#pragma unroll
    for (int e = 0; e < kElements; ++e)
#pragma unroll
      for (int d = (int)kLanes; d < 64; d <<= 1) sum[e] += __shfl_xor(sum[e], d, 64);
  }
  // A finished row, to where it belongs.
  static __device__ __forceinline__ void put(const float (&x)[kElements], float by, uint16_t* row) {
    const uint32_t lane = threadIdx.x & 63u;
    if (lane >= kLanes) return;
#pragma unroll
    for (int n = 0; n < kElements; n += 8)
      *reinterpret_cast<u32x4*>(row + kElements * lane + n) = u32x4{T::pack(x[n] * by, x[n + 1] * by), T::pack(x[n + 2] * by, x[n + 3] * by),
                                                                    T::pack(x[n + 4] * by, x[n + 5] * by), T::pack(x[n + 6] * by, x[n + 7] * by)};
  }
  static __device__ __forceinline__ void put(const float (&x)[kElements], float by, float* row) {
    const uint32_t lane = threadIdx.x & 63u;
    if (lane >= kLanes) return;
#pragma unroll
    for (int n = 0; n < kElements; n += 4) *reinterpret_cast<f32x4*>(row + kElements * lane + n) = f32x4{x[n] * by, x[n + 1] * by, x[n + 2] * by, x[n + 3] * by};
  }

 private:
  template <int CTRL>
  static __device__ __forceinline__ float moved(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
  }
};

// A NaN in every element of every lane?
template <int K>
__device__ __forceinline__ bool all_nan(const float (&x)[K]) {
  bool nan = true;
#pragma unroll
  for (int e = 0; e < K; ++e) nan = nan & (x[e] != x[e]);
  return __builtin_amdgcn_ballot_w64(nan) == ~0ull;
}

// The softmax of one row.
template <class T, int D, int SRC>
struct Row {
  using In = Rows<T, D, kCodes<SRC>>;
  float m = kNoKey, l = 0.f, o[In::kElements] = {};

  // over the keys from .. to - 1 that the row sees, which stands at p (drafts: of a drafted token, what else it sees)
  __device__ __forceinline__ void over_keys(const uint16_t* query, const Source<D, SRC>& src, int32_t p, uint32_t window, uint32_t sinks,
                                            float scale_log2, uint32_t from, uint32_t to, const Drafts* drafts = nullptr) {
    if constexpr (!kDrafts<SRC>) {
      if (p < 0) return;
      if (to > (uint32_t)p + 1u) to = (uint32_t)p + 1u;
    }
    if (from >= to) return;
    float q[In::kElements];
    In::one(query, q);
    for (uint32_t j0 = from; j0 < to; j0 += 64u) {
      if (l != l) return;  // (a weight that is NaN: so is every value)
      const uint32_t j = j0 + In::place(threadIdx.x & 63u);
      bool seen = (j < to) & ((window == 0u) | ((uint32_t)p - j < window) | (j < sinks));
      if constexpr (kDrafts<SRC>) seen = (j < to) & ((int32_t)j < drafts->first ? seen : drafts->sees(j));
      uint32_t row = ~0u;
      if (seen) row = src.row_of(j);
      if constexpr (SRC != kPlain) seen = seen & (row != ~0u);
      const uint64_t all = __builtin_amdgcn_ballot_w64(seen);
      if (all == 0ull) continue;
      const uint32_t some = __builtin_amdgcn_readlane(row, __builtin_ctzll(all));
      row = seen ? row : some;  // (a row that is seen)
      float s = In::products(q, [&](uint32_t lane) __attribute__((always_inline)) { return src.k_at(__shfl(row, (int)lane, 64)); });
      if constexpr (kCodes<SRC>) s *= power_of(src.k_exp[row]);
      s = seen ? s * scale_log2 : -INFINITY;
      const float top = fmaxf(m, wave_max(s)), alpha = __builtin_amdgcn_exp2f(m - top);
      float w = seen ? __builtin_amdgcn_exp2f(s - top) : 0.f;
      m = top;
      l = l * alpha + wave_sum(w);
#pragma unroll
      for (int e = 0; e < In::kElements; ++e) o[e] *= alpha;
      if constexpr (kCodes<SRC>) w *= power_of(src.v_exp[row]);
      In::add(o, w, seen, [&](uint32_t lane) __attribute__((always_inline)) { return src.v_at(__shfl(row, (int)lane, 64)); });
    }
  }
  __device__ __forceinline__ void store(uint16_t* to, float* lse) {
    In::finish(o);
    In::put(o, l == 0.f ? 0.f : 1.0f / l, to);
    if (lse && (threadIdx.x & 63u) == 0u) *lse = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
  // a part of it, to be joined
  __device__ __forceinline__ void store_part(float* values, float* max_and_sum) {
    In::finish(o);
    In::put(o, 1.f, values);
    if ((threadIdx.x & 63u) == 0u) *reinterpret_cast<f32x2*>(max_and_sum) = f32x2{m, l};
  }
};

}  // namespace attn
}  // namespace kp
