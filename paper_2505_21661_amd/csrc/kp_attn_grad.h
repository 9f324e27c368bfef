// What the two kernels of the attention gradient share: their arguments, rows in fp32, tiles in LDS that are read both ways.
#pragma once
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

constexpr int kGradKeys = 128;   // keys of a workgroup of the dk, dv kernel

// fp16 holds little below 2^-14, and P and dS are often smaller: they are rounded to it times a power of two that their
// factors leave room for.  P <= 1 times 2^kShiftP; dS, of the order of |d_o|, times 2^kShiftS over the power of two of the
// largest |d_o| of the row (dq) or of the rows that it is summed with in one step (dk: RowsScale).  What overflows all the
// same is not finite and is taken again in fp32.  bf16 has the exponents of fp32 and needs none of it.
template <class T> constexpr float kShiftP = 0.f;
template <> constexpr float kShiftP<Fp16> = 14.f;
constexpr int kShiftS = 5;

struct GradArgs {
  Heads q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
  float *neg, *delta;  // workspace, [B, Hq, Sq]: kShiftP - lse log2(e), and d_o . o
  float* most;         // workspace, fp16: largest finite |d_o| of every row, [B, Hq, Sq]
  float* part;         // partial dk, dv: [worker][first, last tile][dk, dv][kGradKeys][D]
  uint32_t seqs, hkv, group, n_q, n_k, window, sinks;
  uint32_t row_tiles;  // of one head of keys
  float scale, scale_log2;
};

__device__ __forceinline__ const uint16_t* row_at(const Heads& t, uint32_t seq, uint32_t head, uint32_t token) {
  return t.at + t.seq * (int64_t)seq + t.head * (int64_t)head + t.token * (int64_t)token;
}
__device__ __forceinline__ bool sees(int32_t p, uint32_t j, uint32_t window, uint32_t sinks) {
  return ((int32_t)j <= p) & ((window == 0u) | ((uint32_t)p - j < window) | (j < sinks));
}

// One query row's gradient in fp32, by a wave; only keys that the row sees are touched.  For rows whose sums on the matrix
// instructions are not finite (see Rows).
template <class T, int D>
__device__ __forceinline__ void query_row(const GradArgs& g, uint32_t seq, uint32_t head, uint32_t token, float neg, float delta, uint16_t* out) {
  using R = Rows<T, D, false>;
  const uint32_t hk = head / g.group;
  const int32_t p = (int32_t)g.n_k - (int32_t)g.n_q + (int32_t)token;
  const Span span = span_of(p, p, g.window, g.sinks);
  float q[R::kElements], d_o[R::kElements], dq[R::kElements] = {};
  R::one(row_at(g.q, seq, head, token), q);
  R::one(row_at(g.d_o, seq, head, token), d_o);
  bool nan = false;
  for (int window = 0; window < 2; ++window) {  // the sinks, then the other keys
    const uint32_t to = window ? span.end : span.sink_end;
    for (uint32_t j0 = window ? span.lo : 0u; j0 < to && !nan; j0 += 64u) {
      const uint32_t n = to - j0;
      const bool seen = R::place(threadIdx.x & 63u) < n;
      const auto key = [&](uint32_t lane) __attribute__((always_inline)) { return j0 + (R::place(lane) < n ? R::place(lane) : n - 1u); };
      const auto k = [&](uint32_t lane) __attribute__((always_inline)) { return reinterpret_cast<const uint8_t*>(row_at(g.k, seq, hk, key(lane))); };
      const auto v = [&](uint32_t lane) __attribute__((always_inline)) { return reinterpret_cast<const uint8_t*>(row_at(g.v, seq, hk, key(lane))); };
      const float w = __builtin_amdgcn_exp2f(R::products(q, k) * g.scale_log2 + (neg - kShiftP<T>)), ds = w * (R::products(d_o, v) - delta);
      R::add(dq, ds, seen, k);
      nan = __builtin_amdgcn_ballot_w64(seen && ds != ds) != 0ull || all_nan(dq);  // (so will be all of dq)
    }
  }
  R::finish(dq);
  R::put(dq, g.scale, out);
}

// Adds one key's gradients from the query tokens from .. to - 1, at most 64, of one head, those wanted: of what is NaN for
// good no more is.
template <class T, int D>
__device__ __forceinline__ void key_row(const GradArgs& g, uint32_t seq, uint32_t head, uint32_t j, uint32_t from, uint32_t to,
                                        const float (&k)[8], const float (&v)[8], bool* want_k, bool* want_v, float (&dk)[8], float (&dv)[8]) {
  using R = Rows<T, D, false>;
  uint32_t i = from + R::place(threadIdx.x & 63u);
  const bool seen = i < to && sees((int32_t)g.n_k - (int32_t)g.n_q + (int32_t)i, j, g.window, g.sinks);
  const uint64_t all = __builtin_amdgcn_ballot_w64(seen);
  if (all == 0ull) return;
  const uint32_t some = __builtin_amdgcn_readlane(i, __builtin_ctzll(all));
  i = seen ? i : some;  // (a token that sees it)
  const auto q = [&](uint32_t lane) __attribute__((always_inline)) { return reinterpret_cast<const uint8_t*>(row_at(g.q, seq, head, __shfl(i, (int)lane, 64))); };
  const auto d_o = [&](uint32_t lane) __attribute__((always_inline)) { return reinterpret_cast<const uint8_t*>(row_at(g.d_o, seq, head, __shfl(i, (int)lane, 64))); };
  const size_t stat = ((size_t)seq * g.hkv * g.group + head) * g.n_q + i;
  const float w = __builtin_amdgcn_exp2f(R::products(k, q) * g.scale_log2 + (g.neg[stat] - kShiftP<T>));
  if (*want_k) {
    const float ds = w * (R::products(v, d_o) - g.delta[stat]);
    R::add(dk, ds, seen, q);
    *want_k = __builtin_amdgcn_ballot_w64(seen && ds != ds) == 0ull && !all_nan(dk);
  }
  if (*want_v) {
    R::add(dv, w, seen, d_o);
    *want_v = __builtin_amdgcn_ballot_w64(seen && w != w) == 0ull && !all_nan(dv);
  }
}

__device__ __forceinline__ float power_of_two_in(float x) {  // the largest power of two <= x (1 for 0), as a number
  const uint32_t e = __builtin_bit_cast(uint32_t, x) >> 23;
  return x == 0.f ? 1.f : __builtin_bit_cast(float, (e < 1u ? 1u : e) << 23);
}

// fp16: what dS of the 64 tokens of a step is multiplied by before it is rounded (besides 2^kShiftP, which is in P).  Their
// largest |d_o| sets it, so that a token decides about the precision of those that share a step with it and of nobody else:
// with one scale for all rows of a head and one token 2^20 times the others, 31 % of dk's values are outside the bounds of its
// other roundings (2 x 2100 x 64, the first token).  It moves, and dk with it, where that largest is twice as large or a
// sixteenth, so seldom (no time is lost).  dS is off by at most 2^-26 of the largest |d_o| of its step, besides its relative
// rounding.
struct RowsScale {
  uint32_t top = 127u << 23;  // bits of a power of two (scalar): |d_o| < 2 top
  __device__ __forceinline__ float by() const { return __builtin_bit_cast(float, ((uint32_t)(254 + kShiftS - 14) << 23) - top); }
  // most: of row `lane` of the step, 0 if none of the wave's keys sees it.  What dk has to be multiplied by.
  __device__ __forceinline__ float moved(float most) {
    const float least = __builtin_bit_cast(float, top - (4u << 23));
    if (__builtin_amdgcn_ballot_w64(most >= __builtin_bit_cast(float, top + (1u << 23))) == 0ull &&
        (__builtin_amdgcn_ballot_w64(most >= least) != 0ull || __builtin_amdgcn_ballot_w64(most != 0.f) == 0ull)) return 1.f;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
    const uint32_t before = top;
    top = kp::wave_uniform(__builtin_bit_cast(uint32_t, power_of_two_in(most)));
    return __builtin_bit_cast(float, (127u << 23) + before - top);
  }
};
static_assert(kShiftP<Fp16> == 14.f, "RowsScale::by is 2^(kShiftS - kShiftP) / top");
// Bytes of the statistics of a step's 64 rows in LDS: neg, delta, largest |d_o|.
constexpr uint32_t kStatBytes = 1024u;

// ---- tiles of 64 rows in LDS that are read both ways ---------------------------------------------------------------
// A row's 16-byte chunk c lies at position c ^ swizzle(row).  Read as it lies (32 rows x 16 bytes to a half wave) the 16
// rows of a pass take all banks; read transposed (four rows x 32 bytes to 16 lanes, two such pieces to a pass) so do they.
template <int D>
__device__ __forceinline__ uint32_t swizzle(uint32_t row) {
  if constexpr (D == 128) return ((row & 3u) << 2) | ((row >> 2) & 3u);
  else return (((row >> 1) & 1u) << 2) | ((row >> 2) & 3u);
}
template <int D>
struct TileReader {
  static constexpr uint32_t kRow = 2u * D;
  // LDS byte addresses of row l32's first chunk and of the transposing read's first piece; other chunks are an exclusive or
  // away (the tile begins at a multiple of 256 bytes: kernels that use this have no LDS but the dynamic, which begins at 0)
  uint32_t row0, col0;
  __device__ __forceinline__ TileReader(uint32_t base) {
    const uint32_t lane = threadIdx.x & 63u, h32 = lane >> 5, l32 = lane & 31u, i = lane & 15u, grp = lane >> 4;
    row0 = base + l32 * kRow + ((h32 ^ swizzle<D>(l32)) << 4);
    const uint32_t row = 4u * (grp >> 1) + (i >> 2), d = 16u * (grp & 1u) + 4u * (i & 3u);
    col0 = base + row * kRow + (((d >> 3) ^ swizzle<D>(row)) << 4) + 8u * ((d >> 2) & 1u);
  }
  // rows `from` + l32 (from: a multiple of 32), d = 16 s + 8 h32 .. + 7; buffer: its distance from the first
  __device__ __forceinline__ u32x4 rows(int s, uint32_t from, uint32_t buffer) const {
    return rows_at((row0 ^ (32u * (uint32_t)s)) + buffer, from);
  }
  // d = 32 dt + l32 of the 16 rows from `from` on, in the order of an accumulator's rows
  __device__ __forceinline__ u32x4 cols(int dt, uint32_t from, uint32_t buffer) const {
    // (swizzle(row + 8) = swizzle(row) ^ 2)
    return cols_at((col0 ^ (64u * (uint32_t)dt)) + buffer, (col0 ^ (64u * (uint32_t)dt + 32u)) + buffer, from);
  }
  static __device__ __forceinline__ u32x4 rows_at(uint32_t ofs, uint32_t from) {
    typedef const __attribute__((address_space(3))) u32x4* lds_u32x4;
    return *(lds_u32x4)(uintptr_t)(ofs + from * kRow);
  }
  static __device__ __forceinline__ u32x4 cols_at(uint32_t lo_ofs, uint32_t hi_ofs, uint32_t from) {
    return cols_from(lo_ofs + from * kRow, hi_ofs + (from + 8u) * kRow);
  }
  static __device__ __forceinline__ u32x4 cols_from(uint32_t lo_at, uint32_t hi_at) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)lo_at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)hi_at);
    const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(u32x4, v);
  }
};

// The same of tiles in two buffers: the addresses go from one buffer to the other (an addition per register and step, where
// every read had one).
template <int D>
struct TileCursor {
  uint32_t row[D / 16], col[D / 32][2], by;
  __device__ __forceinline__ TileCursor(uint32_t base, uint32_t buffer_bytes) : by(buffer_bytes) {
    const TileReader<D> rd(base);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) row[s] = rd.row0 ^ (32u * (uint32_t)s);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      col[dt][0] = rd.col0 ^ (64u * (uint32_t)dt);
      col[dt][1] = rd.col0 ^ (64u * (uint32_t)dt + 32u);
    }
  }
  __device__ __forceinline__ u32x4 rows(int s, uint32_t from) const { return TileReader<D>::rows_at(row[s], from); }
  __device__ __forceinline__ u32x4 cols(int dt, uint32_t from) const { return TileReader<D>::cols_at(col[dt][0], col[dt][1], from); }
  __device__ __forceinline__ void to_other() {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) row[s] += by;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) { col[dt][0] += by; col[dt][1] += by; }
    by = 0u - by;
  }
};

// 64 rows from global memory straight to such a tile: 1 KiB to a load of one of WAVES waves.
template <int D, int WAVES>
struct TileLoader {
  static constexpr uint32_t kRow = 2u * D, kChunks = kRow / 16u, kBlockRows = 1024u / kRow;
  static constexpr int NL = (int)(64u * kRow / (1024u * WAVES));
  uint32_t ofs[NL], step, in;  // bytes
  __device__ __forceinline__ TileLoader(int64_t token_step) {
    const uint32_t lane = threadIdx.x & 63u, row = first_row();
    step = (uint32_t)(2 * token_step);
    in = ((lane % kChunks) ^ swizzle<D>(row)) << 4;
  }
  static __device__ __forceinline__ uint32_t first_row() {
    return kBlockRows * (threadIdx.x >> 6) + (threadIdx.x & 63u) / kChunks;
  }
  // rows past `last` are that row again
  __device__ __forceinline__ void upto(uint32_t last) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint32_t row = first_row() + (uint32_t)WAVES * kBlockRows * (uint32_t)i;
      ofs[i] = (row < last ? row : last) * step + in;
    }
  }
  // M0 (the LDS base) is put back; the loads are waited for by hand (see kp_attn_tile)
  __device__ __forceinline__ void load(const uint16_t* base, uint32_t dst) const {
#pragma unroll
    for (int i = 0; i < NL; ++i) load_one(i, base, dst);
  }
  __device__ __forceinline__ void load_one(int i, const uint16_t* base, uint32_t dst) const {
    {
      uint32_t saved_m0;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0) : "v"(ofs[i]), "s"(base), "s"(dst + 1024u * WAVES * (uint32_t)i) : "memory");
    }
  }
  // Row r < mixed is token r, the others token start + r (up to r = left): further apart than 32 bits reach, perhaps.
  __device__ __forceinline__ void load_two(const uint16_t* head, int64_t token_step, uint32_t mixed, uint32_t start, uint32_t left, uint32_t dst) const {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const uint32_t r = first_row() + (uint32_t)WAVES * kBlockRows * (uint32_t)i, token = r < mixed ? r : start + (r < left ? r : left);
      const uint64_t from = (uint64_t)(uintptr_t)(head + token_step * (int64_t)token) + in;
      uint32_t saved_m0;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0) : "v"(from), "s"(dst + 1024u * WAVES * (uint32_t)i) : "memory");
    }
  }
};

// A wave's 32 rows of D accumulators (row l32, d = 32 dt + 8 j + 4 h32 + i), times `by`, through LDS and out as whole rows.
template <class T, int D>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], float by, unsigned char* lds, uint16_t* to, int64_t at, uint64_t rows_out) {
  constexpr uint32_t kRow = 2u * D, kChunks = kRow / 16u, kBlockRows = 1024u / kRow;
  const uint32_t lane = threadIdx.x & 63u, h32 = lane >> 5, l32 = lane & 31u, half = h32 ^ ((l32 >> 3) & 1u);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x2 two = {T::pack(acc[dt][4 * j] * by, acc[dt][4 * j + 1] * by), T::pack(acc[dt][4 * j + 2] * by, acc[dt][4 * j + 3] * by)};
      *reinterpret_cast<u32x2*>(lds + l32 * kRow + (((uint32_t)(4 * dt + j) ^ (l32 & 7u)) << 4) + 8u * half) = two;
    }
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < (int)(32u / kBlockRows); ++i) {
    const uint32_t r = kBlockRows * (uint32_t)i + lane / kChunks, chunk = (lane % kChunks) ^ (r & 7u);
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + 1024u * (uint32_t)i + 16u * lane);
    const int64_t row = (int64_t)(((uint64_t)(uint32_t)__shfl((int)(at >> 32), (int)r, 64) << 32) | (uint32_t)__shfl((int)at, (int)r, 64));
    if ((rows_out >> r) & 1ull) *reinterpret_cast<u32x4*>(to + row + 8u * chunk) = (r & 8u) ? u32x4{v.z, v.w, v.x, v.y} : v;
  }
  asm volatile("" ::: "memory");
}
// A NaN where a value of a lane is not finite, else 0.
template <int N>
__device__ __forceinline__ float odd_of(const f32x16 (&acc)[N]) {
  float odd = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int v = 0; v < 16; ++v) odd = __builtin_fmaf(acc[n][v], 0.f, odd);
  return odd;
}

}  // namespace attn
}  // namespace kp
