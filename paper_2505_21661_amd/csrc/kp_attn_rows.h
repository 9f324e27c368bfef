// Attention of a tile of 128 query rows over the keys they see (the kernel behind kp_attn_window and kp_attn_paged
// wherever there are more than a few rows), and the join of partial results.
//
// The rows of a tile are (token, query head of a group) pairs, token by token: heads that share keys share the tile, so
// that 16 tokens of 8 heads read a key once, and a window costs its keys once per tile.  4 waves of 32 rows; products
// are formed transposed (S^T = K Q^T, O^T = V^T P^T), so that a lane holds all scores of one row: maximum and sum are
// in-lane but for one exchange, P needs no movement between the products, O is rescaled per lane.  K and V tiles of 64
// keys are shared through LDS (K one buffer, V two): 16-bit keys go there directly from global memory, every lane
// fetching the chunk that belongs at its place; e4m3 codes come through registers and are widened on the way.
// A tile begins at the first key that a row of the tile sees, not at a multiple of 64, and past the last one the last is
// read again: nothing outside the visible ranges is touched, whatever the cache holds there.
#pragma once
#include <type_traits>

#include "kp_attn.h"
#include "kp_record.h"

namespace kp {
namespace attn {

constexpr int kThreads = 256;
constexpr int kTileRows = 128, kTileKeys = 64;
// The reference that a row's exponentials are taken against only has to keep them in range: it moves when some score exceeds
// it by more than 2^kSlack, to 2^kBelow under that score.  fp16 holds little below 2^-14: its reference stands so far below
// that the largest weight P lies between 2^11 and 2^15, and a weight 2^-25 of the largest still has ten bits (a first key that
// takes most of the weight, with a small value, over a long even tail: 32768 keys of 2^-25.3 are 7 % off without).  bf16 has the
// exponents of fp32 and needs none of it.
template <class T> constexpr float kBelow = std::is_same<T, Fp16>::value ? 11.f : 0.f;
template <class T> constexpr float kSlack = std::is_same<T, Fp16>::value ? 15.f : 8.f;
// A weight is exp2 of score times scale less the reference, in one rounding, and the reference, a rounded score, may be off by
// half a step of its own: at 2^24 by 1, at 2^33 by 512, which leaves no weight at all.  The sum of a row's weights is made a
// NaN where the reference goes that far, so that the row is taken again with scores and reference rounded alike.
constexpr float kFar = 16777216.f;
__device__ __forceinline__ float sum_unless_far(float l, float reference, float score) {
  return ((__builtin_fabsf(reference) > kFar) & (score > -INFINITY)) ? __builtin_nanf("") : l;
}

template <int D>
constexpr uint32_t tile_lds_bytes() { return 3u * kTileKeys * 2u * D; }

// Where row `flat` of a tile's sequence lies.
struct RowPlace {
  uint32_t token, in_group;
};
__device__ __forceinline__ RowPlace place_of(uint32_t flat, uint32_t group) {
  RowPlace r;
  r.token = group == 1u ? flat : flat / group;
  r.in_group = flat - r.token * group;
  return r;
}

// The larger of a lane's value and that of the lane 32 away.
__device__ __forceinline__ float either_half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// Workgroup `id` of units x per items: which unit (a head of keys, of one sequence or of all), which of its items.
// Workgroups are dealt round-robin to the 8 XCDs, each with its own L2.  All items of a unit go to one XCD where the units
// can be dealt out evenly; as many units as have places at a time (two workgroups per CU) are taken together, the first
// items of all of them first, which are the longest.
__device__ __forceinline__ void unit_of(uint32_t id, uint32_t units, uint32_t per, uint32_t* unit, uint32_t* item) {
  const uint32_t even = (units & 7u) == 0u ? 1u : 0u;
  const uint32_t xcd = even ? id & 7u : 0u, j = even ? id >> 3 : id;
  const uint32_t mine = even ? units >> 3 : units, places = even ? 64u : 512u;
  const uint32_t together = places > per ? places / per : 1u;
  const uint32_t group = j / (together * per), in = j - group * (together * per);
  const uint32_t left = mine - group * together, n = left < together ? left : together;
  const uint32_t block = in / n, u = group * together + in - block * n;
  *unit = even ? u * 8u + xcd : u;
  *item = block;
}

// Index of a row in the partial results, which hold [splits][rows](maximum, sum) and then [splits][rows][D].
template <int ROWS>
__device__ __forceinline__ size_t part_row(const Args& g, uint32_t tile, uint32_t h, uint32_t r) {
  return ((size_t)tile * g.hkv + h) * ROWS + r;
}

// Recording (INSTR: 0 no record sites, 1 generic sites, 3 the same on the constant-rate clock).
template <int INSTR>
__device__ __forceinline__ kp::Ring ring_of(const Args& g, unsigned char* ring_lds, unsigned char* scratch, uint32_t wg) {
  kp::Ring ring = kp::ring_init<true>(reinterpret_cast<uint32_t*>(ring_lds), reinterpret_cast<uint64_t*>(scratch), g.cap_lds, g.region_mask, g.flush,
                                      g.cap_hbm, g.trace, g.n_wg, 4u >> g.group_log2, wg, g.group_log2);
  ring.collab = g.collab;
  if constexpr (INSTR == 3) kp::ring_use_realtime(ring);
  return ring;
}
template <int INSTR>
__device__ __forceinline__ void finish_ring(kp::Ring& ring, const Args& g, uint32_t wg) {
  const kp::TraceGeom tg{g.n_wg, 4u >> g.group_log2, 3, g.cap_hbm, g.flags};
  kp::ring_finish<INSTR == 3>(ring, g.cap_lds, g.trace, tg, wg, g.rec_cost);
}

#define KP_BOUNDARY(ring, end_r, start_r) do { if constexpr (INSTR != 0) kp::site<INSTR>(ring, end_r, start_r); } while (0)

// Per tile of 64 keys a wave has 32 MFMAs (1024 cycles), 33 exponentials (530) and some 160 other vector instructions (640),
// which its partner on the SIMD hides in part: the matrix pipes are busy 48 % of the time at 1.9 GHz (32/8 x 8192 x 128,
// window 1024: 146 us, 890 TFLOP/s of what rows see), 38 % where a tile of rows has 10 tiles of keys (2 x 16/16 x 4000, window
// 512: 55 us, 575), since the first loads and the stores of a workgroup then weigh more; chunks of 512 tokens over up to 8192
// keys in pages, window 2048: 113 us, 750.
// Recorded regions, per tile of 64 keys: 0 K Q^T, with the request of the next keys and values and the lower half's mask and
// maximum between its MFMAs, 1 the rest of the softmax, 2 V^T P^T up to the barrier behind it.
template <class T, int D, int SRC, int INSTR>
__global__ __launch_bounds__(kThreads, 2) void kp_attn_tile(Args g) {
  constexpr uint32_t kRow = 2u * D, kChunks = kRow / 16u, kTile = kTileKeys * kRow;
  constexpr uint32_t kBlockRows = 1024u / kRow;  // rows of the 1 KiB that a wave's load fills
  constexpr int NS = D / 16, ND = D / 32, NL = (int)(kTile / 4096u);
  constexpr bool E4M3 = SRC == kPagedE4m3;
  extern __shared__ __align__(16) unsigned char smem[];  // [K tile][V tile, two buffers][ring]

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = wave_uniform(tid >> 6);
  const uint32_t h32 = lane >> 5, l32 = lane & 31u;

  uint32_t unit, item;
  const uint32_t units = SRC == kPlain ? g.seqs * g.hkv : g.hkv;
  const uint32_t tiles_per = SRC == kPlain ? g.tiles / g.seqs : g.tiles, per = tiles_per * g.splits;
  unit_of(blockIdx.x, units, per, &unit, &item);
  const uint32_t split = item % g.splits;
  uint32_t tile_id = item / g.splits, h = unit;
  if constexpr (SRC == kPlain) {  // the last rows see the most keys
    const uint32_t seq = unit / g.hkv;
    h = unit - seq * g.hkv;
    tile_id = seq * tiles_per + (tiles_per - 1u - tile_id);
  }
  Tile tl;
  const bool there = find_tile<kTileRows, SRC != kPlain>(g, tile_id, &tl);

  kp::Ring ring{};
  if constexpr (INSTR != 0) ring = ring_of<INSTR>(g, smem + 3u * kTile, smem, unit * per + item);
  if (there) {
    const Source<D, SRC> src(g, tl.seq, h);
    const uint32_t last_row = tl.rows - 1u;
    auto position = [&](uint32_t flat) __attribute__((always_inline)) {
      return (int32_t)tl.n_k - (int32_t)tl.n_q + (int32_t)place_of(flat < last_row ? flat : last_row, g.group).token;
    };
    const uint32_t wave_first = tl.first + 32u * wave, flat = wave_first + l32;
    const bool mine = flat <= last_row;
    const RowPlace at = place_of(mine ? flat : last_row, g.group);
    const int32_t p = (int32_t)tl.n_k - (int32_t)tl.n_q + (int32_t)at.token;
    const int32_t p_min = (int32_t)wave_uniform((uint32_t)position(wave_first)), p_max = (int32_t)wave_uniform((uint32_t)position(wave_first + 31u));
    const KeyTiles kt(span_of(position(tl.first), position(tl.first + kTileRows - 1u), g.window, g.sinks));
    const uint32_t t_begin = (uint32_t)((uint64_t)kt.all * split / g.splits), t_end = (uint32_t)((uint64_t)kt.all * (split + 1u) / g.splits);

    const uint32_t q_seq = SRC == kPlain ? tl.seq : 0u, head = h * g.group + at.in_group;
    const int64_t token = (int64_t)tl.q0 + at.token;
    u32x4 qf[NS];  // this lane's row: d = 16 s + 8 h32 .. + 7
    {
      const uint16_t* q = g.q.at + g.q.seq * (int64_t)q_seq + g.q.head * (int64_t)head + g.q.token * token;
#pragma unroll
      for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(q + 16 * s + 8 * h32);
    }

    // ---- the tile that is requested next ----------------------------------------------------------------------
    const uint32_t lds0 = wave_uniform((uint32_t)(uintptr_t)smem + 1024u * wave);
    const uint32_t ld_row = kBlockRows * wave + lane / kChunks, pos = lane % kChunks;
    // chunk c of row r lies at position c ^ swizzle(r): 16 neighbouring rows' 16-byte reads (K), and the four rows of a
    // transposing read (V), cover all banks once
    const uint32_t k_sw = D == 128 ? ld_row & 15u : (ld_row >> 1) & 7u, v_sw = D == 128 ? 4u * (ld_row & 3u) : 4u * ((ld_row >> 1) & 1u);
    const uint32_t k_in = (pos ^ k_sw) << 4, v_in = (pos ^ v_sw) << 4;
    uint32_t k_ofs[NL], v_ofs[NL];        // kPlain: from the tile's first key, bytes
    const uint8_t *k_base = nullptr, *v_base = nullptr;
    uint64_t k_ptr[NL], v_ptr[NL];        // kPaged
    uint32_t ofs_last = 0;                // last row that the offsets were made for
    int32_t page_id = 0;                  // paged: block-table entry of the next tile's key number `lane`
    uint64_t valid = ~0ull, valid_next = ~0ull;  // paged: keys of this and the next tile whose page exists
    u32x4 k8[E4M3 ? D / 64 : 1], v8[E4M3 ? D / 64 : 1];
    float ke[E4M3 ? D / 64 : 1], ve[E4M3 ? D / 64 : 1];
    uint32_t v_into = kTile;              // LDS offset of the V buffer that the next tile goes to

    // the key that tile t's row r is (past the last one that again); FIRST: it may be the first tile
    auto key_of = [&](uint32_t t, uint32_t start, uint32_t r, uint32_t last, auto first_c) __attribute__((always_inline)) {
      uint32_t key = start + (r < last ? r : last);
      if constexpr (decltype(first_c)::value) key = kt.is_mixed(t) && r < kt.mixed ? r : key;
      return key;
    };
    uint32_t next_start = 0, next_limit = 0, next_sinks = g.sinks;  // of the tile that is requested
    auto begin_of = [&](uint32_t t, uint32_t* limit, auto first_c) __attribute__((always_inline)) {
      if constexpr (decltype(first_c)::value) return kt.start_of(t, limit, &next_sinks);
      else return kt.start(t, limit);
    };
    auto load_page_ids = [&](uint32_t t, auto first_c) __attribute__((always_inline)) {
      if constexpr (SRC != kPlain) {
        if (t < t_end) {
          uint32_t limit;
          const uint32_t start = begin_of(t, &limit, first_c);
          page_id = src.table[key_of(t, start, lane, limit - 1u - start, first_c) >> src.page_log2];
        }
      }
    };
    // Where tile t's rows are; its page ids have been asked for before.
    auto locate = [&](uint32_t t, auto first_c) __attribute__((always_inline)) {
      const uint32_t start = next_start = begin_of(t, &next_limit, first_c), left = next_limit - 1u - start, last = left < kTileKeys - 1u ? left : kTileKeys - 1u;
      if constexpr (SRC == kPlain) {
        k_base = src.k + src.k_step * (int64_t)start;
        v_base = src.v + src.v_step * (int64_t)start;
        if (last != ofs_last) {
          ofs_last = last;
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const uint32_t row = ld_row + 4u * kBlockRows * (uint32_t)i, r = row < last ? row : last;
            k_ofs[i] = r * (uint32_t)src.k_step + k_in;
            v_ofs[i] = r * (uint32_t)src.v_step + v_in;
          }
        }
      } else {
        uint32_t row_no = src.row_of_page(page_id, key_of(t, start, lane, last, first_c));
        valid_next = __builtin_amdgcn_ballot_w64(row_no != ~0u);
        if (row_no == ~0u) row_no = 0u;  // (some row of the cache: its scores are masked)
        if constexpr (!E4M3) {
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const uint32_t r = __shfl(row_no, (int)(ld_row + 4u * kBlockRows * (uint32_t)i), 64);
            k_ptr[i] = (uint64_t)(uintptr_t)src.k + (uint64_t)r * kRow + k_in;
            v_ptr[i] = (uint64_t)(uintptr_t)src.v + (uint64_t)r * kRow + v_in;
          }
        } else {
#pragma unroll
          for (int i = 0; i < D / 64; ++i) {
            constexpr uint32_t kPer = D / 16;  // 16-byte chunks of a row of codes
            const uint32_t r = __shfl(row_no, (int)((tid + kThreads * (uint32_t)i) / kPer), 64);
            k8[i] = *reinterpret_cast<const u32x4*>(src.k + (size_t)r * D + 16u * (tid % kPer));
            v8[i] = *reinterpret_cast<const u32x4*>(src.v + (size_t)r * D + 16u * (tid % kPer));
            ke[i] = power_of(src.k_exp[r]);
            ve[i] = power_of(src.v_exp[r]);
          }
        }
        load_page_ids(t + 1u, std::false_type{});
      }
    };
    // One load straight to LDS: M0 (the LDS base) is put back afterwards.  From inline assembly because the compiler would
    // make the next LDS access of any kind wait for such a load; the loads complete in order, and the kernel waits for them
    // itself in front of the barrier that precedes the tile's use.
    auto load_from = [&](const uint8_t* base, uint32_t ofs, uint32_t dst) __attribute__((always_inline)) {
      uint32_t saved_m0;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0) : "v"(ofs), "s"(base), "s"(dst) : "memory");
    };
    auto load_at = [&](uint64_t ptr, uint32_t dst) __attribute__((always_inline)) {
      uint32_t saved_m0;
      asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                   : "=&s"(saved_m0) : "v"(ptr), "s"(dst) : "memory");
    };
    auto load_k = [&](int i) __attribute__((always_inline)) {
      const uint32_t dst = lds0 + 4096u * (uint32_t)i;
      if constexpr (SRC == kPlain) load_from(k_base, k_ofs[i], dst);
      else if constexpr (!E4M3) load_at(k_ptr[i], dst);
    };
    auto load_v = [&](int i) __attribute__((always_inline)) {
      const uint32_t dst = lds0 + v_into + 4096u * (uint32_t)i;
      if constexpr (SRC == kPlain) load_from(v_base, v_ofs[i], dst);
      else if constexpr (!E4M3) load_at(v_ptr[i], dst);
    };
    // e4m3: the codes in registers become 16-bit rows in LDS
    auto widen = [&](const u32x4& codes, float scale, uint32_t base, uint32_t row, uint32_t c, uint32_t sw) __attribute__((always_inline)) {
      u32x4 lo, hi;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        u32x4& to = w < 2 ? lo : hi;
        to[2 * (w & 1)] = T::template from_e4m3<false>(codes[w], scale);
        to[2 * (w & 1) + 1] = T::template from_e4m3<true>(codes[w], scale);
      }
      *reinterpret_cast<u32x4*>(smem + base + row * kRow + (((2u * c) ^ sw) << 4)) = lo;
      *reinterpret_cast<u32x4*>(smem + base + row * kRow + (((2u * c + 1u) ^ sw) << 4)) = hi;
    };
    auto store_codes = [&](bool keys) __attribute__((always_inline)) {
      if constexpr (E4M3) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const uint32_t j = tid + kThreads * (uint32_t)i, row = j / (D / 16), c = j % (D / 16);
          if (keys) widen(k8[i], ke[i], 0u, row, c, D == 128 ? row & 15u : (row >> 1) & 7u);
          else widen(v8[i], ve[i], v_into, row, c, D == 128 ? 4u * (row & 3u) : 4u * ((row >> 1) & 1u));
        }
      }
    };
    auto requested = [&]() __attribute__((always_inline)) {
      v_into ^= kTile ^ (2u * kTile);
    };

    // ---- operand reads: K row 32 tk + l32, chunk 2 s + h32; V for the keys of step (16 keys) and the d of dt --------
    uint32_t k_rd[NS], v_rd[ND];
#pragma unroll
    for (int s = 0; s < NS; ++s)
      k_rd[s] = (uint32_t)(uintptr_t)smem + l32 * kRow + (((2u * (uint32_t)s + h32) ^ (D == 128 ? l32 & 15u : (l32 >> 1) & 7u)) << 4);
    {
      const uint32_t i = lane & 15u, grp = lane >> 4, row = 4u * (grp >> 1) + (i >> 2);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const uint32_t d = 32u * (uint32_t)dt + 16u * (grp & 1u) + 4u * (i & 3u), sw = D == 128 ? 4u * (row & 3u) : 4u * ((row >> 1) & 1u);
        v_rd[dt] = (uint32_t)(uintptr_t)smem + kTile + row * kRow + (((d >> 3) ^ sw) << 4) + 8u * ((d >> 2) & 1u);
      }
    }
    uint32_t v_other = kTile;  // from the V buffer in use to the other one
    auto read_k = [&](int s, int tk) __attribute__((always_inline)) -> u32x4 {
      typedef const __attribute__((address_space(3))) u32x4* lds_u32x4;
      return *(lds_u32x4)(uintptr_t)(k_rd[s] + (uint32_t)tk * 32u * kRow);
    };
    auto read_v = [&](uint32_t step, int dt) __attribute__((always_inline)) -> u32x4 {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
      const uint32_t a = v_rd[dt] + step * (16u * kRow);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(a));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(a + 8u * kRow));
      const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(u32x4, v);
    };

    f32x16 oacc[ND];  // O^T: rows d = 32 dt + 8 j + 4 h32 + i, column = row l32
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) oacc[dt] = f32x16{0};
    float m_run = kNoKey, l_run = 0.f;

    u32x4 kf[NS];  // operands of K Q^T, NS MFMAs ahead
    auto request_k_operands = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < NS; ++n) kf[n] = read_k(n, 0);
    };
    auto tile = [&](uint32_t t, auto more_c) __attribute__((always_inline)) {
      constexpr bool MORE = decltype(more_c)::value;
      const uint32_t start = next_start, limit = next_limit, sinks = next_sinks;
      next_sinks = g.sinks;
      const int32_t end = (int32_t)(start + kTileKeys);  // one past the tile's last key
      bool masked = (end > (int32_t)limit) | (end - 1 > p_min);
      masked = masked | ((g.window != 0u) & (p_max - (int32_t)start >= (int32_t)g.window) & (end > (int32_t)sinks));
      if constexpr (SRC != kPlain) masked = masked | (valid != ~0ull);
      f32x16 sacc[2];
      sacc[0] = f32x16{0}; sacc[1] = f32x16{0};
      float mx = -INFINITY, psum = 0.f;
      u32x4 pw[4];  // P, in accumulator order: one entry per MFMA step of V^T P^T (16 keys)
      auto mask = [&](int tk) __attribute__((always_inline)) {
        if (!masked) return;
        RowMask m(p, limit, (int32_t)(start + 4u * h32), g.window, sinks);
        if ((g.window != 0u) & (start < sinks)) {
          m.apart();
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[tk][v] = m.sees_mixed(32 * tk + 8 * (v >> 2) + (v & 3)) ? sacc[tk][v] : -INFINITY;
        } else {
          m.apart();
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[tk][v] = m.sees(32 * tk + 8 * (v >> 2) + (v & 3)) ? sacc[tk][v] : -INFINITY;
        }
        if constexpr (SRC != kPlain) {
          if (valid != ~0ull) {  // pages that are not there
            const uint64_t there = valid >> (4u * h32);
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[tk][v] = (there >> (32 * tk + 8 * (v >> 2) + (v & 3))) & 1ull ? sacc[tk][v] : -INFINITY;
          }
        }
      };
      auto exps = [&](int pair) __attribute__((always_inline)) {
        const int tk = pair >> 3, v = 2 * (pair & 7);
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[tk][v], g.scale_log2, -m_run));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[tk][v + 1], g.scale_log2, -m_run));
        psum += p0 + p1;  // the sum is of the unrounded probabilities
        pw[pair >> 2][pair & 3] = T::pack(p0, p1);
      };

      // ---- region 0: S^T = K Q^T ------------------------------------------------------------------------------
      if constexpr (MORE) locate(t + 1u, std::false_type{});
      __builtin_amdgcn_s_setprio(2);
      constexpr int kBarrier = NS + 1, kLoads = NS == 8 ? 11 : 6;
#pragma unroll
      for (int n = 0; n < 2 * NS; ++n) {  // the lower 32 keys, then the upper ones, whose operands are requested meanwhile
        const int s = n % NS, tk = n / NS;
        sacc[tk] = T::mfma32(kf[s], qf[s], sacc[tk]);
        if (tk == 0) kf[s] = read_k(s, 1);
        if (MORE && tk == 0 && (s & 1)) load_v(s >> 1);
        if (MORE && n >= kLoads && n < kLoads + NL) load_k(n - kLoads);
        if (tk == 1) {  // the maximum of the lower half
          if (s == 0) mask(0);
#pragma unroll
          for (int v = s * (16 / NS); v < (s + 1) * (16 / NS); v += 2) mx = fmaxf(fmaxf(mx, sacc[0][v]), sacc[0][v + 1]);
        }
        __builtin_amdgcn_sched_barrier(0);
        // every wave has read this K tile
        if (MORE && n == kBarrier) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
      __builtin_amdgcn_s_setprio(0);
      KP_BOUNDARY(ring, 0, 1);

      // ---- region 1: online softmax (this lane: 32 of the tile's 64 keys) -----------------------------------------
      u32x4 vf[4];  // operands of V^T P^T, four MFMAs ahead
#pragma unroll
      for (int m = 0; m < 4; ++m) vf[m] = read_v((uint32_t)(m / ND), m % ND);
      mask(1);
#pragma unroll
      for (int v = 0; v < 16; v += 2) mx = fmaxf(fmaxf(mx, sacc[1][v]), sacc[1][v + 1]);
      mx = either_half_max(mx);
      // O and l are rescaled when some row's reference has to move
      const float mx_s = mx * g.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx_s > m_run + kSlack<T>) != 0ull) {
        const float m_new = fmaxf(m_run, mx_s - kBelow<T>);
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run = sum_unless_far(l_run * alpha, m_new, mx_s);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
        m_run = m_new;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) exps(i);
      l_run += psum;
      KP_BOUNDARY(ring, 1, 2);
      if constexpr (MORE && E4M3) { store_codes(true); store_codes(false); }
      __builtin_amdgcn_s_setprio(1);

      // ---- region 2: O^T += V^T P^T ---------------------------------------------------------------------------------
      // The key order inside a step follows the accumulator layout of S^T, so P needs no movement; V is read to match.
      auto pv = [&](int m) __attribute__((always_inline)) {
        oacc[m % ND] = T::mfma32(vf[m & 3], pw[m / ND], oacc[m % ND]);
      };
#pragma unroll
      for (int m = 0; m < 4 * ND - 4; ++m) {
        pv(m);
        vf[m & 3] = read_v((uint32_t)((m + 4) / ND), (m + 4) % ND);
        __builtin_amdgcn_sched_barrier(0);
      }
      // Every wave has read this V tile, and the next K and V tiles have landed.  The last four MFMAs come behind the
      // barrier, under the first operand reads of the next tile.
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if constexpr (MORE) request_k_operands();
#pragma unroll
      for (int m = 4 * ND - 4; m < 4 * ND; ++m) pv(m);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) v_rd[dt] += v_other;
      v_other = 0u - v_other;
      if constexpr (MORE) { requested(); valid = valid_next; }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (MORE) KP_BOUNDARY(ring, 2, 0); else KP_BOUNDARY(ring, 2, kp::kNoRegion);
    };
    if (t_begin < t_end) {
      load_page_ids(t_begin, std::true_type{});
      ofs_last = ~0u;
      bool loaded = false;
      if constexpr (SRC == kPlain) {
        if (kt.is_mixed(t_begin)) {  // (the distance between its keys may take more than 32 bits)
          next_start = begin_of(t_begin, &next_limit, std::true_type{});
          const uint32_t last = next_limit - 1u - next_start;
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int64_t key = (int64_t)key_of(t_begin, next_start, ld_row + 4u * kBlockRows * (uint32_t)i, last, std::true_type{});
            load_at((uint64_t)(uintptr_t)(src.k + src.k_step * key) + k_in, lds0 + 4096u * (uint32_t)i);
            load_at((uint64_t)(uintptr_t)(src.v + src.v_step * key) + v_in, lds0 + v_into + 4096u * (uint32_t)i);
          }
          loaded = true;
        }
      }
      if (!loaded) {
        locate(t_begin, std::true_type{});
#pragma unroll
        for (int i = 0; i < NL; ++i) { load_k(i); load_v(i); }
      }
      store_codes(true);
      store_codes(false);
      requested();
      valid = valid_next;
      __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own count of outstanding loads)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      constexpr std::true_type yes{};
      constexpr std::false_type no{};
      KP_BOUNDARY(ring, kp::kNoRegion, 0);
      request_k_operands();
      for (uint32_t t = t_begin; t + 1u < t_end; ++t) tile(t, yes);
      tile(t_end - 1u, no);
    }

    // ---- the rows leave -----------------------------------------------------------------------------------------------
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    const int64_t o_at = g.o.seq * (int64_t)q_seq + g.o.head * (int64_t)head + g.o.token * token;
    const int64_t lse_at = g.lse_seq * (int64_t)q_seq + g.lse_head * (int64_t)head + token;
    // 0 where all values are finite, else a NaN
    float odd = l_tot * 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) odd = __builtin_fmaf(oacc[dt][v], 0.f, odd);
    uint64_t again = __builtin_amdgcn_ballot_w64(odd != odd && mine);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    float* const part_ml = g.part;
    const size_t part_rows = (size_t)g.tiles * g.hkv * kTileRows;
    if (g.splits > 1u) {
      const size_t row = split * part_rows + part_row<kTileRows>(g, tile_id, h, 32u * wave + l32);
      if (mine) {
        if (h32 == 0) *reinterpret_cast<f32x2*>(part_ml + 2 * row) = f32x2{m_run, l_tot};
        float* o = g.part + 2 * g.splits * part_rows + row * D;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4*>(o + 32 * dt + 8 * j + 4 * h32) = f32x4{oacc[dt][4 * j], oacc[dt][4 * j + 1], oacc[dt][4 * j + 2], oacc[dt][4 * j + 3]};
      }
    } else {
      if (g.lse && mine && h32 == 0) g.lse[lse_at] = l_tot == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
      const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
      // Through LDS (32 rows of a wave: every wave is past its last operand read), whole rows leave.  Chunk c of row r at
      // position c ^ r % 8, its halves swapped where r / 8 is odd: 16 lanes of an 8-byte write hit all banks once.
      unsigned char* const sO = smem + 32u * kRow * wave;
      const uint32_t half = h32 ^ ((l32 >> 3) & 1u);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u32x2 two;
          two.x = T::pack(oacc[dt][4 * j + 0] * inv, oacc[dt][4 * j + 1] * inv);
          two.y = T::pack(oacc[dt][4 * j + 2] * inv, oacc[dt][4 * j + 3] * inv);
          *reinterpret_cast<u32x2*>(sO + l32 * kRow + (((uint32_t)(4 * dt + j) ^ (l32 & 7u)) << 4) + 8u * half) = two;
        }
      uint16_t* const o = const_cast<uint16_t*>(g.o.at);
#pragma unroll
      for (int i = 0; i < (int)(32u / kBlockRows); ++i) {
        const uint32_t r = kBlockRows * (uint32_t)i + lane / kChunks, chunk = (lane % kChunks) ^ (r & 7u);
        const u32x4 v = *reinterpret_cast<const u32x4*>(sO + 1024u * (uint32_t)i + 16u * lane);
        const int64_t to = (int64_t)(((uint64_t)(uint32_t)__shfl((int)(o_at >> 32), (int)r, 64) << 32) | (uint32_t)__shfl((int)o_at, (int)r, 64));
        if (wave_first + r <= last_row) *reinterpret_cast<u32x4*>(o + to + 8u * chunk) = (r & 8u) ? u32x4{v.z, v.w, v.x, v.y} : v;
      }
    }
    // Rows with a value that is not finite, taken again (see Row).
    if (again != 0ull) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // their first results have left
      for (; again != 0ull; again &= again - 1ull) {
        const uint32_t r = (uint32_t)__builtin_ctzll(again);
        const RowPlace a = place_of(wave_first + r, g.group);
        const uint32_t hd = h * g.group + a.in_group;
        const int64_t tok = (int64_t)tl.q0 + a.token;
        const uint16_t* const q = g.q.at + g.q.seq * (int64_t)q_seq + g.q.head * (int64_t)hd + g.q.token * tok;
        Row<T, D, SRC> row;
        for (uint32_t t = t_begin; t < t_end; ++t) {
          uint32_t limit, unused;
          const int32_t at = (int32_t)tl.n_k - (int32_t)tl.n_q + (int32_t)a.token;
          const uint32_t start = kt.start_of(t, &limit, &unused), to = start + kTileKeys, mixed = kt.is_mixed(t) ? kt.mixed : 0u;
          if (mixed != 0u) row.over_keys(q, src, at, g.window, g.sinks, g.scale_log2, 0u, mixed);
          row.over_keys(q, src, at, g.window, g.sinks, g.scale_log2, start + mixed, to < limit ? to : limit);
        }
        if (g.splits > 1u) {
          const size_t to = split * part_rows + part_row<kTileRows>(g, tile_id, h, 32u * wave + r);
          row.store_part(g.part + 2 * g.splits * part_rows + to * D, part_ml + 2 * to);
        } else {
          row.store(const_cast<uint16_t*>(g.o.at) + g.o.seq * (int64_t)q_seq + g.o.head * (int64_t)hd + g.o.token * tok,
                    g.lse ? g.lse + g.lse_seq * (int64_t)q_seq + g.lse_head * (int64_t)hd + tok : nullptr);
        }
      }
    }
  }
  if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, unit * per + item);
}

// Bound by latency: 3 to 6 us for up to 4 MB of parts.
// Joins the partial results of a row: D / 4 lanes to a row, 4 elements to a lane.  ROWS: of a tile of the kernel that made
// them.  WIDE: the workgroup has one row, whose parts its groups of lanes share, eight at a time to a group.
constexpr uint32_t kJoinAtOnce = 8;  // parts of a group whose loads are in flight together
template <class T, int D, int ROWS, bool PAGED, bool WIDE>
__global__ __launch_bounds__(kThreads) void kp_attn_join(Args g) {
  constexpr uint32_t kLanes = D / 4, kGroups = kThreads / kLanes, kPer = WIDE ? 1u : kGroups;  // rows of a workgroup
  const uint32_t blocks = ROWS / kPer, unit = blockIdx.x / blocks, block = blockIdx.x - unit * blocks;
  const uint32_t group = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  const uint32_t tile_id = unit / g.hkv, h = unit - tile_id * g.hkv, r = WIDE ? block : block * kPer + group;
  Tile tl;
  if (!find_tile<ROWS, PAGED>(g, tile_id, &tl)) return;
  const uint32_t flat = tl.first + r;
  if (flat >= tl.rows) return;
  const size_t rows = (size_t)g.tiles * g.hkv * ROWS, row = part_row<ROWS>(g, tile_id, h, r);
  float m = kNoKey, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr uint32_t kAtOnce = kJoinAtOnce;
  for (uint32_t s0 = WIDE ? group * kAtOnce : 0u; s0 < g.splits; s0 += WIDE ? kGroups * kAtOnce : kAtOnce) {
    f32x2 ml[kAtOnce];
    f32x4 part[kAtOnce];
    float top = m;
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) {
      const size_t at = (s0 + i < g.splits ? s0 + i : g.splits - 1u) * rows + row;
      ml[i] = *reinterpret_cast<const f32x2*>(g.part + 2 * at);
      part[i] = *reinterpret_cast<const f32x4*>(g.part + 2 * g.splits * rows + at * D + 4u * c);
    }
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i].x);
    const float before = __builtin_amdgcn_exp2f(m - top);
    l *= before;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= before;
    m = top;
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i) {
      if ((s0 + i >= g.splits) | (ml[i].y == 0.f)) continue;
      const float w = __builtin_amdgcn_exp2f(ml[i].x - m);
      l = __builtin_fmaf(ml[i].y, w, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(part[i][e], w, o[e]);
    }
  }
  if constexpr (WIDE) {
    __shared__ float group_m[kGroups], group_l[kGroups];
    __shared__ f32x4 group_o[kGroups][kLanes];
    if (c == 0) { group_m[group] = m; group_l[group] = l; }
    group_o[group][c] = o;
    __syncthreads();
    if (group != 0u) return;
    float top = m;
    for (uint32_t i = 1; i < kGroups; ++i) top = fmaxf(top, group_m[i]);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (uint32_t i = 0; i < kGroups; ++i) {
      if (group_l[i] == 0.f) continue;
      const float w = __builtin_amdgcn_exp2f(group_m[i] - top);
      l = __builtin_fmaf(group_l[i], w, l);
      const f32x4 part = group_o[i][c];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(part[e], w, o[e]);
    }
    m = top;
  }
  const RowPlace at = place_of(flat, g.group);
  const uint32_t head = h * g.group + at.in_group, seq = PAGED ? 0u : tl.seq;
  const int64_t token = (int64_t)tl.q0 + at.token;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  uint16_t* to = const_cast<uint16_t*>(g.o.at) + g.o.seq * (int64_t)seq + g.o.head * (int64_t)head + g.o.token * token + 4u * c;
  *reinterpret_cast<u32x2*>(to) = u32x2{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
  if (g.lse && c == 0) g.lse[g.lse_seq * (int64_t)seq + g.lse_head * (int64_t)head + token] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace attn
}  // namespace kp
