// Attention of few query rows over many keys (single tokens): a tile of 16 rows, the keys dealt out to the waves.
//
// With one token per sequence there are as many rows per head of keys as query heads in its group, and every key is used
// once per row: the time is that of reading the cache.  A workgroup takes a run of a sequence's keys (a split) of one head;
// its 4 waves take steps of 32 keys in turn, each with a softmax of its own, and join at the end through LDS; the splits
// join in kp_attn_join.  Products as in kp_attn_rows.h with the 16x16x32 shape: K goes from memory to the operand
// registers as it lies (a lane reads 16-byte pieces of one key's row), V through 8 KiB of LDS per wave, which the
// transposing read needs; both are asked for a step ahead.
// Bound by memory: 64 tokens of 32/8 heads of 128 over up to 16384 keys of e4m3, 1409 MB, take 238 us with the join (5920
// GB/s, 96 % of what reading alone reaches); 16 tokens of 16/2 heads over a window of 4096, 67 MB, 17.7 us (14 of them this
// kernel); small calls by latency (4 tokens over up to 700 keys: 8 us; an empty kernel takes 3.8 a launch).
#pragma once
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

constexpr int kFewRows = 16, kFewKeys = 32;

// Recorded regions, per step of 32 keys: 0 K Q^T and the request of the next keys, 1 mask and softmax, 2 V to LDS, the
// request of the next values, V^T P^T.
template <class T, int D, int SRC, int INSTR>
__global__ __launch_bounds__(kThreads, 2) void kp_attn_few(Args g) {
  constexpr bool E4M3 = SRC == kPagedE4m3;
  constexpr uint32_t kRow = 2u * D;
  constexpr int NS = D / 32;                    // MFMA steps of K Q^T
  constexpr int NT = D / 16;                    // tiles of 16 d
  constexpr int KL = E4M3 ? D / 64 : D / 32;    // 16-byte loads of a lane per 16 keys
  constexpr uint32_t kVPer = E4M3 ? D / 16 : D / 8;          // lanes to a row of V
  constexpr int VL = (int)(kFewKeys * kVPer / 64u);          // loads of a lane per step
  constexpr uint32_t kWaveLds = kFewKeys * kRow;
  __shared__ __align__(16) unsigned char smem[4u * kWaveLds];
  __shared__ float join_m[4][kFewRows], join_l[4][kFewRows];
  __shared__ uint32_t again_rows;
  extern __shared__ __align__(16) unsigned char ring_lds[];

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = wave_uniform(tid >> 6), r16 = lane & 15u, g4 = lane >> 4;
  // (splits of a tile next to one another: they share the tile's queries; heads are dealt to the XCDs as they come)
  const uint32_t units = SRC == kPlain ? g.seqs * g.hkv : g.hkv, tiles_per = SRC == kPlain ? g.tiles / g.seqs : g.tiles;
  uint32_t unit, item;
  unit_of(blockIdx.x, units, tiles_per * g.splits, &unit, &item);
  const uint32_t split = item % g.splits;
  uint32_t tile_id = item / g.splits, h = unit;
  if constexpr (SRC == kPlain) {
    const uint32_t seq = unit / g.hkv;
    h = unit - seq * g.hkv;
    tile_id = seq * tiles_per + tile_id;
  }
  Tile tl;
  const bool there = find_tile<kFewRows, SRC != kPlain>(g, tile_id, &tl);
  const uint32_t recorded = unit * (tiles_per * g.splits) + item;  // number of the workgroup in a trace
  kp::Ring ring{};
  if constexpr (INSTR != 0) ring = ring_of<INSTR>(g, ring_lds, smem, recorded);
  if (!there) {
    if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
    return;
  }
  const Source<D, SRC> src(g, tl.seq, h);
  const uint32_t last_row = tl.rows - 1u, flat = tl.first + r16;
  const bool mine = flat <= last_row;
  const RowPlace at = place_of(mine ? flat : last_row, g.group);
  const int32_t p0 = (int32_t)tl.n_k - (int32_t)tl.n_q, p = p0 + (int32_t)at.token;
  const int32_t p_min = p0 + (int32_t)place_of(tl.first, g.group).token;
  const int32_t p_max = p0 + (int32_t)place_of(tl.first + kFewRows - 1u < last_row ? tl.first + kFewRows - 1u : last_row, g.group).token;
  const Span span = span_of(p_min, p_max, g.window, g.sinks);
  const uint32_t sink_steps = (span.sink_end + kFewKeys - 1u) / kFewKeys;
  const uint32_t all = sink_steps + (span.end > span.lo ? (span.end - span.lo + kFewKeys - 1u) / kFewKeys : 0u);
  const uint32_t t_begin = (uint32_t)((uint64_t)all * split / g.splits), t_end = (uint32_t)((uint64_t)all * (split + 1u) / g.splits);
  auto step_start = [&](uint32_t t, uint32_t* limit) __attribute__((always_inline)) {
    *limit = t < sink_steps ? span.sink_end : span.end;
    return t < sink_steps ? t * kFewKeys : span.lo + (t - sink_steps) * kFewKeys;
  };

  // Queries of row r16.  The d that a lane's operand of step s stands for: 16-bit keys 32 s + 8 g4 .. + 7; codes, of which a
  // lane reads 16 at a time, 64 (s / 2) + 16 g4 + 8 (s % 2) .. + 7.
  const uint32_t q_seq = SRC == kPlain ? tl.seq : 0u, head = h * g.group + at.in_group;
  const int64_t token = (int64_t)tl.q0 + at.token;
  u32x4 qf[NS];
  {
    const uint16_t* q = g.q.at + g.q.seq * (int64_t)q_seq + g.q.head * (int64_t)head + g.q.token * token;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(q + (E4M3 ? 64u * (s / 2) + 16u * g4 + 8u * (s % 2) : 32u * s + 8u * g4));
  }

  unsigned char* const sV = smem + kWaveLds * wave;
  u32x4 kr[2][KL], vr[VL];
  uint32_t k_e[2], v_e[VL];
  int32_t page_id = 0;        // of key number lane % 32 of the next step
  uint64_t valid = 0, valid_next = 0;
  auto load_page_ids = [&](uint32_t t) __attribute__((always_inline)) {
    if constexpr (SRC != kPlain) {
      if (t < t_end) {
        uint32_t limit;
        const uint32_t start = step_start(t, &limit), last = limit - 1u - start, l = lane & 31u;
        page_id = src.table[(start + (l < last ? l : last)) >> src.page_log2];
      }
    }
  };
  // Asks for step t's keys (its page ids have been asked for before), and for its values.
  uint32_t row_no = 0;
  auto locate = [&](uint32_t t) __attribute__((always_inline)) {
    uint32_t limit;
    const uint32_t start = step_start(t, &limit), last = limit - 1u - start, l = lane & 31u, j = start + (l < last ? l : last);
    if constexpr (SRC == kPlain) {
      row_no = j;
    } else {
      row_no = src.row_of_page(page_id, j);
      valid_next = __builtin_amdgcn_ballot_w64(row_no != ~0u);
      if (row_no == ~0u) row_no = 0u;  // (some row of the cache: its scores are masked)
      load_page_ids(t + 4u);
    }
  };
  auto load_k = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t r = __shfl(row_no, (int)(16u * n + r16), 64);
      const uint8_t* row = src.k_at(r) + 16u * g4;
#pragma unroll
      for (int i = 0; i < KL; ++i) kr[n][i] = *reinterpret_cast<const u32x4*>(row + 64 * i);
      if constexpr (E4M3) k_e[n] = src.k_exp[r];
    }
  };
  // Values go past the caches, whole lines at a time; of a line of keys a load takes half, and the other half is to be there
  // for the next (64 tokens over up to 16384 keys: 238 us, all through the caches 261, nothing 247).  That suits sequences of
  // one tile with pages of their own, whose values are read once; those of a longer run of tokens in a batch of single ones,
  // or of a shared page, come from memory for every tile that sees them.
  auto load_v = [&](uint32_t rows) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const uint32_t r = __shfl(rows, (int)((64u / kVPer) * i + lane / kVPer), 64);
      vr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src.v_at(r) + 16u * (lane % kVPer)));
      if constexpr (E4M3) v_e[i] = src.v_exp[r];
    }
  };
  // V tile: chunk c of row r at position c ^ swizzle(r), as in kp_attn_tile
  auto swizzle = [&](uint32_t row) __attribute__((always_inline)) { return D == 128 ? 4u * (row & 3u) : 4u * ((row >> 1) & 1u); };
  auto store_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const uint32_t row = (64u / kVPer) * i + lane / kVPer, c = lane % kVPer, sw = swizzle(row);
      if constexpr (!E4M3) {
        *reinterpret_cast<u32x4*>(sV + row * kRow + ((c ^ sw) << 4)) = vr[i];
      } else {
        const float scale = power_of(v_e[i]);
        u32x4 lo, hi;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          u32x4& to = w < 2 ? lo : hi;
          to[2 * (w & 1)] = T::template from_e4m3<false>(vr[i][w], scale);
          to[2 * (w & 1) + 1] = T::template from_e4m3<true>(vr[i][w], scale);
        }
        *reinterpret_cast<u32x4*>(sV + row * kRow + (((2u * c) ^ sw) << 4)) = lo;
        *reinterpret_cast<u32x4*>(sV + row * kRow + (((2u * c + 1u) ^ sw) << 4)) = hi;
      }
    }
  };
  uint32_t v_rd[NT];
  {
    const uint32_t row = 4u * g4 + (r16 >> 2);
#pragma unroll
    for (int dt = 0; dt < NT; ++dt) {
      const uint32_t d = 16u * (uint32_t)dt + 4u * (r16 & 3u);
      v_rd[dt] = (uint32_t)(uintptr_t)sV + row * kRow + (((d >> 3) ^ swizzle(row)) << 4) + 8u * ((d >> 2) & 1u);
    }
  }
  auto read_v = [&](int dt) __attribute__((always_inline)) -> u32x4 {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_rd[dt]));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(v_rd[dt] + 16u * kRow));
    const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(u32x4, v);
  };

  f32x4 oacc[NT];  // O^T: d = 16 dt + 4 g4 + i, column = row r16
#pragma unroll
  for (int dt = 0; dt < NT; ++dt) oacc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_run = kNoKey, l_run = 0.f;

  const uint32_t t_first = t_begin + wave;
  if (t_first < t_end) {
    load_page_ids(t_first);
    locate(t_first);
    load_k();
    load_v(row_no);
    valid = valid_next;
    KP_BOUNDARY(ring, kp::kNoRegion, 0);
    for (uint32_t t = t_first; t < t_end; t += 4u) {
      const bool more = t + 4u < t_end;
      uint32_t limit;
      const uint32_t start = step_start(t, &limit);
      const int32_t end = (int32_t)(start + kFewKeys);
      // S^T = K Q^T: keys 16 n + 4 g4 + i, column = row r16
      f32x4 sacc[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        sacc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!E4M3) {
#pragma unroll
          for (int s = 0; s < NS; ++s) sacc[n] = T::mfma16(kr[n][s], qf[s], sacc[n]);
        } else {
          const float scale = power_of(k_e[n]);
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            u32x4 a;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              a[2 * w] = T::template from_e4m3<false>(kr[n][s / 2][2 * (s % 2) + w], scale);
              a[2 * w + 1] = T::template from_e4m3<true>(kr[n][s / 2][2 * (s % 2) + w], scale);
            }
            sacc[n] = T::mfma16(a, qf[s], sacc[n]);
          }
        }
      }
      if (more) {
        locate(t + 4u);
        load_k();
      }
      KP_BOUNDARY(ring, 0, 1);
      bool masked = end > (int32_t)limit || end - 1 > p_min;
      if (g.window != 0u) masked = masked || (p_max - (int32_t)start >= (int32_t)g.window && end > (int32_t)g.sinks);
      if constexpr (SRC != kPlain) masked = masked || valid != ~0ull;
      if (masked) {
        const RowMask m(p, limit, (int32_t)(start + 4u * g4), g.window, g.sinks);
        const uint32_t there = SRC != kPlain ? (uint32_t)valid >> (4u * g4) : ~0u;  // keys whose page exists
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = 16 * n + i;
            // (& and |: short cuts become branches)
            const bool seen = (m.sees(c) | ((g.window != 0u) & (c <= m.sink))) & (((there >> c) & 1u) != 0u);
            sacc[n][i] = seen ? sacc[n][i] : -INFINITY;
          }
      }
      float mx = fmaxf(fmaxf(fmaxf(sacc[0][0], sacc[0][1]), fmaxf(sacc[0][2], sacc[0][3])), fmaxf(fmaxf(sacc[1][0], sacc[1][1]), fmaxf(sacc[1][2], sacc[1][3])));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = either_half_max(mx);
      const float mx_s = mx * g.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx_s > m_run + kSlack<T>) != 0ull) {
        const float m_new = fmaxf(m_run, mx_s - kBelow<T>), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        l_run = sum_unless_far(l_run * alpha, m_new, mx_s);
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) oacc[dt][i] *= alpha;
        m_run = m_new;
      }
      u32x4 pw;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[n][i], g.scale_log2, -m_run));
          l_run += w[i];
        }
        pw[2 * n] = T::pack(w[0], w[1]);
        pw[2 * n + 1] = T::pack(w[2], w[3]);
      }
      KP_BOUNDARY(ring, 1, 2);
      // O^T += V^T P^T; the LDS accesses of one wave are in order, the fences keep the compiler to it
      store_v();
      asm volatile("" ::: "memory");
      if (more) load_v(row_no);
#pragma unroll
      for (int dt = 0; dt < NT; ++dt) oacc[dt] = T::mfma16(read_v(dt), pw, oacc[dt]);
      asm volatile("" ::: "memory");
      valid = valid_next;
      if (more) KP_BOUNDARY(ring, 2, 0); else KP_BOUNDARY(ring, 2, kp::kNoRegion);
    }
  }
  float l_tot = l_run + __shfl_xor(l_run, 16, 64);
  l_tot += __shfl_xor(l_tot, 32, 64);

  // ---- the four waves' softmaxes become one -----------------------------------------------------------------------
  if (g4 == 0) { join_m[wave][r16] = m_run; join_l[wave][r16] = l_tot; }
  if (tid == 0) again_rows = 0u;
  __syncthreads();
  const float m_all = fmaxf(fmaxf(join_m[0][r16], join_m[1][r16]), fmaxf(join_m[2][r16], join_m[3][r16]));
  const float by = __builtin_amdgcn_exp2f(m_run - m_all);
  float* const sO = reinterpret_cast<float*>(smem) + wave * (kFewRows * D);  // [wave][row][d]: as large as the V tiles
  // 16-byte piece e of row r at piece e ^ r: 16 rows' writes cover all banks
#pragma unroll
  for (int dt = 0; dt < NT; ++dt)
    *reinterpret_cast<f32x4*>(sO + r16 * D + 4u * ((4u * (uint32_t)dt + g4) ^ r16)) = f32x4{oacc[dt][0] * by, oacc[dt][1] * by, oacc[dt][2] * by, oacc[dt][3] * by};
  __syncthreads();
  constexpr uint32_t kPieces = D / 64;  // 16-byte pieces of a thread: 16 threads to a row
  const uint32_t row = tid >> 4, c = tid & 15u;
  float m = join_m[0][row], l = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) m = fmaxf(m, join_m[w][row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) l = __builtin_fmaf(join_l[w][row], __builtin_amdgcn_exp2f(join_m[w][row] - m), l);
  f32x4 o[kPieces];
  float odd = l * 0.f;
#pragma unroll
  for (uint32_t e = 0; e < kPieces; ++e) {
    o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const f32x4 part = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem) + w * (kFewRows * D) + row * D + 4u * ((kPieces * c + e) ^ row));
#pragma unroll
      for (int i = 0; i < 4; ++i) o[e][i] += part[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = __builtin_fmaf(o[e][i], 0.f, odd);
  }
  const uint32_t out_flat = tl.first + row;
  const size_t part_rows = (size_t)g.tiles * g.hkv * kFewRows, part_at = split * part_rows + part_row<kFewRows>(g, tile_id, h, row);
  if (out_flat <= last_row) {
    if (odd != odd) atomicOr(&again_rows, 1u << row);
    if (g.splits > 1u) {
      if (c == 0) *reinterpret_cast<f32x2*>(g.part + 2 * part_at) = f32x2{m, l};
#pragma unroll
      for (uint32_t e = 0; e < kPieces; ++e) *reinterpret_cast<f32x4*>(g.part + 2 * g.splits * part_rows + part_at * D + 4u * (kPieces * c + e)) = o[e];
    } else {
      const RowPlace a = place_of(out_flat, g.group);
      const uint32_t hd = h * g.group + a.in_group;
      const int64_t tok = (int64_t)tl.q0 + a.token;
      uint16_t* to = const_cast<uint16_t*>(g.o.at) + g.o.seq * (int64_t)q_seq + g.o.head * (int64_t)hd + g.o.token * tok + 4u * kPieces * c;
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (uint32_t e = 0; e < kPieces; ++e) reinterpret_cast<u32x2*>(to)[e] = u32x2{T::pack(o[e][0] * inv, o[e][1] * inv), T::pack(o[e][2] * inv, o[e][3] * inv)};
      if (g.lse && c == 0) g.lse[g.lse_seq * (int64_t)q_seq + g.lse_head * (int64_t)hd + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
  }
  __syncthreads();  // (waits for the stores of the rows that are taken again)
  for (uint32_t again = again_rows >> wave; again != 0u; again &= again - 1u) {  // rows with a value that is not finite
    const uint32_t r = wave + (uint32_t)__builtin_ctz(again);
    if ((r - wave) % 4u != 0u) continue;
    const RowPlace a = place_of(tl.first + r, g.group);
    const uint32_t hd = h * g.group + a.in_group;
    const int64_t tok = (int64_t)tl.q0 + a.token;
    const uint16_t* const q = g.q.at + g.q.seq * (int64_t)q_seq + g.q.head * (int64_t)hd + g.q.token * tok;
    Row<T, D, SRC> rr;
    for (int window = 0; window < 2; ++window) {  // the sinks of this split, then its other keys
      const uint32_t from = window ? max(t_begin, sink_steps) : t_begin, to = window ? t_end : min(t_end, sink_steps);
      if (from >= to) continue;
      uint32_t limit;
      const uint32_t start = step_start(from, &limit), end = start + (to - from) * kFewKeys;
      rr.over_keys(q, src, p0 + (int32_t)a.token, g.window, g.sinks, g.scale_log2, start, end < limit ? end : limit);
    }
    if (g.splits > 1u) {
      const size_t to = split * part_rows + part_row<kFewRows>(g, tile_id, h, r);
      rr.store_part(g.part + 2 * g.splits * part_rows + to * D, g.part + 2 * to);
    } else {
      rr.store(const_cast<uint16_t*>(g.o.at) + g.o.seq * (int64_t)q_seq + g.o.head * (int64_t)hd + g.o.token * tok,
               g.lse ? g.lse + g.lse_seq * (int64_t)q_seq + g.lse_head * (int64_t)hd + tok : nullptr);
    }
  }
  if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
}

}  // namespace attn
}  // namespace kp
