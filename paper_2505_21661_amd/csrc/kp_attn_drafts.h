// Attention of a tree's drafted tokens over many keys: tiles of 16 rows that a wave has together, the keys dealt out to the waves.
//
// A handful of drafted tokens, times the query heads that share keys, are some tens of rows, too few for the tiles of kp_attn_tile and
// more than the 16 of kp_attn_few, whose way of going about it this is: a workgroup takes a run of a sequence's keys (a split) of one head;
// its 4 waves take steps of 32 keys in turn, each with softmaxes of its own, and join at the end through LDS; the splits join in
// kp_attn_join.  A wave uses the keys and values that it has fetched, and widened, for all of its tiles of rows: K as it lies
// in memory, in the operand registers; V through 8 KiB of LDS per wave, which the transposing read needs; both are asked for a
// step ahead.
#pragma once
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

constexpr int kDraftKeys = 32, kDraftTiles = 2, kDraftRows = 16 * kDraftTiles;

// Recorded regions, per step of 32 keys: 0 K Q^T and the request of the next keys, 1 mask and softmax, 2 V to LDS, the
// request of the next values, V^T P^T.
template <class T, int D, int SRC, int INSTR>
__global__ __launch_bounds__(kThreads, 2) void kp_attn_drafts(Args g) {
  constexpr bool E4M3 = kCodes<SRC>;
  constexpr int RT = kDraftTiles, ROWS = kDraftRows;
  constexpr uint32_t kRow = 2u * D;
  constexpr int NS = D / 32;                    // MFMA steps of K Q^T
  constexpr int NT = D / 16;                    // tiles of 16 d
  constexpr int KL = E4M3 ? D / 64 : D / 32;    // 16-byte loads of a lane per 16 keys
  constexpr uint32_t kVPer = E4M3 ? D / 16 : D / 8;          // lanes to a row of V
  constexpr int VL = (int)(kDraftKeys * kVPer / 64u);          // loads of a lane per step
  constexpr uint32_t kWaveLds = kDraftKeys * kRow;
  __shared__ __align__(16) unsigned char smem[4u * kWaveLds];
  __shared__ float join_m[4][ROWS], join_l[4][ROWS];
  __shared__ uint32_t again_rows;
  extern __shared__ __align__(16) unsigned char ring_lds[];

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = wave_uniform(tid >> 6), r16 = lane & 15u, g4 = lane >> 4;
  // (splits of a tile next to one another: they share the tile's queries; heads are dealt to the XCDs as they come)
  uint32_t unit, item;
  unit_of(blockIdx.x, g.hkv, g.tiles * g.splits, &unit, &item);
  const uint32_t split = item % g.splits, tile_id = item / g.splits, h = unit;
  Tile tl;
  const bool there = find_tile<ROWS, true>(g, tile_id, &tl);
  const uint32_t recorded = unit * (g.tiles * g.splits) + item;  // number of the workgroup in a trace
  kp::Ring ring{};
  if constexpr (INSTR != 0) ring = ring_of<INSTR>(g, ring_lds, smem, recorded);
  if (!there) {
    if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
    return;
  }
  const Source<D, SRC> src(g, tl.seq, h);
  const uint32_t last_row = tl.rows - 1u;
  const uint32_t tiles = wave_uniform((min(tl.rows - tl.first, (uint32_t)ROWS) + 15u) / 16u);  // of 16 rows that there are
  // Positions are in the order of the tree: the first is the context's end, and any may be the last.
  const int32_t context = (int32_t)tl.n_k - (int32_t)tl.n_q;
  RowPlace at[RT];
  int32_t p[RT], p_max = context;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t flat = tl.first + 16u * (uint32_t)rt + r16;
    at[rt] = place_of(flat <= last_row ? flat : last_row, g.group);
    p[rt] = draft_position(g, tl, at[rt].token);
    p_max = max(p_max, p[rt]);
  }
  p_max = (int32_t)wave_uniform((uint32_t)last_of_wave(p_max));
  const Span span = span_of(context, (int32_t)tl.n_k - 1, g.window, g.sinks);
  const uint32_t sink_steps = (span.sink_end + kDraftKeys - 1u) / kDraftKeys;
  const uint32_t all = sink_steps + (span.end > span.lo ? (span.end - span.lo + kDraftKeys - 1u) / kDraftKeys : 0u);
  const uint32_t t_begin = (uint32_t)((uint64_t)all * split / g.splits), t_end = (uint32_t)((uint64_t)all * (split + 1u) / g.splits);
  auto step_start = [&](uint32_t t, uint32_t* limit) __attribute__((always_inline)) {
    *limit = t < sink_steps ? span.sink_end : span.end;
    return t < sink_steps ? t * kDraftKeys : span.lo + (t - sink_steps) * kDraftKeys;
  };

  // Queries of row r16 of each tile.  The d that a lane's operand of step s stands for: 16-bit keys 32 s + 8 g4 .. + 7; codes, of
  // which a lane reads 16 at a time, 64 (s / 2) + 16 g4 + 8 (s % 2) .. + 7.
  u32x4 qf[RT][NS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t head = h * g.group + at[rt].in_group;
    const int64_t token = (int64_t)tl.q0 + at[rt].token;
    const uint16_t* q = g.q.at + g.q.head * (int64_t)head + g.q.token * token;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[rt][s] = *reinterpret_cast<const u32x4*>(q + (E4M3 ? 64u * (s / 2) + 16u * g4 + 8u * (s % 2) : 32u * s + 8u * g4));
  }

  unsigned char* const sV = smem + kWaveLds * wave;
  u32x4 kr[2][KL], vr[VL];
  uint32_t k_e[2], v_e[VL];
  int32_t page_id = 0;        // of key number lane % 32 of the next step
  uint64_t valid = 0, valid_next = 0;
  auto load_page_ids = [&](uint32_t t) __attribute__((always_inline)) {
    if (t < t_end) {
      uint32_t limit;
      const uint32_t start = step_start(t, &limit), last = limit - 1u - start, l = lane & 31u;
      page_id = src.table[(start + (l < last ? l : last)) >> src.page_log2];
    }
  };
  // Where step t's keys are; their page ids have been asked for before.
  uint32_t row_no = 0;
  auto locate = [&](uint32_t t) __attribute__((always_inline)) {
    uint32_t limit;
    const uint32_t start = step_start(t, &limit), last = limit - 1u - start, l = lane & 31u;
    row_no = src.row_of_page(page_id, start + (l < last ? l : last));
    valid_next = __builtin_amdgcn_ballot_w64(row_no != ~0u);
    if (row_no == ~0u) row_no = 0u;  // (some row of the cache: its scores are masked)
    load_page_ids(t + 4u);
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
  // Values go past the caches, whole lines at a time (see kp_attn_few), but those of a sequence with more than one tile, whose workgroups
  // run side by side and find them there.
  const bool shared = tl.rows > (uint32_t)ROWS;
  auto load_v = [&](uint32_t rows) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const uint32_t r = __shfl(rows, (int)((64u / kVPer) * i + lane / kVPer), 64);
      const u32x4* const from = reinterpret_cast<const u32x4*>(src.v_at(r) + 16u * (lane % kVPer));
      if (shared) vr[i] = *from; else vr[i] = __builtin_nontemporal_load(from);
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

  f32x4 oacc[RT][NT];  // O^T: d = 16 dt + 4 g4 + i, column = row r16
  float m_run[RT], l_run[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m_run[rt] = kNoKey;
    l_run[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < NT; ++dt) oacc[rt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

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
      const int32_t end = (int32_t)(start + kDraftKeys);
      // S^T = K Q^T: keys 16 n + 4 g4 + i, column = row r16
      f32x4 sacc[RT][2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) sacc[rt][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float scale = E4M3 ? power_of(k_e[n]) : 1.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          u32x4 a;
          if constexpr (E4M3) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              a[2 * w] = T::template from_e4m3<false>(kr[n][s / 2][2 * (s % 2) + w], scale);
              a[2 * w + 1] = T::template from_e4m3<true>(kr[n][s / 2][2 * (s % 2) + w], scale);
            }
          } else {
            a = kr[n][s];
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            if (rt == 0 || (uint32_t)rt < tiles) sacc[rt][n] = T::mfma16(a, qf[rt][s], sacc[rt][n]);
        }
      }
      if (more) {
        locate(t + 4u);
        load_k();
      }
      KP_BOUNDARY(ring, 0, 1);
      bool masked = end > (int32_t)limit || end > context;
      if (g.window != 0u) masked = masked || (p_max - (int32_t)start >= (int32_t)g.window && end > (int32_t)g.sinks);
      masked = masked || valid != ~0ull;
      u32x4 pw[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (rt != 0 && (uint32_t)rt >= tiles) continue;
        if (masked) {
          const RowMask m(p[rt], context < (int32_t)limit ? (uint32_t)context : limit, (int32_t)(start + 4u * g4), g.window, g.sinks);
          const uint32_t drafts = end > context ? Drafts(g, tl, at[rt].token).of(start) >> (4u * g4) : 0u;
          const uint32_t there = (uint32_t)valid >> (4u * g4);  // keys whose page exists
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int c = 16 * n + i;
              // (& and |: short cuts become branches)
              const bool seen = (m.sees(c) | ((g.window != 0u) & (c <= m.sink)) | (((drafts >> c) & 1u) != 0u)) & (((there >> c) & 1u) != 0u);
              sacc[rt][n][i] = seen ? sacc[rt][n][i] : -INFINITY;
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(sacc[rt][0][0], sacc[rt][0][1]), fmaxf(sacc[rt][0][2], sacc[rt][0][3])),
                         fmaxf(fmaxf(sacc[rt][1][0], sacc[rt][1][1]), fmaxf(sacc[rt][1][2], sacc[rt][1][3])));
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = either_half_max(mx);
        const float mx_s = mx * g.scale_log2;
        if (__builtin_amdgcn_ballot_w64(mx_s > m_run[rt] + kSlack<T>) != 0ull) {
          const float m_new = fmaxf(m_run[rt], mx_s - kBelow<T>), alpha = __builtin_amdgcn_exp2f(m_run[rt] - m_new);
          l_run[rt] = sum_unless_far(l_run[rt] * alpha, m_new, mx_s);
#pragma unroll
          for (int dt = 0; dt < NT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) oacc[rt][dt][i] *= alpha;
          m_run[rt] = m_new;
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[rt][n][i], g.scale_log2, -m_run[rt]));
            l_run[rt] += w[i];
          }
          pw[rt][2 * n] = T::pack(w[0], w[1]);
          pw[rt][2 * n + 1] = T::pack(w[2], w[3]);
        }
      }
      KP_BOUNDARY(ring, 1, 2);
      // O^T += V^T P^T; the LDS accesses of one wave are in order, the fences keep the compiler to it
      store_v();
      asm volatile("" ::: "memory");
      if (more) load_v(row_no);
#pragma unroll
      for (int dt = 0; dt < NT; ++dt) {
        const u32x4 v = read_v(dt);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          if (rt == 0 || (uint32_t)rt < tiles) oacc[rt][dt] = T::mfma16(v, pw[rt], oacc[rt][dt]);
      }
      asm volatile("" ::: "memory");
      valid = valid_next;
      if (more) KP_BOUNDARY(ring, 2, 0); else KP_BOUNDARY(ring, 2, kp::kNoRegion);
    }
  }

  // ---- the four waves' softmaxes become one -----------------------------------------------------------------------
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float l_tot = l_run[rt] + __shfl_xor(l_run[rt], 16, 64);
    l_tot += __shfl_xor(l_tot, 32, 64);
    if (g4 == 0) { join_m[wave][16 * rt + r16] = m_run[rt]; join_l[wave][16 * rt + r16] = l_tot; }
  }
  if (tid == 0) again_rows = 0u;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();  // (of a second tile: the first one's values have been read)
    if (rt != 0 && (uint32_t)rt >= tiles) continue;
    const uint32_t jr = 16u * (uint32_t)rt + r16;
    const float m_all = fmaxf(fmaxf(join_m[0][jr], join_m[1][jr]), fmaxf(join_m[2][jr], join_m[3][jr]));
    const float by = __builtin_amdgcn_exp2f(m_run[rt] - m_all);
    float* const sO = reinterpret_cast<float*>(smem) + wave * (16 * D);  // [wave][row][d]: as large as the V tiles
    // 16-byte piece e of row r at piece e ^ r: 16 rows' writes cover all banks
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
      *reinterpret_cast<f32x4*>(sO + r16 * D + 4u * ((4u * (uint32_t)dt + g4) ^ r16)) = f32x4{oacc[rt][dt][0] * by, oacc[rt][dt][1] * by, oacc[rt][dt][2] * by, oacc[rt][dt][3] * by};
    __syncthreads();
    constexpr uint32_t kPieces = D / 64;  // 16-byte pieces of a thread: 16 threads to a row
    const uint32_t in_tile = tid >> 4, row = 16u * (uint32_t)rt + in_tile, c = tid & 15u;
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
        const f32x4 part = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem) + w * (16 * D) + in_tile * D + 4u * ((kPieces * c + e) ^ in_tile));
#pragma unroll
        for (int i = 0; i < 4; ++i) o[e][i] += part[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) odd = __builtin_fmaf(o[e][i], 0.f, odd);
    }
    const uint32_t out_flat = tl.first + row;
    const size_t part_rows = (size_t)g.tiles * g.hkv * ROWS, part_at = split * part_rows + part_row<ROWS>(g, tile_id, h, row);
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
        uint16_t* to = const_cast<uint16_t*>(g.o.at) + g.o.head * (int64_t)hd + g.o.token * tok + 4u * kPieces * c;
        const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
        for (uint32_t e = 0; e < kPieces; ++e) reinterpret_cast<u32x2*>(to)[e] = u32x2{T::pack(o[e][0] * inv, o[e][1] * inv), T::pack(o[e][2] * inv, o[e][3] * inv)};
        if (g.lse && c == 0) g.lse[g.lse_head * (int64_t)hd + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
  }
  __syncthreads();  // (waits for the stores of the rows that are taken again)
  for (uint32_t again = again_rows >> wave; again != 0u; again &= again - 1u) {  // rows with a value that is not finite
    const uint32_t r = wave + (uint32_t)__builtin_ctz(again);
    if ((r - wave) % 4u != 0u) continue;
    const RowPlace a = place_of(tl.first + r, g.group);
    const uint32_t hd = h * g.group + a.in_group;
    const int64_t tok = (int64_t)tl.q0 + a.token;
    const uint16_t* const q = g.q.at + g.q.head * (int64_t)hd + g.q.token * tok;
    const int32_t stands = draft_position(g, tl, a.token);
    const Drafts drafts(g, tl, a.token);
    Row<T, D, SRC> rr;
    for (int window = 0; window < 2; ++window) {  // the sinks of this split, then its other keys
      const uint32_t from = window ? max(t_begin, sink_steps) : t_begin, to = window ? t_end : min(t_end, sink_steps);
      if (from >= to) continue;
      uint32_t limit;
      const uint32_t start = step_start(from, &limit), end = start + (to - from) * kDraftKeys;
      rr.over_keys(q, src, stands, g.window, g.sinks, g.scale_log2, start, end < limit ? end : limit, &drafts);
    }
    if (g.splits > 1u) {
      const size_t part_rows = (size_t)g.tiles * g.hkv * ROWS, to = split * part_rows + part_row<ROWS>(g, tile_id, h, r);
      rr.store_part(g.part + 2 * g.splits * part_rows + to * D, g.part + 2 * to);
    } else {
      rr.store(const_cast<uint16_t*>(g.o.at) + g.o.head * (int64_t)hd + g.o.token * tok,
               g.lse ? g.lse + g.lse_head * (int64_t)hd + tok : nullptr);
    }
  }
  if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
}

}  // namespace attn
}  // namespace kp
