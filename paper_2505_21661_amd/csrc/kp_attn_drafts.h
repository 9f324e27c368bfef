// Attention of a tree's drafted tokens over many keys: a tile of 32 rows, the keys dealt out to the waves.
//
// A handful of drafted tokens, times the query heads that share keys, are some tens of rows, too few for the tiles of kp_attn_tile and
// more than the 16 of kp_attn_few, whose way of going about it this is: a workgroup takes a run of a sequence's keys (a split) of one head;
// its 4 waves take blocks of 32 keys in turn, each with softmaxes of its own, and join at the end through LDS; the splits join in
// kp_attn_join.  Products as in kp_attn_tile (S^T = K Q^T, O^T = V^T P^T, a lane has half of a row's scores), but that K goes
// from memory to the operand registers as it lies and V through 8 KiB of LDS per wave; both are asked for a block ahead.
// Blocks begin at multiples of 32 keys, and pages hold at least 16 (kp_attn_tile has the others): either half of a block lies in one
// page, whose place is a scalar, and a load takes no more than the row's number in the half.
// The weights that multiply values are rounded to the type, as the matrix instructions take them (those that are summed up are not): the one
// rounding besides the result's, as in kp_attn_tile.
// Per block a wave has 16 MFMAs (512 cycles) and some 240 other instructions (950).  64 sequences of one tile of 32 rows each, 32/8 heads of 128,
// over 16384 keys of e4m3: with pages of their own 390 us, 2.16 GB, which is memory (5550 GB/s; 16 bits 741, 5800), with pages that they
// share, out of the caches, 207: 1.6 us for a block of each of a SIMD's two waves (16 bits 305, 2.4).  With unequal lengths and more than a tile to a
// sequence it is neither alone: 32 sequences of up to 16 tokens (1.8 tiles each) over up to 16384 keys of e4m3, 749 MB, take 187 us and
// 10 for the join (3800 GB/s), of which the 162528 blocks out of the caches would be some 130, and the longest sequences' last
// workgroups 20 % more than the mean.  3 sequences of up to 7 tokens over 700 keys take 9.8 us, which is latency.
#pragma once
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

constexpr int kDraftKeys = 32, kDraftRows = 32, kDraftPage = 16;

// A record site whose sample is waited for: the loop below has two bodies, between which its registers move.
#define KP_SITE(ring, end_r, start_r) do { if constexpr (INSTR != 0) { kp::site<INSTR>(ring, end_r, start_r); kp::sample_landed(ring); } } while (0)

// Recorded regions, per block of 32 keys: 0 K Q^T, V to LDS and the requests of the next keys and values, 1 mask and softmax,
// 2 V^T P^T.
template <class T, int D, int SRC, int INSTR>
__global__ __launch_bounds__(kThreads, 2) void kp_attn_drafts(Args g) {
  constexpr bool E4M3 = kCodes<SRC>;
  constexpr uint32_t kRow = 2u * D, kBytes = E4M3 ? D : 2 * D;  // of a row in LDS, and in the cache
  constexpr int NS = D / 16, ND = D / 32;       // MFMA steps of K Q^T, tiles of 32 d
  constexpr int KL = E4M3 ? NS / 2 : NS;        // 16-byte loads of a lane of its key
  constexpr uint32_t kVPer = E4M3 ? D / 16 : D / 8, kVRows = 64u / kVPer;  // lanes to a row of V, rows of a load
  constexpr int VL = (int)(kDraftKeys / kVRows);             // loads of a lane per block
  constexpr uint32_t kWaveLds = kDraftKeys * kRow;
  __shared__ __align__(16) unsigned char smem[4u * kWaveLds];
  __shared__ float join_m[4][kDraftRows], join_l[4][kDraftRows];
  __shared__ uint32_t again_rows;
  extern __shared__ __align__(16) unsigned char ring_lds[];

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = wave_uniform(tid >> 6), l32 = lane & 31u, h32 = lane >> 5;
  // (splits of a tile next to one another: they share the tile's queries; heads are dealt to the XCDs as they come)
  uint32_t unit, item;
  unit_of(blockIdx.x, g.hkv, g.tiles * g.splits, &unit, &item);
  const uint32_t split = item % g.splits, tile_id = item / g.splits, h = unit;
  Tile tl;
  const bool there = find_tile<kDraftRows, true>(g, tile_id, &tl);
  const uint32_t recorded = unit * (g.tiles * g.splits) + item;  // number of the workgroup in a trace
  kp::Ring ring{};
  if constexpr (INSTR != 0) ring = ring_of<INSTR>(g, ring_lds, smem, recorded);
  if (!there) {
    if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
    return;
  }
  const Source<D, SRC> src(g, tl.seq, h);
  const uint32_t last_row = tl.rows - 1u, flat = tl.first + l32;
  const RowPlace at = place_of(flat <= last_row ? flat : last_row, g.group);
  // Positions are in the order of the tree: the first is the context's end, and any may be the last.
  const int32_t context = (int32_t)tl.n_k - (int32_t)tl.n_q, p = draft_position(g, tl, at.token);
  const int32_t p_max = (int32_t)wave_uniform((uint32_t)last_of_wave(p));
  const Span span = span_of(context, (int32_t)tl.n_k - 1, g.window, g.sinks);
  // Blocks of the sinks, then those of the window that are not among them.
  const uint32_t sink_blocks = (span.sink_end + 31u) / 32u, window_block = max(span.lo / 32u, sink_blocks), end_block = (span.end + 31u) / 32u;
  const uint32_t all = sink_blocks + (end_block > window_block ? end_block - window_block : 0u);
  const uint32_t t_begin = (uint32_t)((uint64_t)all * split / g.splits), t_end = (uint32_t)((uint64_t)all * (split + 1u) / g.splits);
  auto block_of = [&](uint32_t t) __attribute__((always_inline)) { return t < sink_blocks ? t : t - sink_blocks + window_block; };

  // This lane's query.  The d that an operand of step s stands for: 16-bit keys 16 s + 8 h32 .. + 7; codes, of which a lane reads
  // 16 at a time, 32 (s / 2) + 16 h32 + 8 (s % 2) .. + 7.
  u32x4 qf[NS];
  {
    const uint16_t* q = g.q.at + g.q.head * (int64_t)(h * g.group + at.in_group) + g.q.token * ((int64_t)tl.q0 + at.token);
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(q + (E4M3 ? 32u * (s / 2) + 16u * h32 + 8u * (s % 2) : 16u * s + 8u * h32));
  }

  unsigned char* const sV = smem + kWaveLds * wave;
  u32x4 kr[KL], vr[VL];
  uint32_t k_e = 0, v_e[VL];
  // Where the halves of a block are, as the wave's blocks come: lane l has the pages of the l-th of 64.
  const uint32_t t_first = t_begin + wave;
  int32_t pages[2] = {0, 0};
  auto load_pages = [&](uint32_t t) __attribute__((always_inline)) {
    const uint32_t mine = t + 4u * lane, key = 32u * block_of(mine < t_end ? mine : t_end - 1u), last = span.end - 1u;
    pages[0] = src.table[key >> src.page_log2];
    pages[1] = src.table[(key + 16u < last ? key + 16u : last) >> src.page_log2];
  };
  // The block that is requested: its first key, which of its keys' pages there are, and of either half the cache's row and which of
  // 16 keys are read (what lies between the sinks and the window or behind the last key is not: those of the other half or of the
  // border are taken in its place).
  uint32_t next_key = 0, next_valid = 0, half_row[2], half_first[2], half_last[2];
  auto locate = [&](uint32_t t) __attribute__((always_inline)) {
    const uint32_t l = (t - t_first) / 4u;
    if ((l & 63u) == 0u) load_pages(t);
    const uint32_t key = next_key = 32u * block_of(t), end = t < sink_blocks && span.lo > key + 31u ? span.sink_end : span.end;
    const uint32_t left = end - 1u - key, last = left < 31u ? left : 31u;
    const int32_t ahead = (int32_t)span.lo - (int32_t)key;  // keys in front of the window
    const uint32_t first = t >= sink_blocks && ahead > 0 ? (uint32_t)ahead : 0u;
    next_valid = 0u;
#pragma unroll
    for (uint32_t n = 0; n < 2; ++n) {
      const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages[n], (int)(l & 63u)), in = (key + 16u * n) & ((1u << src.page_log2) - 1u);
      const bool there = page < src.n_pages;
      half_row[n] = there ? ((page * src.hkv + src.head) << src.page_log2) + in : 0u;  // (some rows: their scores are masked)
      next_valid |= there ? 0xFFFFu << (16u * n) : 0u;
      half_first[n] = n == 0 ? (first < 15u ? first : 15u) : (first > 16u ? first - 16u : 0u);
      half_last[n] = n == 0 ? (last < 15u ? last : 15u) : (last > 16u ? last - 16u : 0u);
    }
    if (last < 16u) { half_row[1] = half_row[0]; half_first[1] = half_first[0]; half_last[1] = half_last[0]; }
    if (first >= 16u) { half_row[0] = half_row[1]; half_first[0] = half_first[1]; half_last[0] = half_last[1]; }
  };
  auto within = [&](uint32_t row, uint32_t first, uint32_t last) __attribute__((always_inline)) { return min(max(row, first), last); };
  auto load_k = [&]() __attribute__((always_inline)) {
    const bool upper = l32 >= 16u;
    const uint32_t row = (upper ? half_row[1] : half_row[0]) + within(l32 & 15u, upper ? half_first[1] : half_first[0], upper ? half_last[1] : half_last[0]);
    const uint8_t* const from = src.k + (size_t)row * kBytes + 16u * h32;
#pragma unroll
    for (int i = 0; i < KL; ++i) kr[i] = *reinterpret_cast<const u32x4*>(from + 32 * i);
    if constexpr (E4M3) k_e = src.k_exp[row];
  };
  // (not past the caches, as kp_attn_few has them: a sequence's other tiles, whose workgroups run side by side, find them there)
  auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      constexpr uint32_t kHalf = 16u / kVRows;  // loads of a half
      const int n = i / (int)kHalf;
      const uint32_t row = within(kVRows * ((uint32_t)i % kHalf) + lane / kVPer, half_first[n], half_last[n]);
      vr[i] = *reinterpret_cast<const u32x4*>(src.v + (size_t)half_row[n] * kBytes + (row * kBytes + 16u * (lane % kVPer)));
      if constexpr (E4M3) v_e[i] = (src.v_exp + half_row[n])[row];
    }
  };
  // V tile: chunk c of row r at position c ^ swizzle(r), as in kp_attn_tile
  auto swizzle = [&](uint32_t row) __attribute__((always_inline)) { return D == 128 ? 4u * (row & 3u) : 4u * ((row >> 1) & 1u); };
  auto store_v = [&](int i) __attribute__((always_inline)) {
    const uint32_t row = kVRows * (uint32_t)i + lane / kVPer, c = lane % kVPer, sw = swizzle(row);
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
  };
  uint32_t v_rd[ND];
  {
    const uint32_t i = lane & 15u, grp = lane >> 4, row = 4u * (grp >> 1) + (i >> 2);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
      const uint32_t d = 32u * (uint32_t)dt + 16u * (grp & 1u) + 4u * (i & 3u);
      v_rd[dt] = (uint32_t)(uintptr_t)sV + row * kRow + (((d >> 3) ^ swizzle(row)) << 4) + 8u * ((d >> 2) & 1u);
    }
  }
  auto read_v = [&](int step, int dt) __attribute__((always_inline)) -> u32x4 {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    const uint32_t a = v_rd[dt] + (uint32_t)step * (16u * kRow);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(a + 8u * kRow));
    const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(u32x4, v);
  };

  f32x16 oacc[ND];  // O^T: d = 32 dt + 8 j + 4 h32 + i, column = row l32
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) oacc[dt] = f32x16{0};
  float m_run = kNoKey, l_run = 0.f;

  // One block; MORE: another one follows.
  uint32_t key = 0, valid = 0;
  auto block = [&](uint32_t t, auto more_c) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_c)::value;
    // S^T = K Q^T: keys 8 (v / 4) + 4 h32 + v % 4, column = row l32; values to LDS meanwhile (the LDS accesses of one wave are
    // in order, the fences keep the compiler to it)
    f32x16 sacc = f32x16{0};
    const float scale = E4M3 ? power_of(k_e) : 1.f;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      u32x4 a;
      if constexpr (E4M3) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          a[2 * w] = T::template from_e4m3<false>(kr[s / 2][2 * (s % 2) + w], scale);
          a[2 * w + 1] = T::template from_e4m3<true>(kr[s / 2][2 * (s % 2) + w], scale);
        }
      } else {
        a = kr[s];
      }
      sacc = T::mfma32(a, qf[s], sacc);
#pragma unroll
      for (int i = s * VL / NS; i < (s + 1) * VL / NS; ++i) store_v(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("" ::: "memory");
    const uint32_t start = key, there = valid >> (4u * h32);
    const int32_t end = (int32_t)(start + kDraftKeys);
    bool masked = (end > context) | (valid != ~0u);
    masked = masked | ((g.window != 0u) & (p_max - (int32_t)start >= (int32_t)g.window) & (end > (int32_t)g.sinks));
    if constexpr (MORE) {
      locate(t + 4u);
      load_k();
      load_v();
      key = next_key;
      valid = next_valid;
    }
    KP_SITE(ring, 0, 1);
    if (masked) {
      const RowMask m(p, (uint32_t)context, (int32_t)(start + 4u * h32), g.window, g.sinks);
      const uint32_t drafts = end > context ? Drafts(g, tl, at.token).of(start) >> (4u * h32) : 0u;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int c = 8 * (v >> 2) + (v & 3);
        // (& and |: short cuts become branches)
        const bool seen = (m.sees(c) | ((g.window != 0u) & (c <= m.sink)) | (((drafts >> c) & 1u) != 0u)) & (((there >> c) & 1u) != 0u);
        sacc[v] = seen ? sacc[v] : -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; v += 2) mx = fmaxf(fmaxf(mx, sacc[v]), sacc[v + 1]);
    mx = either_half_max(mx);
    const float mx_s = mx * g.scale_log2;
    if (__builtin_amdgcn_ballot_w64(mx_s > m_run + kSlack<T>) != 0ull) {
      const float m_new = fmaxf(m_run, mx_s - kBelow<T>), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run = sum_unless_far(l_run * alpha, m_new, mx_s);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
      m_run = m_new;
    }
    u32x4 vf[4];  // operands of V^T P^T, four MFMAs ahead
#pragma unroll
    for (int n = 0; n < 4; ++n) vf[n] = read_v(n / ND, n % ND);
    u32x4 pw[2];
    float psum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
      const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v], g.scale_log2, -m_run));
      const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v + 1], g.scale_log2, -m_run));
      psum += w0 + w1;
      pw[v >> 3][(v >> 1) & 3] = T::pack(w0, w1);
    }
    l_run += psum;
    KP_SITE(ring, 1, 2);
    // O^T += V^T P^T: the keys of a step in the order of the scores
#pragma unroll
    for (int n = 0; n < 2 * ND; ++n) {
      oacc[n % ND] = T::mfma32(vf[n & 3], pw[n / ND], oacc[n % ND]);
      if (n + 4 < 2 * ND) vf[n & 3] = read_v((n + 4) / ND, (n + 4) % ND);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (MORE) KP_SITE(ring, 2, 0); else KP_SITE(ring, 2, kp::kNoRegion);
  };
  if (t_first < t_end) {
    locate(t_first);
    load_k();
    load_v();
    key = next_key;
    valid = next_valid;
    KP_SITE(ring, kp::kNoRegion, 0);
    uint32_t t = t_first;
    for (; t + 4u < t_end; t += 4u) block(t, std::true_type{});
    block(t, std::false_type{});
  }

  // ---- the four waves' softmaxes become one -----------------------------------------------------------------------
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (h32 == 0) { join_m[wave][l32] = m_run; join_l[wave][l32] = l_tot; }
  if (tid == 0) again_rows = 0u;
  __syncthreads();
  const float m_all = fmaxf(fmaxf(join_m[0][l32], join_m[1][l32]), fmaxf(join_m[2][l32], join_m[3][l32]));
  const float by = __builtin_amdgcn_exp2f(m_run - m_all);
  constexpr uint32_t kHalfD = D / 2, kPieces = kHalfD / 4, kMine = kPieces / 8;  // 16-byte pieces of half a row, of a thread: 8 to a row
  const uint32_t row = tid >> 3, c = tid & 7u;
  float m = join_m[0][row], l = 0.f;
#pragma unroll
  for (int w = 1; w < 4; ++w) m = fmaxf(m, join_m[w][row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) l = __builtin_fmaf(join_l[w][row], __builtin_amdgcn_exp2f(join_m[w][row] - m), l);
  const uint32_t out_flat = tl.first + row;
  const RowPlace to = place_of(out_flat <= last_row ? out_flat : last_row, g.group);
  const int64_t o_at = g.o.head * (int64_t)(h * g.group + to.in_group) + g.o.token * ((int64_t)tl.q0 + to.token);
  const size_t part_rows = (size_t)g.tiles * g.hkv * kDraftRows, part_at = split * part_rows + part_row<kDraftRows>(g, tile_id, h, row);
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  float odd = l * 0.f;
  float* const sO = reinterpret_cast<float*>(smem);  // [wave][row][half of D]: as large as the V tiles
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
    // 16-byte piece e of row r at piece e ^ r: neighbouring rows' writes cover all banks
#pragma unroll
    for (int dt = half * ND / 2; dt < (half + 1) * ND / 2; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t e = 8u * (uint32_t)(dt - half * ND / 2) + 2u * (uint32_t)j + h32;
        *reinterpret_cast<f32x4*>(sO + (wave * kDraftRows + l32) * kHalfD + 4u * (e ^ (l32 & (kPieces - 1u)))) =
            f32x4{oacc[dt][4 * j] * by, oacc[dt][4 * j + 1] * by, oacc[dt][4 * j + 2] * by, oacc[dt][4 * j + 3] * by};
      }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
      const uint32_t e = kMine * c + i;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (uint32_t w = 0; w < 4; ++w) {
        const f32x4 part = *reinterpret_cast<const f32x4*>(sO + (w * kDraftRows + row) * kHalfD + 4u * (e ^ (row & (kPieces - 1u))));
#pragma unroll
        for (int n = 0; n < 4; ++n) o[n] += part[n];
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) odd = __builtin_fmaf(o[n], 0.f, odd);
      if (out_flat > last_row) continue;
      const uint32_t d = kHalfD * (uint32_t)half + 4u * e;
      if (g.splits > 1u) *reinterpret_cast<f32x4*>(g.part + 2 * g.splits * part_rows + part_at * D + d) = o;
      else *reinterpret_cast<u32x2*>(const_cast<uint16_t*>(g.o.at) + o_at + d) = u32x2{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
    }
  }
  if (out_flat <= last_row) {
    if (odd != odd) atomicOr(&again_rows, 1u << row);
    if (c == 0) {
      if (g.splits > 1u) *reinterpret_cast<f32x2*>(g.part + 2 * part_at) = f32x2{m, l};
      else if (g.lse) g.lse[g.lse_head * (int64_t)(h * g.group + to.in_group) + tl.q0 + to.token] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
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
    for (int window = 0; window < 2; ++window) {  // the sinks' blocks of this split, then the others
      const uint32_t from = window ? max(t_begin, sink_blocks) : t_begin, to = window ? t_end : min(t_end, sink_blocks);
      if (from < to) rr.over_keys(q, src, stands, g.window, g.sinks, g.scale_log2, 32u * block_of(from), min(32u * (block_of(to - 1u) + 1u), span.end), &drafts);
    }
    if (g.splits > 1u) {
      const size_t to = split * part_rows + part_row<kDraftRows>(g, tile_id, h, r);
      rr.store_part(g.part + 2 * g.splits * part_rows + to * D, g.part + 2 * to);
    } else {
      rr.store(const_cast<uint16_t*>(g.o.at) + g.o.head * (int64_t)hd + g.o.token * tok, g.lse ? g.lse + g.lse_head * (int64_t)hd + tok : nullptr);
    }
  }
  if constexpr (INSTR != 0) finish_ring<INSTR>(ring, g, recorded);
}

#undef KP_SITE

}  // namespace attn
}  // namespace kp
