// Gradients of attention with a sliding window and sinks (kp_attn_window_grad).
//
// With P_ij = exp2(scale log2(e) q_i.k_j - lse_i log2(e)) and delta_i = d_o_i . o_i (= sum_j P_ij d_o_i . v_j):
//   dS_ij = P_ij (d_o_i . v_j - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij d_o_i.
// Two kernels, both of which form S and d_o v^T for themselves: one goes over the keys of a tile of query rows (dq), the
// other over the query rows that see a tile of keys (dk, dv).  That is seven products instead of the five that one kernel
// would need, which would have to add up dq with atomics, in an order that changes from run to run.
#include "kp_attn_host.h"
#include "kp_grad_keys.h"

using namespace kp::attn;

namespace {
constexpr int32_t kFewSeen = 16;

// 32/8 x 8192 x 128, window 1024: 198 us, 980 TFLOP/s of three products, the matrix pipes busy 57 % of the time at 1.9 GHz;
// the vector work of dS is the rest.
// dq of a tile of 128 rows, and delta and lse for the kernel after it.  Tiles, rows and keys as in kp_attn_tile; K and V
// tiles in two buffers each.  Per 32 keys: S^T = K Q^T, dP^T = V dO^T, dS^T from them, dq^T += K^T dS^T.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void kp_grad_query(GradArgs g) {
  constexpr uint32_t kTile = 64u * 2u * D;
  constexpr int NS = D / 16, ND = D / 32;
  constexpr bool kScaled = std::is_same<T, Fp16>::value;
  extern __shared__ __align__(16) unsigned char smem[];  // two buffers of [K tile][V tile]
  const uint32_t lane = threadIdx.x & 63u, wave = kp::wave_uniform(threadIdx.x >> 6), h32 = lane >> 5, l32 = lane & 31u;
  uint32_t unit, item;
  unit_of(blockIdx.x, g.seqs * g.hkv, g.row_tiles, &unit, &item);
  const uint32_t seq = unit / g.hkv, hk = unit - seq * g.hkv, first = (g.row_tiles - 1u - item) * kTileRows;
  const uint32_t last_row = g.n_q * g.group - 1u, wave_first = first + 32u * wave, flat = wave_first + l32;
  const bool mine = flat <= last_row;
  const int32_t off = (int32_t)g.n_k - (int32_t)g.n_q;
  auto position = [&](uint32_t f) __attribute__((always_inline)) { return off + (int32_t)place_of(f < last_row ? f : last_row, g.group).token; };
  const RowPlace at = place_of(mine ? flat : last_row, g.group);
  const uint32_t head = hk * g.group + at.in_group;
  const int32_t p = off + (int32_t)at.token, p_min = (int32_t)kp::wave_uniform((uint32_t)position(wave_first)), p_max = (int32_t)kp::wave_uniform((uint32_t)position(wave_first + 31u));
  const KeyTiles kt(span_of(position(first), position(first + kTileRows - 1u), g.window, g.sinks));
  const uint32_t tiles = kt.all;

  u32x4 qf[NS], dof[NS];
  float delta = 0.f, most = 0.f;
  {
    const uint16_t *q = row_at(g.q, seq, head, at.token), *d_o = row_at(g.d_o, seq, head, at.token), *o = row_at(g.o, seq, head, at.token);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = *reinterpret_cast<const u32x4*>(q + 16 * s + 8 * h32);
      dof[s] = *reinterpret_cast<const u32x4*>(d_o + 16 * s + 8 * h32);
      const u32x4 of = *reinterpret_cast<const u32x4*>(o + 16 * s + 8 * h32);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float a = T::to_float(dof[s][w] & 0xFFFFu), b = T::to_float(dof[s][w] >> 16);
        delta = __builtin_fmaf(a, T::to_float(of[w] & 0xFFFFu), __builtin_fmaf(b, T::to_float(of[w] >> 16), delta));
        if constexpr (kScaled) {
          most = fmaxf(most, __builtin_fabsf(a) < INFINITY ? __builtin_fabsf(a) : 0.f);
          most = fmaxf(most, __builtin_fabsf(b) < INFINITY ? __builtin_fabsf(b) : 0.f);
        }
      }
    }
  }
  delta += __shfl_xor(delta, 32, 64);
  const size_t row_no = ((size_t)seq * g.hkv * g.group + head) * g.n_q + at.token;
  // (a row that sees nothing: any finite number, so that its scores of -inf give 0)
  const float lse = g.lse[row_no], neg = lse == -INFINITY ? 0.f : kShiftP<T> - lse * kLog2e;
  if (mine && h32 == 0) g.neg[row_no] = neg;
  float row_scale = 1.f;  // dS is rounded times this
  if constexpr (kScaled) {
    most = either_half_max(most);
    row_scale = __builtin_ldexpf(1.0f, kShiftS) / power_of_two_in(most);
    if (mine && h32 == 0) g.most[row_no] = most;
  }
  const float neg_p = kScaled ? neg - kShiftP<T> : neg;

  TileCursor<D> rd((uint32_t)(uintptr_t)smem, 2u * kTile);
  TileLoader<D, 4> lk(g.k.token), lv(g.v.token);
  const uint32_t lds0 = kp::wave_uniform((uint32_t)(uintptr_t)smem + 1024u * wave);
  const uint16_t *k_head = row_at(g.k, seq, hk, 0), *v_head = row_at(g.v, seq, hk, 0);
  uint32_t loaded_last = ~0u, into = 0u;  // `into`: LDS offset of the buffer that the next tiles go to
  uint32_t next_start = 0, next_limit = 0, next_sinks = g.sinks;  // of the tile that is requested
  auto request_at = [&](uint32_t start, uint32_t limit) __attribute__((always_inline)) {
    const uint32_t left = limit - 1u - start, last = left < 63u ? left : 63u;
    if (last != loaded_last) { loaded_last = last; lk.upto(last); lv.upto(last); }
    lk.load(k_head + g.k.token * (int64_t)start, lds0 + into);
    lv.load(v_head + g.v.token * (int64_t)start, lds0 + into + kTile);
    into ^= 2u * kTile;
  };
  auto request = [&](uint32_t t) __attribute__((always_inline)) {
    next_start = kt.start(t, &next_limit);
    request_at(next_start, next_limit);
  };
  auto request_first = [&]() __attribute__((always_inline)) {
    next_start = kt.start_of(0u, &next_limit, &next_sinks);
    if (!kt.is_mixed(0u)) { request_at(next_start, next_limit); return; }
    const uint32_t left = next_limit - 1u - next_start;
    lk.load_two(k_head, g.k.token, kt.mixed, next_start, left, lds0 + into);
    lv.load_two(v_head, g.v.token, kt.mixed, next_start, left, lds0 + into + kTile);
    into ^= 2u * kTile;
  };

  f32x16 acc[ND];  // dq^T: rows d, column = row l32
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) acc[dt] = f32x16{0};
  // The operands of the three products come out of LDS LA MFMAs ahead, in one set of registers.
  constexpr int LA = 4;
  u32x4 ra[LA];
  // operand n of the half tile tk: K rows, V rows, K^T; from 3 NS on the half after it
  auto fetch = [&](int n, int tk) __attribute__((always_inline)) {
    if (n >= 3 * NS) { n -= 3 * NS; tk ^= 1; }
    if (n < NS) return rd.rows(n, 32u * (uint32_t)tk);
    if (n < 2 * NS) return rd.rows(n - NS, 64u + 32u * (uint32_t)tk);
    return rd.cols((n - 2 * NS) % ND, 32u * (uint32_t)tk + 16u * (uint32_t)((n - 2 * NS) / ND));
  };
  float lacks = 0.f;
  // Over all keys; CHECK: with the sum of dS.
  auto over_keys = [&](auto check_c) __attribute__((always_inline)) {
    constexpr bool CHECK = decltype(check_c)::value;
    request_first();
    __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own count of outstanding loads)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int n = 0; n < LA; ++n) ra[n] = fetch(n, 0);
    for (uint32_t t = 0; t < tiles; ++t) {
      const uint32_t start = next_start, limit = next_limit, sinks = next_sinks;
      next_sinks = g.sinks;
      if (t + 1u < tiles) request(t + 1u);
      const int32_t end = (int32_t)(start + 64u);
      bool masked = (end > (int32_t)limit) | (end - 1 > p_min);
      masked = masked | ((g.window != 0u) & (p_max - (int32_t)start >= (int32_t)g.window) & (end > (int32_t)sinks));
#pragma unroll
      for (int tk = 0; tk < 2; ++tk) {
        f32x16 sacc = f32x16{0}, dp = f32x16{0};
        __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (int n = 0; n < 2 * NS; ++n) {
          if (n < NS) sacc = T::mfma32(ra[n % LA], qf[n], sacc);
          else dp = T::mfma32(ra[n % LA], dof[n - NS], dp);
          ra[n % LA] = fetch(n + LA, tk);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (masked) {
          RowMask m(p, limit, (int32_t)(start + 4u * h32), g.window, sinks);
          if ((g.window != 0u) & (start < sinks)) {
            m.apart();
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[v] = m.sees_mixed(32 * tk + 8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
          } else {
            m.apart();
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[v] = m.sees(32 * tk + 8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
          }
        }
        u32x4 ds[2];
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v + e], g.scale_log2, neg_p));
            x[e] = w * (dp[v + e] - delta);
            if constexpr (CHECK) lacks += x[e];
            if constexpr (kScaled) x[e] *= row_scale;
          }
          ds[v >> 3][(v >> 1) & 3] = T::pack(x[0], x[1]);
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int n = 2 * NS; n < 3 * NS; ++n) {
          const int s = n - 2 * NS;
          // behind the tile's last operand read: every wave has read these tiles, and the next ones have landed
          if (tk == 1 && s == NS - LA) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            rd.to_other();
          }
          acc[s % ND] = T::mfma32(ra[n % LA], ds[s / ND], acc[s % ND]);
          ra[n % LA] = fetch(n + LA, tk);  // (behind the last tile: not used)
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
      }
    }
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  // delta comes from an o that was rounded; the exact one makes sum_j dS_ij = 0, so the sum of a row's dS is what it lacks.
  // That enters dq as half a step of the type over the square root of the number of keys that count: with 2, 4, 8, 16, 32 and
  // 64 keys dq's error is 1.54, 1.25, 1.13, 1.07, 1.05 and 1.04 times what it is without (bf16, D = 64).  Rows that see up to
  // kFewSeen keys, whatever their tile and group, have it put right: the tiles that hold such rows are gone over twice, first for
  // the sum, which takes 3 to 9 % of a training pass where the window is that short and each head has keys of its own.
  const bool few = (g.window != 0u) & (g.window + g.sinks <= (uint32_t)kFewSeen);
  if ((few | (position(first) < kFewSeen)) & (tiles != 0u)) {
    over_keys(yes);
    lacks += __shfl_xor(lacks, 32, 64);
    // (a value that the row does not see may be in it)
    delta += ((few | (p < kFewSeen)) & (__builtin_fabsf(lacks) < INFINITY)) ? lacks : 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) acc[dt] = f32x16{0};
  }
  if (tiles != 0u) over_keys(no);
  if (mine && h32 == 0) g.delta[row_no] = delta;
  uint64_t again = __builtin_amdgcn_ballot_w64(odd_of<ND>(acc) != 0.f && mine);
  again = (again | again >> 32) & 0xFFFFFFFFull;
  const uint64_t rows_out = __builtin_amdgcn_ballot_w64(mine) & 0xFFFFFFFFull;
  __syncthreads();  // (the tiles' room is used below)
  uint16_t* const dq = const_cast<uint16_t*>(g.dq.at);
  store_rows<T, D>(acc, kScaled ? g.scale / row_scale : g.scale, smem + 64u * D * wave, dq, g.dq.seq * (int64_t)seq + g.dq.head * (int64_t)head + g.dq.token * (int64_t)at.token, rows_out);
  if (again != 0ull) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // their first results have left
    for (; again != 0ull; again &= again - 1ull) {
      const int r = __builtin_ctzll(again);
      const RowPlace a = place_of(wave_first + (uint32_t)r, g.group);
      query_row<T, D>(g, seq, hk * g.group + a.in_group, a.token, __shfl(neg, r, 64), __shfl(delta, r, 64), const_cast<uint16_t*>(row_at(g.dq, seq, hk * g.group + a.in_group, a.token)));
    }
  }
}

// Tiles of a call, its workers and its workspace.
struct GradPlan {
  bool too_many;  // the steps of a line are counted in 32 bits
  long long lines, units, row_tiles, key_tiles, sink_tiles, workers, whole, split;  // split: key tiles that kp_grad_join looks at
  size_t rows, most_at, part_at, bytes;  // rows: query rows; byte offsets into the workspace
};
GradPlan plan_grad(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  GradPlan p{};
  window = window_of(window);
  sinks = sinks_of(sinks);
  const long long group = Hq / Hkv, head_steps = (Sq + 63) / 64;
  p.units = (long long)B * Hkv;
  p.row_tiles = (group * Sq + kTileRows - 1) / kTileRows;
  p.key_tiles = (Sk + kGradKeys - 1) / kGradKeys;
  // steps of 64 tokens of an ordinary key tile (an estimate)
  long long steps = window > 0 ? ((long long)window + kGradKeys + 62) / 64 + 1 : head_steps;
  steps = (steps < head_steps ? steps : head_steps) * group;
  const long long saves = D == 64 ? 14 : 7;  // steps that a worker has to save for its tile to be split
  // tiles with sinks: where their steps are not many more, they are as the others
  p.sink_tiles = window > 0 && head_steps * group - steps >= saves ? ((long long)sinks + kGradKeys - 1) / kGradKeys : 0;
  if (p.sink_tiles > p.key_tiles) p.sink_tiles = p.key_tiles;
  const long long lines = p.lines = p.units % 8 == 0 ? 8 : 1, plain = p.units / lines * (p.key_tiles - p.sink_tiles);
  const long long sink_steps = head_steps * group * (p.units / lines) * p.sink_tiles, all = lines * (steps * plain + sink_steps);
  p.too_many = all / lines >= (1ll << 30);
  // One worker per CU, or two (D = 64).  Where there are fewer tiles than that, a worker per tile saves the second tile of a
  // worker's piece and the sums of parts (some 14 us, as much as 14 steps of D = 64 or 7 of 128); splitting them saves steps.
  // (D = 64: 2 x 12/4 x 1153, window 250, saves 18 of them and takes 37 us split, 44 whole;
  // 8/8 x 4096, window 1024, saves 10: 70 split, 56 whole.)
  const long long chip = D == 64 ? kMostWorkers : kChip;
  p.workers = chip;
  // The tiles with sinks go to more workers, as many as they keep busy for as long (6/3 x 1489 x 128, window 20, 148 sinks:
  // 63 us without, 40 with; 5 x 6/2 x 637 x 64, window 49, 4 sinks: 46 and 36).
  if (plain > 0 && lines * plain < chip && steps - all / chip < saves) {
    const long long more = plain + sink_steps / steps;
    p.workers = lines * (more < chip / lines ? more : chip / lines);
  }
  if (all < p.workers) p.workers = all / lines * lines;
  if (p.workers < lines) p.workers = lines;
  // Whole rounds, and one that is not full if what it lacks can be made up for by the tiles with sinks, or is little.
  const long long places = p.workers / lines, lacks = (places - plain % places) % places;
  p.whole = lacks * steps <= sink_steps + places * steps / 16 ? plain : plain / places * places;
  p.split = p.units * p.sink_tiles + lines * (plain - p.whole);
  p.rows = (size_t)B * (size_t)Hq * (size_t)Sq;
  const auto up = [](size_t n) { return (n + 15) & ~(size_t)15; };
  p.most_at = up(8 * p.rows);
  p.part_at = up(p.most_at + 4 * p.rows);
  p.bytes = p.part_at + (size_t)p.workers * (2u * 2u * kGradKeys * 4u) * (size_t)D;
  return p;
}

template <class T, int D>
kp_status launch_grad(GradArgs& g, const GradPlan& p, hipStream_t st) {
  constexpr uint32_t kTile = 64u * 2u * D;
  hipLaunchKernelGGL((kp_grad_query<T, D>), dim3((uint32_t)(p.units * p.row_tiles)), dim3(kThreads), 4u * kTile, st, g);
  KP_HIP_TRY(hipGetLastError());
  KeyPlan plan{};
  plan.n_q = g.n_q; plan.n_k = g.n_k; plan.window = g.window; plan.sinks = g.sinks; plan.group = g.group;
  plan.lines = (uint32_t)p.lines; plan.units = (uint32_t)(p.units / p.lines); plan.workers = (uint32_t)(p.workers / p.lines);
  plan.sink_tiles = (uint32_t)p.sink_tiles; plan.per_unit = (uint32_t)(p.key_tiles - p.sink_tiles);
  plan.whole = (uint32_t)p.whole; plan.rest = (uint32_t)(p.split / p.lines);
  plan.deal();
  if constexpr (D == 64) {
    hipLaunchKernelGGL((kp_grad_keys<T, D>), dim3((uint32_t)p.workers), dim3(kThreads), 4u * kTile + 2u * kStatBytes, st, g, plan);
  } else {
    static thread_local int attr_dev = -1;  // the attribute is kept per device
    int dev = 0;
    KP_HIP_TRY(hipGetDevice(&dev));
    if (attr_dev != dev) {
      KP_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kp_grad_keys_pairs<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)pairs_lds_bytes<D>()));
      attr_dev = dev;
    }
    hipLaunchKernelGGL((kp_grad_keys_pairs<T, D>), dim3((uint32_t)p.workers), dim3(kPairThreads), pairs_lds_bytes<D>(), st, g, plan);
  }
  KP_HIP_TRY(hipGetLastError());
  if (p.split > 0) {
    hipLaunchKernelGGL((kp_grad_join<T, D>), dim3((uint32_t)(p.split * (kGradKeys / kJoinRows<D>)), 2), dim3(kThreads), 0, st, g, plan);
    KP_HIP_TRY(hipGetLastError());
  }
  return KP_OK;
}

bool sizes_ok(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  return B > 0 && Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && Sq > 0 && Sk > 0 && (D == 64 || D == 128) && window >= 0 && sinks >= 0 && Sq < kMostTokens &&
         Sk < kMostTokens && (long long)B * Hq < (1ll << 31);
}

}  // namespace

extern "C" size_t kp_attn_window_grad_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  if (!sizes_ok(B, Hq, Hkv, Sq, Sk, D, window, sinks)) return 0;
  return plan_grad(B, Hq, Hkv, Sq, Sk, D, window, sinks).bytes;
}

extern "C" kp_status kp_attn_window_grad(const kp_heads* q, const kp_heads* k, const kp_heads* v, const kp_heads* o,
                                         const float* lse, const kp_heads* d_o, const kp_heads* dq, const kp_heads* dk,
                                         const kp_heads* dv, int B, int Hq, int Hkv, int Sq, int Sk, int D, int type,
                                         int window, int sinks, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, type, window, sinks, scale)) return s;
  if (B < 1 || Sq < 1 || Sk < 1) return kp::fail(KP_ERR_INVALID_ARG, "B, Sq and Sk must be positive");
  if (!sizes_ok(B, Hq, Hkv, Sq, Sk, D, window, sinks)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^30 or more tokens, or 2^31 heads");
  const struct { const char* name; const kp_heads* t; bool query, written; } all[] = {
      {"q", q, true, false}, {"k", k, false, false}, {"v", v, false, false}, {"o", o, true, false}, {"d_o", d_o, true, false},
      {"dq", dq, true, true}, {"dk", dk, false, true}, {"dv", dv, false, true}};
  for (const auto& a : all)
    if (kp_status s = check_heads(a.name, a.t, B, a.query ? Hq : Hkv, a.query ? Sq : Sk, D, a.written)) return s;
  if (!lse || ((uintptr_t)lse & 3u)) return kp::fail(KP_ERR_INVALID_ARG, "lse must be device memory, 4-byte aligned");
  const GradPlan p = plan_grad(B, Hq, Hkv, Sq, Sk, D, window, sinks);
  if (p.too_many || p.units * p.row_tiles >= kMostGroups || p.split * 32 >= kMostGroups) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^23 or more workgroups, or 2^30 or more steps");
  if (kp_status s = check_workspace(workspace, workspace_bytes, p.bytes)) return s;
  GradArgs g{};
  g.q = heads_of(q, B, Hq, Sq); g.o = heads_of(o, B, Hq, Sq); g.d_o = heads_of(d_o, B, Hq, Sq); g.dq = heads_of(dq, B, Hq, Sq);
  g.k = heads_of(k, B, Hkv, Sk); g.v = heads_of(v, B, Hkv, Sk); g.dk = heads_of(dk, B, Hkv, Sk); g.dv = heads_of(dv, B, Hkv, Sk);
  g.lse = lse;
  char* const ws = static_cast<char*>(workspace);
  g.neg = reinterpret_cast<float*>(ws); g.delta = g.neg + p.rows;
  g.most = reinterpret_cast<float*>(ws + p.most_at); g.part = reinterpret_cast<float*>(ws + p.part_at);
  g.row_tiles = (uint32_t)p.row_tiles;
  g.seqs = (uint32_t)B; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)Sq; g.n_k = (uint32_t)Sk;
  g.window = (uint32_t)window_of(window); g.sinks = (uint32_t)sinks_of(sinks); g.scale = scale; g.scale_log2 = scale * kLog2e;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (type == KP_FP16) return D == 64 ? launch_grad<Fp16, 64>(g, p, st) : launch_grad<Fp16, 128>(g, p, st);
  return D == 64 ? launch_grad<Bf16, 64>(g, p, st) : launch_grad<Bf16, 128>(g, p, st);
}
