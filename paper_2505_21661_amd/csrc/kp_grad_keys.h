// Gradients of keys and values: the plan of the work, the kernels of a key tile, the sum of its parts.
#pragma once
#include "kp_attn_grad.h"

namespace kp {
namespace attn {

// Query tokens that see keys of key tile `kt`: [from, to).
struct Tokens {
  uint32_t from, to;
};
// How the key tiles of a call are dealt to its workers (workgroups).  Where the heads of keys can be dealt out to the 8 XCDs
// (and their L2s) evenly, each XCD's workers have heads of their own (a line; otherwise there is one).  Of a line's tiles
// every worker takes as many whole as there are for all, side by side, so that the rows that neighbouring tiles share are in
// L2 when they are asked for (with a run of tiles of its own for every worker 80 % of the requests missed it, this way
// 50 %), forwards and backwards in turn, since without a window the first are the longest.  What is left over, and the
// tiles that hold sinks, which all later tokens see, stand in a line step by step (64 tokens of one query head), of which
// every worker takes a piece that makes up for what its whole tiles are short of the others': a tile that does not lie
// whole in one piece leaves a partial sum for every worker that has a part, first or last in its piece, and kp_grad_join
// adds them up in order.  The host makes the plan (on the device it took 4 us at the start of every worker).
constexpr uint32_t kChip = 256, kMostWorkers = 2u * kChip;  // CUs; workers: one per CU, or two (D = 64)
constexpr uint32_t kTileCost = 4;  // steps' worth of time that a tile takes besides its steps
struct KeyPlan {
  uint32_t n_q, n_k, window, sinks, group;
  uint32_t lines, units, workers;          // lines; of each: heads, workers
  uint32_t sink_tiles, per_unit;           // of a head: tiles with sinks, the others
  uint32_t whole, rest;                    // of a line: tiles that are taken whole, tiles that are split
  uint32_t edge[kMostWorkers + 1];         // first step of every worker's piece of the latter, and one past the last

  __host__ __device__ Tokens tokens(uint32_t kt) const {
    const int32_t k0 = (int32_t)(kt * kGradKeys), k1 = k0 + kGradKeys < (int32_t)n_k ? k0 + kGradKeys : (int32_t)n_k;
    const int32_t first = k0 + (int32_t)n_q - (int32_t)n_k, last = k1 - 1 + (int32_t)n_q - (int32_t)n_k;  // tokens at the first and last key
    Tokens t;
    t.from = first < 0 ? 0u : (first < (int32_t)n_q ? (uint32_t)first : n_q);
    const int32_t end = window == 0u || k0 < (int32_t)sinks || last >= (int32_t)n_q ? (int32_t)n_q : last + (int32_t)window;
    t.to = end > (int32_t)n_q ? n_q : (end > (int32_t)t.from ? (uint32_t)end : t.from);
    return t;
  }
  __host__ __device__ uint32_t steps(uint32_t kt) const {
    const Tokens t = tokens(kt);
    return (t.to - t.from + 63u) / 64u * group;
  }
  // the n-th of a line's tiles that are not sinks': head (of the line) and tile; the n-th that is split
  __host__ __device__ void plain_tile(uint32_t n, uint32_t* unit, uint32_t* kt) const {
    *unit = units == 1u ? 0u : n / per_unit;
    *kt = sink_tiles + (n - *unit * per_unit);
  }
  __host__ __device__ void split_tile(uint32_t n, uint32_t* unit, uint32_t* kt) const {
    if (n < units * sink_tiles) {
      *unit = n / sink_tiles;
      *kt = n - *unit * sink_tiles;
    } else {
      plain_tile(whole + (n - units * sink_tiles), unit, kt);
    }
  }
  __host__ __device__ uint32_t split_steps(uint32_t n) const {
    uint32_t unit, kt;
    split_tile(n, &unit, &kt);
    return steps(kt);
  }
  // the n-th whole tile of a worker, if below `whole`
  __host__ __device__ uint32_t whole_tile(uint32_t worker, uint32_t n) const {
    return n * workers + ((n & 1u) ? workers - 1u - worker : worker);
  }
  __host__ void deal() {
    uint32_t total = 0;
    for (uint32_t n = 0; n < rest; ++n) total += split_steps(n);
    uint64_t all = total, before = 0;
    for (uint32_t w = 0; w < workers; ++w) all += edge[w] = cost(w);
    const uint32_t each = (uint32_t)((all + workers - 1u) / workers);  // (what all are short of it is the total or more)
    for (uint32_t w = 0; w < workers; ++w) {
      const uint32_t has = edge[w];
      edge[w] = before < total ? (uint32_t)before : total;
      before += has < each ? each - has : 0u;
    }
    edge[workers] = total;
  }

 private:
  __host__ uint32_t cost(uint32_t worker) const {
    uint32_t sum = 0;
    for (uint32_t n = 0; n * workers < whole; ++n) {
      const uint32_t tile = whole_tile(worker, n);
      if (tile >= whole) continue;  // (the last round may not be full)
      uint32_t unit, kt;
      plain_tile(tile, &unit, &kt);
      sum += steps(kt) + kTileCost;
    }
    return sum;
  }
};

__device__ __forceinline__ uint32_t sum_up_to_lane(uint32_t x) {
  const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(x, d, 64);
    if (lane >= (uint32_t)d) x += up;
  }
  return x;
}

// What a worker does, one key tile (or a part of one) after the other.
struct KeyWork {
  uint32_t unit, key_tile, s_begin, s_end, steps_per_head, slot;  // steps [s_begin, s_end) of the tile; slot: of its partial sums
  Tokens tok;
  bool whole;

  __device__ __forceinline__ KeyWork(const KeyPlan& plan) {
    line = plan.lines == 1u ? 0u : blockIdx.x & 7u;
    worker = blockIdx.x / plan.lines;
    // workgroups that come to CUs that have one already: the last of them beside the first (tiles without a window, the
    // longest with the shortest: 4 x 32/8 x 2048 x 64 takes 315 us, 375 in order)
    const uint32_t once = kChip / plan.lines;
    if (worker >= once) worker = plan.workers - 1u - (worker - once);
    round = 0u; split_no = 0u; s_from = 0u;
    at = plan.edge[worker];
    to = plan.edge[worker + 1u];
    first = true;
    if (at >= to) return;
    // the split tile that the piece begins in
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;
    for (uint32_t t0 = 0; t0 < plan.rest; t0 += 64u) {
      const uint32_t steps = t0 + lane < plan.rest ? plan.split_steps(t0 + lane) : 0u, sum = before + sum_up_to_lane(steps);
      const uint64_t past = __builtin_amdgcn_ballot_w64(sum > at);
      if (past != 0ull) {
        const int l = __builtin_ctzll(past);
        split_no = t0 + (uint32_t)l;
        s_from = at - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(steps, l));
        break;
      }
      before = __builtin_amdgcn_readlane(sum, 63);
    }
  }
  __device__ __forceinline__ bool next(const KeyPlan& plan) {
    for (;;) {
      const bool rounds = round * plan.workers < plan.whole;  // first the whole tiles
      if (!rounds && at >= to) return false;
      const uint32_t tile = plan.whole_tile(worker, round);
      uint32_t u;
      if (rounds) {
        ++round;
        if (tile >= plan.whole) continue;
        plan.plain_tile(tile, &u, &key_tile);
      } else {
        plan.split_tile(split_no++, &u, &key_tile);
      }
      unit = u * plan.lines + line;
      tok = plan.tokens(key_tile);
      steps_per_head = (tok.to - tok.from + 63u) / 64u;
      const uint32_t steps = steps_per_head * plan.group;
      s_begin = rounds ? 0u : s_from;
      s_end = rounds || steps - s_begin <= to - at ? steps : s_begin + (to - at);
      slot = first && s_begin != 0u ? 0u : 1u;
      whole = s_begin == 0u && s_end == steps;
      if (rounds) return true;
      at += s_end - s_begin;
      s_from = 0u;
      first = false;
      if (s_begin < s_end) return true;  // (otherwise a tile that no token sees: kp_grad_join's)
    }
  }

  __device__ __forceinline__ size_t part_at(const KeyPlan& plan) const { return 2u * (size_t)(worker * plan.lines + line) + slot; }

 private:
  uint32_t line, worker, round, split_no, s_from, at, to;
  bool first;
};

// Largest |d_o| (at `most`) of row `lane` of the step that starts at `start`, 0 if it sees none of the keys k0 .. k1.
__device__ __forceinline__ float most_of_row(const GradArgs& g, const Tokens& tok, uint32_t start, int32_t k0, int32_t k1, const float* most) {
  const uint32_t token = start + (threadIdx.x & 63u);
  const int32_t p = (int32_t)g.n_k - (int32_t)g.n_q + (int32_t)token;
  const bool sees_some = (token < tok.to) & (p >= k0) & ((g.window == 0u) | (k0 < (int32_t)g.sinks) | (p - k1 < (int32_t)g.window));
  return sees_some ? most[threadIdx.x & 63u] : 0.f;
}

// The keys of 32 (from j0 on) whose dk or dv are not finite, those taken again over the same steps, in fp32; `mine`: of which
// keys this wave does so.
template <class T, int D>
__device__ __forceinline__ void keys_again(const GradArgs& g, const KeyWork& work, uint32_t seq, uint32_t hk, uint32_t j0, uint32_t again_k, uint32_t again_v, uint32_t mine, float* part) {
  using R = Rows<T, D, false>;
  for (uint32_t again = (again_k | again_v) & mine; again != 0u; again &= again - 1u) {
    const uint32_t r = (uint32_t)__builtin_ctz(again), key = j0 + r;
    const bool need_k = ((again_k >> r) & 1u) != 0u, need_v = ((again_v >> r) & 1u) != 0u;
    float k[8], v[8], dk[8] = {}, dv[8] = {};
    R::one(row_at(g.k, seq, hk, key), k);
    R::one(row_at(g.v, seq, hk, key), v);
    bool want_k = need_k, want_v = need_v;
    for (uint32_t step = work.s_begin; step < work.s_end && (want_k || want_v); ++step) {
      const uint32_t in_group = step / work.steps_per_head, first = work.tok.from + (step - in_group * work.steps_per_head) * 64u;
      key_row<T, D>(g, seq, hk * g.group + in_group, key, first, first + 64u < work.tok.to ? first + 64u : work.tok.to, k, v, &want_k, &want_v, dk, dv);
    }
    R::finish(dk);
    R::finish(dv);
    if (work.whole) {
      if (need_k) R::put(dk, g.scale, const_cast<uint16_t*>(row_at(g.dk, seq, hk, key)));
      if (need_v) R::put(dv, 1.f, const_cast<uint16_t*>(row_at(g.dv, seq, hk, key)));
    } else {
      if (need_k) R::put(dk, g.scale, part + r * D);
      if (need_v) R::put(dv, 1.f, part + kGradKeys * D + r * D);
    }
  }
}
// Keys (rows l32 of the wave) for which some lane's `odd` is not 0.
__device__ __forceinline__ uint32_t odd_keys(float odd, bool mine) {
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(mine && odd != 0.f);
  return (uint32_t)(lanes | lanes >> 32);
}

// dk and dv of 128 keys from a run of the query rows that see them.  A step is 64 tokens of one query head, whose Q and dO
// tiles are in LDS, three buffers each, with the rows' lse and delta.
// 8 waves, two to a group of 32 keys.  K and V rows, dk and dv of 32 keys of D = 128 would fill the registers of a wave that
// has a SIMD for itself (which issues too slowly: 2200 cycles for 32 rows, of which the matrix pipes need 1024); so the two
// waves of a group share the rows in the first two products, 32 each, give each other P and dS through LDS, and share d in
// the last two.  S^T = K Q^T and dP^T = V dO^T have a row to a lane, with its lse and delta; P and dS go to LDS as
// [row][key] and are read transposed, for dv^T += dO^T P and dk^T += Q^T dS, which have a key to a lane.
// S and dP are formed a step ahead: the exponentials stand between the MFMAs of dP, the rest of the vector work between
// those of dv.
// 32/8 x 8192 x 128, window 1024: 343 us, 755 TFLOP/s of four products, the matrix pipes busy 46 % of the time at 1.6 GHz, the
// lowest clock of these kernels: it is bound by power as much as by the vector and scalar instructions between its MFMAs.
constexpr int kPairThreads = 512;
template <int D> constexpr uint32_t pairs_lds_bytes() { return 3u * (4u * 64u * D + kStatBytes) + 24u * 2048u; }
template <class T, int D>
__global__ __launch_bounds__(kPairThreads, 2) void kp_grad_keys_pairs(GradArgs g, KeyPlan plan) {
  constexpr uint32_t kRow = 2u * D, kTile = 64u * kRow, kBuffer = 2u * kTile;
  constexpr int NS = D / 16, NH = D / 64;  // NH: tiles of 32 d of a wave
  constexpr int LA = 4;                    // operands come out of LDS this many MFMAs ahead
  constexpr bool kScaled = std::is_same<T, Fp16>::value;
  extern __shared__ __align__(16) unsigned char smem[];
  // [three buffers of Q tile, dO tile][P of every wave: 2 KiB][dS, twice][three times neg, delta, largest |d_o| of 64 rows]
  constexpr uint32_t kShared = 3u * kBuffer, kSharedDs = kShared + 8u * 2048u, kStats = kSharedDs + 16u * 2048u;
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = kp::wave_uniform(tid >> 6), h32 = lane >> 5, l32 = lane & 31u;
  const uint32_t group_no = wave & 3u, hf = wave >> 2;  // of 32 keys; the wave's half of the rows and of d
  const int32_t off = (int32_t)g.n_k - (int32_t)g.n_q;
  const uint32_t j_last = g.n_k - 1u;
  KeyWork work(plan);
  const TileReader<D> rd((uint32_t)(uintptr_t)smem);
  TileLoader<D, 8> lq(g.q.token), ld(g.d_o.token);
  const uint32_t lds0 = kp::wave_uniform((uint32_t)(uintptr_t)smem + 1024u * wave);
  // What the waves of a group share, [32 rows][32 keys] each: the 8-byte piece n of row r at n ^ r / 4 % 8, so that 32 rows'
  // writes and four rows' transposing reads cover all banks once.
  const uint32_t shared_wr = 2048u * wave + 64u * l32 + ((h32 ^ ((l32 >> 2) & 7u)) << 3);
  uint32_t shared_own, shared_other;
  {
    const uint32_t i = lane & 15u, grp = lane >> 4, row = 4u * (grp >> 1) + (i >> 2), piece = 4u * (grp & 1u) + (i & 3u);
    shared_own = (uint32_t)(uintptr_t)smem + 2048u * wave + 64u * row + ((piece ^ (row >> 2)) << 3);
    shared_other = shared_own ^ 8192u;
  }
  while (work.next(plan)) {
    const uint32_t unit = work.unit, key_tile = work.key_tile, seq = unit / g.hkv, hk = unit - seq * g.hkv;
    const Tokens tok = work.tok;
    const uint32_t steps_per_head = work.steps_per_head, s_begin = work.s_begin, s_end = work.s_end;
    const bool whole = work.whole;
    const uint32_t j0 = key_tile * kGradKeys + 32u * group_no, j = j0 + l32, j_in = j < j_last ? j : j_last;
    u32x4 kf[NS], vf[NS];
    {
      const uint16_t *k = row_at(g.k, seq, hk, j_in), *v = row_at(g.v, seq, hk, j_in);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        kf[s] = *reinterpret_cast<const u32x4*>(k + 16 * s + 8 * h32);
        vf[s] = *reinterpret_cast<const u32x4*>(v + 16 * s + 8 * h32);
      }
    }
    RowsScale scale;     // fp16: of dS that is formed
    float dk_by = 1.f;   // what takes dk to that scale

    // ---- requests: the next step's head, first token, place ---------------------------------------------------------
    uint32_t loaded_last = ~0u, into = 0u;  // `into`: buffer that it goes to
    auto after = [](uint32_t buffer) __attribute__((always_inline)) { return buffer == 2u ? 0u : buffer + 1u; };
    const uint32_t head_steps = steps_per_head == 0u ? 1u : steps_per_head;
    uint32_t ask_group = s_begin / head_steps, ask_start = tok.from + (s_begin - ask_group * head_steps) * 64u;
    uint32_t asked = s_begin;    // number of the step that is requested next
    uint32_t start = ask_start;  // first token of the step whose S and dP are formed
    const uint16_t *ask_q, *ask_do;
    const float* ask_stat;
    auto ask_at = [&]() __attribute__((always_inline)) {
      const uint32_t head = hk * g.group + ask_group;
      ask_q = row_at(g.q, seq, head, ask_start);
      ask_do = row_at(g.d_o, seq, head, ask_start);
      ask_stat = (wave == 0u ? g.neg : wave == 1u ? g.delta : g.most) + ((size_t)seq * g.hkv * g.group + head) * g.n_q + ask_start;
    };
    ask_at();
    constexpr int NL = TileLoader<D, 8>::NL, kAsks = 2 * NL + 2;
    // The request in kAsks parts, to stand between MFMAs.
    auto ask = [&](int part) __attribute__((always_inline)) {
      if (part == 0) {
        const uint32_t left = tok.to - 1u - ask_start, last = left < 63u ? left : 63u;
        if (last != loaded_last) { loaded_last = last; lq.upto(last); ld.upto(last); }
      }
      if (part >= kAsks) return;
      if (part < NL) {
        lq.load_one(part, ask_q, lds0 + into * kBuffer);
      } else if (part < 2 * NL) {
        ld.load_one(part - NL, ask_do, lds0 + into * kBuffer + kTile);
      } else if (part == 2 * NL) {
        if (wave < (kScaled ? 3u : 2u)) {  // the rows' neg (wave 0), delta (wave 1), largest |d_o| (wave 2): 4 bytes to a lane
          const uint32_t ofs = 4u * (lane < loaded_last ? lane : loaded_last), dst = kp::wave_uniform((uint32_t)(uintptr_t)smem + kStats + into * kStatBytes + 256u * wave);
          uint32_t saved_m0;
          asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                       : "=&s"(saved_m0) : "v"(ofs), "s"(ask_stat), "s"(dst) : "memory");
        }
      } else {
        into = after(into);
        if (++asked >= s_end) return;  // (past the last step: that one again, of no use)
        ask_start += 64u;
        if (ask_start < tok.to) {
          ask_q += 64 * g.q.token;
          ask_do += 64 * g.d_o.token;
          ask_stat += 64;
        } else {  // the next head's first
          ask_start = tok.from;
          ++ask_group;
          ask_at();
        }
      }
    };
    auto request = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int part = 0; part < kAsks; ++part) ask(part);
    };
    auto wait_all = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    f32x16 dk[NH], dv[NH];  // transposed: rows d = 32 (NH hf + dt) + .., column = key l32
#pragma unroll
    for (int dt = 0; dt < NH; ++dt) { dk[dt] = f32x16{0}; dv[dt] = f32x16{0}; }
    u32x4 ra[LA];
    f32x16 sacc, dp;
    float w[16], neg, delta;  // of the wave's 32 rows of the next step, row l32
    float most = 0.f;         // fp16: of all its 64, row `lane`
    u32x2 pw[4], ds[4];  // P and dS: keys 8 i + 4 h32 .. + 3 of row l32
    uint32_t ds_now = 0u;  // which of the two dS in LDS is this step's
    uint32_t now = 0u, next = 0u;  // buffers of the step at hand and of the one whose S and dP are formed
    // Keeps a value that is not used before the next block of code where it is made: the compiler would move it there.
    auto stay = [](auto& x) __attribute__((always_inline)) { asm volatile("" : "+v"(x)); };
    // operands in the order of their use: Q and dO rows of the next step (this wave's half), dO^T and then Q^T of this one
    // (first of this wave's rows, then of the other's); behind them the next step's
    // LDS addresses of those in the buffers at hand: rows by operand, transposed pieces by half of the rows, dt, half of the keys
    uint32_t row_at_lds[NS], col_at_lds[2][NH][2];
#pragma unroll
    for (int n = 0; n < NS; ++n) row_at_lds[n] = (rd.row0 + 32u * hf * kRow) ^ (32u * (uint32_t)n);
#pragma unroll
    for (int dt = 0; dt < NH; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        col_at_lds[e >> 1][dt][e & 1] = ((rd.col0 ^ (64u * NH * hf)) + 32u * (hf ^ (uint32_t)(e >> 1)) * kRow) ^ (64u * (uint32_t)dt + 32u * (uint32_t)(e & 1));
    auto step_rows = [&]() __attribute__((always_inline)) {
      const uint32_t by = next == 2u ? 0u - 2u * kBuffer : kBuffer;
      next = after(next);
#pragma unroll
      for (int n = 0; n < NS; ++n) row_at_lds[n] += by;
    };
    auto step_cols = [&]() __attribute__((always_inline)) {
      const uint32_t by = now == 2u ? 0u - 2u * kBuffer : kBuffer;
      now = after(now);
#pragma unroll
      for (int dt = 0; dt < NH; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) col_at_lds[e >> 1][dt][e & 1] += by;
    };
    auto fetch = [&](int n) __attribute__((always_inline)) -> u32x4 {
      if (n >= 4 * NS) n -= 4 * NS;
      if (n < NS) return rd.rows_at(row_at_lds[n], 0u);
      if (n < 2 * NS) return rd.rows_at(row_at_lds[n - NS], 64u);
      const int m = (n - 2 * NS) % NS, ks = m / NH, dt = m % NH;
      return rd.cols_at(col_at_lds[ks / 2][dt][0], col_at_lds[ks / 2][dt][1], (n < 3 * NS ? 64u : 0u) + 16u * (uint32_t)(ks & 1));
    };
    // S of the wave's 32 rows of the step that starts at `start`: what is not visible becomes -inf
    auto hide = [&]() __attribute__((always_inline)) {
      const int32_t first = (int32_t)(start + 32u * hf), last = first + 31, k0 = (int32_t)j0, k1 = k0 + 31;
      if ((last >= (int32_t)tok.to) | (off + first < k1) | ((g.window != 0u) & (k1 >= (int32_t)g.sinks) & (off + last - k0 >= (int32_t)g.window))) {
        const int32_t token = first + (int32_t)l32;
        RowMask m(token < (int32_t)tok.to ? off + token : -1, g.n_k, k0 + 4 * (int32_t)h32, g.window, g.sinks);
        if ((g.window == 0u) | (k0 >= (int32_t)g.sinks)) {
          m.apart();
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = m.sees(8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
        } else if (off + first - k1 >= (int32_t)g.window) {  // sinks alone are left
          m.apart();
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = 8 * (v >> 2) + (v & 3) <= m.sink ? sacc[v] : -INFINITY;
        } else {
          m.apart();
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = m.sees_mixed(8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
        }
      }
    };
    auto load_stats = [&]() __attribute__((always_inline)) {
      const float* const st = reinterpret_cast<const float*>(smem + kStats + next * kStatBytes + 128u * hf) + l32;
      neg = st[0];
      delta = st[64];
      if constexpr (kScaled) most = most_of_row(g, tok, start, (int32_t)j0, (int32_t)j0 + 31, reinterpret_cast<const float*>(smem + kStats + next * kStatBytes + 512u));
    };
    auto exponential = [&](int v) __attribute__((always_inline)) {
      w[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v], g.scale_log2, neg));
      stay(w[v]);
    };
    auto finish = [&](int v) __attribute__((always_inline)) {  // elements v, v + 1
      float x0 = w[v] * (dp[v] - delta), x1 = w[v + 1] * (dp[v + 1] - delta);
      if constexpr (kScaled) { x0 *= scale.by(); x1 *= scale.by(); }
      pw[v >> 2][(v >> 1) & 1] = T::pack(w[v], w[v + 1]);
      ds[v >> 2][(v >> 1) & 1] = T::pack(x0, x1);
    };
    auto share_p = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x2*>(smem + kShared + (shared_wr ^ (16u * (uint32_t)i))) = pw[i];
    };
    auto share_ds = [&](uint32_t which, int i) __attribute__((always_inline)) {
      *reinterpret_cast<u32x2*>(smem + kSharedDs + which * 16384u + (shared_wr ^ (16u * (uint32_t)i))) = ds[i];
    };
    // operand ks of the last products: 16 rows each, two of this wave's and two of the other's; key l32
    auto shared_at = [&](uint32_t region, int ks) __attribute__((always_inline)) {
      const uint32_t a = ks < 2 ? shared_own : shared_other, x = 32u * (uint32_t)(ks & 1), rows = 1024u * (uint32_t)(ks & 1);
      return TileReader<D>::cols_from((a ^ x) + region + rows, (a ^ (x + 16u)) + region + rows + 512u);
    };
    auto shared_p = [&](int ks) __attribute__((always_inline)) { return shared_at(kShared, ks); };
    auto shared_ds = [&](int ks) __attribute__((always_inline)) { return shared_at(kSharedDs + ds_now * 16384u, ks); };
    constexpr int kPer = 16 / NS;  // elements between two MFMAs

    if (s_begin < s_end) {
    request();
    request();
    __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own count of outstanding loads)
    wait_all();
    sacc = f32x16{0}; dp = f32x16{0};
#pragma unroll
    for (int n = 0; n < LA; ++n) ra[n] = fetch(n);
#pragma unroll
    for (int n = 0; n < 2 * NS; ++n) {
      if (n < NS) sacc = T::mfma32(kf[n], ra[n % LA], sacc); else dp = T::mfma32(vf[n - NS], ra[n % LA], dp);
      if (n + LA < 2 * NS) ra[n % LA] = fetch(n + LA);
    }
    hide();
    load_stats();
    if constexpr (kScaled) scale.moved(most);  // (dk is 0)
#pragma unroll
    for (int v = 0; v < 16; ++v) exponential(v);
#pragma unroll
    for (int v = 0; v < 16; v += 2) finish(v);
    share_p();
#pragma unroll
    for (int i = 0; i < 4; ++i) share_ds(0u, i);
    wait_all();
    step_rows();
#pragma unroll
    for (int n = 0; n < LA; ++n) ra[n] = fetch(n);
    for (uint32_t step = s_begin; step < s_end; ++step) {
      start += 64u;
      if (start >= tok.to) start = tok.from;
      u32x4 rb[2];  // operands of P and dS, one ahead
      // S and dP of the next step (behind the last: of no use), its exponentials; the one after that is asked for, into the
      // buffer of the step before this one
      sacc = f32x16{0}; dp = f32x16{0};
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        sacc = T::mfma32(kf[n], ra[n % LA], sacc);
        ra[n % LA] = fetch(n + LA);
        if (n == 0) load_stats();
        ask(n);
        if (n == NS - 1) {
#pragma unroll
          for (int part = NS; part < kAsks; ++part) ask(part);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      hide();
      if constexpr (kScaled) dk_by = scale.moved(most);
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        dp = T::mfma32(vf[n], ra[n % LA], dp);
        stay(dp);
        ra[n % LA] = fetch(NS + n + LA);
#pragma unroll
        for (int v = kPer * n; v < kPer * (n + 1); ++v) exponential(v);
        if (n == NS - 1) rb[0] = shared_p(0);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int ks = n / NH;
        if (n % NH == 0) rb[(ks + 1) & 1] = ks < 3 ? shared_p(ks + 1) : shared_ds(0);
        dv[n % NH] = T::mfma32(ra[n % LA], rb[ks & 1], dv[n % NH]);
        ra[n % LA] = fetch(2 * NS + n + LA);
#pragma unroll
        for (int v = kPer * n; v < kPer * (n + 1); v += 2) finish(v);
        if (kPer * (n + 1) % 4 == 0) share_ds(ds_now ^ 1u, kPer * (n + 1) / 4 - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // every wave has read this step's P
      share_p();
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        const int ks = n / NH;
        if (n % NH == 0 && ks < 3) rb[(ks + 1) & 1] = shared_ds(ks + 1);
        // behind the last operand of this step: P and dS of the next are there, so are its successor's tiles
        if (n == NS - LA) {
          wait_all();
          step_cols();
          step_rows();
        }
        dk[n % NH] = T::mfma32(ra[n % LA], rb[ks & 1], dk[n % NH]);
        ra[n % LA] = fetch(3 * NS + n + LA);
        __builtin_amdgcn_sched_barrier(0);
      }
      ds_now ^= 1u;
      if constexpr (kScaled) {
        if (dk_by != 1.f) {
#pragma unroll
          for (int dt = 0; dt < NH; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) dk[dt][v] *= dk_by;
        }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what was asked for past the end has landed too)
    }

    const float by_k = kScaled ? g.scale / (scale.by() * __builtin_ldexpf(1.0f, (int)kShiftP<T>)) : g.scale;
    const float by_v = kScaled ? __builtin_ldexpf(1.0f, -(int)kShiftP<T>) : 1.f;
    // what both waves of a group, each with half of d, have to take again, of which each takes every other key
    uint32_t* const again = reinterpret_cast<uint32_t*>(smem + kStats + 768u);  // (behind a step's statistics)
    const uint32_t odd_k = odd_keys(odd_of<NH>(dk), j <= j_last), odd_v = odd_keys(odd_of<NH>(dv), j <= j_last);
    if (lane == 0u) { again[2u * wave] = odd_k; again[2u * wave + 1u] = odd_v; }
    float* const part = g.part + work.part_at(plan) * (2u * kGradKeys * D) + (size_t)(32u * group_no) * D;
    __syncthreads();  // (the tiles' room is used below)
    const uint32_t again_k = kp::wave_uniform(odd_k | again[2u * (wave ^ 4u)]), again_v = kp::wave_uniform(odd_v | again[2u * (wave ^ 4u) + 1u]);
    if (!whole) {
      if (j <= j_last) {  // (3 x 64/8 x 5 x 128: 26 us for both kernels and the join, 37 with the rows that are no keys)
#pragma unroll
        for (int dt = 0; dt < NH; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float* const out = part + l32 * D + 32u * (NH * hf + (uint32_t)dt) + 8 * i + 4 * h32;
            *reinterpret_cast<f32x4*>(out) = f32x4{dk[dt][4 * i] * by_k, dk[dt][4 * i + 1] * by_k, dk[dt][4 * i + 2] * by_k, dk[dt][4 * i + 3] * by_k};
            *reinterpret_cast<f32x4*>(out + kGradKeys * D) = f32x4{dv[dt][4 * i] * by_v, dv[dt][4 * i + 1] * by_v, dv[dt][4 * i + 2] * by_v, dv[dt][4 * i + 3] * by_v};
          }
      }
    } else {
      // Through LDS as in store_rows, the dk tile and behind it the dv tile: [128 keys][D]
      unsigned char* const to_lds = smem + 32u * group_no * kRow + l32 * kRow;
      const uint32_t half = h32 ^ ((l32 >> 3) & 1u);
#pragma unroll
      for (int dt = 0; dt < NH; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at_lds = (((4u * (NH * hf + (uint32_t)dt) + (uint32_t)i) ^ (l32 & 7u)) << 4) + 8u * half;
          *reinterpret_cast<u32x2*>(to_lds + at_lds) = u32x2{T::pack(dk[dt][4 * i] * by_k, dk[dt][4 * i + 1] * by_k), T::pack(dk[dt][4 * i + 2] * by_k, dk[dt][4 * i + 3] * by_k)};
          *reinterpret_cast<u32x2*>(to_lds + kGradKeys * kRow + at_lds) = u32x2{T::pack(dv[dt][4 * i] * by_v, dv[dt][4 * i + 1] * by_v), T::pack(dv[dt][4 * i + 2] * by_v, dv[dt][4 * i + 3] * by_v)};
        }
      __syncthreads();
      constexpr uint32_t kChunks = kRow / 16u;
#pragma unroll
      for (uint32_t i = 0; i < 2u * kGradKeys * kChunks / kPairThreads; ++i) {
        const uint32_t n = tid + i * kPairThreads, r = n / kChunks % kGradKeys, chunk = (n % kChunks) ^ (r & 7u), key = key_tile * kGradKeys + r;
        const u32x4 v = *reinterpret_cast<const u32x4*>(smem + 16u * n);
        const Heads& out = n < kGradKeys * kChunks ? g.dk : g.dv;
        if (key <= j_last) *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(row_at(out, seq, hk, key)) + 8u * chunk) = (r & 8u) ? u32x4{v.z, v.w, v.x, v.y} : v;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the results have left, before some are put right
    __syncthreads();  // (and the next tile's rows go to the same room)
    keys_again<T, D>(g, work, seq, hk, j0, again_k, again_v, hf == 0u ? 0x55555555u : 0xAAAAAAAAu, part);
  }
}

// The same for D = 64, where a wave's 32 keys leave room for two waves on a SIMD: 4 waves, each with all rows of a step, two
// workgroups on a CU that overlap one another.  S = Q K^T and dP = dO V^T have a key to a lane, as dv^T += dO^T P and
// dk^T += Q^T dS need it.  (The kernel above takes 33 us where this one takes 22: 2 x 12/4 x 1153 x 64, window 250.)
// There a worker has 3 or 4 steps, and the start of a workgroup, its first loads and its partial sums (39 MB in all) are most
// of the time; 32/8 x 8192, no window, takes 1105 us with the kernel of the queries (fp16 1270), 870 TFLOP/s.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void kp_grad_keys(GradArgs g, KeyPlan plan) {
  constexpr uint32_t kTile = 64u * 2u * D, kBuffer = 2u * kTile;
  constexpr int NS = D / 16, ND = D / 32;
  constexpr bool kScaled = std::is_same<T, Fp16>::value;
  extern __shared__ __align__(16) unsigned char smem[];  // two buffers of [Q tile][dO tile], then two of [neg][delta][largest |d_o|] of 64 rows
  constexpr uint32_t kStats = 2u * kBuffer;
  const uint32_t lane = threadIdx.x & 63u, wave = kp::wave_uniform(threadIdx.x >> 6), h32 = lane >> 5, l32 = lane & 31u;
  const int32_t off = (int32_t)g.n_k - (int32_t)g.n_q;
  const uint32_t j_last = g.n_k - 1u;
  KeyWork work(plan);
  TileCursor<D> rd((uint32_t)(uintptr_t)smem, kBuffer);
  TileLoader<D, 4> lq(g.q.token), ld(g.d_o.token);
  const uint32_t lds0 = kp::wave_uniform((uint32_t)(uintptr_t)smem + 1024u * wave);
  while (work.next(plan)) {
    const uint32_t unit = work.unit, seq = unit / g.hkv, hk = unit - seq * g.hkv;
    const Tokens tok = work.tok;
    const uint32_t steps_per_head = work.steps_per_head, s_begin = work.s_begin, s_end = work.s_end;
    const uint32_t j0 = work.key_tile * kGradKeys + 32u * wave, j = j0 + l32, j_in = j < j_last ? j : j_last;
    u32x4 kf[NS], vf[NS];
    {
      const uint16_t *k = row_at(g.k, seq, hk, j_in), *v = row_at(g.v, seq, hk, j_in);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        kf[s] = *reinterpret_cast<const u32x4*>(k + 16 * s + 8 * h32);
        vf[s] = *reinterpret_cast<const u32x4*>(v + 16 * s + 8 * h32);
      }
    }
    RowsScale scale;  // fp16: of dS and dk
    uint32_t loaded_last = ~0u, into = 0u;  // `into`: buffer that the next step goes to
    if (rd.by != kBuffer) rd.to_other();    // (an odd number of steps before: back to the first)
    const uint32_t head_steps = steps_per_head == 0u ? 1u : steps_per_head;
    uint32_t ask_group = s_begin / head_steps, ask_start = tok.from + (s_begin - ask_group * head_steps) * 64u;
    uint32_t start = ask_start;  // first token of the step at hand
    auto request = [&]() __attribute__((always_inline)) {
      const uint32_t head = hk * g.group + ask_group, left = tok.to - 1u - ask_start, last = left < 63u ? left : 63u;
      if (last != loaded_last) { loaded_last = last; lq.upto(last); ld.upto(last); }
      lq.load(row_at(g.q, seq, head, ask_start), lds0 + into);
      ld.load(row_at(g.d_o, seq, head, ask_start), lds0 + into + kTile);
      if (wave < (kScaled ? 3u : 2u)) {  // the rows' neg (wave 0), delta (wave 1), largest |d_o| (wave 2): 4 bytes to a lane
        const float* from = (wave == 0u ? g.neg : wave == 1u ? g.delta : g.most) + ((size_t)seq * g.hkv * g.group + head) * g.n_q + ask_start;
        const uint32_t ofs = 4u * (lane < last ? lane : last), dst = kp::wave_uniform((uint32_t)(uintptr_t)smem + kStats + (into != 0u ? kStatBytes : 0u) + 256u * wave);
        uint32_t saved_m0;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved_m0) : "v"(ofs), "s"(from), "s"(dst) : "memory");
      }
      into ^= kBuffer;
      ask_start += 64u;
      if (ask_start >= tok.to) { ask_start = tok.from; ++ask_group; }
    };

    f32x16 dk[ND], dv[ND];  // transposed: rows d, column = key l32
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) { dk[dt] = f32x16{0}; dv[dt] = f32x16{0}; }
    u32x4 ra[NS];  // operands, a product ahead
    if (s_begin < s_end) {
      request();
      __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own count of outstanding loads)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      uint32_t stats = kStats;
#pragma unroll
      for (int s = 0; s < NS; ++s) ra[s] = rd.rows(s, 0u);
      for (uint32_t step = s_begin; step < s_end; ++step) {
        float most = 0.f;
        if constexpr (kScaled) most = most_of_row(g, tok, start, (int32_t)j0, (int32_t)j0 + 31, reinterpret_cast<const float*>(smem + stats + 512u));
        if (step + 1u < s_end) request();
        if constexpr (kScaled) {
          const float by = scale.moved(most);
          if (by != 1.f) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
              for (int v = 0; v < 16; ++v) dk[dt][v] *= by;
          }
        }
        auto next_buffer = [&]() __attribute__((always_inline)) {
          // every wave has read these tiles, and the next ones have landed
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          rd.to_other();
        };
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
          // rows of this half: tokens first .. last, positions p0 .. p1; this wave's keys: k0 .. k1
          const int32_t first = (int32_t)start + 32 * rt, last = first + 31, p0 = off + first, p1 = off + (last < (int32_t)tok.to ? last : (int32_t)tok.to - 1);
          const int32_t k0 = (int32_t)j0, k1 = (int32_t)(j0 + 31u < j_last ? j0 + 31u : j_last);
          const bool none = (first >= (int32_t)tok.to) | (k0 > (int32_t)j_last) | (p1 < k0) |
                            ((g.window != 0u) & (k0 >= (int32_t)g.sinks) & (p0 - k1 >= (int32_t)g.window));
          if (none) {
            if (rt == 1) next_buffer();
#pragma unroll
            for (int s = 0; s < NS; ++s) ra[s] = rd.rows(s, rt == 0 ? 32u : 0u);
            continue;
          }
          f32x16 sacc = f32x16{0}, dp = f32x16{0};
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            sacc = T::mfma32(ra[s], kf[s], sacc);
            ra[s] = rd.rows(s, 64u + 32u * (uint32_t)rt);  // dO
            __builtin_amdgcn_sched_barrier(0);
          }
          f32x4 neg[4], delta[4];  // of rows 8 i + 4 h32 .. + 3
          const unsigned char* const st = smem + stats + 128u * (uint32_t)rt + 16u * h32;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            neg[i] = *reinterpret_cast<const f32x4*>(st + 32 * i);
            delta[i] = *reinterpret_cast<const f32x4*>(st + 256 + 32 * i);
          }
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            dp = T::mfma32(ra[s], vf[s], dp);
            ra[s] = rd.cols(s % ND, 64u + 32u * (uint32_t)rt + 16u * (uint32_t)(s / ND));  // dO^T
            __builtin_amdgcn_sched_barrier(0);
          }
          if ((last >= (int32_t)tok.to) | (p0 < k1) | ((g.window != 0u) & (k1 >= (int32_t)g.sinks) & (p1 - k0 >= (int32_t)g.window))) {
            asm volatile("");  // (a branch: no selects where nothing is masked)
            // tokens of the key's lane: from its own position to the end, or to the window's
            const int32_t base = first + 4 * (int32_t)h32, lo = (int32_t)j - off - base;
            int32_t hi = (int32_t)tok.to - 1 - base;
            const int32_t w = (int32_t)j - off - base + ((int32_t)g.window - 1);
            hi = ((g.window != 0u) & (j >= g.sinks) & (w < hi)) ? w : hi;
            const uint32_t from = hi < lo ? 1u << 30 : (uint32_t)lo, count = hi < lo ? 0u : (uint32_t)(hi - lo);
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[v] = (uint32_t)(8 * (v >> 2) + (v & 3)) - from <= count ? sacc[v] : -INFINITY;
          }
          u32x4 pw[2], ds[2];
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            float w[2], x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v + e], g.scale_log2, neg[v >> 2][(v & 3) + e]));
              x[e] = w[e] * (dp[v + e] - delta[v >> 2][(v & 3) + e]);
              if constexpr (kScaled) x[e] *= scale.by();
            }
            pw[v >> 3][(v >> 1) & 3] = T::pack(w[0], w[1]);
            ds[v >> 3][(v >> 1) & 3] = T::pack(x[0], x[1]);
          }
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            dv[s % ND] = T::mfma32(ra[s], pw[s / ND], dv[s % ND]);
            ra[s] = rd.cols(s % ND, 32u * (uint32_t)rt + 16u * (uint32_t)(s / ND));  // Q^T
            __builtin_amdgcn_sched_barrier(0);
          }
          if (rt == 1) next_buffer();
#pragma unroll
          for (int s = 0; s < NS; ++s) {
            dk[s % ND] = T::mfma32(ra[s], ds[s / ND], dk[s % ND]);
            ra[s] = rd.rows(s, rt == 0 ? 32u : 0u);  // Q: the other half, or the next step's (the last time: not used)
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        stats ^= kStatBytes;
        start += 64u;
        if (start >= tok.to) start = tok.from;
      }
    }

    const float by_k = kScaled ? g.scale / (scale.by() * __builtin_ldexpf(1.0f, (int)kShiftP<T>)) : g.scale;
    const float by_v = kScaled ? __builtin_ldexpf(1.0f, -(int)kShiftP<T>) : 1.f;
    const bool mine = j <= j_last;
    const uint32_t again_k = odd_keys(odd_of<ND>(dk), mine), again_v = odd_keys(odd_of<ND>(dv), mine);
    const uint64_t rows_out = __builtin_amdgcn_ballot_w64(mine) & 0xFFFFFFFFull;
    float* const part = g.part + work.part_at(plan) * (2u * kGradKeys * D) + (size_t)(32u * wave) * D;
    __syncthreads();  // (the tiles' room is used below)
    if (!work.whole) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* const out = part + l32 * D + 32 * dt + 8 * i + 4 * h32;
          *reinterpret_cast<f32x4*>(out) = f32x4{dk[dt][4 * i] * by_k, dk[dt][4 * i + 1] * by_k, dk[dt][4 * i + 2] * by_k, dk[dt][4 * i + 3] * by_k};
          *reinterpret_cast<f32x4*>(out + kGradKeys * D) = f32x4{dv[dt][4 * i] * by_v, dv[dt][4 * i + 1] * by_v, dv[dt][4 * i + 2] * by_v, dv[dt][4 * i + 3] * by_v};
        }
    } else {
      store_rows<T, D>(dk, by_k, smem + 64u * D * wave, const_cast<uint16_t*>(g.dk.at), g.dk.seq * (int64_t)seq + g.dk.head * (int64_t)hk + g.dk.token * (int64_t)j_in, rows_out);
      store_rows<T, D>(dv, by_v, smem + 64u * D * wave, const_cast<uint16_t*>(g.dv.at), g.dv.seq * (int64_t)seq + g.dv.head * (int64_t)hk + g.dv.token * (int64_t)j_in, rows_out);
    }
    if ((again_k | again_v) != 0u) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // their first results have left
      keys_again<T, D>(g, work, seq, hk, j0, again_k, again_v, ~0u, part);
    }
    __syncthreads();  // (the next tile's rows go to the same room)
  }
}

// Bound by latency: 5 to 8 us.
// Adds up the parts of the split key tiles that do not lie whole in one worker's piece: D / 4 lanes to a row, a row to a lane;
// blockIdx.y: dk or dv.
template <int D> constexpr int kJoinRows = kThreads / (D / 4);
template <class T, int D>
__global__ __launch_bounds__(kThreads) void kp_grad_join(GradArgs g, KeyPlan plan) {
  constexpr uint32_t kLanes = D / 4, kBlocks = kGradKeys / kJoinRows<D>;
  __shared__ const float* from[kMostWorkers];  // where the tile's parts are
  __shared__ uint32_t counted;
  const uint32_t tile = blockIdx.x / kBlocks, line = tile % plan.lines, no = tile / plan.lines, lane = threadIdx.x & 63u;
  uint32_t u, kt;
  plan.split_tile(no, &u, &kt);
  const uint32_t unit = u * plan.lines + line, n = plan.steps(kt);
  if (threadIdx.x < 64u) {  // a wave finds them: the tile's first step in the line, then the workers whose pieces reach into it
    uint32_t begin = 0, parts = 0;
    for (uint32_t t0 = 0; t0 < no; t0 += 64u) begin += __builtin_amdgcn_readlane(sum_up_to_lane(t0 + lane < no ? plan.split_steps(t0 + lane) : 0u), 63);
    for (uint32_t w0 = 0; w0 < plan.workers; w0 += 64u) {
      const uint32_t w = w0 + lane, a = w < plan.workers ? plan.edge[w] : 0u, b = w < plan.workers ? plan.edge[w + 1u] : 0u;
      const bool has = (n != 0u) & (a < b) & (a < begin + n) & (b > begin);  // (a piece may go on past a tile without steps)
      const uint64_t all = __builtin_amdgcn_ballot_w64(has);
      const uint32_t at = parts + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0u));
      if (has) from[at] = g.part + (2u * (size_t)(w * plan.lines + line) + (a > begin ? 0u : 1u)) * (2u * kGradKeys * D) + (size_t)blockIdx.y * (kGradKeys * D);
      parts += (uint32_t)__builtin_popcountll(all);
    }
    if (lane == 0u) counted = parts;
  }
  __syncthreads();
  const uint32_t parts = counted;
  if (parts == 1u) return;  // one worker has all of it and has written it (none: no token sees the tile)
  const uint32_t seq = unit / g.hkv, hk = unit - seq * g.hkv;
  const uint32_t c = threadIdx.x % kLanes, row = (blockIdx.x % kBlocks) * kJoinRows<D> + threadIdx.x / kLanes, j = kt * kGradKeys + row;
  if (j >= g.n_k) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (uint32_t i = 0; i < parts; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(from[i] + row * D + 4u * c);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  const Heads& out = blockIdx.y ? g.dv : g.dk;
  *reinterpret_cast<u32x2*>(const_cast<uint16_t*>(row_at(out, seq, hk, j)) + 4u * c) = u32x2{T::pack(sum[0], sum[1]), T::pack(sum[2], sum[3])};
}

}  // namespace attn
}  // namespace kp
