// Queries and keys normed per head and turned by their positions: forward, gradient, and forward into a paged cache.
//
// A row x of D values, r = 1 / sqrt(mean x^2 + eps), u = x r w (without weights u = x); pair m of u, values (a, b), becomes
//   (a cos - b sin, a sin + b cos),  angle = position on the pair's axis * freq[m],
// and a value y_n = r (x_n A_n + x_p B_n) for its partner p, with A_n = w_n cos and B_n = -+w_p sin the same for all heads of a
// token.  The gradient turns d_y back, g = R^T d_y, and passes the norm: d_w += g n, d_x = r (w g - n mean(w g n)), n = x r.
// D / 8 lanes have a row, 16 bytes each; a thread keeps its token, whose A and B it makes once, and goes from head to head.
#include <type_traits>

#include "kp_cache_row.h"
#include "kp_attn_host.h"

namespace {
using namespace kp::attn;

constexpr uint32_t kThreads = 256;

struct RotateArgs {
  Heads x[2], y[2];          // queries and keys (gradient: d_y and d_x); y is written
  Heads in[2];               // gradient: what was normed
  const void* weight[2];
  float* d_weight[2];
  uint32_t heads[2], chunk;  // chunk: heads (of queries, keys and values, one behind the other) that a workgroup takes
  uint32_t tokens, per_seq;  // tokens of all sequences, and of one
  uint32_t tile_log2, tiles; // tokens side by side in a workgroup, and how many times as many there are
  uint32_t heads_first;      // neighbouring threads have neighbouring heads, not tokens
  float eps;
  uint32_t fp32_weights;
  const int32_t* at;
  int64_t axis_step, seq_step;
  const float* freq;
  const uint8_t* axis;
  uint32_t pairs, axes;
  float* part;               // gradient: sums of d_w of each workgroup
  // into a cache: v, and where keys and values go
  Heads v;
  const int64_t* slots;
  uint8_t *k_cache, *v_cache, *k_exp, *v_exp;
  uint32_t page_log2;
  uint64_t n_slots;
};

// Sum over the D / 8 lanes of a row, in all of them.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int D>
__device__ __forceinline__ float row_sum(float s) {
  s += moved<0xB1>(s);  // from the next lane, the next two, the next four, the next eight
  s += moved<0x4E>(s);
  s += moved<0x141>(s);
  if constexpr (D == 128) s += moved<0x140>(s);
  return s;
}

// cos and sin of position * freq.  The angle in turns is taken in 64 bits, its fraction in 32 as a whole number (the low word of a
// double whose last place is 2^-32 turns), of which the nearest quarter goes off; what is left, up to an eighth of a turn, goes into the
// Taylor series (they end 2^-29 and 2^-32 from the functions).  With |freq| <= 1 off by at most 2^-21 for any position of 31 bits.
__device__ __forceinline__ void turn_of(int32_t position, double freq_turns, float* cos, float* sin) {
  const double at = (double)position, whole = __builtin_rint(at * freq_turns), part = __builtin_fma(at, freq_turns, -whole);
  const uint32_t u = (uint32_t)__builtin_bit_cast(uint64_t, __builtin_fma(part, 4294967296.0, 6755399441055744.0));
  const uint32_t q = (u + 0x20000000u) >> 30;
  const float z = (float)(int32_t)(u - (q << 30)) * 1.4629180792671596e-09f, z2 = z * z;  // 2 pi / 2^32
  const float s = z * __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = (q & 1u) ? s : c, b = (q & 1u) ? c : s;
  *cos = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) ^ (((q + 1u) & 2u) << 30));
  *sin = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, b) ^ ((q & 2u) << 30));
}

template <class T>
__device__ __forceinline__ void widen(const u32x4& raw, float (&x)[8]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    x[2 * w] = T::to_float(raw[w] & 0xFFFFu);
    x[2 * w + 1] = T::to_float(raw[w] >> 16);
  }
}
template <class T>
__device__ __forceinline__ u32x4 narrow(const float (&x)[8]) {
  return u32x4{T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7])};
}
// 8 weights from number n on; ones where there are none
template <class T>
__device__ __forceinline__ void weights_of(const void* weight, bool fp32, uint32_t n, float (&w)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = 1.f;
  if (!weight) return;
  if (fp32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = static_cast<const float*>(weight)[n + e];
  } else {
    widen<T>(*reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(weight) + n), w);
  }
}

// The sine of a value that is not turned, being in no pair or in one whose axis is not there: one that no angle gives (they are 0 or 2^-30 and
// more).  Nothing of a partner may come to such a value, which an infinity or a NaN does through any factor.
constexpr float kStays = 0x1p-149f;

// What a lane needs for its values 8 c .. 8 c + 7 of a row, and how it meets their partners.
template <bool ADJACENT>
struct Turn {
  bool turned;    // its values belong to pairs
  bool lower;     // (not ADJACENT) they are the first of their pairs
  uint32_t far;   // (not ADJACENT) lanes from one half of the pairs to the other
  bool some_stay; // a lane of the wave has a pair that is not turned
  float cos[8], sin[8];

  __device__ __forceinline__ Turn(const RotateArgs& g, uint32_t c) : turned(8u * c < 2u * g.pairs), lower(8u * c < g.pairs), far(g.pairs / 8u) {}
  __device__ __forceinline__ uint32_t partner_of(uint32_t x) const { return ADJACENT || !turned ? x : (lower ? x + far : x - far); }
  __device__ __forceinline__ void angles(const RotateArgs& g, uint32_t c, uint32_t seq, uint32_t token) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { cos[e] = 1.f; sin[e] = ADJACENT && !(e & 1) ? -kStays : kStays; }
    bool stays = false;
    if (turned) stays = pairs_of(g, c, seq, token);
    some_stay = __builtin_amdgcn_ballot_w64(stays) != 0ull;
  }
  __device__ __forceinline__ bool pairs_of(const RotateArgs& g, uint32_t c, uint32_t seq, uint32_t token) {
    bool stays = false;
    const uint32_t first = ADJACENT ? 4u * c : (lower ? 8u * c : 8u * c - g.pairs);
    const int32_t* at = g.at + g.seq_step * (int64_t)seq + token;
#pragma unroll
    for (int i = 0; i < (ADJACENT ? 4 : 8); ++i) {
      const uint32_t axis = g.axis ? g.axis[first + i] : 0u;
      if (axis >= g.axes) { stays = true; continue; }
      float co, si;
      turn_of(at[g.axis_step * (int64_t)axis], (double)g.freq[first + i] * 0.15915494309189535, &co, &si);
      if constexpr (ADJACENT) { cos[2 * i] = cos[2 * i + 1] = co; sin[2 * i] = -si; sin[2 * i + 1] = si; }
      else { cos[i] = co; sin[i] = lower ? -si : si; }
    }
    return stays;
  }
  // The partners of a row's values, in the type; 0 where a value stays.  y_e = u_e cos + u_partner sin.
  __device__ __forceinline__ u32x4 partners(const u32x4& raw) const {
    u32x4 other;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t x;
      if constexpr (ADJACENT) x = raw[w] << 16 | raw[w] >> 16;
      else x = (uint32_t)__shfl((int)raw[w], (int)partner_of(threadIdx.x & 63u), 64);
      other[w] = turned ? x : 0u;
    }
    if (some_stay) {
#pragma unroll
      for (int e = ADJACENT ? 1 : 0; e < 8; e += ADJACENT ? 2 : 1) {
        float s = sin[e];
        asm volatile("" : "+v"(s));  // (compared here, not ahead of the loop over heads: there are no registers to keep it in)
        other[e >> 1] &= s != kStays ? ~0u : ADJACENT ? 0u : e & 1 ? 0xFFFFu : 0xFFFF0000u;
      }
    }
    return other;
  }
};

// 1 / sqrt(mean x^2 + eps) of a row.  Squares of bf16 may pass the range of fp32: such a row is taken 2^-96 as large, and eps 2^-192;
// x becomes x times the factor.
template <class T, int D>
__device__ __forceinline__ float norm_of(float (&x)[8], float eps, float* factor) {
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
  ss = row_sum<D>(ss);
  *factor = 1.f;
  if constexpr (std::is_same<T, Bf16>::value) {
    const bool far = ss > 0x1p100f;
    if (__builtin_amdgcn_ballot_w64(far) != 0ull) {
      const float by = far ? 0x1p-96f : 1.f;
      float small = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) { x[e] *= by; small = __builtin_fmaf(x[e], x[e], small); }
      small = row_sum<D>(small);
      if (far) { ss = small; eps = eps * 0x1p-96f * 0x1p-96f; *factor = by; }  // (one factor of 2^-192 would be 0)
    }
  }
  return __builtin_amdgcn_rsqf(__builtin_fmaf(ss, 1.0f / D, eps));
}

// Which rows of a workgroup's tokens and heads a thread has: token `token` of the tile, heads `head`, head + step, ..
struct Mine {
  uint32_t token, head, slot, c;
};
template <int D>
__device__ __forceinline__ Mine mine_of(const RotateArgs& g) {
  constexpr uint32_t kLanes = D / 8, kSlots = kThreads / kLanes;
  Mine m;
  m.c = threadIdx.x % kLanes;
  m.slot = threadIdx.x / kLanes;
  const uint32_t step_log2 = __builtin_ctz(kSlots) - g.tile_log2;
  m.token = g.heads_first ? m.slot >> step_log2 : m.slot & ((1u << g.tile_log2) - 1u);
  m.head = g.heads_first ? m.slot & ((1u << step_log2) - 1u) : m.slot >> g.tile_log2;
  return m;
}

// Goes over heads first .. end - 1 of a tensor, `step` apart: load(i, head, there) of a few at a time, then work(i, head, there).
template <uint32_t AT_ONCE, class Load, class Work>
__device__ __forceinline__ void over_heads(uint32_t first, uint32_t end, uint32_t step, uint32_t mine, Load load, Work work) {
  for (uint32_t h0 = first; h0 < end; h0 += step * AT_ONCE) {
#pragma unroll
    for (uint32_t i = 0; i < AT_ONCE; ++i) {
      const uint32_t h = h0 + step * i + mine;
      if (h0 + step * i < end) load(i, h < end ? h : end - 1u);
    }
#pragma unroll
    for (uint32_t i = 0; i < AT_ONCE; ++i) {
      const uint32_t h = h0 + step * i + mine;
      if (h0 + step * i < end) work(i, h < end ? h : end - 1u, h < end);
    }
  }
}

// Bound by memory.  In sequences of 8192 tokens with 32/8 heads of 128 of bf16 side by side, four of them on three axes, 671 MB take
// 149.5 us (4490 GB/s; a copy 5120).  What counts is the order of the rows: neighbouring lanes take those that are neighbours in memory, heads
// of a token here; with tokens in their place, 8 KB apart and so on few of the L2's channels, 173 us.  Eight rows of a thread in
// flight 148, four 161 (into a cache, whose rows take more registers: four 39.7 us for 12001 tokens, eight 45).  Rows are read past
// the caches, once: 161 us and 39.7, through them 163 and 44.  (Compared before pairs without an axis had their mark: 148 then.)
// 12001 tokens of 16/8 heads of 128 into a cache: in 16 bits 40 to 42 us with neighbours for pairs and 54 with halves, however many are
// turned, 197 MB; into e4m3 45 to 47 and 60, 172 MB.  Halves take registers for 8 sines and cosines, where neighbours share 4: three
// workgroups to a compute unit and four rounds of them, four and three with neighbours.
// WRITE: 0 keys go to a tensor, 1 to a cache in 16 bits, 2 to one of e4m3 codes; so do values then.
template <class T, int D, bool ADJACENT, int WRITE>
__global__ __launch_bounds__(kThreads) void kp_norm_rotate_rows(RotateArgs g) {
  constexpr uint32_t kSlots = kThreads / (D / 8), kAtOnce = WRITE == 0 ? 8 : 4;
  const Mine m = mine_of<D>(g);
  const uint32_t step = kSlots >> g.tile_log2;
  const uint32_t begin = blockIdx.y * g.chunk, end = begin + g.chunk;  // of the heads of all tensors, one behind the other
  Turn<ADJACENT> turn(g, m.c);
  for (uint32_t t = blockIdx.x; t < g.tiles; t += gridDim.x) {
    const uint32_t n = (t << g.tile_log2) + m.token, at = n < g.tokens ? n : g.tokens - 1u;
    const uint32_t seq = at / g.per_seq, token = at - seq * g.per_seq;
    int64_t slot = 0;
    if constexpr (WRITE != 0) slot = g.slots[at];
    turn.angles(g, m.c, seq, token);
    uint32_t before = 0;  // heads of the tensors ahead
#pragma unroll
    for (int w = 0; w < (WRITE != 0 ? 3 : 2); ++w) {
      const uint32_t heads = g.heads[w == 0 ? 0 : 1], first = begin > before ? begin - before : 0u, last = end > before ? min(end - before, heads) : 0u;
      before += heads;
      if (first >= last) continue;
      const Heads src = w == 2 ? g.v : g.x[w & 1], dst = g.y[w & 1];
      const uint16_t* const from = src.at + src.seq * (int64_t)seq + src.token * (int64_t)token + 8u * m.c;
      uint16_t* const to = const_cast<uint16_t*>(dst.at) + dst.seq * (int64_t)seq + dst.token * (int64_t)token + 8u * m.c;
      const bool cached = WRITE != 0 && w != 0, normed = w != 2 && g.weight[w & 1] != nullptr;
      const bool there = n < g.tokens && (!cached || (slot >= 0 && (uint64_t)slot < g.n_slots));
      float a[8], b[8];
      if (w != 2) {
        weights_of<T>(g.weight[w & 1], g.fp32_weights != 0u, 8u * m.c, a);
        weights_of<T>(g.weight[w & 1], g.fp32_weights != 0u, 8u * turn.partner_of(m.c), b);
        if constexpr (ADJACENT)
#pragma unroll
          for (int e = 0; e < 8; e += 2) { const float x = b[e]; b[e] = b[e + 1]; b[e + 1] = x; }
#pragma unroll
        for (int e = 0; e < 8; ++e) { a[e] *= turn.cos[e]; b[e] = __builtin_fabsf(turn.sin[e]) == kStays ? -0.f : b[e] * turn.sin[e]; }  // (-0: what it is added to keeps its sign)
      }
      u32x4 raw[kAtOnce];
      over_heads<kAtOnce>(
          first, last, step, m.head, [&](uint32_t i, uint32_t h) __attribute__((always_inline)) { raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + src.head * (int64_t)h)); },
          [&](uint32_t i, uint32_t h, bool is_head) __attribute__((always_inline)) {
            u32x4 out = raw[i];
            if (w != 2) {
              float x[8], o[8], y[8], r = 1.f, factor = 1.f;
              widen<T>(raw[i], x);
              widen<T>(turn.partners(raw[i]), o);
              if (normed) r = norm_of<T, D>(x, g.eps, &factor);
              const float r_o = r * factor;
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(r * x[e], a[e], (r_o * o[e]) * b[e]);
              out = narrow<T>(y);
            }
            if (!there || !is_head) return;
            if (cached) {
              const uint32_t row = row_of_slot((uint64_t)slot, h, g.heads[1], g.page_log2);
              put_row<T, D, WRITE == 2>(out, w == 2 ? g.v_cache : g.k_cache, w == 2 ? g.v_exp : g.k_exp, row, m.c);
            } else {
              *reinterpret_cast<u32x4*>(to + dst.head * (int64_t)h) = out;
            }
          });
    }
  }
}

// Bound by memory: 8192 tokens of 32/8 heads of 128, 252 MB, take 52 us with the join (4810 GB/s; the kernel 48.6 of them); before the join had eight loads in flight 59, with 512, 1024 and 256
// workgroups instead of 768 67, 74 and 98.
template <class T, int D, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void kp_norm_rotate_back(RotateArgs g) {
  constexpr uint32_t kSlots = kThreads / (D / 8), kBackAtOnce = 4;
  __shared__ float sums[kSlots][D];
  const Mine m = mine_of<D>(g);
  const uint32_t step = kSlots >> g.tile_log2;
  const uint32_t begin = blockIdx.y * g.chunk, end = begin + g.chunk;
  Turn<ADJACENT> turn(g, m.c);
  float dw[2][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;
  for (uint32_t t = blockIdx.x; t < g.tiles; t += gridDim.x) {
    const uint32_t n = (t << g.tile_log2) + m.token, at = n < g.tokens ? n : g.tokens - 1u;
    const uint32_t seq = at / g.per_seq, token = at - seq * g.per_seq;
    turn.angles(g, m.c, seq, token);
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t heads = g.heads[w], first = begin > before ? begin - before : 0u, last = end > before ? min(end - before, heads) : 0u;
      before += heads;
      if (first >= last) continue;
      const Heads src = g.x[w], in = g.in[w], dst = g.y[w];
      const bool normed = g.weight[w] != nullptr;
      const uint16_t* const from = src.at + src.seq * (int64_t)seq + src.token * (int64_t)token + 8u * m.c;
      const uint16_t* const from_x = normed ? in.at + in.seq * (int64_t)seq + in.token * (int64_t)token + 8u * m.c : from;
      uint16_t* const to = const_cast<uint16_t*>(dst.at) + dst.seq * (int64_t)seq + dst.token * (int64_t)token + 8u * m.c;
      float weight[8];
      weights_of<T>(g.weight[w], g.fp32_weights != 0u, 8u * m.c, weight);
      u32x4 raw[kBackAtOnce], raw_x[kBackAtOnce];
      over_heads<kBackAtOnce>(
          first, last, step, m.head,
          [&](uint32_t i, uint32_t h) __attribute__((always_inline)) {
            raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + src.head * (int64_t)h));
            if (normed) raw_x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from_x + in.head * (int64_t)h));
          },
          [&](uint32_t i, uint32_t h, bool is_head) __attribute__((always_inline)) {
            const bool there = n < g.tokens && is_head;
            float d[8], o[8], y[8];
            widen<T>(raw[i], d);
            widen<T>(turn.partners(raw[i]), o);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(d[e], turn.cos[e], -o[e] * turn.sin[e]);
            if (normed) {
              float x[8], factor, dot = 0.f;
              widen<T>(raw_x[i], x);
              const float r = norm_of<T, D>(x, g.eps, &factor);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                x[e] *= r;
                dw[w][e] = there ? __builtin_fmaf(y[e], x[e], dw[w][e]) : dw[w][e];
                y[e] *= weight[e];
                dot = __builtin_fmaf(y[e], x[e], dot);
              }
              dot = row_sum<D>(dot) * (1.0f / D);
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = r * factor * __builtin_fmaf(-x[e], dot, y[e]);
            }
            if (there) *reinterpret_cast<u32x4*>(to + dst.head * (int64_t)h) = narrow<T>(y);
          });
    }
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    if (!g.weight[w]) continue;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[m.slot][8u * m.c + e] = dw[w][e];
    __syncthreads();
    if (threadIdx.x < (uint32_t)D) {
      float s = 0.f;
      for (uint32_t i = 0; i < kSlots; ++i) s += sums[i][threadIdx.x];
      g.part[((size_t)w * gridDim.x * gridDim.y + blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = s;
    }
  }
}

// The workgroups' sums of d_w, added up: 32 values of a head to a workgroup, blockIdx.y: queries' or keys'.
constexpr uint32_t kJoinRows = 32;
__global__ __launch_bounds__(32 * kJoinRows) void kp_norm_rotate_join(RotateArgs g, uint32_t rows, uint32_t D) {
  __shared__ float sums[kJoinRows][33];
  const uint32_t w = blockIdx.y, c = threadIdx.x & 31u, r = threadIdx.x >> 5;
  if (!g.weight[w]) return;
  const uint32_t d = 32u * blockIdx.x + c;
  const float* const part = g.part + (size_t)w * rows * D + d;
  float s = 0.f;
#pragma unroll 8
  for (uint32_t i = r; i < rows; i += kJoinRows) s += part[(size_t)i * D];
  sums[r][c] = s;
  __syncthreads();
  if (r != 0u) return;
  for (uint32_t i = 1; i < kJoinRows; ++i) s += sums[i][c];
  g.d_weight[w][d] = s;
}

// ---- the host -------------------------------------------------------------------------------------------------------

kp_status check_sizes(int B, int Hq, int Hk, int S, int D, int type, int weight_type, float eps, bool normed) {
  if (B < 0 || Hq < 0 || Hk < 0 || S < 0) return kp::fail(KP_ERR_INVALID_ARG, "B, Hq, Hk and S must not be negative");
  if (type != KP_BF16 && type != KP_FP16) return kp::fail(KP_ERR_INVALID_ARG, "type must be KP_BF16 or KP_FP16");
  if (normed && weight_type != type && weight_type != KP_FP32) return kp::fail(KP_ERR_INVALID_ARG, "weight_type must be the type or KP_FP32");
  if (normed && !(eps >= 1e-30f && eps <= 1e30f)) return kp::fail(KP_ERR_INVALID_ARG, "eps must be from 1e-30 to 1e30");
  if (D != 64 && D != 128) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "D = %d must be 64 or 128", D);
  if ((long long)B * S >= kMostTokens) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^30 or more tokens");
  if (Hq > (1 << 16) || Hk > (1 << 16)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "more than 2^16 heads");
  return KP_OK;
}

kp_status check_weight(const char* name, const void* w) {
  return (uintptr_t)w & 15u ? kp::fail(KP_ERR_INVALID_ARG, "%s must be 16-byte aligned", name) : KP_OK;
}

kp_status check_turns(const kp_turns* t, int D) {
  if (!t || t->pairs == 0) return KP_OK;
  if (t->pairs < 0 || 2 * (long long)t->pairs > D) return kp::fail(KP_ERR_INVALID_ARG, "turns: pairs must be from 0 to D / 2");
  if (t->pairs & 7) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "turns: pairs must be a multiple of 8");
  if (t->axes < 1 || t->axes > 255) return kp::fail(KP_ERR_INVALID_ARG, "turns: axes must be from 1 to 255");
  if (t->adjacent != 0 && t->adjacent != 1) return kp::fail(KP_ERR_INVALID_ARG, "turns: adjacent must be 0 or 1");
  if (!t->at || ((uintptr_t)t->at & 3u)) return kp::fail(KP_ERR_INVALID_ARG, "turns: at must be device memory, 4-byte aligned");
  if (!t->freq || ((uintptr_t)t->freq & 3u)) return kp::fail(KP_ERR_INVALID_ARG, "turns: freq must be device memory, 4-byte aligned");
  if (t->axis_step < 0 || t->seq_step < 0) return kp::fail(KP_ERR_INVALID_ARG, "turns: negative steps");
  return KP_OK;
}

// `out` may be the tensor that it is made of, but then every row has to lie where it was.
kp_status check_pair(const char* in_name, const char* out_name, const kp_heads* in, const kp_heads* out, int B, int H, int S, int D) {
  if (kp_status s = check_heads(in_name, in, B, H, S, D, false)) return s;
  if (kp_status s = check_heads(out_name, out, B, H, S, D, true)) return s;
  if (in->at == out->at && ((B > 1 && in->seq != out->seq) || (H > 1 && in->head != out->head) || (S > 1 && in->token != out->token)))
    return kp::fail(KP_ERR_INVALID_ARG, "%s lies where %s does, with other strides", out_name, in_name);
  return KP_OK;
}

void set_turns(RotateArgs& g, const kp_turns* t) {
  if (!t || t->pairs == 0) return;
  g.at = t->at; g.axis_step = t->axis_step; g.seq_step = t->seq_step;
  g.freq = t->freq; g.axis = t->axis; g.pairs = (uint32_t)t->pairs; g.axes = (uint32_t)t->axes;
}

// Tokens and heads of a workgroup.
constexpr uint32_t kWanted = 1024, kBackWanted = 768, kMostTiles = 1u << 16;  // (a workgroup goes on with further tiles)
struct RotatePlan {
  uint32_t groups, chunks;  // of tokens, of heads
};
RotatePlan plan_rows(RotateArgs& g, int tokens, int per_seq, int Hq, int Hk, int Hv, int D, bool heads_first) {
  const uint32_t slots = kThreads / (uint32_t)(D / 8), rows = slots / 4u;  // of a workgroup, of a wave
  g.tokens = (uint32_t)tokens; g.per_seq = (uint32_t)per_seq;
  g.heads[0] = (uint32_t)Hq; g.heads[1] = (uint32_t)Hk;
  g.heads_first = heads_first;
  uint32_t most = slots;
  if (heads_first) {
    uint32_t step = 1u;
    while (step < rows && step < (uint32_t)(Hq > Hk ? Hq : Hk)) step *= 2u;
    most = slots / step;
  }
  while ((1u << g.tile_log2) < most && (1u << g.tile_log2) < g.tokens) ++g.tile_log2;
  g.tiles = (g.tokens + (1u << g.tile_log2) - 1u) >> g.tile_log2;
  const uint32_t all = (uint32_t)(Hq + Hk + Hv), step = slots >> g.tile_log2;
  RotatePlan p;
  g.chunk = (all + step - 1u) / step * step;
  while (g.chunk > step && (uint64_t)g.tiles * ((all + g.chunk - 1u) / g.chunk) < kWanted) g.chunk = (g.chunk / step + 1u) / 2u * step;
  p.chunks = (all + g.chunk - 1u) / g.chunk;
  p.groups = g.tiles < kMostTiles ? g.tiles : kMostTiles;
  return p;
}

// Do heads of a token lie closer together than tokens of a head?  As the first tensor has it.
bool heads_first(const RotateArgs& g) {
  const Heads& x = g.x[g.x[0].at ? 0 : 1];
  return x.head < x.token;
}

#define KP_PICK_ADJACENT(T, D, ...) do { if (adjacent) KP_LAUNCH(T, D, true, ##__VA_ARGS__); else KP_LAUNCH(T, D, false, ##__VA_ARGS__); } while (0)
#define KP_PICK_D(T, ...) do { if (D == 64) KP_PICK_ADJACENT(T, 64, ##__VA_ARGS__); else KP_PICK_ADJACENT(T, 128, ##__VA_ARGS__); } while (0)
#define KP_PICK_TYPE(...) do { if (type == KP_FP16) KP_PICK_D(Fp16, ##__VA_ARGS__); else KP_PICK_D(Bf16, ##__VA_ARGS__); } while (0)

}  // namespace

extern "C" kp_status kp_norm_rotate(const kp_heads* q, const kp_heads* k, const void* q_weight, const void* k_weight, int weight_type,
                                    float eps, const kp_turns* turns, const kp_heads* q_out, const kp_heads* k_out, int B, int Hq,
                                    int Hk, int S, int D, int type, void* stream) {
  kp::clear_error();
  if (kp_status s = check_sizes(B, Hq, Hk, S, D, type, weight_type, eps, q_weight || k_weight)) return s;
  if (kp_status s = check_weight("q_weight", q_weight)) return s;
  if (kp_status s = check_weight("k_weight", k_weight)) return s;
  if (B == 0 || S == 0 || (Hq == 0 && Hk == 0)) return KP_OK;
  if (kp_status s = check_turns(turns, D)) return s;
  RotateArgs g{};
  if (Hq > 0) {
    if (kp_status s = check_pair("q", "q_out", q, q_out, B, Hq, S, D)) return s;
    g.x[0] = heads_of(q, B, Hq, S); g.y[0] = heads_of(q_out, B, Hq, S);
  }
  if (Hk > 0) {
    if (kp_status s = check_pair("k", "k_out", k, k_out, B, Hk, S, D)) return s;
    g.x[1] = heads_of(k, B, Hk, S); g.y[1] = heads_of(k_out, B, Hk, S);
  }
  g.weight[0] = q_weight; g.weight[1] = k_weight; g.fp32_weights = weight_type == KP_FP32; g.eps = eps;
  set_turns(g, turns);
  const RotatePlan plan = plan_rows(g, B * S, S, Hq, Hk, 0, D, heads_first(g));
  const bool adjacent = g.pairs && turns->adjacent;
  const dim3 grid(plan.groups, plan.chunks);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define KP_LAUNCH(T, D, A) hipLaunchKernelGGL((kp_norm_rotate_rows<T, D, A, 0>), grid, dim3(kThreads), 0, st, g)
  KP_PICK_TYPE();
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}

extern "C" kp_status kp_norm_rotate_write(const kp_heads* q, const kp_heads* k, const kp_heads* v, const void* q_weight,
                                          const void* k_weight, int weight_type, float eps, const kp_turns* turns, const kp_heads* q_out,
                                          const int64_t* slots, int T, int Hq, const kp_cache* cache, void* stream) {
  kp::clear_error();
  if (kp_status s = check_cache(cache)) return s;
  const int Hk = cache->Hkv, D = cache->D, type = cache->type;
  if (kp_status s = check_sizes(1, Hq, Hk, T, D, type, weight_type, eps, q_weight || k_weight)) return s;
  if (kp_status s = check_weight("q_weight", q_weight)) return s;
  if (kp_status s = check_weight("k_weight", k_weight)) return s;
  if (T == 0) return KP_OK;
  if (kp_status s = check_turns(turns, D)) return s;
  if (!slots || ((uintptr_t)slots & 7u)) return kp::fail(KP_ERR_INVALID_ARG, "slots must be device memory, 8-byte aligned");
  RotateArgs g{};
  if (Hq > 0) {
    if (kp_status s = check_pair("q", "q_out", q, q_out, 1, Hq, T, D)) return s;
    g.x[0] = heads_of(q, 1, Hq, T); g.y[0] = heads_of(q_out, 1, Hq, T);
  }
  if (kp_status s = check_heads("k", k, 1, Hk, T, D, false)) return s;
  if (kp_status s = check_heads("v", v, 1, Hk, T, D, false)) return s;
  g.x[1] = heads_of(k, 1, Hk, T); g.v = heads_of(v, 1, Hk, T);
  g.weight[0] = q_weight; g.weight[1] = k_weight; g.fp32_weights = weight_type == KP_FP32; g.eps = eps;
  set_turns(g, turns);
  g.slots = slots;
  g.k_cache = static_cast<uint8_t*>(cache->k); g.v_cache = static_cast<uint8_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp; g.page_log2 = log2_of(cache->page);
  g.n_slots = (uint64_t)cache->n_pages * (uint64_t)cache->page;
  const RotatePlan plan = plan_rows(g, T, T, Hq, Hk, Hk, D, heads_first(g));
  const bool adjacent = g.pairs && turns->adjacent;
  const dim3 grid(plan.groups, plan.chunks);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define KP_LAUNCH(T, D, A, W) hipLaunchKernelGGL((kp_norm_rotate_rows<T, D, A, W>), grid, dim3(kThreads), 0, st, g)
  if (cache->cache_type == KP_CACHE_E4M3) KP_PICK_TYPE(2); else KP_PICK_TYPE(1);
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}

// The gradient: each workgroup leaves its sums of d_w, so that there are fewer, each with more tiles.
static RotatePlan plan_back(RotateArgs& g, int tokens, int per_seq, int Hq, int Hk, int D, bool heads_first) {
  RotatePlan p = plan_rows(g, tokens, per_seq, Hq, Hk, 0, D, heads_first);
  const uint32_t most = kBackWanted / p.chunks;
  if (p.groups > most) p.groups = most > 1u ? most : 1u;
  return p;
}

extern "C" size_t kp_norm_rotate_grad_bytes(int B, int Hq, int Hk, int S, int D) {
  if (check_sizes(B, Hq, Hk, S, D, KP_BF16, KP_BF16, 1.f, true) || B == 0 || S == 0 || (Hq == 0 && Hk == 0)) return 0;
  size_t rows = 0;
  for (int first = 0; first < 2; ++first) {
    RotateArgs g{};
    const RotatePlan p = plan_back(g, B * S, S, Hq, Hk, D, first != 0);
    const size_t n = (size_t)p.groups * p.chunks;
    rows = n > rows ? n : rows;
  }
  return 2 * rows * (size_t)D * sizeof(float);
}

extern "C" kp_status kp_norm_rotate_grad(const kp_heads* q, const kp_heads* k, const void* q_weight, const void* k_weight, int weight_type,
                                         float eps, const kp_turns* turns, const kp_heads* d_q_out, const kp_heads* d_k_out,
                                         const kp_heads* dq, const kp_heads* dk, float* dq_weight, float* dk_weight, int B, int Hq, int Hk,
                                         int S, int D, int type, void* workspace, size_t workspace_bytes, void* stream) {
  kp::clear_error();
  if (kp_status s = check_sizes(B, Hq, Hk, S, D, type, weight_type, eps, q_weight || k_weight)) return s;
  if (kp_status s = check_weight("q_weight", q_weight)) return s;
  if (kp_status s = check_weight("k_weight", k_weight)) return s;
  if ((q_weight && (!dq_weight || ((uintptr_t)dq_weight & 3u))) || (k_weight && (!dk_weight || ((uintptr_t)dk_weight & 3u))))
    return kp::fail(KP_ERR_INVALID_ARG, "dq_weight and dk_weight must be device memory, 4-byte aligned, where there are weights");
  const bool rows = B > 0 && S > 0;
  if (rows)
    if (kp_status s = check_turns(turns, D)) return s;
  RotateArgs g{};
  if (rows && Hq > 0) {
    if (kp_status s = check_pair("d_q_out", "dq", d_q_out, dq, B, Hq, S, D)) return s;
    g.x[0] = heads_of(d_q_out, B, Hq, S); g.y[0] = heads_of(dq, B, Hq, S);
    if (q_weight) {
      if (kp_status s = check_pair("q", "dq", q, dq, B, Hq, S, D)) return s;
      g.in[0] = heads_of(q, B, Hq, S);
    }
  }
  if (rows && Hk > 0) {
    if (kp_status s = check_pair("d_k_out", "dk", d_k_out, dk, B, Hk, S, D)) return s;
    g.x[1] = heads_of(d_k_out, B, Hk, S); g.y[1] = heads_of(dk, B, Hk, S);
    if (k_weight) {
      if (kp_status s = check_pair("k", "dk", k, dk, B, Hk, S, D)) return s;
      g.in[1] = heads_of(k, B, Hk, S);
    }
  }
  g.weight[0] = q_weight; g.weight[1] = k_weight; g.fp32_weights = weight_type == KP_FP32; g.eps = eps;
  g.d_weight[0] = dq_weight; g.d_weight[1] = dk_weight;
  RotatePlan plan{};
  if (rows && (Hq > 0 || Hk > 0)) {
    set_turns(g, turns);
    plan = plan_back(g, B * S, S, Hq, Hk, D, heads_first(g));
  }
  if (q_weight || k_weight)
    if (kp_status s = check_workspace(workspace, workspace_bytes, kp_norm_rotate_grad_bytes(B, Hq, Hk, S, D))) return s;
  g.part = static_cast<float*>(workspace);
  const bool adjacent = g.pairs && turns->adjacent;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (plan.groups) {
    const dim3 grid(plan.groups, plan.chunks);
#define KP_LAUNCH(T, D, A) hipLaunchKernelGGL((kp_norm_rotate_back<T, D, A>), grid, dim3(kThreads), 0, st, g)
    KP_PICK_TYPE();
#undef KP_LAUNCH
    KP_HIP_TRY(hipGetLastError());
  }
  if (q_weight || k_weight) {
    hipLaunchKernelGGL(kp_norm_rotate_join, dim3((uint32_t)D / 32u, 2), dim3(32 * kJoinRows), 0, st, g, plan.groups * plan.chunks, (uint32_t)D);
    KP_HIP_TRY(hipGetLastError());
  }
  return KP_OK;
}
