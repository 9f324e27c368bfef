// Gradients of attention with a sliding window and sinks (kp_attn_window_grad).
//
// With P_ij = exp2(scale log2(e) q_i.k_j - lse_i log2(e)) and delta_i = d_o_i . o_i (= sum_j P_ij d_o_i . v_j):
//   dS_ij = P_ij (d_o_i . v_j - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij d_o_i.
// Two kernels, both of which form S and d_o v^T for themselves: one goes over the keys of a tile of query rows (dq), the
// other over the query rows that see a tile of keys (dk, dv).  That is seven products instead of the five that one kernel
// would need, which would have to add up dq with atomics, in an order that changes from run to run.
#include "kp_attn_host.h"
#include "kp_attn_rows.h"

using namespace kp::attn;

namespace {

constexpr int kGradKeys = 128;   // keys of a workgroup of the dk, dv kernel

// fp16 holds little below 2^-14, and P and dS are often smaller: they are rounded to it times a power of two that their
// factors leave room for.  P <= 1 times 2^kShiftP; dS, of the order of |d_o|, times 2^kShiftS over the power of two of the
// largest |d_o| of the row (dq) or of all rows of the key's heads (dk).  What overflows all the same is not finite and is
// taken again in fp32.  bf16 has the exponents of fp32 and needs none of it.
template <class T> constexpr float kShiftP = 0.f;
template <> constexpr float kShiftP<Fp16> = 14.f;
constexpr int kShiftS = 5;

struct GradArgs {
  Heads q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
  float *neg, *delta;  // workspace, [B, Hq, Sq]: kShiftP - lse log2(e), and d_o . o
  float* most;         // fp16: largest finite |d_o| of every row tile, [B, Hkv, row tiles]
  float* part;         // partial dk, dv: [worker][first, last tile][dk, dv][kGradKeys][D]
  uint32_t seqs, hkv, group, n_q, n_k, window, sinks;
  uint32_t row_tiles, key_tiles, sink_tiles;  // of one head of keys; sink_tiles: key tiles that all later tokens see, for their sinks
  uint32_t workers;               // workgroups of kp_grad_keys; a multiple of 8 where B Hkv is one
  uint32_t whole;                 // tiles of a line that are taken whole
  float scale, scale_log2;
};

__device__ __forceinline__ const uint16_t* row_at(const Heads& t, uint32_t seq, uint32_t head, uint32_t token) {
  return t.at + t.seq * (int64_t)seq + t.head * (int64_t)head + t.token * (int64_t)token;
}
__device__ __forceinline__ bool sees(int32_t p, uint32_t j, uint32_t window, uint32_t sinks) {
  return ((int32_t)j <= p) & ((window == 0u) | ((uint32_t)p - j < window) | (j < sinks));
}
template <class T, int E>
__device__ __forceinline__ void load_row(const uint16_t* at, float (&out)[E]) {
  row_elements<T, E>(reinterpret_cast<const uint8_t*>(at), threadIdx.x & 63u, out);
}
template <int E>
__device__ __forceinline__ float dot(const float (&a)[E], const float (&b)[E]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) s = __builtin_fmaf(a[e], b[e], s);
  return wave_sum(s);
}
template <class T, int E>
__device__ __forceinline__ void put_row(uint16_t* at, const float (&x)[E], float by) {
  const uint32_t lane = threadIdx.x & 63u;
  if constexpr (E == 1) at[lane] = (uint16_t)T::pack(x[0] * by, 0.f);
  else reinterpret_cast<uint32_t*>(at)[lane] = T::pack(x[0] * by, x[1] * by);
}

// One query row's gradient in fp32, by a wave; only keys that the row sees are touched.  For rows whose sums on the matrix
// instructions are not finite (as in kp_attn.h).
template <class T, int D>
__device__ __forceinline__ void query_row(const GradArgs& g, uint32_t seq, uint32_t head, uint32_t token, float neg, float delta, float (&dq)[D / 64]) {
  constexpr int E = D / 64;
  const uint32_t hk = head / g.group;
  float q[E], d_o[E];
  load_row<T, E>(row_at(g.q, seq, head, token), q);
  load_row<T, E>(row_at(g.d_o, seq, head, token), d_o);
#pragma unroll
  for (int e = 0; e < E; ++e) dq[e] = 0.f;
  const int32_t p = (int32_t)g.n_k - (int32_t)g.n_q + (int32_t)token;
  for (int32_t j = 0; j <= p; ++j) {
    if (!sees(p, (uint32_t)j, g.window, g.sinks)) { j = p - (int32_t)g.window; continue; }
    float k[E], v[E];
    load_row<T, E>(row_at(g.k, seq, hk, (uint32_t)j), k);
    load_row<T, E>(row_at(g.v, seq, hk, (uint32_t)j), v);
    const float w = __builtin_amdgcn_exp2f(dot<E>(q, k) * g.scale_log2 + (neg - kShiftP<T>)), ds = w * (dot<E>(d_o, v) - delta);
#pragma unroll
    for (int e = 0; e < E; ++e) dq[e] = __builtin_fmaf(ds, k[e], dq[e]);
  }
}

// Adds one key's gradients from the query tokens from .. to - 1 of one head.
template <class T, int D>
__device__ __forceinline__ void key_row(const GradArgs& g, uint32_t seq, uint32_t head, uint32_t j, uint32_t from, uint32_t to,
                                        const float (&k)[D / 64], const float (&v)[D / 64], float (&dk)[D / 64], float (&dv)[D / 64]) {
  constexpr int E = D / 64;
  for (uint32_t i = from; i < to; ++i) {
    if (!sees((int32_t)g.n_k - (int32_t)g.n_q + (int32_t)i, j, g.window, g.sinks)) continue;
    float q[E], d_o[E];
    load_row<T, E>(row_at(g.q, seq, head, i), q);
    load_row<T, E>(row_at(g.d_o, seq, head, i), d_o);
    const size_t at = ((size_t)seq * g.hkv * g.group + head) * g.n_q + i;
    const float w = __builtin_amdgcn_exp2f(dot<E>(q, k) * g.scale_log2 + (g.neg[at] - kShiftP<T>)), ds = w * (dot<E>(d_o, v) - g.delta[at]);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dk[e] = __builtin_fmaf(ds, q[e], dk[e]);
      dv[e] = __builtin_fmaf(w, d_o[e], dv[e]);
    }
  }
}

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
__device__ __forceinline__ float power_of_two_in(float x) {  // the largest power of two <= x (1 for 0), as a number
  const uint32_t e = __builtin_bit_cast(uint32_t, x) >> 23;
  return x == 0.f ? 1.f : __builtin_bit_cast(float, (e < 1u ? 1u : e) << 23);
}

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
  const int32_t p = off + (int32_t)at.token, p_min = position(wave_first), p_max = position(wave_first + 31u);
  const Span span = span_of(position(first), position(first + kTileRows - 1u), g.window, g.sinks);
  const uint32_t sink_tiles = (span.sink_end + 63u) / 64u, tiles = sink_tiles + (span.end > span.lo ? (span.end - span.lo + 63u) / 64u : 0u);

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
    float all = mine ? most : 0.f;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) all = fmaxf(all, __shfl_xor(all, d, 64));
    float* const most_of = reinterpret_cast<float*>(smem);
    if (lane == 0) most_of[wave] = all;
    __syncthreads();
    if (threadIdx.x == 0) g.most[(size_t)unit * g.row_tiles + (g.row_tiles - 1u - item)] = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3]));
    __syncthreads();  // (the tiles go there)
  }
  const float neg_p = kScaled ? neg - kShiftP<T> : neg;

  TileReader<D> rd((uint32_t)(uintptr_t)smem);
  TileLoader<D, 4> lk(g.k.token), lv(g.v.token);
  const uint32_t lds0 = kp::wave_uniform((uint32_t)(uintptr_t)smem + 1024u * wave);
  const uint16_t *k_head = row_at(g.k, seq, hk, 0), *v_head = row_at(g.v, seq, hk, 0);
  uint32_t loaded_last = ~0u, into = 0u;  // `into`: LDS offset of the buffer that the next tiles go to
  auto tile_start = [&](uint32_t t, uint32_t* limit) __attribute__((always_inline)) {
    *limit = t < sink_tiles ? span.sink_end : span.end;
    return t < sink_tiles ? t * 64u : span.lo + (t - sink_tiles) * 64u;
  };
  auto request = [&](uint32_t t) __attribute__((always_inline)) {
    uint32_t limit;
    const uint32_t start = tile_start(t, &limit), left = limit - 1u - start, last = left < 63u ? left : 63u;
    if (last != loaded_last) { loaded_last = last; lk.upto(last); lv.upto(last); }
    lk.load(k_head + g.k.token * (int64_t)start, lds0 + into);
    lv.load(v_head + g.v.token * (int64_t)start, lds0 + into + kTile);
    into ^= 2u * kTile;
  };

  f32x16 acc[ND];  // dq^T: rows d, column = row l32
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) acc[dt] = f32x16{0};
  // The operands of the three products come out of LDS LA MFMAs ahead, in one set of registers.
  constexpr int LA = 4;
  u32x4 ra[LA];
  uint32_t buffer = 0u;
  // operand n of the half tile tk: K rows, V rows, K^T; from 3 NS on the half after it
  auto fetch = [&](int n, int tk) __attribute__((always_inline)) {
    if (n >= 3 * NS) { n -= 3 * NS; tk ^= 1; }
    if (n < NS) return rd.rows(n, 32u * (uint32_t)tk, buffer);
    if (n < 2 * NS) return rd.rows(n - NS, 64u + 32u * (uint32_t)tk, buffer);
    return rd.cols((n - 2 * NS) % ND, 32u * (uint32_t)tk + 16u * (uint32_t)((n - 2 * NS) / ND), buffer);
  };
  float lacks = 0.f;
  // Over all keys; CHECK: with the sum of dS.
  auto over_keys = [&](auto check_c) __attribute__((always_inline)) {
    constexpr bool CHECK = decltype(check_c)::value;
    request(0u);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // (the compiler's own count of outstanding loads)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int n = 0; n < LA; ++n) ra[n] = fetch(n, 0);
    for (uint32_t t = 0; t < tiles; ++t) {
      if (t + 1u < tiles) request(t + 1u);
      uint32_t limit;
      const uint32_t start = tile_start(t, &limit);
      const int32_t end = (int32_t)(start + 64u);
      bool masked = (end > (int32_t)limit) | (end - 1 > p_min);
      masked = masked | ((g.window != 0u) & (p_max - (int32_t)start >= (int32_t)g.window) & (end > (int32_t)g.sinks));
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
          const RowMask m(p, limit, (int32_t)(start + 4u * h32), g.window, g.sinks);
          if ((g.window != 0u) & (start < g.sinks)) {
            asm volatile("");  // (branches: no selects where nothing is masked)
#pragma unroll
            for (int v = 0; v < 16; ++v) sacc[v] = m.sees_mixed(32 * tk + 8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
          } else {
            asm volatile("");
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
            buffer ^= 2u * kTile;
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
  // That enters dq as half a step of the type over the square root of the number of keys that count, which shows where a
  // row sees a few: tiles of up to 128 keys are gone over twice, first for the sum.
  if (tiles - 1u < 2u) {
    over_keys(yes);
    lacks += __shfl_xor(lacks, 32, 64);
    delta += __builtin_fabsf(lacks) < INFINITY ? lacks : 0.f;  // (a value that the row does not see may be in it)
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
      float out[D / 64];
      query_row<T, D>(g, seq, hk * g.group + a.in_group, a.token, __shfl(neg, r, 64), __shfl(delta, r, 64), out);
      put_row<T, D / 64>(const_cast<uint16_t*>(row_at(g.dq, seq, hk * g.group + a.in_group, a.token)), out, g.scale);
    }
  }
}

// Query tokens that see keys of key tile `kt`: [from, to).
struct Tokens {
  uint32_t from, to;
};
__device__ __forceinline__ Tokens tokens_of(const GradArgs& g, uint32_t kt) {
  const int64_t off = (int64_t)g.n_k - (int64_t)g.n_q, k0 = (int64_t)kt * kGradKeys;
  const int64_t k1 = k0 + kGradKeys < (int64_t)g.n_k ? k0 + kGradKeys : (int64_t)g.n_k;  // one past the last key
  int64_t from = k0 - off, to = g.window != 0u && k0 >= (int64_t)g.sinks ? k1 - 1 + (int64_t)g.window - off : (int64_t)g.n_q;
  from = from < 0 ? 0 : from;
  to = to > (int64_t)g.n_q ? (int64_t)g.n_q : to;
  Tokens t;
  t.from = from < (int64_t)g.n_q ? (uint32_t)from : g.n_q;
  t.to = to > from ? (uint32_t)to : t.from;
  return t;
}

// How the key tiles are dealt to the workers (a workgroup per CU).  Where the heads of keys can be dealt out to the 8 XCDs
// (and their L2s) evenly, each XCD's workers have heads of their own (a line).  Of a line's tiles every worker takes as many
// whole as there are for all, side by side, so that the rows that neighbouring tiles share are in L2 when they are asked
// for (with a run of tiles of its own for every worker 80 % of the requests missed it, this way 50 %), forwards and backwards in turn, since without a window the first are the longest.  What is left over, and the tiles that
// hold sinks, which all later tokens see, stand in a line step by step (64 tokens of one query head), of which every worker
// takes a piece that makes up for what its whole tiles are short of the others': a tile that does not lie whole in one piece
// leaves a partial sum for every worker that has a part, first or last in its piece, and kp_grad_join adds them up in order.
constexpr uint32_t kMostWorkers = 256, kTileCost = 4;  // kTileCost: steps' worth of time that a tile takes besides its steps
struct Line {
  uint32_t lines, number, units, workers;  // lines, this one, its heads and workers
  uint32_t sink_tiles, per_unit;           // of a head: tiles with sinks, the others
  uint32_t whole, rest;                    // tiles that are taken whole, tiles that are split
  uint32_t total;                          // steps of the latter
  // the n-th of the tiles that are not sinks'; the n-th that is split
  __device__ __forceinline__ void plain_tile(uint32_t n, uint32_t* unit, uint32_t* kt) const {
    const uint32_t u = n / per_unit;
    *unit = u * lines + number;
    *kt = sink_tiles + (n - u * per_unit);
  }
  __device__ __forceinline__ void split_tile(uint32_t n, uint32_t* unit, uint32_t* kt) const {
    if (n < units * sink_tiles) {
      const uint32_t u = n / sink_tiles;
      *unit = u * lines + number;
      *kt = n - u * sink_tiles;
    } else {
      plain_tile(whole + (n - units * sink_tiles), unit, kt);
    }
  }
};
__device__ __forceinline__ uint32_t steps_of(const GradArgs& g, uint32_t kt) {
  const Tokens t = tokens_of(g, kt);
  return (t.to - t.from + 63u) / 64u * g.group;
}
__device__ __forceinline__ uint32_t split_steps(const GradArgs& g, const Line& l, uint32_t n) {
  uint32_t unit, kt;
  l.split_tile(n, &unit, &kt);
  return steps_of(g, kt);
}
__device__ __forceinline__ uint32_t sum_over_wave(uint32_t x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += (uint32_t)__shfl_xor((int)x, d, 64);
  return kp::wave_uniform(x);
}
__device__ __forceinline__ uint32_t sum_up_to_lane(uint32_t x) {
  const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(x, d, 64);
    if (lane >= (uint32_t)d) x += up;
  }
  return x;
}
// Steps of the split tiles before number n, by a wave.
__device__ __forceinline__ uint32_t steps_before(const GradArgs& g, const Line& l, uint32_t n) {
  uint32_t sum = 0;
  for (uint32_t t0 = 0; t0 < n; t0 += 64u) {
    const uint32_t t = t0 + (threadIdx.x & 63u);
    sum += sum_over_wave(t < n ? split_steps(g, l, t) : 0u);
  }
  return sum;
}
__device__ __forceinline__ Line line_of(const GradArgs& g, uint32_t number, uint32_t lines) {
  Line l;
  l.lines = lines; l.number = number;
  l.units = g.seqs * g.hkv / lines; l.workers = g.workers / lines;
  l.sink_tiles = g.sink_tiles; l.per_unit = g.key_tiles - g.sink_tiles;
  const uint32_t plain = l.units * l.per_unit;
  l.whole = g.whole;
  l.rest = l.units * l.sink_tiles + (plain - l.whole);
  l.total = steps_before(g, l, l.rest);
  return l;
}
// The n-th whole tile of a worker.
__device__ __forceinline__ uint32_t whole_tile(const Line& l, uint32_t worker, uint32_t n) {
  return n * l.workers + ((n & 1u) ? l.workers - 1u - worker : worker);
}
// What a worker's whole tiles cost, in steps.
__device__ __forceinline__ uint32_t whole_cost(const GradArgs& g, const Line& l, uint32_t worker) {
  uint32_t sum = 0;
  for (uint32_t n = 0; n * l.workers < l.whole; ++n) {
    const uint32_t tile = whole_tile(l, worker, n);
    if (tile >= l.whole) continue;  // (the last round may not be full)
    uint32_t unit, kt;
    l.plain_tile(tile, &unit, &kt);
    sum += steps_of(g, kt) + kTileCost;
  }
  return sum;
}
// Calls f(worker, first step of its piece, one past its last) for 64 workers at a time, one to a lane of the wave.
template <class F>
__device__ __forceinline__ void for_pieces(const GradArgs& g, const Line& l, F f) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t all = l.total;
  for (uint32_t w0 = 0; w0 < l.workers; w0 += 64u) all += sum_over_wave(w0 + lane < l.workers ? whole_cost(g, l, w0 + lane) : 0u);
  const uint32_t each = (all + l.workers - 1u) / l.workers;  // (what all are short of it is the line's total or more)
  uint32_t before = 0;
  for (uint32_t w0 = 0; w0 < l.workers; w0 += 64u) {
    uint32_t short_of = 0;
    if (w0 + lane < l.workers) {
      const uint32_t has = whole_cost(g, l, w0 + lane);
      short_of = has < each ? each - has : 0u;
    }
    const uint32_t up_to = before + sum_up_to_lane(short_of), from = up_to - short_of;
    f(w0 + lane, from < l.total ? from : l.total, up_to < l.total ? up_to : l.total);
    before = __builtin_amdgcn_readlane(up_to, 63);
  }
}
// The split tile that step number x of the line belongs to, and the step's number in it.
__device__ __forceinline__ void split_at(const GradArgs& g, const Line& line, uint32_t x, uint32_t* n, uint32_t* in) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t before = 0;
  for (uint32_t t0 = 0; t0 < line.rest; t0 += 64u) {
    const uint32_t steps = t0 + lane < line.rest ? split_steps(g, line, t0 + lane) : 0u, sum = before + sum_up_to_lane(steps);
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum > x);
    if (past != 0ull) {
      const int l = __builtin_ctzll(past);
      *n = t0 + (uint32_t)l;
      *in = x - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(steps, l));
      return;
    }
    before = __builtin_amdgcn_readlane(sum, 63);
  }
  *n = line.rest;  // (not reached: x is a step of the line)
  *in = 0u;
}
__device__ __forceinline__ uint32_t lines_of(const GradArgs& g) { return ((g.seqs * g.hkv) & 7u) == 0u ? 8u : 1u; }

// dk and dv of 128 keys from a run of the query rows that see them.  A step is 64 tokens of one query head, whose Q and dO
// tiles are in LDS, three buffers each, with the rows' lse and delta.
// 8 waves, two to a group of 32 keys.  K and V rows, dk and dv of 32 keys of D = 128 would fill the registers of a wave that
// has a SIMD for itself (which issues too slowly: 2200 cycles for 32 rows, of which the matrix pipes need 1024); so the two
// waves of a group share the rows in the first two products, 32 each, give each other P and dS through LDS, and share d in
// the last two.  S^T = K Q^T and dP^T = V dO^T have a row to a lane, with its lse and delta; P and dS go to LDS as
// [row][key] and are read transposed, for dv^T += dO^T P and dk^T += Q^T dS, which have a key to a lane.
// S and dP are formed a step ahead: the exponentials stand between the MFMAs of dP, the rest of the vector work between
// those of dv.
constexpr int kKeysThreads = 512;
template <class T, int D>
__global__ __launch_bounds__(kKeysThreads, 2) void kp_grad_keys(GradArgs g) {
  constexpr uint32_t kRow = 2u * D, kTile = 64u * kRow, kBuffer = 2u * kTile;
  constexpr int NS = D / 16, NH = D / 64;  // NH: tiles of 32 d of a wave
  constexpr int LA = 4;                    // operands come out of LDS this many MFMAs ahead
  constexpr bool kScaled = std::is_same<T, Fp16>::value;
  extern __shared__ __align__(16) unsigned char smem[];
  // [three buffers of Q tile, dO tile][P of every wave: 2 KiB][dS, twice][three times neg, delta of 64 rows]
  constexpr uint32_t kShared = 3u * kBuffer, kSharedDs = kShared + 8u * 2048u, kStats = kSharedDs + 16u * 2048u;
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = kp::wave_uniform(tid >> 6), h32 = lane >> 5, l32 = lane & 31u;
  const uint32_t group_no = wave & 3u, hf = wave >> 2;  // of 32 keys; the wave's half of the rows and of d
  const Line line = line_of(g, lines_of(g) == 8u ? blockIdx.x & 7u : 0u, lines_of(g));
  const uint32_t worker = blockIdx.x / line.lines;
  const int32_t off = (int32_t)g.n_k - (int32_t)g.n_q;
  const uint32_t j_last = g.n_k - 1u;
  uint32_t at = 0u, to = 0u;  // its piece of the line
  for_pieces(g, line, [&](uint32_t w, uint32_t from, uint32_t end) __attribute__((always_inline)) {
    const uint64_t mine = __builtin_amdgcn_ballot_w64(w == worker);
    if (mine != 0ull) {
      at = __builtin_amdgcn_readlane(from, __builtin_ctzll(mine));
      to = __builtin_amdgcn_readlane(end, __builtin_ctzll(mine));
    }
  });
  uint32_t round = 0u, split_no = 0u, s_from = 0u;
  if (at < to) split_at(g, line, at, &split_no, &s_from);
  bool first_piece = true;

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
  while (round * line.workers < line.whole || at < to) {
    uint32_t unit, key_tile;
    const bool rounds = round * line.workers < line.whole;  // first the whole tiles
    if (rounds && whole_tile(line, worker, round) >= line.whole) {
      ++round;
      continue;
    }
    if (rounds) line.plain_tile(whole_tile(line, worker, round), &unit, &key_tile);
    else line.split_tile(split_no, &unit, &key_tile);
    const uint32_t seq = unit / g.hkv, hk = unit - seq * g.hkv;
    const Tokens tok = tokens_of(g, key_tile);
    const uint32_t steps_per_head = (tok.to - tok.from + 63u) / 64u, steps = steps_per_head * g.group;
    const uint32_t s_begin = rounds ? 0u : s_from, s_end = rounds || steps - s_begin <= to - at ? steps : s_begin + (to - at);
    const uint32_t slot = first_piece && s_begin != 0u ? 0u : 1u;
    if (rounds) {
      ++round;
    } else {
      at += s_end - s_begin;
      s_from = 0u;
      ++split_no;
      first_piece = false;
      if (s_begin == s_end) continue;  // (a tile that no token sees: kp_grad_join's)
    }
    const bool whole = s_begin == 0u && s_end == steps;

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
    float ds_scale = 1.f;  // dS is rounded times this (and 2^kShiftP, which is in P)
    if constexpr (kScaled) {
      float most = 0.f;
      for (uint32_t i = lane; i < g.row_tiles; i += 64u) most = fmaxf(most, g.most[(size_t)unit * g.row_tiles + i]);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
      ds_scale = __builtin_ldexpf(1.0f, kShiftS - (int)kShiftP<T>) / power_of_two_in(most);
    }

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
      ask_stat = (wave == 0u ? g.neg : g.delta) + ((size_t)seq * g.hkv * g.group + head) * g.n_q + ask_start;
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
        if (wave < 2u) {  // the rows' neg (wave 0) and delta (wave 1): 4 bytes to a lane
          const uint32_t ofs = 4u * (lane < loaded_last ? lane : loaded_last), dst = kp::wave_uniform((uint32_t)(uintptr_t)smem + kStats + into * 512u + 256u * wave);
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
    u32x2 pw[4], ds[4];  // P and dS: keys 8 i + 4 h32 .. + 3 of row l32
    uint32_t ds_now = 0u;  // which of the two dS in LDS is this step's
    uint32_t now = 0u, next = 0u;  // buffers of the step at hand and of the one whose S and dP are formed
    // Keeps a value that is not used before the next block of code where it is made: the compiler would move it there.
    auto stay = [](auto& x) __attribute__((always_inline)) { asm volatile("" : "+v"(x)); };
    // operands in the order of their use: Q and dO rows of the next step (this wave's half), dO^T and then Q^T of this one
    // (first of this wave's rows, then of the other's); behind them the next step's
    const uint32_t row_own = rd.row0 + 32u * hf * kRow, col_own = (rd.col0 ^ (64u * NH * hf)) + 32u * hf * kRow;
    const uint32_t col_other = (rd.col0 ^ (64u * NH * hf)) + 32u * (hf ^ 1u) * kRow;
    auto fetch = [&](int n) __attribute__((always_inline)) -> u32x4 {
      if (n >= 4 * NS) n -= 4 * NS;
      if (n < NS) return rd.rows_at((row_own ^ (32u * (uint32_t)n)) + next * kBuffer, 0u);
      if (n < 2 * NS) return rd.rows_at((row_own ^ (32u * (uint32_t)(n - NS))) + next * kBuffer, 64u);
      const int m = (n - 2 * NS) % NS, ks = m / NH, dt = m % NH;
      const uint32_t c = ks < 2 ? col_own : col_other, from = (n < 3 * NS ? 64u : 0u) + 16u * (uint32_t)(ks & 1);
      return rd.cols_at((c ^ (64u * (uint32_t)dt)) + now * kBuffer, (c ^ (64u * (uint32_t)dt + 32u)) + now * kBuffer, from);
    };
    // S of the wave's 32 rows of the step that starts at `start`: what is not visible becomes -inf
    auto hide = [&]() __attribute__((always_inline)) {
      const int32_t first = (int32_t)(start + 32u * hf), last = first + 31, k0 = (int32_t)j0, k1 = k0 + 31;
      if ((last >= (int32_t)tok.to) | (off + first < k1) | ((g.window != 0u) & (k1 >= (int32_t)g.sinks) & (off + last - k0 >= (int32_t)g.window))) {
        const int32_t token = first + (int32_t)l32;
        const RowMask m(token < (int32_t)tok.to ? off + token : -1, g.n_k, k0 + 4 * (int32_t)h32, g.window, g.sinks);
        if ((g.window == 0u) | (k0 >= (int32_t)g.sinks)) {
          asm volatile("");  // (branches: no selects where nothing is masked)
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = m.sees(8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
        } else if (off + first - k1 >= (int32_t)g.window) {  // sinks alone are left
          asm volatile("");
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = 8 * (v >> 2) + (v & 3) <= m.sink ? sacc[v] : -INFINITY;
        } else {
          asm volatile("");
#pragma unroll
          for (int v = 0; v < 16; ++v) sacc[v] = m.sees_mixed(8 * (v >> 2) + (v & 3)) ? sacc[v] : -INFINITY;
        }
      }
    };
    auto load_stats = [&]() __attribute__((always_inline)) {
      const float* const st = reinterpret_cast<const float*>(smem + kStats + next * 512u + 128u * hf) + l32;
      neg = st[0];
      delta = st[64];
    };
    auto exponential = [&](int v) __attribute__((always_inline)) {
      w[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[v], g.scale_log2, neg));
      stay(w[v]);
    };
    auto finish = [&](int v) __attribute__((always_inline)) {  // elements v, v + 1
      float x0 = w[v] * (dp[v] - delta), x1 = w[v + 1] * (dp[v + 1] - delta);
      if constexpr (kScaled) { x0 *= ds_scale; x1 *= ds_scale; }
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
#pragma unroll
    for (int v = 0; v < 16; ++v) exponential(v);
#pragma unroll
    for (int v = 0; v < 16; v += 2) finish(v);
    share_p();
#pragma unroll
    for (int i = 0; i < 4; ++i) share_ds(0u, i);
    wait_all();
    next = 1u;
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
          now = now == 2u ? 0u : now + 1u;
          next = next == 2u ? 0u : next + 1u;
        }
        dk[n % NH] = T::mfma32(ra[n % LA], rb[ks & 1], dk[n % NH]);
        ra[n % LA] = fetch(3 * NS + n + LA);
        __builtin_amdgcn_sched_barrier(0);
      }
      ds_now ^= 1u;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (what was asked for past the end has landed too)
    }

    const float by_k = kScaled ? g.scale / (ds_scale * __builtin_ldexpf(1.0f, (int)kShiftP<T>)) : g.scale;
    const float by_v = kScaled ? __builtin_ldexpf(1.0f, -(int)kShiftP<T>) : 1.f;
    uint64_t again = __builtin_amdgcn_ballot_w64((odd_of<NH>(dk) != 0.f || odd_of<NH>(dv) != 0.f) && j <= j_last);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    float* const part = g.part + (2u * (size_t)(worker * line.lines + line.number) + slot) * (2u * kGradKeys * D) + (size_t)(32u * group_no) * D;
    __syncthreads();  // (the tiles' room is used below)
    if (!whole) {
#pragma unroll
      for (int dt = 0; dt < NH; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* const out = part + l32 * D + 32u * (NH * hf + (uint32_t)dt) + 8 * i + 4 * h32;
          *reinterpret_cast<f32x4*>(out) = f32x4{dk[dt][4 * i] * by_k, dk[dt][4 * i + 1] * by_k, dk[dt][4 * i + 2] * by_k, dk[dt][4 * i + 3] * by_k};
          *reinterpret_cast<f32x4*>(out + kGradKeys * D) = f32x4{dv[dt][4 * i] * by_v, dv[dt][4 * i + 1] * by_v, dv[dt][4 * i + 2] * by_v, dv[dt][4 * i + 3] * by_v};
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
      for (uint32_t i = 0; i < 2u * kGradKeys * kChunks / kKeysThreads; ++i) {
        const uint32_t n = tid + i * kKeysThreads, r = n / kChunks % kGradKeys, chunk = (n % kChunks) ^ (r & 7u), key = key_tile * kGradKeys + r;
        const u32x4 v = *reinterpret_cast<const u32x4*>(smem + 16u * n);
        const Heads& out = n < kGradKeys * kChunks ? g.dk : g.dv;
        if (key <= j_last) *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(row_at(out, seq, hk, key)) + 8u * chunk) = (r & 8u) ? u32x4{v.z, v.w, v.x, v.y} : v;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the results have left, before some are put right
    __syncthreads();  // (and the next tile's rows go to the same room)
    for (; again != 0ull; again &= again - 1ull) {
      const uint32_t r = (uint32_t)__builtin_ctzll(again), key = j0 + r;
      constexpr int E = D / 64;
      float k[E], v[E], out_k[E] = {}, out_v[E] = {};
      load_row<T, E>(row_at(g.k, seq, hk, key), k);
      load_row<T, E>(row_at(g.v, seq, hk, key), v);
      for (uint32_t step = s_begin; step < s_end; ++step) {
        const uint32_t in_group = step / steps_per_head, first = tok.from + (step - in_group * steps_per_head) * 64u;
        key_row<T, D>(g, seq, hk * g.group + in_group, key, first, first + 64u < tok.to ? first + 64u : tok.to, k, v, out_k, out_v);
      }
      if (!whole) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          part[r * D + lane * E + e] = out_k[e] * g.scale;
          part[kGradKeys * D + r * D + lane * E + e] = out_v[e];
        }
      } else {
        put_row<T, E>(const_cast<uint16_t*>(row_at(g.dk, seq, hk, key)), out_k, g.scale);
        put_row<T, E>(const_cast<uint16_t*>(row_at(g.dv, seq, hk, key)), out_v, 1.f);
      }
    }
  }
}

// Adds up the parts of the split key tiles that do not lie whole in one worker's piece: D / 4 lanes to a row, a row to a lane;
// blockIdx.y: dk or dv.
template <int D> constexpr int kJoinRows = kThreads / (D / 4);
template <class T, int D>
__global__ __launch_bounds__(kThreads) void kp_grad_join(GradArgs g) {
  constexpr uint32_t kLanes = D / 4, kBlocks = kGradKeys / kJoinRows<D>;
  __shared__ const float* from[kMostWorkers];  // where the tile's parts are
  __shared__ uint32_t edge[kMostWorkers + 64u], ends[2], counts[4];  // where the workers' pieces begin; the first and the last that have a part
  const uint32_t lines = lines_of(g), tile = blockIdx.x / kBlocks;
  const Line line = line_of(g, tile % lines, lines);
  uint32_t unit, kt;
  line.split_tile(tile / lines, &unit, &kt);
  const uint32_t n = steps_of(g, kt);
  const uint32_t begin = steps_before(g, line, tile / lines), end = begin + n;
  if (threadIdx.x < 64u)
    for_pieces(g, line, [&](uint32_t w, uint32_t first, uint32_t last) __attribute__((always_inline)) {
      edge[w] = first;
      if (w + 1u == line.workers) edge[line.workers] = last;
    });
  __syncthreads();
  uint32_t parts = 0u;
  if (n != 0u) {
    if (threadIdx.x < line.workers) {
      if (edge[threadIdx.x] <= begin && begin < edge[threadIdx.x + 1u]) ends[0] = threadIdx.x;
      if (edge[threadIdx.x] < end && end <= edge[threadIdx.x + 1u]) ends[1] = threadIdx.x;
    }
    __syncthreads();
    if (ends[0] == ends[1]) return;  // one worker has all of it
    // their places, in the order of the workers, without those whose piece is empty
    const uint32_t w = ends[0] + threadIdx.x;
    const bool has = w <= ends[1] && edge[w] < edge[w + 1u];
    const uint64_t all = __builtin_amdgcn_ballot_w64(has);
    if ((threadIdx.x & 63u) == 0u) counts[threadIdx.x >> 6] = (uint32_t)__builtin_popcountll(all);
    __syncthreads();
    uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0u));
    for (uint32_t i = 0; i < (threadIdx.x >> 6); ++i) before += counts[i];
    parts = counts[0] + counts[1] + counts[2] + counts[3];
    if (has) {
      const size_t slot = 2u * (size_t)(w * line.lines + line.number) + (edge[w] > begin ? 0u : 1u);
      from[before] = g.part + slot * (2u * kGradKeys * D) + (size_t)blockIdx.y * (kGradKeys * D);
    }
    __syncthreads();
  }
  const uint32_t seq = unit / g.hkv, hk = unit - seq * g.hkv;
  const uint32_t c = threadIdx.x % kLanes, row = (blockIdx.x % kBlocks) * kJoinRows<D> + threadIdx.x / kLanes, j = kt * kGradKeys + row;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (uint32_t i = 0; i < parts; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(from[i] + row * D + 4u * c);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += x[e];
  }
  const Heads& out = blockIdx.y ? g.dv : g.dk;
  if (j < g.n_k) *reinterpret_cast<u32x2*>(const_cast<uint16_t*>(row_at(out, seq, hk, j)) + 4u * c) = u32x2{T::pack(sum[0], sum[1]), T::pack(sum[2], sum[3])};
}

// Tiles of a call, its workers and its workspace.
struct GradPlan {
  bool too_many;  // the steps of a line are counted in 32 bits
  long long units, row_tiles, key_tiles, sink_tiles, workers, whole, split;  // split: key tiles that kp_grad_join looks at
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
  const long long lines = p.units % 8 == 0 ? 8 : 1, plain = p.units / lines * (p.key_tiles - p.sink_tiles);
  const long long all = steps * lines * plain + head_steps * group * p.units * p.sink_tiles;
  p.too_many = all / lines >= (1ll << 30);
  // One worker per CU.  Where there are fewer tiles than that, a worker per tile saves the second tile of a worker's piece
  // and the sums of parts (some 14 us, as much as 14 steps of D = 64 or 7 of 128); splitting them saves steps.
  p.workers = kMostWorkers;
  if (plain > 0 && lines * plain < p.workers && steps - all / p.workers < saves) p.workers = lines * plain;
  if (all < p.workers) p.workers = all / lines * lines;
  if (p.workers < lines) p.workers = lines;
  // Whole rounds, and one that is not full if what it lacks can be made up for by the tiles with sinks, or is little.
  const long long places = p.workers / lines, lacks = (places - plain % places) % places;
  p.whole = lacks * steps <= head_steps * group * (p.units / lines) * p.sink_tiles + places * steps / 16 ? plain : plain / places * places;
  p.split = p.units * p.sink_tiles + lines * (plain - p.whole);
  p.rows = (size_t)B * (size_t)Hq * (size_t)Sq;
  const auto up = [](size_t n) { return (n + 15) & ~(size_t)15; };
  p.most_at = up(8 * p.rows);
  p.part_at = up(p.most_at + 4 * (size_t)(p.units * p.row_tiles));
  p.bytes = p.part_at + (size_t)p.workers * (2u * 2u * kGradKeys * 4u) * (size_t)D;
  return p;
}

template <class T, int D>
kp_status launch_grad(GradArgs& g, const GradPlan& p, hipStream_t st) {
  constexpr uint32_t kTile = 64u * 2u * D, kKeysLds = 6u * kTile + 24u * 2048u + 1536u;
  if constexpr (kKeysLds > 64u * 1024u) {
    static thread_local int attr_dev = -1;  // the attribute is kept per device
    int dev = 0;
    KP_HIP_TRY(hipGetDevice(&dev));
    if (attr_dev != dev) {
      KP_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kp_grad_keys<T, D>), hipFuncAttributeMaxDynamicSharedMemorySize, kKeysLds));
      attr_dev = dev;
    }
  }
  hipLaunchKernelGGL((kp_grad_query<T, D>), dim3((uint32_t)(p.units * p.row_tiles)), dim3(kThreads), 4u * kTile, st, g);
  KP_HIP_TRY(hipGetLastError());
  hipLaunchKernelGGL((kp_grad_keys<T, D>), dim3((uint32_t)p.workers), dim3(kKeysThreads), kKeysLds, st, g);
  KP_HIP_TRY(hipGetLastError());
  if (p.split > 0) {
    hipLaunchKernelGGL((kp_grad_join<T, D>), dim3((uint32_t)(p.split * (kGradKeys / kJoinRows<D>)), 2), dim3(kThreads), 0, st, g);
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
  g.row_tiles = (uint32_t)p.row_tiles; g.key_tiles = (uint32_t)p.key_tiles; g.sink_tiles = (uint32_t)p.sink_tiles; g.workers = (uint32_t)p.workers; g.whole = (uint32_t)p.whole;
  g.seqs = (uint32_t)B; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)Sq; g.n_k = (uint32_t)Sk;
  g.window = (uint32_t)window_of(window); g.sinks = (uint32_t)sinks_of(sinks); g.scale = scale; g.scale_log2 = scale * kLog2e;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (type == KP_FP16) return D == 64 ? launch_grad<Fp16, 64>(g, p, st) : launch_grad<Fp16, 128>(g, p, st);
  return D == 64 ? launch_grad<Bf16, 64>(g, p, st) : launch_grad<Bf16, 128>(g, p, st);
}
