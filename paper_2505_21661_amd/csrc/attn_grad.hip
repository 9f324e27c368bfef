// Gradients of attention with a sliding window and sinks (kp_attn_window_grad).
//
// With P_ij = exp2(scale log2(e) q_i.k_j - lse_i log2(e)) and delta_i = d_o_i . o_i (= sum_j P_ij d_o_i . v_j):
//   dS_ij = P_ij (d_o_i . v_j - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij d_o_i.
#include "kp_attn_host.h"

using namespace kp::attn;

namespace {

constexpr int kThreads = 256;

struct GradArgs {
  Heads q, k, v, o, d_o, dq, dk, dv;
  const float* lse;
  float *lse2, *delta;  // workspace, [B, Hq, Sq]: lse * log2(e) and d_o . o
  uint32_t seqs, hkv, group, n_q, n_k, window, sinks;
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

// One query row's gradient in fp32, by a wave; only keys that the row sees are touched.
template <class T, int D>
__device__ void query_row(const GradArgs& g, uint32_t seq, uint32_t head, uint32_t token, float lse2, float delta, float (&dq)[D / 64]) {
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
    const float w = __builtin_amdgcn_exp2f(dot<E>(q, k) * g.scale_log2 - lse2), ds = w * (dot<E>(d_o, v) - delta);
#pragma unroll
    for (int e = 0; e < E; ++e) dq[e] = __builtin_fmaf(ds, k[e], dq[e]);
  }
}

// One key's gradients from the query tokens from .. to - 1 of every head of its group.
template <class T, int D>
__device__ void key_row(const GradArgs& g, uint32_t seq, uint32_t hk, uint32_t j, uint32_t head_from, uint32_t head_to, uint32_t from, uint32_t to,
                        float (&dk)[D / 64], float (&dv)[D / 64]) {
  constexpr int E = D / 64;
  float k[E], v[E];
  load_row<T, E>(row_at(g.k, seq, hk, j), k);
  load_row<T, E>(row_at(g.v, seq, hk, j), v);
#pragma unroll
  for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
  for (uint32_t head = head_from; head < head_to; ++head)
    for (uint32_t i = from; i < to; ++i) {
      const int32_t p = (int32_t)g.n_k - (int32_t)g.n_q + (int32_t)i;
      if (!sees(p, j, g.window, g.sinks)) continue;
      float q[E], d_o[E];
      load_row<T, E>(row_at(g.q, seq, head, i), q);
      load_row<T, E>(row_at(g.d_o, seq, head, i), d_o);
      const size_t at = ((size_t)seq * g.hkv * g.group + head) * g.n_q + i;
      const float w = __builtin_amdgcn_exp2f(dot<E>(q, k) * g.scale_log2 - g.lse2[at]), ds = w * (dot<E>(d_o, v) - g.delta[at]);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dk[e] = __builtin_fmaf(ds, q[e], dk[e]);
        dv[e] = __builtin_fmaf(w, d_o[e], dv[e]);
      }
    }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void kp_grad_query_rows(GradArgs g) {
  constexpr int E = D / 64;
  const uint64_t row = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
  if (row >= (uint64_t)g.seqs * g.hkv * g.group * g.n_q) return;
  const uint32_t token = (uint32_t)(row % g.n_q), bh = (uint32_t)(row / g.n_q), seq = bh / (g.hkv * g.group), head = bh % (g.hkv * g.group);
  float o[E], d_o[E], dq[E];
  load_row<T, E>(row_at(g.o, seq, head, token), o);
  load_row<T, E>(row_at(g.d_o, seq, head, token), d_o);
  const float delta = dot<E>(o, d_o), lse2 = g.lse[row] * kLog2e;
  if ((threadIdx.x & 63u) == 0) { g.lse2[row] = lse2; g.delta[row] = delta; }
  query_row<T, D>(g, seq, head, token, lse2, delta, dq);
  put_row<T, E>(const_cast<uint16_t*>(row_at(g.dq, seq, head, token)), dq, g.scale);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void kp_grad_key_rows(GradArgs g) {
  constexpr int E = D / 64;
  const uint64_t row = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
  if (row >= (uint64_t)g.seqs * g.hkv * g.n_k) return;
  const uint32_t j = (uint32_t)(row % g.n_k), bh = (uint32_t)(row / g.n_k), seq = bh / g.hkv, hk = bh % g.hkv;
  float dk[E], dv[E];
  key_row<T, D>(g, seq, hk, j, hk * g.group, (hk + 1u) * g.group, 0u, g.n_q, dk, dv);
  put_row<T, E>(const_cast<uint16_t*>(row_at(g.dk, seq, hk, j)), dk, g.scale);
  put_row<T, E>(const_cast<uint16_t*>(row_at(g.dv, seq, hk, j)), dv, 1.f);
}

bool sizes_ok(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  return B > 0 && Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && Sq > 0 && Sk > 0 && (D == 64 || D == 128) && window >= 0 && sinks >= 0 && Sq < kMostTokens &&
         Sk < kMostTokens && (long long)B * Hq < (1ll << 31);
}

}  // namespace

extern "C" size_t kp_attn_window_grad_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  if (!sizes_ok(B, Hq, Hkv, Sq, Sk, D, window, sinks)) return 0;
  return (size_t)B * (size_t)Hq * (size_t)Sq * 8;
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
  if (kp_status s = check_workspace(workspace, workspace_bytes, kp_attn_window_grad_bytes(B, Hq, Hkv, Sq, Sk, D, window, sinks))) return s;
  GradArgs g{};
  g.q = heads_of(q, B, Hq, Sq); g.o = heads_of(o, B, Hq, Sq); g.d_o = heads_of(d_o, B, Hq, Sq); g.dq = heads_of(dq, B, Hq, Sq);
  g.k = heads_of(k, B, Hkv, Sk); g.v = heads_of(v, B, Hkv, Sk); g.dk = heads_of(dk, B, Hkv, Sk); g.dv = heads_of(dv, B, Hkv, Sk);
  g.lse = lse;
  const size_t rows = (size_t)B * (size_t)Hq * (size_t)Sq;
  g.lse2 = static_cast<float*>(workspace); g.delta = g.lse2 + rows;
  g.seqs = (uint32_t)B; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)Sq; g.n_k = (uint32_t)Sk;
  g.window = (uint32_t)window; g.sinks = (uint32_t)sinks; g.scale = scale; g.scale_log2 = scale * kLog2e;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const size_t keys = (size_t)B * (size_t)Hkv * (size_t)Sk;
  if ((rows + 3) / 4 >= (1ull << 31) || (keys + 3) / 4 >= (1ull << 31)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^31 or more workgroups");
#define KP_LAUNCH(T, D)                                                                                              \
  do {                                                                                                               \
    hipLaunchKernelGGL((kp_grad_query_rows<T, D>), dim3((uint32_t)((rows + 3) / 4)), dim3(kThreads), 0, st, g);      \
    hipLaunchKernelGGL((kp_grad_key_rows<T, D>), dim3((uint32_t)((keys + 3) / 4)), dim3(kThreads), 0, st, g);        \
  } while (0)
  if (type == KP_BF16) { if (D == 64) KP_LAUNCH(Bf16, 64); else KP_LAUNCH(Bf16, 128); }
  else { if (D == 64) KP_LAUNCH(Fp16, 64); else KP_LAUNCH(Fp16, 128); }
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}
