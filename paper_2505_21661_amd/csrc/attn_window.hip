// Attention with a sliding window and sinks over keys that lie in one piece (kp_attn_window).
#include "kp_attn_host.h"
#include "kp_attn_launch.h"

using namespace kp::attn;

namespace {
kp_status check_sizes(int B, int Hq, int Hkv, int Sq, int Sk, int D) {
  if (B < 1 || Sq < 1 || Sk < 1 || Hq < 1) return kp::fail(KP_ERR_INVALID_ARG, "B, Hq, Sq and Sk must be positive");
  if (Sq >= kMostTokens || Sk >= kMostTokens) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^30 or more tokens");
  if ((long long)B * Hq >= (1ll << 31) || (long long)Hq / Hkv * Sq >= (1ll << 31)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^31 or more rows of one head");
  return KP_OK;
}
}  // namespace

static Plan plan_window(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  const long long rows = (long long)(Hq / Hkv) * Sq;
  window = window_of(window);
  sinks = sinks_of(sinks);
  return plan_of(B, rows * B, most_keys_of(Sk, Sq < kTileRows ? Sq : kTileRows, window, sinks), Hkv, D, true);
}

extern "C" size_t kp_attn_window_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks) {
  if (Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128) || window < 0 || sinks < 0 || check_sizes(B, Hq, Hkv, Sq, Sk, D)) return 0;
  return plan_window(B, Hq, Hkv, Sq, Sk, D, window, sinks).bytes;
}

extern "C" kp_status kp_attn_window_launch_shape(int B, int Hq, int Hkv, int Sq, int Sk, int D, int window, int sinks, int* n_wg,
                                                 int* waves_per_wg, int* n_regions) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, KP_BF16, window, sinks, 1.f)) return s;
  if (kp_status s = check_sizes(B, Hq, Hkv, Sq, Sk, D)) return s;
  return launch_shape(plan_window(B, Hq, Hkv, Sq, Sk, D, window, sinks), n_wg, waves_per_wg, n_regions);
}

extern "C" kp_status kp_attn_window(const kp_heads* q, const kp_heads* k, const kp_heads* v, const kp_heads* o, float* lse,
                                    int B, int Hq, int Hkv, int Sq, int Sk, int D, int type, int window, int sinks,
                                    float scale, void* workspace, size_t workspace_bytes, uint32_t region_mask, void* trace_buf,
                                    size_t trace_cap, void* stream) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, type, window, sinks, scale)) return s;
  if (kp_status s = check_sizes(B, Hq, Hkv, Sq, Sk, D)) return s;
  if (kp_status s = check_heads("q", q, B, Hq, Sq, D, false)) return s;
  if (kp_status s = check_heads("k", k, B, Hkv, Sk, D, false)) return s;
  if (kp_status s = check_heads("v", v, B, Hkv, Sk, D, false)) return s;
  if (kp_status s = check_heads("o", o, B, Hq, Sq, D, true)) return s;
  if ((uintptr_t)lse & 3u) return kp::fail(KP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  const Plan plan = plan_window(B, Hq, Hkv, Sq, Sk, D, window, sinks);
  if (kp_status s = check_workspace(workspace, workspace_bytes, plan.bytes)) return s;
  Args g{};
  g.q = heads_of(q, B, Hq, Sq); g.o = heads_of(o, B, Hq, Sq);
  g.k = heads_of(k, B, Hkv, Sk); g.v = heads_of(v, B, Hkv, Sk);
  g.lse = lse; g.lse_seq = (int64_t)Hq * Sq; g.lse_head = Sq;
  g.seqs = (uint32_t)B; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)Sq; g.n_k = (uint32_t)Sk;
  g.window = (uint32_t)window_of(window); g.sinks = (uint32_t)sinks_of(sinks); g.scale_log2 = scale * kLog2e;
  g.part = static_cast<float*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (type == KP_FP16) return D == 64 ? launch<Fp16, 64, kPlain>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<Fp16, 128, kPlain>(g, plan, region_mask, trace_buf, trace_cap, st);
  return D == 64 ? launch<Bf16, 64, kPlain>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<Bf16, 128, kPlain>(g, plan, region_mask, trace_buf, trace_cap, st);
}
