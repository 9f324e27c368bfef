// Attention of new tokens over a paged cache (kp_attn_paged).
#include "kp_attn_host.h"
#include "kp_attn_launch.h"

using namespace kp::attn;

static Plan plan_paged(int T, int n_seqs, int Hq, int Hkv, int D, long long most, int window, int sinks) {
  window = window_of(window);
  sinks = sinks_of(sinks);
  const long long rows = (long long)(Hq / Hkv) * T, tokens = T < kTileRows ? T : kTileRows;
  return plan_of(n_seqs, rows, most_keys_of(most, tokens, window, sinks), Hkv, D, false);
}

extern "C" size_t kp_attn_paged_bytes(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window, int sinks) {
  if (T < 1 || n_seqs < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128) || table_width < 0 || page < 1 || window < 0 || sinks < 0) return 0;
  return plan_paged(T, n_seqs, Hq, Hkv, D, (long long)table_width * page, window, sinks).bytes;
}

extern "C" kp_status kp_attn_paged_launch_shape(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window,
                                                int sinks, int* n_wg, int* waves_per_wg, int* n_regions) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, KP_BF16, window, sinks, 1.f)) return s;
  if (T < 1 || n_seqs < 1 || table_width < 0 || page < 1) return kp::fail(KP_ERR_INVALID_ARG, "T, n_seqs and page must be positive, table_width not negative");
  return launch_shape(plan_paged(T, n_seqs, Hq, Hkv, D, (long long)table_width * page, window, sinks), n_wg, waves_per_wg, n_regions);
}

extern "C" kp_status kp_attn_paged(const kp_heads* q, const kp_cache* cache, const int32_t* block_table, int table_width,
                                   const int32_t* lens, const int32_t* starts, const kp_heads* o, float* lse, int T, int n_seqs,
                                   int Hq, int window, int sinks, float scale, void* workspace, size_t workspace_bytes, uint32_t region_mask, void* trace_buf,
                                    size_t trace_cap, void* stream) {
  kp::clear_error();
  if (kp_status s = check_cache(cache)) return s;
  const int Hkv = cache->Hkv, D = cache->D;
  if (kp_status s = check_common(Hq, Hkv, D, cache->type, window, sinks, scale)) return s;
  if (T < 0 || n_seqs < 0 || table_width < 0) return kp::fail(KP_ERR_INVALID_ARG, "T, n_seqs and table_width must not be negative");
  if (T == 0 || n_seqs == 0) return KP_OK;
  if (T >= kMostTokens || n_seqs >= kMostTokens || (long long)Hq / Hkv * T >= (1ll << 31)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^30 or more tokens, or 2^31 rows of one head");
  if ((long long)table_width * cache->page >= kMostTokens) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "a block table of 2^30 or more tokens");
  if (!lens || !starts || ((uintptr_t)lens & 3u) || ((uintptr_t)starts & 3u)) return kp::fail(KP_ERR_INVALID_ARG, "lens and starts must be device memory, 4-byte aligned");
  if (table_width > 0 && (!block_table || ((uintptr_t)block_table & 3u))) return kp::fail(KP_ERR_INVALID_ARG, "block_table must be device memory, 4-byte aligned");
  if (kp_status s = check_heads("q", q, 1, Hq, T, D, false)) return s;
  if (kp_status s = check_heads("o", o, 1, Hq, T, D, true)) return s;
  if ((uintptr_t)lse & 3u) return kp::fail(KP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  const Plan plan = plan_paged(T, n_seqs, Hq, Hkv, D, (long long)table_width * cache->page, window, sinks);
  if (kp_status s = check_workspace(workspace, workspace_bytes, plan.bytes)) return s;
  Args g{};
  g.q = heads_of(q, 1, Hq, T); g.o = heads_of(o, 1, Hq, T);
  g.k.at = static_cast<const uint16_t*>(cache->k); g.v.at = static_cast<const uint16_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp;
  g.lse = lse; g.lse_head = T;
  g.table = block_table; g.lens = lens; g.starts = starts;
  g.table_width = (uint32_t)table_width; g.page_log2 = log2_of(cache->page); g.n_pages = (uint32_t)cache->n_pages;
  g.seqs = (uint32_t)n_seqs; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)T; g.n_k = (uint32_t)(table_width * cache->page);
  g.window = (uint32_t)window_of(window); g.sinks = (uint32_t)sinks_of(sinks); g.scale_log2 = scale * kLog2e;
  g.part = static_cast<float*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3;
#define KP_PICK(T) (D == 64 ? (e4m3 ? launch<T, 64, kPagedE4m3>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<T, 64, kPaged>(g, plan, region_mask, trace_buf, trace_cap, st)) \
                            : (e4m3 ? launch<T, 128, kPagedE4m3>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<T, 128, kPaged>(g, plan, region_mask, trace_buf, trace_cap, st)))
  return cache->type == KP_FP16 ? KP_PICK(Fp16) : KP_PICK(Bf16);
#undef KP_PICK
}
