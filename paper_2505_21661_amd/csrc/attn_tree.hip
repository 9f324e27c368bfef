// Attention of drafted tokens, each of which sees its ancestors, over a paged cache (kp_attn_tree).
#include "kp_attn_host.h"
#include "kp_attn_launch.h"

using namespace kp::attn;

static Plan plan_tree(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window, int sinks) {
  const long long rows = (long long)(Hq / Hkv) * T, tokens = T < kTileRows ? T : kTileRows;
  const long long most_keys = most_keys_of((long long)table_width * page, tokens, window_of(window), sinks_of(sinks));
  Plan p{};
  p.few = rows <= 64ll * n_seqs && page >= kDraftPage;
  const long long per_tile = p.few ? kDraftRows : kTileRows;
  p.tiles = rows / per_tile + n_seqs;
  p.units = p.tiles * Hkv;
  split_keys(p, p.few ? 2048 : 512, most_keys, per_tile, D);
  return p;
}

extern "C" size_t kp_attn_tree_bytes(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window, int sinks) {
  if (T < 1 || n_seqs < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128) || table_width < 0 || page < 1 || window < 0 || sinks < 0) return 0;
  return plan_tree(T, n_seqs, Hq, Hkv, D, table_width, page, window, sinks).bytes;
}

extern "C" kp_status kp_attn_tree_launch_shape(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window,
                                               int sinks, int* n_wg, int* waves_per_wg, int* n_regions) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, KP_BF16, window, sinks, 1.f)) return s;
  if (T < 1 || n_seqs < 1 || table_width < 0 || page < 1) return kp::fail(KP_ERR_INVALID_ARG, "T, n_seqs and page must be positive, table_width not negative");
  return launch_shape(plan_tree(T, n_seqs, Hq, Hkv, D, table_width, page, window, sinks), n_wg, waves_per_wg, n_regions);
}

extern "C" kp_status kp_attn_tree(const kp_heads* q, const kp_cache* cache, const int32_t* block_table, int table_width,
                                  const int32_t* lens, const int32_t* starts, const int64_t* seen, int words, const int32_t* depth,
                                  const kp_heads* o, float* lse, int T, int n_seqs, int Hq, int window, int sinks, float scale,
                                  void* workspace, size_t workspace_bytes, uint32_t region_mask, void* trace_buf, size_t trace_cap,
                                  void* stream) {
  kp::clear_error();
  Args g{};
  if (kp_status s = check_paged(g, q, cache, block_table, table_width, lens, starts, o, lse, T, n_seqs, Hq, window, sinks, scale)) return s;
  if (words < 0 || words > (1 << 24)) return kp::fail(KP_ERR_INVALID_ARG, "words must be from 0 to 2^24");
  if (T == 0 || n_seqs == 0) return KP_OK;
  if ((words > 0 && !seen) || ((uintptr_t)seen & 7u)) return kp::fail(KP_ERR_INVALID_ARG, "seen must be device memory, 8-byte aligned");
  if ((uintptr_t)depth & 3u) return kp::fail(KP_ERR_INVALID_ARG, "depth must be device memory, 4-byte aligned");
  const Plan plan = plan_tree(T, n_seqs, Hq, cache->Hkv, cache->D, table_width, cache->page, window, sinks);
  if (kp_status s = check_workspace(workspace, workspace_bytes, plan.bytes)) return s;
  g.part = static_cast<float*>(workspace);
  g.seen = reinterpret_cast<const uint32_t*>(seen); g.depth = depth; g.words = (uint32_t)words;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int D = cache->D;
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3;
#define KP_PICK(T) (D == 64 ? (e4m3 ? launch<T, 64, kTreeE4m3>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<T, 64, kTree>(g, plan, region_mask, trace_buf, trace_cap, st)) \
                            : (e4m3 ? launch<T, 128, kTreeE4m3>(g, plan, region_mask, trace_buf, trace_cap, st) : launch<T, 128, kTree>(g, plan, region_mask, trace_buf, trace_cap, st)))
  return cache->type == KP_FP16 ? KP_PICK(Fp16) : KP_PICK(Bf16);
#undef KP_PICK
}
