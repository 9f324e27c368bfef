// Attention of new tokens over a paged cache (kp_attn_paged).
#include "kp_attn_host.h"
#include "kp_attn_rows.h"

using namespace kp::attn;

extern "C" size_t kp_attn_paged_bytes(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int window, int sinks) { return 0; }

extern "C" kp_status kp_attn_paged(const kp_heads* q, const kp_cache* cache, const int32_t* block_table, int table_width,
                                   const int32_t* lens, const int32_t* starts, const kp_heads* o, float* lse, int T, int n_seqs,
                                   int Hq, int window, int sinks, float scale, void* workspace, size_t workspace_bytes, void* stream) {
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
  if (kp_status s = check_workspace(workspace, workspace_bytes, kp_attn_paged_bytes(T, n_seqs, Hq, Hkv, D, table_width, cache->page, window, sinks))) return s;
  Args g{};
  g.q = heads_of(q, 1, Hq, T); g.o = heads_of(o, 1, Hq, T);
  g.k.at = static_cast<const uint16_t*>(cache->k); g.v.at = static_cast<const uint16_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp;
  g.lse = lse; g.lse_head = T;
  g.table = block_table; g.lens = lens; g.starts = starts;
  g.table_width = (uint32_t)table_width; g.page_log2 = log2_of(cache->page); g.n_pages = (uint32_t)cache->n_pages;
  g.seqs = (uint32_t)n_seqs; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)T; g.n_k = (uint32_t)(table_width * cache->page);
  g.window = (uint32_t)window; g.sinks = (uint32_t)sinks; g.scale_log2 = scale * kLog2e;
  const long long tiles = (long long)g.group * T / 16 + n_seqs, grid = tiles * Hkv;
  if (grid >= (1ll << 31)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^31 or more workgroups");
  g.tiles = (uint32_t)tiles;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3, fp16 = cache->type == KP_FP16;
#define KP_LAUNCH(T, D, S) hipLaunchKernelGGL((kp_attn_row_by_row<T, D, S>), dim3((uint32_t)grid), dim3(kThreads), 0, st, g)
#define KP_PICK(T) do { if (D == 64) { if (e4m3) KP_LAUNCH(T, 64, kPagedE4m3); else KP_LAUNCH(T, 64, kPaged); } else { if (e4m3) KP_LAUNCH(T, 128, kPagedE4m3); else KP_LAUNCH(T, 128, kPaged); } } while (0)
  if (fp16) KP_PICK(Fp16); else KP_PICK(Bf16);
#undef KP_PICK
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}
