// Attention of drafted tokens, each of which sees its ancestors, over a paged cache (kp_attn_tree).
#include "kp_attn_host.h"
#include "kp_attn_launch.h"

using namespace kp::attn;

// Which kernel: tiles of 32 rows (kp_attn_drafts) up to so many rows of a sequence on average, and where there is so little work
// that its latency counts.  32 sequences over up to 16384 keys, 32/8 heads of 128, by rows on average, in us (32 rows / 128):
//   e4m3     33: 190 / 289   44: 201 / 271   66: 268 / 281   88: 320 / 282      16 bits  33: 326 / 340   44: 353 / 309   66: 458 / 324
// 3 sequences over up to 700 keys: 9.8 / 16, whatever their rows.
// Into how many runs the keys of a tile are split: of 128 rows so that all workgroups have a place at once (24 drafted tokens at most: 293
// us in two runs, 404 in one, 324 in three); where one run takes more than half of the places, so that they come to three rounds, which
// evens out what long sequences have more than others (40 tokens: 478 us in one run, 391 in two, 341 in four), as long as
// a run has 4096 keys.  Of 32 rows further (three runs 200 us, two 204, six 209).
static Plan plan_tree(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int cache_type, int window, int sinks) {
  const long long rows = (long long)(Hq / Hkv) * T, tokens = T < kTileRows ? T : kTileRows, places = 512;
  const long long most_keys = most_keys_of((long long)table_width * page, tokens, window_of(window), sinks_of(sinks));
  // Tiles of 128 rows that there may be, for sequences of half to one and a half times as many rows as they have on average.
  long long tiles = 0;
  for (int i = 1; i < 16; i += 2) tiles += ((8 + i) * rows + (16ll * kTileRows * n_seqs - 1)) / (16ll * kTileRows * n_seqs);
  tiles = (tiles * n_seqs + 7) / 8;
  Plan p{};
  p.few = page >= kDraftPage && (rows <= (cache_type == KP_CACHE_E4M3 ? 64ll : 40ll) * n_seqs || (most_keys < 1536 && tiles * Hkv <= places / 4));
  const long long per_tile = p.few ? kDraftRows : kTileRows;
  p.tiles = rows / per_tile + n_seqs;
  p.units = p.tiles * Hkv;
  if (p.few) {
    split_keys(p, p.units, 2048, most_keys, 512, per_tile, D);
  } else {
    split_keys(p, tiles * Hkv, places, most_keys, 512, per_tile, D);
    if (p.splits == 1) split_keys(p, tiles * Hkv, 3 * places, most_keys, 4096, per_tile, D);
  }
  return p;
}

extern "C" size_t kp_attn_tree_bytes(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int cache_type, int window, int sinks) {
  if (T < 1 || n_seqs < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128) || table_width < 0 || page < 1 || window < 0 || sinks < 0) return 0;
  return plan_tree(T, n_seqs, Hq, Hkv, D, table_width, page, cache_type, window, sinks).bytes;
}

extern "C" kp_status kp_attn_tree_launch_shape(int T, int n_seqs, int Hq, int Hkv, int D, int table_width, int page, int cache_type,
                                               int window, int sinks, int* n_wg, int* waves_per_wg, int* n_regions) {
  kp::clear_error();
  if (kp_status s = check_common(Hq, Hkv, D, KP_BF16, window, sinks, 1.f)) return s;
  if (T < 1 || n_seqs < 1 || table_width < 0 || page < 1) return kp::fail(KP_ERR_INVALID_ARG, "T, n_seqs and page must be positive, table_width not negative");
  return launch_shape(plan_tree(T, n_seqs, Hq, Hkv, D, table_width, page, cache_type, window, sinks), n_wg, waves_per_wg, n_regions);
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
  const Plan plan = plan_tree(T, n_seqs, Hq, cache->Hkv, cache->D, table_width, cache->page, cache->cache_type, window, sinks);
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
