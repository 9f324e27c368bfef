// Checks of the attention operators' arguments, on the host.
#pragma once
#include "kp_attn.h"

namespace kp {
namespace attn {

constexpr int64_t kMostTokens = 1 << 30, kMostStep = 1 << 24;
constexpr int64_t kMostGroups = 1 << 23;  // workgroups of a launch: its threads are counted in 32 bits

inline uint32_t log2_of(int pow2) { return (uint32_t)__builtin_ctz((unsigned)pow2); }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0u; }

// Strides and alignment of a tensor of heads; `written`: its rows must not overlap.  With one sequence, head or token
// the stride between them means nothing.
inline kp_status check_heads(const char* name, const kp_heads* t, int64_t seqs, int64_t heads, int64_t tokens, int D, bool written) {
  if (!t || !t->at) return fail(KP_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(t->at)) return fail(KP_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  int64_t stride[3] = {t->seq, t->head, t->token}, count[3] = {seqs, heads, tokens};
  for (int i = 0; i < 3; ++i) {
    if (count[i] <= 1) continue;
    if (stride[i] < 0) return fail(KP_ERR_INVALID_ARG, "%s has a negative stride", name);
    if (stride[i] & 7) return fail(KP_ERR_INVALID_ARG, "strides of %s must be multiples of 8 elements", name);
    if (stride[i] > ((int64_t)1 << 40)) return fail(KP_ERR_UNSUPPORTED_SHAPE, "%s has a stride above 2^40 elements", name);
  }
  if (tokens > 1 && t->token >= kMostStep) return fail(KP_ERR_UNSUPPORTED_SHAPE, "%s has 2^24 or more elements between tokens", name);
  if (written) {
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2 - i; ++j)
        if (stride[order[j]] > stride[order[j + 1]]) { const int x = order[j]; order[j] = order[j + 1]; order[j + 1] = x; }
    int64_t extent = D;
    for (int i = 0; i < 3; ++i) {
      if (count[order[i]] <= 1) continue;
      if (stride[order[i]] < extent) return fail(KP_ERR_INVALID_ARG, "rows of %s overlap", name);
      extent = stride[order[i]] * (count[order[i]] - 1) + extent;
    }
  }
  return KP_OK;
}

inline Heads heads_of(const kp_heads* t, int64_t seqs, int64_t heads, int64_t tokens) {
  Heads h;
  h.at = static_cast<const uint16_t*>(t->at);
  h.seq = seqs > 1 ? t->seq : 0;
  h.head = heads > 1 ? t->head : 0;
  h.token = tokens > 1 ? t->token : 0;
  return h;
}

inline kp_status check_common(int Hq, int Hkv, int D, int type, int window, int sinks, float scale) {
  if (Hq < 1 || Hkv < 1 || Hq % Hkv) return fail(KP_ERR_INVALID_ARG, "Hq = %d must be a multiple of Hkv = %d, both positive", Hq, Hkv);
  if (type != KP_BF16 && type != KP_FP16) return fail(KP_ERR_INVALID_ARG, "type must be KP_BF16 or KP_FP16");
  if (window < 0 || sinks < 0) return fail(KP_ERR_INVALID_ARG, "window and sinks must not be negative");
  if (!(scale > 0.f) || scale > 1e30f) return fail(KP_ERR_INVALID_ARG, "scale must be positive and finite");
  if (D != 64 && D != 128) return fail(KP_ERR_UNSUPPORTED_SHAPE, "D = %d must be 64 or 128", D);
  if (Hq / Hkv > (1 << 16)) return fail(KP_ERR_UNSUPPORTED_SHAPE, "more than 2^16 query heads per head of keys");
  return KP_OK;
}

// There are fewer than 2^30 tokens: a window of as many hides nothing, and more sinks are no more.
inline int window_of(int window) { return window >= kMostTokens ? 0 : window; }
inline int sinks_of(int sinks) { return sinks < kMostTokens ? sinks : (int)kMostTokens; }

inline kp_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need == 0) return KP_OK;
  if (!workspace) return fail(KP_ERR_INVALID_ARG, "workspace is NULL: %zu bytes are needed", need);
  if (!aligned16(workspace)) return fail(KP_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  if (have < need) return fail(KP_ERR_INVALID_ARG, "workspace holds %zu bytes, %zu are needed", have, need);
  return KP_OK;
}

inline kp_status check_cache(const kp_cache* c) {
  if (!c) return fail(KP_ERR_INVALID_ARG, "cache is NULL");
  if (!c->k || !c->v) return fail(KP_ERR_INVALID_ARG, "cache: k or v is NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(KP_ERR_INVALID_ARG, "cache: k and v must be 16-byte aligned");
  if (c->cache_type != KP_CACHE_SAME && c->cache_type != KP_CACHE_E4M3) return fail(KP_ERR_INVALID_ARG, "cache: cache_type must be KP_CACHE_SAME or KP_CACHE_E4M3");
  if (c->cache_type == KP_CACHE_E4M3 && (!c->k_exp || !c->v_exp)) return fail(KP_ERR_INVALID_ARG, "cache: an e4m3 cache needs k_exp and v_exp");
  if (c->type != KP_BF16 && c->type != KP_FP16) return fail(KP_ERR_INVALID_ARG, "cache: type must be KP_BF16 or KP_FP16");
  if (c->n_pages < 1 || c->Hkv < 1 || c->page < 1 || !is_pow2((unsigned long long)c->page)) return fail(KP_ERR_INVALID_ARG, "cache: n_pages and Hkv must be positive, page a power of two");
  if (c->D != 64 && c->D != 128) return fail(KP_ERR_UNSUPPORTED_SHAPE, "D = %d must be 64 or 128", c->D);
  // rows are numbered in 32 bits, and all ones is no row
  if ((unsigned long long)c->n_pages * (unsigned long long)c->Hkv > 0xFFFFFFFFull / (unsigned long long)c->page) return fail(KP_ERR_UNSUPPORTED_SHAPE, "cache of 2^32 or more rows");
  return KP_OK;
}

// A call over a paged cache: its arguments checked and put into `g`, as far as there is anything to do.
inline kp_status check_paged(Args& g, const kp_heads* q, const kp_cache* cache, const int32_t* block_table, int table_width, const int32_t* lens,
                             const int32_t* starts, const kp_heads* o, float* lse, int T, int n_seqs, int Hq, int window, int sinks, float scale) {
  if (kp_status s = check_cache(cache)) return s;
  const int Hkv = cache->Hkv, D = cache->D;
  if (kp_status s = check_common(Hq, Hkv, D, cache->type, window, sinks, scale)) return s;
  if (T < 0 || n_seqs < 0 || table_width < 0) return fail(KP_ERR_INVALID_ARG, "T, n_seqs and table_width must not be negative");
  if (T == 0 || n_seqs == 0) return KP_OK;
  if (T >= kMostTokens || n_seqs >= kMostTokens || (long long)Hq / Hkv * T >= (1ll << 31)) return fail(KP_ERR_UNSUPPORTED_SHAPE, "2^30 or more tokens, or 2^31 rows of one head");
  if ((long long)table_width * cache->page >= kMostTokens) return fail(KP_ERR_UNSUPPORTED_SHAPE, "a block table of 2^30 or more tokens");
  if (!lens || !starts || ((uintptr_t)lens & 3u) || ((uintptr_t)starts & 3u)) return fail(KP_ERR_INVALID_ARG, "lens and starts must be device memory, 4-byte aligned");
  if (table_width > 0 && (!block_table || ((uintptr_t)block_table & 3u))) return fail(KP_ERR_INVALID_ARG, "block_table must be device memory, 4-byte aligned");
  if (kp_status s = check_heads("q", q, 1, Hq, T, D, false)) return s;
  if (kp_status s = check_heads("o", o, 1, Hq, T, D, true)) return s;
  if ((uintptr_t)lse & 3u) return fail(KP_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  g.q = heads_of(q, 1, Hq, T); g.o = heads_of(o, 1, Hq, T);
  g.k.at = static_cast<const uint16_t*>(cache->k); g.v.at = static_cast<const uint16_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp;
  g.lse = lse; g.lse_head = T;
  g.table = block_table; g.lens = lens; g.starts = starts;
  g.table_width = (uint32_t)table_width; g.page_log2 = log2_of(cache->page); g.n_pages = (uint32_t)cache->n_pages;
  g.seqs = (uint32_t)n_seqs; g.hkv = (uint32_t)Hkv; g.group = (uint32_t)(Hq / Hkv); g.n_q = (uint32_t)T; g.n_k = (uint32_t)(table_width * cache->page);
  g.window = (uint32_t)window_of(window); g.sinks = (uint32_t)sinks_of(sinks); g.scale_log2 = scale * kLog2e;
  return KP_OK;
}

// Which kernel takes a call, on how many row tiles, and into how many runs the keys of a tile are split.
struct Plan {
  bool few;
  long long tiles, splits, units;  // units: heads of keys (of all sequences where a tile belongs to one)
  size_t bytes;                    // workspace
};
// Into how many runs the keys of `units` go, for about `want` workgroups, a run of `least` keys or more.
inline void split_keys(Plan& p, long long units, long long want, long long most_keys, long long least, long long per_tile, int D) {
  const long long runs = most_keys < 1536 ? 1 : most_keys / least;
  p.splits = units * 2 > want ? 1 : want / units;
  if (p.splits > runs) p.splits = runs;
  if (p.splits > 256) p.splits = 256;
  if (p.splits < 1) p.splits = 1;
  p.bytes = p.splits > 1 ? (size_t)p.splits * (size_t)(p.units * per_tile) * (size_t)(D + 2) * 4 : 0;
}
// rows: query rows of a head of keys, of all `seqs` sequences; most_keys: keys that a row tile may have to go over;
// even: every sequence has rows / seqs of them.
inline Plan plan_of(long long seqs, long long rows, long long most_keys, int Hkv, int D, bool even) {
  Plan p{};
  p.few = rows <= 16 * seqs;
  const long long per_tile = p.few ? 16 : 128;
  p.tiles = even ? (rows / seqs + per_tile - 1) / per_tile * seqs : rows / per_tile + seqs;
  p.units = p.tiles * Hkv;
  // Joining the parts takes 6 us more, in which a workgroup gets through some 1000 keys: fewer than 1536 are not split, and
  // a run has 512.  Tiles of 128 rows are split to fill the chip (two workgroups per CU: 6 chunks of up to 512 tokens over
  // 8192 keys, 672 workgroups, 125 us, split in two 149); few rows further, since the sequences differ in length (64 tokens
  // over up to 16384 keys, 1024 workgroups 277 us, 4096 261, 8192 267).
  split_keys(p, p.units, p.few ? 4096 : 512, most_keys, 512, per_tile, D);
  return p;
}
// Keys that the rows of a tile may see: all there are, or the window of its tokens and the sinks.
inline long long most_keys_of(long long n_k, long long tokens, int window, int sinks) {
  const long long w = (long long)window + sinks + tokens;
  return window > 0 && w < n_k ? w : n_k;
}

// Workgroups, waves and regions that a recording of the planned call has.
inline kp_status launch_shape(const Plan& plan, int* n_wg, int* waves_per_wg, int* n_regions) {
  if (plan.units * plan.splits >= kMostGroups) return fail(KP_ERR_UNSUPPORTED_SHAPE, "2^23 or more workgroups");
  if (n_wg) *n_wg = (int)(plan.units * plan.splits);
  if (waves_per_wg) *waves_per_wg = 4;
  if (n_regions) *n_regions = 3;
  return KP_OK;
}

}  // namespace attn
}  // namespace kp
