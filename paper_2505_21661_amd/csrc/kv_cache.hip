// A paged cache of keys and values: new rows quantised (or copied) into their slots, whole sequences read back.
#include "kp_cache_row.h"
#include "kp_attn_host.h"

namespace {
using namespace kp::attn;

constexpr int kThreads = 256;

struct WriteArgs {
  Heads k, v;
  const int64_t* slots;
  uint8_t *k_cache, *v_cache, *k_exp, *v_exp;
  uint32_t tokens, hkv, page_log2, run_log2;
  uint64_t n_slots;
};

// D / 8 lanes to a row, 16 bytes to a lane, kWriteRows rows one after the other, all of whose loads are in flight together;
// blockIdx.y: keys or values.  Rows are taken for one head from a run of tokens, then for the next: a run's rows lie side by
// side in the cache, where rows in the order that they come in (all heads of a token) leave pieces of D bytes and single
// exponents.  (Nothing orders the rows of a slot that two tokens name: the caller's to avoid.)  They are read once, past the caches (nontemporal), so that what stays there is the cache that is read next.
// Bound by memory: 32749 tokens of 8 heads of 128, 202 MB, take 39 us (5150 GB/s, what a copy reaches); in runs of 32 and 64
// tokens 40 and 43, token by token 44, that through the caches 47.6; with 8 rows 42.5, with 2 42.9, with 1 51.
constexpr uint32_t kWriteRows = 4, kMostRunLog2 = 4;
template <class T, int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void kp_cache_write_rows(WriteArgs g) {
  constexpr uint32_t kLanes = D / 8, kStep = kThreads / kLanes;
  const uint32_t r0 = blockIdx.x * (kStep * kWriteRows) + threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  const Heads src = blockIdx.y ? g.v : g.k;
  uint8_t* const cache = blockIdx.y ? g.v_cache : g.k_cache;
  int64_t slot[kWriteRows];
  uint32_t head[kWriteRows];
  u32x4 raw[kWriteRows];
#pragma unroll
  for (uint32_t i = 0; i < kWriteRows; ++i) {
    const uint32_t r = r0 + kStep * i, rest = r >> g.run_log2, run = rest / g.hkv;
    const uint32_t at = (run << g.run_log2) + (r & ((1u << g.run_log2) - 1u)), token = at < g.tokens ? at : g.tokens - 1u;
    head[i] = rest - run * g.hkv;
    slot[i] = at < g.tokens ? g.slots[token] : -1;
    raw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src.at + src.token * (int64_t)token + src.head * (int64_t)head[i] + 8u * c));
  }
#pragma unroll
  for (uint32_t i = 0; i < kWriteRows; ++i) {
    if (slot[i] < 0 || (uint64_t)slot[i] >= g.n_slots) continue;  // (the same for all lanes of a row)
    put_row<T, D, E4M3>(raw[i], cache, blockIdx.y ? g.v_exp : g.k_exp, row_of_slot((uint64_t)slot[i], head[i], g.hkv, g.page_log2), c);
  }
}

struct ReadArgs {
  Heads k, v;
  const uint8_t *k_cache, *v_cache, *k_exp, *v_exp;
  const int32_t *table, *starts;
  uint32_t table_width, seqs, tokens, hkv, page_log2, n_pages;
};

constexpr uint32_t kReadTokens = 8;  // tokens of a workgroup (8: 106 us at the sizes below, 16: 109, 32: 120, 4: 113)

// 16 bytes of the cache to a lane; blockIdx.y: keys or values.  Bound by memory, most of it writes: 16 sequences of up to
// 8192 tokens of 8 heads of 128 out of e4m3, 510 MB, take 106 us (4800 GB/s); through the caches 109.
template <class T, int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void kp_cache_read_rows(ReadArgs g) {
  constexpr uint32_t kPer = E4M3 ? 16 : 8, kLanes = D / kPer;
  __shared__ uint32_t page_row[kReadTokens], state[kReadTokens];  // state: 0 no sequence's token, 1 zeros, 2 a row
  const uint32_t t0 = blockIdx.x * kReadTokens;
  if (threadIdx.x < kReadTokens) {
    const uint32_t t = t0 + threadIdx.x;
    uint32_t found = 0, row = 0;
    if (t < g.tokens) {
      uint32_t a = 0, b = g.seqs + 1;  // the first start above t lies in [a, b]
      while (a < b) {
        const uint32_t m = (a + b) >> 1;
        if (g.starts[m] > (int32_t)t) b = m; else a = m + 1;
      }
      if (a > 0 && a <= g.seqs) {
        found = 1;
        const int32_t start = g.starts[a - 1];
        const uint32_t at = t - (start < 0 ? 0u : (uint32_t)start), block = at >> g.page_log2;
        if (block < g.table_width) {
          const uint32_t page = (uint32_t)g.table[(size_t)(a - 1) * g.table_width + block];
          if (page < g.n_pages) {
            found = 2;
            row = ((page * g.hkv) << g.page_log2) + (at & ((1u << g.page_log2) - 1u));
          }
        }
      }
    }
    state[threadIdx.x] = found;
    page_row[threadIdx.x] = row;
  }
  __syncthreads();
  const Heads dst = blockIdx.y ? g.v : g.k;
  const uint8_t* const cache = blockIdx.y ? g.v_cache : g.k_cache;
  const uint8_t* const exps = blockIdx.y ? g.v_exp : g.k_exp;
  const uint32_t c = threadIdx.x % kLanes;
#pragma unroll 4
  for (uint32_t i = threadIdx.x / kLanes; i < kReadTokens * g.hkv; i += kThreads / kLanes) {
    const uint32_t tl = i / g.hkv, head = i - tl * g.hkv, how = state[tl];
    if (how == 0) continue;
    const uint32_t row = page_row[tl] + (head << g.page_log2);
    uint16_t* out = const_cast<uint16_t*>(dst.at) + dst.token * (int64_t)(t0 + tl) + dst.head * (int64_t)head + kPer * c;
    u32x4 raw = {0, 0, 0, 0};
    if (how == 2) raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(cache + (size_t)row * (E4M3 ? D : 2 * D) + 16u * c));
    if constexpr (!E4M3) {
      *reinterpret_cast<u32x4*>(out) = raw;
    } else {
      const float scale = how == 2 ? power_of(exps[row]) : 1.f;
      u32x4 lo, hi;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        u32x4& to = w < 2 ? lo : hi;
        to[2 * (w & 1)] = T::template from_e4m3<false>(raw[w], scale);
        to[2 * (w & 1) + 1] = T::template from_e4m3<true>(raw[w], scale);
      }
      *reinterpret_cast<u32x4*>(out) = lo;
      *reinterpret_cast<u32x4*>(out + 8) = hi;
    }
  }
}

}  // namespace

extern "C" kp_status kp_cache_write(const kp_heads* k, const kp_heads* v, const int64_t* slots, int T, const kp_cache* cache, void* stream) {
  kp::clear_error();
  if (kp_status s = check_cache(cache)) return s;
  if (T < 0) return kp::fail(KP_ERR_INVALID_ARG, "T must not be negative");
  if (T == 0) return KP_OK;
  if (!slots || ((uintptr_t)slots & 7u)) return kp::fail(KP_ERR_INVALID_ARG, "slots must be device memory, 8-byte aligned");
  if (kp_status s = check_heads("k", k, 1, cache->Hkv, T, cache->D, false)) return s;
  if (kp_status s = check_heads("v", v, 1, cache->Hkv, T, cache->D, false)) return s;
  if (T >= kMostTokens || (long long)T * cache->Hkv >= (1ll << 28)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^28 or more rows in one call");
  WriteArgs g{};
  g.k = heads_of(k, 1, cache->Hkv, T); g.v = heads_of(v, 1, cache->Hkv, T);
  g.slots = slots;
  g.k_cache = static_cast<uint8_t*>(cache->k); g.v_cache = static_cast<uint8_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp;
  g.tokens = (uint32_t)T; g.hkv = (uint32_t)cache->Hkv; g.page_log2 = log2_of(cache->page);
  while (g.run_log2 < kMostRunLog2 && 2u << g.run_log2 <= g.tokens) ++g.run_log2;
  g.n_slots = (uint64_t)cache->n_pages * (uint64_t)cache->page;
  const uint32_t per = kThreads / (cache->D / 8) * kWriteRows, runs = (g.tokens + (1u << g.run_log2) - 1u) >> g.run_log2;
  const dim3 grid(((runs * g.hkv << g.run_log2) + per - 1) / per, 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3, fp16 = cache->type == KP_FP16;
#define KP_LAUNCH(T, D, E) hipLaunchKernelGGL((kp_cache_write_rows<T, D, E>), grid, dim3(kThreads), 0, st, g)
#define KP_PICK(D) do { if (!e4m3) KP_LAUNCH(Bf16, D, false); else if (fp16) KP_LAUNCH(Fp16, D, true); else KP_LAUNCH(Bf16, D, true); } while (0)
  if (cache->D == 64) KP_PICK(64); else KP_PICK(128);
#undef KP_PICK
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}

extern "C" kp_status kp_cache_read(const kp_cache* cache, const int32_t* block_table, int table_width, const int32_t* starts,
                                   int n_seqs, int T, const kp_heads* k, const kp_heads* v, void* stream) {
  kp::clear_error();
  if (kp_status s = check_cache(cache)) return s;
  if (T < 0 || n_seqs < 0 || table_width < 0) return kp::fail(KP_ERR_INVALID_ARG, "T, n_seqs and table_width must not be negative");
  if (T == 0 || n_seqs == 0) return KP_OK;
  if (!starts || ((uintptr_t)starts & 3u)) return kp::fail(KP_ERR_INVALID_ARG, "starts must be device memory, 4-byte aligned");
  if (table_width > 0 && (!block_table || ((uintptr_t)block_table & 3u))) return kp::fail(KP_ERR_INVALID_ARG, "block_table must be device memory, 4-byte aligned");
  if (kp_status s = check_heads("k", k, 1, cache->Hkv, T, cache->D, true)) return s;
  if (kp_status s = check_heads("v", v, 1, cache->Hkv, T, cache->D, true)) return s;
  if (T >= kMostTokens || n_seqs >= kMostTokens || (T + kReadTokens - 1) / kReadTokens >= kMostGroups || (long long)T * cache->Hkv >= (1ll << 31)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^27 or more tokens or 2^31 rows in one call");
  ReadArgs g{};
  g.k = heads_of(k, 1, cache->Hkv, T); g.v = heads_of(v, 1, cache->Hkv, T);
  g.k_cache = static_cast<const uint8_t*>(cache->k); g.v_cache = static_cast<const uint8_t*>(cache->v);
  g.k_exp = cache->k_exp; g.v_exp = cache->v_exp;
  g.table = block_table; g.starts = starts; g.table_width = (uint32_t)table_width; g.seqs = (uint32_t)n_seqs;
  g.tokens = (uint32_t)T; g.hkv = (uint32_t)cache->Hkv; g.page_log2 = log2_of(cache->page); g.n_pages = (uint32_t)cache->n_pages;
  const dim3 grid((g.tokens + kReadTokens - 1) / kReadTokens, 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3, fp16 = cache->type == KP_FP16;
#define KP_LAUNCH(T, D, E) hipLaunchKernelGGL((kp_cache_read_rows<T, D, E>), grid, dim3(kThreads), 0, st, g)
#define KP_PICK(D) do { if (!e4m3) KP_LAUNCH(Bf16, D, false); else if (fp16) KP_LAUNCH(Fp16, D, true); else KP_LAUNCH(Bf16, D, true); } while (0)
  if (cache->D == 64) KP_PICK(64); else KP_PICK(128);
#undef KP_PICK
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}
