// Rows of a paged cache that move from slot to slot (kp_cache_move): codes and exponents as they are.
//
// Nothing is computed: the time is that of reading and writing the rows.  A row of a head lies in one piece of 64 to 256
// bytes, 16 of them to a lane.
#include "kp_attn_host.h"
#include "kp_cache_row.h"

namespace {
using namespace kp::attn;

constexpr uint32_t kThreads = 256;

struct MoveArgs {
  const int64_t *from, *to;
  const int32_t* starts;
  uint8_t *half[2], *exps[2];  // keys, values
  uint32_t moves, groups, hkv, page_log2, run_log2;
  uint64_t n_slots;
};

__device__ __forceinline__ bool moves(const MoveArgs& g, int64_t from, int64_t to) {
  return from >= 0 && to >= 0 && (uint64_t)from < g.n_slots && (uint64_t)to < g.n_slots && from != to;
}

// Moves that have nothing to do with one another: any order.  Rows are taken for one head from a run of moves, then for the
// next, since the slots of a page lie side by side for a head; blockIdx.y: keys or values.
constexpr uint32_t kRows = 4, kMostRunLog2 = 4;
template <uint32_t BYTES, bool E4M3>
__global__ __launch_bounds__(kThreads) void kp_cache_move_apart(MoveArgs g) {
  constexpr uint32_t kLanes = BYTES / 16u, kStep = kThreads / kLanes;
  const uint32_t r0 = blockIdx.x * (kStep * kRows) + threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  uint8_t* const half = g.half[blockIdx.y];
  uint8_t* const exps = g.exps[blockIdx.y];
  uint32_t to[kRows];
  u32x4 raw[kRows];
  uint8_t e[kRows];
  bool there[kRows];
#pragma unroll
  for (uint32_t i = 0; i < kRows; ++i) {
    const uint32_t r = r0 + kStep * i, rest = r >> g.run_log2, run = rest / g.hkv, head = rest - run * g.hkv;
    const uint32_t at = (run << g.run_log2) + (r & ((1u << g.run_log2) - 1u)), move = at < g.moves ? at : g.moves - 1u;
    const int64_t a = g.from[move], b = g.to[move];
    there[i] = at < g.moves && moves(g, a, b);
    const uint32_t row = there[i] ? row_of_slot((uint64_t)a, head, g.hkv, g.page_log2) : 0u;
    to[i] = there[i] ? row_of_slot((uint64_t)b, head, g.hkv, g.page_log2) : 0u;
    raw[i] = *reinterpret_cast<const u32x4*>(half + (size_t)row * BYTES + 16u * c);
    if constexpr (E4M3) e[i] = exps[row];
  }
#pragma unroll
  for (uint32_t i = 0; i < kRows; ++i) {
    if (!there[i]) continue;
    *reinterpret_cast<u32x4*>(half + (size_t)to[i] * BYTES + 16u * c) = raw[i];
    if constexpr (E4M3)
      if (c == 0) exps[to[i]] = e[i];
  }
}

// Groups of moves in order: a workgroup has one head of one group, of 128 bytes of its rows, and takes them in runs, each read whole
// before it is written; what a later run reads, no earlier one writes, so that it is asked for a run ahead, and its slots two.
// blockIdx: group, head, keys or values and which 128 bytes.
// Bound by memory: 24 sequences of up to 4001 tokens of 8 heads of 128 in bf16 that lose a third, 334 MB, take 86 us (3850 GB/s, a copy
// 5120); whole rows to a workgroup, nothing asked for ahead, 190; runs of 256 rows 86.
constexpr uint32_t kPasses = 4;
template <uint32_t BYTES, bool E4M3>
__global__ __launch_bounds__(kThreads) void kp_cache_move_groups(MoveArgs g) {
  constexpr uint32_t kPart = BYTES < 128u ? BYTES : 128u, kLanes = kPart / 16u, kStep = kThreads / kLanes, kRun = kStep * kPasses;
  static_assert(kRun >= KP_MOVE_RUN, "a run takes a whole short group");
  const uint32_t slot = threadIdx.x / kLanes, head = blockIdx.y, part = blockIdx.z >> 1;
  uint8_t* const half = g.half[blockIdx.z & 1u] + part * kPart + 16u * (threadIdx.x % kLanes);
  uint8_t* const exps = g.exps[blockIdx.z & 1u];
  const bool has_exp = E4M3 && threadIdx.x % kLanes == 0u;
  const uint32_t begin = clamp_to(g.starts[blockIdx.x], 0u, g.moves), end = clamp_to(g.starts[blockIdx.x + 1u], begin, g.moves);
  if (begin >= end) return;
  struct Slots {
    int64_t from[kPasses], to[kPasses];
  };
  struct Rows {
    u32x4 raw[kPasses];
    uint32_t to[kPasses], e[kPasses];  // to: all ones, none
  };
  auto ask_slots = [&](uint32_t m0, Slots& s) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      const uint32_t m = m0 + kStep * i + slot, at = m < end ? m : end - 1u;
      s.from[i] = g.from[at];
      s.to[i] = m < end ? g.to[at] : -1;
    }
  };
  auto ask_rows = [&](const Slots& s, Rows& r) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      const bool there = moves(g, s.from[i], s.to[i]);
      const uint32_t row = there ? row_of_slot((uint64_t)s.from[i], head, g.hkv, g.page_log2) : 0u;
      r.to[i] = there ? row_of_slot((uint64_t)s.to[i], head, g.hkv, g.page_log2) : ~0u;
      if (there) r.raw[i] = *reinterpret_cast<const u32x4*>(half + (size_t)row * BYTES);
      if (there && has_exp) r.e[i] = exps[row];
    }
  };
  // every wave has its rows in registers before any of them is written
  auto put = [&](Rows& r) __attribute__((always_inline)) {
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      asm volatile("" : "+v"(r.raw[i])::"memory");
      if constexpr (E4M3) asm volatile("" : "+v"(r.e[i])::"memory");
    }
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      if (r.to[i] == ~0u) continue;
      *reinterpret_cast<u32x4*>(half + (size_t)r.to[i] * BYTES) = r.raw[i];
      if (has_exp) exps[r.to[i]] = (uint8_t)r.e[i];
    }
  };
  Slots s;
  Rows now, next;
  ask_slots(begin, s);
  ask_rows(s, now);
  if (end - begin > kRun) ask_slots(begin + kRun, s);
  for (uint32_t m0 = begin;;) {
    if (end - m0 <= kRun) { put(now); break; }
    ask_rows(s, next);
    if (end - m0 > 2u * kRun) ask_slots(m0 + 2u * kRun, s);
    put(now);
    m0 += kRun;
    if (end - m0 <= kRun) { put(next); break; }
    ask_rows(s, now);
    if (end - m0 > 2u * kRun) ask_slots(m0 + 2u * kRun, s);
    put(next);
    m0 += kRun;
  }
}

}  // namespace

extern "C" kp_status kp_cache_move(const int64_t* from, const int64_t* to, int N, const int32_t* starts, int n_groups, const kp_cache* cache,
                                   void* stream) {
  kp::clear_error();
  if (kp_status s = check_cache(cache)) return s;
  if (N < 0 || n_groups < 0) return kp::fail(KP_ERR_INVALID_ARG, "N and n_groups must not be negative");
  if (N == 0 || (starts && n_groups == 0)) return KP_OK;
  if (!from || !to || (((uintptr_t)from | (uintptr_t)to) & 7u)) return kp::fail(KP_ERR_INVALID_ARG, "from and to must be device memory, 8-byte aligned");
  if ((uintptr_t)starts & 3u) return kp::fail(KP_ERR_INVALID_ARG, "starts must be device memory, 4-byte aligned");
  if ((long long)N * cache->Hkv >= (1ll << 28)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^28 or more rows in one call");
  if (starts && ((long long)n_groups * cache->Hkv * 4 >= kMostGroups || cache->Hkv > 65535)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^21 or more groups and heads in one call");
  MoveArgs g{};
  g.from = from; g.to = to; g.starts = starts;
  g.half[0] = static_cast<uint8_t*>(cache->k); g.half[1] = static_cast<uint8_t*>(cache->v);
  g.exps[0] = cache->k_exp; g.exps[1] = cache->v_exp;
  g.moves = (uint32_t)N; g.groups = (uint32_t)n_groups; g.hkv = (uint32_t)cache->Hkv; g.page_log2 = log2_of(cache->page);
  g.n_slots = (uint64_t)cache->n_pages * (uint64_t)cache->page;
  while (g.run_log2 < kMostRunLog2 && 2u << g.run_log2 <= g.moves) ++g.run_log2;
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3;
  const uint32_t bytes = (uint32_t)cache->D * (e4m3 ? 1u : 2u), per = kThreads / (bytes / 16u) * kRows, runs = (g.moves + (1u << g.run_log2) - 1u) >> g.run_log2;
  const dim3 apart(((runs * g.hkv << g.run_log2) + per - 1u) / per, 2), groups(g.groups, g.hkv, bytes > 128u ? 4u : 2u);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define KP_LAUNCH(B, E) do { if (starts) hipLaunchKernelGGL((kp_cache_move_groups<B, E>), groups, dim3(kThreads), 0, st, g); \
                             else hipLaunchKernelGGL((kp_cache_move_apart<B, E>), apart, dim3(kThreads), 0, st, g); } while (0)
  if (e4m3) { if (cache->D == 64) KP_LAUNCH(64, true); else KP_LAUNCH(128, true); }
  else if (cache->D == 64) KP_LAUNCH(128, false); else KP_LAUNCH(256, false);
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}
