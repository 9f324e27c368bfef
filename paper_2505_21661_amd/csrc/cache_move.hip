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

// Groups of moves in order: a workgroup has one head of one group, and takes its rows in runs, each read whole before it is
// written.  blockIdx: group, head, keys or values.
constexpr uint32_t kPasses = 8;
template <uint32_t BYTES, bool E4M3>
__global__ __launch_bounds__(kThreads) void kp_cache_move_groups(MoveArgs g) {
  constexpr uint32_t kLanes = BYTES / 16u, kStep = kThreads / kLanes, kRun = kStep * kPasses;
  static_assert(kRun >= KP_MOVE_RUN, "a run takes a whole short group");
  const uint32_t slot = threadIdx.x / kLanes, c = threadIdx.x % kLanes, head = blockIdx.y;
  uint8_t* const half = g.half[blockIdx.z];
  uint8_t* const exps = g.exps[blockIdx.z];
  const uint32_t begin = clamp_to(g.starts[blockIdx.x], 0u, g.moves), end = clamp_to(g.starts[blockIdx.x + 1u], begin, g.moves);
  for (uint32_t m0 = begin; m0 < end; m0 += kRun) {
    uint32_t to[kPasses];
    u32x4 raw[kPasses];
    uint8_t e[kPasses];
    bool there[kPasses];
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      const uint32_t m = m0 + kStep * i + slot;
      there[i] = false;
      if (m0 + kStep * i >= end) continue;
      const int64_t a = g.from[m < end ? m : end - 1u], b = g.to[m < end ? m : end - 1u];
      there[i] = m < end && moves(g, a, b);
      const uint32_t row = there[i] ? row_of_slot((uint64_t)a, head, g.hkv, g.page_log2) : 0u;
      to[i] = there[i] ? row_of_slot((uint64_t)b, head, g.hkv, g.page_log2) : 0u;
      raw[i] = *reinterpret_cast<const u32x4*>(half + (size_t)row * BYTES + 16u * c);
      if constexpr (E4M3) e[i] = exps[row];
    }
    // every wave's rows are in its registers before any of them is written
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kPasses; ++i) {
      if (!there[i]) continue;
      *reinterpret_cast<u32x4*>(half + (size_t)to[i] * BYTES + 16u * c) = raw[i];
      if constexpr (E4M3)
        if (c == 0) exps[to[i]] = e[i];
    }
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
  if (starts && ((long long)n_groups * cache->Hkv * 2 >= kMostGroups || cache->Hkv > 65535)) return kp::fail(KP_ERR_UNSUPPORTED_SHAPE, "2^22 or more groups and heads in one call");
  MoveArgs g{};
  g.from = from; g.to = to; g.starts = starts;
  g.half[0] = static_cast<uint8_t*>(cache->k); g.half[1] = static_cast<uint8_t*>(cache->v);
  g.exps[0] = cache->k_exp; g.exps[1] = cache->v_exp;
  g.moves = (uint32_t)N; g.groups = (uint32_t)n_groups; g.hkv = (uint32_t)cache->Hkv; g.page_log2 = log2_of(cache->page);
  g.n_slots = (uint64_t)cache->n_pages * (uint64_t)cache->page;
  while (g.run_log2 < kMostRunLog2 && 2u << g.run_log2 <= g.moves) ++g.run_log2;
  const bool e4m3 = cache->cache_type == KP_CACHE_E4M3;
  const uint32_t bytes = (uint32_t)cache->D * (e4m3 ? 1u : 2u), per = kThreads / (bytes / 16u) * kRows, runs = (g.moves + (1u << g.run_log2) - 1u) >> g.run_log2;
  const dim3 apart(((runs * g.hkv << g.run_log2) + per - 1u) / per, 2), groups(g.groups, g.hkv, 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define KP_LAUNCH(B, E) do { if (starts) hipLaunchKernelGGL((kp_cache_move_groups<B, E>), groups, dim3(kThreads), 0, st, g); \
                             else hipLaunchKernelGGL((kp_cache_move_apart<B, E>), apart, dim3(kThreads), 0, st, g); } while (0)
  if (e4m3) { if (cache->D == 64) KP_LAUNCH(64, true); else KP_LAUNCH(128, true); }
  else if (cache->D == 64) KP_LAUNCH(128, false); else KP_LAUNCH(256, false);
#undef KP_LAUNCH
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}
