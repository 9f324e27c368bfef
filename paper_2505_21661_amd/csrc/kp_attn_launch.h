// Launches the attention kernels of a call that has been checked.
#pragma once
#include "kp_attn_few.h"
#include "kp_attn_host.h"
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

// The recording arguments of a call on n_wg workgroups of 4 waves and 3 regions; *ring_bytes: LDS that the records take
// (0: nothing is recorded).
inline kp_status recording(Args& g, const Plan& plan, uint32_t region_mask, void* trace_buf, size_t trace_cap, size_t* ring_bytes) {
  const uint32_t regions = region_mask & ~(KP_MASK_FLUSH | KP_MASK_WAVE_GROUP | KP_MASK_REALTIME | KP_MASK_COLLAB);
  *ring_bytes = 0;
  if (region_mask & KP_MASK_PHASES) return fail(KP_ERR_INVALID_ARG, "KP_MASK_PHASES belongs to the GEMM");
  if (regions == 0) return KP_OK;
  if (!trace_buf) return fail(KP_ERR_INVALID_ARG, "trace_buf is NULL but region_mask enables regions");
  if (regions >> 3) return fail(KP_ERR_INVALID_ARG, "region_mask enables regions this kernel does not have (3 regions)");
  if (!aligned16(trace_buf)) return fail(KP_ERR_INVALID_ARG, "trace_buf must be 16-byte aligned");
  g.group_log2 = (region_mask & KP_MASK_WAVE_GROUP) ? 2u : 0u;
  const size_t streams = 4u >> g.group_log2, cap_wave = trace_cap / streams;
  if (trace_cap % streams || !is_pow2(cap_wave) || cap_wave < 2 || cap_wave > (1u << 19))
    return fail(KP_ERR_TRACE_TOO_SMALL, "trace_cap/streams = %zu must be a power of two >= 2", cap_wave);
  g.region_mask = regions; g.flush = region_mask >> 31;
  g.collab = (region_mask & KP_MASK_COLLAB) ? 1u : 0u;
  g.flags = (g.flush ? KP_FLAG_FLUSH : 0u) | ((region_mask & KP_MASK_REALTIME) ? KP_FLAG_REALTIME : 0u) | (g.collab ? KP_FLAG_HW_IDS : 0u);
  g.trace = trace_buf; g.n_wg = (uint32_t)(plan.units * plan.splits); g.rec_cost = rec_cost();
  g.cap_hbm = (uint32_t)cap_wave;
  g.cap_lds = g.flush && cap_wave > 64 ? 64u : (uint32_t)cap_wave;
  *ring_bytes = (size_t)g.cap_lds * 8 * streams;
  if (*ring_bytes > 16 * 1024) return fail(KP_ERR_UNSUPPORTED_SHAPE, "LDS ring of %zu bytes exceeds the 16 KiB budget", *ring_bytes);
  return KP_OK;
}

template <class T, int D, int SRC, int INSTR>
kp_status launch_as(const Args& g, const Plan& plan, size_t ring_bytes, hipStream_t st) {
  const dim3 grid((uint32_t)(plan.units * plan.splits)), block(kThreads);
  if (plan.few) hipLaunchKernelGGL((kp_attn_few<T, D, SRC, INSTR>), grid, block, ring_bytes, st, g);
  else hipLaunchKernelGGL((kp_attn_tile<T, D, SRC, INSTR>), grid, block, tile_lds_bytes<D>() + ring_bytes, st, g);
  KP_HIP_TRY(hipGetLastError());
  return KP_OK;
}

template <class T, int D, int SRC>
kp_status launch(Args& g, const Plan& plan, uint32_t region_mask, void* trace_buf, size_t trace_cap, hipStream_t st) {
  constexpr long long kJoinRows = kThreads / (D / 4);
  if (plan.units * plan.splits >= kMostGroups) return fail(KP_ERR_UNSUPPORTED_SHAPE, "2^23 or more workgroups");
  g.tiles = (uint32_t)plan.tiles;
  g.splits = (uint32_t)plan.splits;
  size_t ring_bytes = 0;
  if (kp_status s = recording(g, plan, region_mask, trace_buf, trace_cap, &ring_bytes)) return s;
  if (kp_status s = ring_bytes == 0 ? launch_as<T, D, SRC, 0>(g, plan, 0, st)
                    : (region_mask & KP_MASK_REALTIME) ? launch_as<T, D, SRC, 3>(g, plan, ring_bytes, st) : launch_as<T, D, SRC, 1>(g, plan, ring_bytes, st))
    return s;
  if (plan.splits > 1) {
    constexpr bool kPages = SRC != kPlain;
    const bool wide = plan.splits > (long long)kJoinAtOnce;
    const dim3 grid((uint32_t)(plan.units * (plan.few ? kFewRows : kTileRows) / (wide ? 1 : kJoinRows))), block(kThreads);
    if (plan.few && wide) hipLaunchKernelGGL((kp_attn_join<T, D, kFewRows, kPages, true>), grid, block, 0, st, g);
    else if (plan.few) hipLaunchKernelGGL((kp_attn_join<T, D, kFewRows, kPages, false>), grid, block, 0, st, g);
    else if (wide) hipLaunchKernelGGL((kp_attn_join<T, D, kTileRows, kPages, true>), grid, block, 0, st, g);
    else hipLaunchKernelGGL((kp_attn_join<T, D, kTileRows, kPages, false>), grid, block, 0, st, g);
    KP_HIP_TRY(hipGetLastError());
  }
  return KP_OK;
}

}  // namespace attn
}  // namespace kp
