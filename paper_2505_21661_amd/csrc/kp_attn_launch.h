// Launches the attention kernels of a call that has been checked.
#pragma once
#include "kp_attn_few.h"
#include "kp_attn_host.h"
#include "kp_attn_rows.h"

namespace kp {
namespace attn {

template <class T, int D, int SRC>
kp_status launch(Args& g, const Plan& plan, hipStream_t st) {
  const long long grid = plan.units * plan.splits;
  constexpr long long kJoinRows = kThreads / (D / 4);
  if (grid >= (1ll << 31) || plan.units * (kTileRows / kJoinRows) >= (1ll << 31)) return fail(KP_ERR_UNSUPPORTED_SHAPE, "2^31 or more workgroups");
  g.tiles = (uint32_t)plan.tiles;
  g.splits = (uint32_t)plan.splits;
  if (plan.few) hipLaunchKernelGGL((kp_attn_few<T, D, SRC>), dim3((uint32_t)grid), dim3(kThreads), 0, st, g);
  else hipLaunchKernelGGL((kp_attn_tile<T, D, SRC, 0>), dim3((uint32_t)grid), dim3(kThreads), tile_lds_bytes<D>(), st, g);
  KP_HIP_TRY(hipGetLastError());
  if (plan.splits > 1) {
    if (plan.few) hipLaunchKernelGGL((kp_attn_join<T, D, kFewRows, SRC != kPlain>), dim3((uint32_t)(plan.units * kFewRows / kJoinRows)), dim3(kThreads), 0, st, g);
    else hipLaunchKernelGGL((kp_attn_join<T, D, kTileRows, SRC != kPlain>), dim3((uint32_t)(plan.units * kTileRows / kJoinRows)), dim3(kThreads), 0, st, g);
    KP_HIP_TRY(hipGetLastError());
  }
  return KP_OK;
}

}  // namespace attn
}  // namespace kp
