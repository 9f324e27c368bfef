// Attention of a tile of query rows over the keys they see (the kernels behind kp_attn_window and kp_attn_paged).
#pragma once
#include "kp_attn.h"

namespace kp {
namespace attn {

constexpr int kThreads = 256;

// Where row `flat` (token by token, query heads of a group within a token) of a tile's sequence lies.
struct RowPlace {
  uint32_t token, in_group;
};
__device__ __forceinline__ RowPlace place_of(uint32_t flat, uint32_t group) {
  RowPlace r;
  r.token = group == 1u ? flat : flat / group;
  r.in_group = flat - r.token * group;
  return r;
}

template <class T, int D, int SRC>
__global__ __launch_bounds__(kThreads) void kp_attn_row_by_row(Args g) {
  constexpr int kRows = 16;
  const uint32_t h = blockIdx.x % g.hkv, lane = threadIdx.x & 63u;
  Tile tile;
  if (!find_tile<kRows, SRC != kPlain>(g, blockIdx.x / g.hkv, &tile)) return;
  const Source<D, SRC> src(g, tile.seq, h);
  for (uint32_t r = threadIdx.x >> 6; r < kRows; r += kThreads / 64) {
    const uint32_t flat = tile.first + r;
    if (flat >= tile.rows) break;
    const RowPlace at = place_of(flat, g.group);
    const uint32_t head = h * g.group + at.in_group, seq = SRC == kPlain ? tile.seq : 0u;
    const int64_t token = (int64_t)tile.q0 + at.token;
    float q[D / 64];
    row_elements<T, D / 64>(reinterpret_cast<const uint8_t*>(g.q.at + g.q.seq * seq + g.q.head * head + g.q.token * token), lane, q);
    Row<D / 64> row;
    row_over_keys<T, D, SRC>(row, q, src, (int32_t)tile.n_k - (int32_t)tile.n_q + (int32_t)at.token, g.window, g.sinks, g.scale_log2, 0u, tile.n_k);
    store_row<T, D / 64>(row, const_cast<uint16_t*>(g.o.at) + g.o.seq * seq + g.o.head * head + g.o.token * token,
                         g.lse ? g.lse + g.lse_seq * seq + g.lse_head * head + token : nullptr);
  }
}

}  // namespace attn
}  // namespace kp
