// All scores of queries against rows (include/hps_mx4.h: hps_mx4_scores).
//
// One wave computes 32 queries x 32 rows; lanes lie along the rows, so that each store of a register writes
// 32 neighbouring scores of a query.
#pragma once

#include "mx4.hpp"

namespace hps {

template <int WIDTH, bool BIAS, bool BF16>
__global__ void __launch_bounds__(kMxThreads)
mx_scores(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, void* __restrict__ out, u64 stride,
          u32 row_tiles) {
  const u32 lane = lane_id(), half = lane / 32, wave = threadIdx.x / kWave;
  const u32 row_tile = blockIdx.x % row_tiles, query_tile = blockIdx.x / row_tiles;
  const u32 row = (row_tile * (kMxThreads / kWave) + wave) * kMxTile + lane % 32, query0 = query_tile * kMxTile;
  if (row - lane % 32 >= rows.n) return;
  const MxTile d = mx_products_once<WIDTH>(queries, min(query0 + lane % 32, queries.n - 1), rows, min(row, rows.n - 1), blocks);
  if (row >= rows.n) return;
  const float b = BIAS ? mx_bias(bias, row) : 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const u32 q = query0 + mx_row_of(r, half);
    if (q >= queries.n) continue;
    const float s = mx_score<BIAS>(d[r], scale, b);
    if (BF16) static_cast<uint16_t*>(out)[q * stride + row] = (uint16_t)bf16_nearest(s);
    else static_cast<float*>(out)[q * stride + row] = s;
  }
}

}  // namespace hps
