// The gradient of log probabilities and entropy with respect to the queries (include/hps_mx4.h: hps_mx4_logprobs_backward).
//
// With p_r = exp(s_r - lse), U the sum of the upstream gradients u_g of the given rows' log probabilities
// and h that of the entropy H:  dL/ds_r = c_r + (u_g where r is given),  c_r = -p_r (U + h (log p_r + H)),
// d query = scale * (sum_r c_r row_r + sum_g u_g row_g).
// mx_gradient: a workgroup takes 32 queries, a part of the rows and 64 of the columns; it works c out for 32 rows
// at a time (as mx_softmax does their scores) and adds c row to its sums.  mx_gradient_end adds the parts and the given rows.
#pragma once

#include "mx4_logprobs.hpp"

namespace hps {

constexpr u32 kMxGradColumns = 64;

// One value of a held row.
__device__ __forceinline__ float mx_value(const MxHeld& m, u32 row, u32 col, u32 row_bytes, u32 blocks) {
  const u32 codes = m.codes[(u64)row * row_bytes + col / 2] >> (4 * (col & 1u)) & 15u;
  return mx_decode(codes, m.scales[(u64)row * blocks + col / kMxBlock]).v[0];
}

// The upstream gradient of a given row, 0 where it has no part in it.
template <bool BIAS>
__device__ __forceinline__ float mx_upstream(const i32* given, const float* d_logp, u64 at, u32 n_rows, const float* bias) {
  const i32 g = given[at];
  if (g < 0 || (u32)g >= n_rows) return 0.f;
  if (BIAS && mx_bias(bias, (u32)g) == -kMxInf) return 0.f;
  return d_logp[at];
}

template <int WIDTH, bool BIAS>
__global__ void __launch_bounds__(kMxThreads)
mx_gradient(MxHeld queries, MxHeld rows, u32 dim, u32 blocks, u32 row_bytes, float scale, const float* __restrict__ bias,
            const float* __restrict__ lse, const float* __restrict__ entropy, const i32* __restrict__ given, const float* __restrict__ d_logp,
            u32 n_given, const float* __restrict__ d_entropy, u32 part_rows, float* __restrict__ parts) {
  __shared__ float s_c[kMxTile][kMxTile + 1];
  __shared__ float s_w[kMxTile][kMxGradColumns];
  const u32 lane = lane_id(), half = lane / 32, wave = threadIdx.x / kWave;
  const u32 part = blockIdx.x, query0 = blockIdx.y * kMxTile, col0 = blockIdx.z * kMxGradColumns;
  const u32 mine = min(query0 + lane % 32, queries.n - 1);
  float u_all = 0.f;
  for (u32 g = 0; g < n_given; ++g) u_all += mx_upstream<BIAS>(given, d_logp, (u64)mine * n_given + g, rows.n, bias);
  const float q_lse = lse[mine], h = d_entropy ? d_entropy[mine] : 0.f, q_entropy = d_entropy ? entropy[mine] : 0.f;
  float sum[8] = {};
  const u32 first = part * part_rows, end = min(rows.n - first, part_rows) + first;
  for (u32 row0 = first; row0 < end; row0 += kMxTile) {
    __syncthreads();
    if (wave == 0) {
      const MxTile d = mx_products_once<WIDTH>(rows, min(row0 + lane % 32, rows.n - 1), queries, mine, blocks);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const u32 i = mx_row_of(r, half), row = row0 + i;
        const float s = row < end ? mx_score<BIAS>(d[r], scale, BIAS ? mx_bias(bias, row) : 0.f) : -kMxInf;
        const float t = s - q_lse, p = expf(t);
        // (p is 0 for rows that are out and for those far below, whose log p may be too large to multiply with)
        s_c[i][lane % 32] = s == -kMxInf || p == 0.f ? 0.f : -p * (u_all + h * (t + q_entropy));
      }
    }
    for (u32 i = threadIdx.x; i < kMxTile * kMxGradColumns; i += kMxThreads) {
      const u32 row = row0 + i / kMxGradColumns, col = col0 + i % kMxGradColumns;
      // (a row that is out adds nothing, also where it stands for NaN)
      const bool in = row < end && col < dim && !(BIAS && mx_bias(bias, row) == -kMxInf);
      s_w[i / kMxGradColumns][i % kMxGradColumns] = in ? mx_value(rows, row, col, row_bytes, blocks) : 0.f;
    }
    __syncthreads();
    const u32 q = threadIdx.x % 32, c0 = threadIdx.x / 32 * 8;
    for (u32 i = 0; i < kMxTile; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += s_c[i][q] * s_w[i][c0 + k];
  }
  const u32 q = query0 + threadIdx.x % 32, c0 = col0 + threadIdx.x / 32 * 8;
  if (q < queries.n)
    for (int k = 0; k < 8; ++k)
      if (c0 + k < dim) parts[((u64)part * queries.n + q) * dim + c0 + k] = sum[k];
}

template <bool BIAS>
__global__ void __launch_bounds__(kMxThreads)
mx_gradient_end(MxHeld rows, u32 n_queries, u32 dim, u32 blocks, u32 row_bytes, float scale, const float* __restrict__ bias,
                const i32* __restrict__ given, const float* __restrict__ d_logp, u32 n_given, const float* __restrict__ parts,
                u32 n_parts, float* __restrict__ out) {
  const u64 total = (u64)n_queries * dim;
  for (u64 i = (u64)blockIdx.x * kMxThreads + threadIdx.x; i < total; i += (u64)gridDim.x * kMxThreads) {
    const u32 query = (u32)(i / dim), col = (u32)(i - (u64)query * dim);
    float sum = 0.f;
    for (u32 p = 0; p < n_parts; ++p) sum += parts[p * total + i];
    for (u32 g = 0; g < n_given; ++g) {
      const u64 at = (u64)query * n_given + g;
      const float u = mx_upstream<BIAS>(given, d_logp, at, rows.n, bias);
      if (u != 0.f) sum += u * mx_value(rows, (u32)given[at], col, row_bytes, blocks);
    }
    out[i] = scale * sum;
  }
}

}  // namespace hps
