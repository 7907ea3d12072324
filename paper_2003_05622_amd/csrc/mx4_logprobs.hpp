// Log probabilities over the scores of each query, none of which is stored (include/hps_mx4.h: hps_mx4_logprobs).
//
// One pass over the rows.  mx_softmax: a wave holds 32 queries, one per lane of either half, and goes through a
// part of the rows, 32 at a time; the matrix instruction leaves every lane with 16 rows' products for its query, so
// the running maximum m, the sum l = sum e^(s - m) and e = sum e^(s - m) (s - m) are the lane's own
// registers.  log-sum-exp = m + log l, entropy = log l - e / l.  For the best rows it notes the highest score of
// each group of `group` neighbouring rows.
//
// mx_finish, a workgroup per query: joins the parts; takes the `top` best groups by their highest
// score, the earlier group first among equals; scores the rows of these groups again and takes the best.  No
// other group can hold one of the best rows: each of the chosen groups has a row that comes before all rows of a group
// that was not chosen (its highest score is higher, or equal and its row number lower).
#pragma once

#include "mx4.hpp"

namespace hps {

constexpr float kMxLog2e = 1.44269504088896340736f;
constexpr float kMxLn2 = 0.69314718055994530942f;
constexpr float kMxInf = __builtin_huge_valf();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

struct MxPart {        // what a part of the rows adds to a query, m in scores
  float m, l, e;
};
__device__ __forceinline__ MxPart mx_no_part() { return {-3.402823466e38f, 0.f, 0.f}; }
__device__ __forceinline__ MxPart mx_join(const MxPart& a, const MxPart& b) {
  const float m = fmaxf(a.m, b.m);
  MxPart s = {m, 0.f, 0.f};
  // (a part without rows adds nothing, whatever its m)
  if (a.l != 0.f) {
    const float d = a.m - m, f = expf(d);
    s.l += a.l * f;
    s.e += f == 0.f ? 0.f : (a.e + a.l * d) * f;
  }
  if (b.l != 0.f) {
    const float d = b.m - m, f = expf(d);
    s.l += b.l * f;
    s.e += f == 0.f ? 0.f : (b.e + b.l * d) * f;
  }
  return s;
}

template <int WIDTH, bool BIAS>
__global__ void __launch_bounds__(kWave)
mx_softmax(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, u32 part_rows, u32 group,
           u32 n_groups, MxPart* __restrict__ parts, float* __restrict__ highest) {
  const u32 lane = lane_id(), half = lane / 32;
  const u32 query = blockIdx.y * kMxTile + lane % 32, part = blockIdx.x;
  const u32 q = min(query, queries.n - 1);
  const u32 first = part * part_rows, end = min(rows.n - first, part_rows) + first;
  MxPart sum = mx_no_part();
  float high = -kMxInf;
  for (u32 row0 = first; row0 < end; row0 += kMxTile) {
    const MxTile d = mx_products<WIDTH>(rows, min(row0 + lane % 32, rows.n - 1), queries, q, blocks);
    float s[16], most = -kMxInf;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const u32 row = row0 + mx_row_of(r, half);
      s[r] = row < end ? mx_score<BIAS>(d[r], scale, BIAS ? mx_bias(bias, row) : 0.f) : -kMxInf;
      most = fmaxf(most, s[r]);
    }
    high = fmaxf(high, most);
    const float m = fmaxf(sum.m, most);
    if (sum.l != 0.f) {
      const float by = sum.m - m, f = exp2_fast(by * kMxLog2e);
      sum.e = f == 0.f ? 0.f : (sum.e + sum.l * by) * f;
      sum.l *= f;
    }
    sum.m = m;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float t = s[r] - m, p = exp2_fast(t * kMxLog2e);
      sum.l += p;
      sum.e += p * fmaxf(t, -1e30f);
    }
    if (highest && ((row0 - first + kMxTile) % group == 0 || row0 + kMxTile >= end)) {
      high = fmaxf(high, __shfl_xor(high, 32, kWave));
      if (half == 0 && query < queries.n) highest[(u64)query * n_groups + row0 / group] = high;
      high = -kMxInf;
    }
  }
  const MxPart other = {__shfl_xor(sum.m, 32, kWave), __shfl_xor(sum.l, 32, kWave), __shfl_xor(sum.e, 32, kWave)};
  sum = mx_join(sum, other);
  if (half == 0 && query < queries.n) parts[(u64)query * gridDim.x + part] = sum;
}

// ---- the best of many, 64 at a time -----------------------------------------------------------
// A candidate is a score and a number in one 64-bit word that is larger the better it comes: the score in the
// order of whole numbers, below it the number's complement.  0 is none.
__device__ __forceinline__ u64 mx_candidate(float score, u32 number) {
  const u32 b = __float_as_uint(score + 0.f);          // (-0 and 0 are equal)
  return (u64)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (u32)~number;
}
__device__ __forceinline__ float mx_candidate_score(u64 c) {
  const u32 b = (u32)(c >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7FFFFFFFu : ~b);
}
__device__ __forceinline__ u32 mx_candidate_number(u64 c) { return ~(u32)c; }

__device__ __forceinline__ u64 mx_exchange(u64 c, u32 distance, bool larger) {
  const u64 o = __shfl_xor((unsigned long long)c, (int)distance, kWave);
  return (o > c) == larger ? o : c;
}
// Lane i gets the i-th largest of the wave's 64 candidates.
__device__ __forceinline__ u64 mx_sort(u64 c) {
  const u32 lane = lane_id();
#pragma unroll
  for (u32 run = 2; run <= 64; run *= 2)
#pragma unroll
    for (u32 d = run / 2; d; d /= 2) c = mx_exchange(c, d, ((lane & run) == 0) == ((lane & d) == 0));
  return c;
}
// Of two lists in descending order the 64 largest, in descending order.
__device__ __forceinline__ u64 mx_merge(u64 a, u64 b) {
  const u32 lane = lane_id();
  const u64 r = __shfl((unsigned long long)b, 63 - (int)lane, kWave);
  u64 c = a > r ? a : r;
#pragma unroll
  for (u32 d = 32; d; d /= 2) c = mx_exchange(c, d, (lane & d) == 0);
  return c;
}
// Adds 64 candidates to a list of which the first `top` count.
__device__ __forceinline__ void mx_offer(u64* list, u64 c, u32 top) {
  const u64 least = __shfl((unsigned long long)*list, (int)top - 1, kWave);
  if (__any(c > least)) *list = mx_merge(*list, mx_sort(c));
}

constexpr int kMxFinishWaves = 4;

// The product of one query with the row each lane names (below n).
template <int WIDTH>
__device__ __forceinline__ float mx_dots(const MxHeld& queries, u32 query, const MxHeld& rows, u32 row, u32 blocks) {
  const u32 lane = lane_id();
  const u32 low = (u32)__shfl((int)row, (int)(lane % 32), kWave), high = (u32)__shfl((int)row, (int)(lane % 32 + 32), kWave);
  const MxTile a = mx_products<WIDTH>(queries, query, rows, low, blocks);
  const MxTile b = mx_products<WIDTH>(queries, query, rows, high, blocks);
  return lane < 32 ? a[0] : b[0];
}

template <int WIDTH, bool BIAS>
__global__ void __launch_bounds__(kMxFinishWaves * kWave)
mx_finish(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, const MxPart* __restrict__ parts,
          u32 n_parts, const float* __restrict__ highest, u32 group, u32 n_groups, const i32* __restrict__ given, u32 n_given,
          u32 top, float* __restrict__ lse_out, float* __restrict__ entropy_out, float* __restrict__ logp_out,
          i32* __restrict__ top_index, float* __restrict__ top_logp) {
  __shared__ u64 s_list[kMxFinishWaves][kWave];
  __shared__ MxPart s_part[kMxFinishWaves];
  const u32 lane = lane_id(), wave = threadIdx.x / kWave, query = blockIdx.x;
  // join the parts: every wave some, then every wave all waves'
  MxPart sum = mx_no_part();
  for (u32 i = threadIdx.x; i < n_parts; i += kMxFinishWaves * kWave) sum = mx_join(sum, parts[(u64)query * n_parts + i]);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const MxPart o = {__shfl_xor(sum.m, d, kWave), __shfl_xor(sum.l, d, kWave), __shfl_xor(sum.e, d, kWave)};
    sum = mx_join(sum, o);
  }
  if (lane == 0) s_part[wave] = sum;
  u64 best = 0;
  if (top) {
    for (u32 i0 = wave * kWave; i0 < n_groups; i0 += kMxFinishWaves * kWave) {
      const u32 g = i0 + lane;
      const float h = g < n_groups ? highest[(u64)query * n_groups + g] : 0.f;
      mx_offer(&best, g < n_groups ? mx_candidate(h, g) : 0, top);
    }
    s_list[wave][lane] = best;
  }
  __syncthreads();
  sum = s_part[0];
#pragma unroll
  for (int w = 1; w < kMxFinishWaves; ++w) sum = mx_join(sum, s_part[w]);
  const bool empty = sum.l == 0.f;
  const float lse = empty ? -kMxInf : sum.m + logf(sum.l);
  if (threadIdx.x == 0) {
    lse_out[query] = lse;
    entropy_out[query] = empty ? 0.f : logf(sum.l) - sum.e / sum.l;
  }
  if (top) {
    best = s_list[0][lane];
#pragma unroll
    for (int w = 1; w < kMxFinishWaves; ++w) best = mx_merge(best, s_list[w][lane]);
    __syncthreads();
    u64 list = 0;
    for (u32 i = wave; i < top; i += kMxFinishWaves) {
      const u64 c = __shfl((unsigned long long)best, (int)i, kWave);
      if (c == 0) break;
      const u32 g = mx_candidate_number(c);
      for (u32 k = 0; k < group; k += kWave) {
        const u32 row = g * group + k + lane;
        const bool in = k + lane < group && row < rows.n;
        const u32 at = in ? row : rows.n - 1;
        const float dot = mx_dots<WIDTH>(queries, query, rows, at, blocks);
        const float s = mx_score<BIAS>(dot, scale, BIAS ? mx_bias(bias, at) : 0.f);
        // (a NaN and a row taken out are no candidates)
        mx_offer(&list, in && s > -kMxInf ? mx_candidate(s, row) : 0, top);
      }
    }
    s_list[wave][lane] = list;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 1; w < kMxFinishWaves; ++w) list = mx_merge(list, s_list[w][lane]);
      if (lane < top) {
        top_index[(u64)query * top + lane] = list ? (i32)mx_candidate_number(list) : -1;
        top_logp[(u64)query * top + lane] = list ? mx_candidate_score(list) - lse : -kMxInf;
      }
    }
  }
  for (u32 i0 = wave * kWave; i0 < n_given; i0 += kMxFinishWaves * kWave) {
    const u32 i = i0 + lane;
    const i32 g = i < n_given ? given[(u64)query * n_given + i] : -1;
    const bool in = g >= 0 && (u32)g < rows.n;
    const u32 at = in ? (u32)g : rows.n - 1;
    const float dot = mx_dots<WIDTH>(queries, query, rows, at, blocks);
    const float s = mx_score<BIAS>(dot, scale, BIAS ? mx_bias(bias, at) : 0.f);
    if (i < n_given)
      logp_out[(u64)query * n_given + i] = g < 0 ? 0.f : !in ? __uint_as_float(0x7FC00000u) : s == -kMxInf ? s : s - lse;
  }
}

// Without a row: nothing to sum, nothing to take.
__global__ void __launch_bounds__(kMxThreads)
mx_no_rows(u32 n_queries, const i32* __restrict__ given, u32 n_given, u32 top, float* __restrict__ lse_out, float* __restrict__ entropy_out,
           float* __restrict__ logp_out, i32* __restrict__ top_index, float* __restrict__ top_logp) {
  for (u64 i = (u64)blockIdx.x * kMxThreads + threadIdx.x; i < (u64)n_queries * max(max(n_given, top), 1u); i += (u64)gridDim.x * kMxThreads) {
    if (i < n_queries) { lse_out[i] = -kMxInf; entropy_out[i] = 0.f; }
    if (i < (u64)n_queries * n_given) logp_out[i] = given[i] < 0 ? 0.f : __uint_as_float(0x7FC00000u);
    if (i < (u64)n_queries * top) { top_index[i] = -1; top_logp[i] = -kMxInf; }
  }
}

}  // namespace hps
