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
//
// What bounds them.  mx_softmax: the vector unit; 64 scores take one exponential (8 cycles) and, of 4 cycles each, half a
// maximum, two multiply-adds and an addition: 180 us for 1024 queries and 1 M rows at the 2.0 GHz the GPU keeps then, 215 measured
// (93 % busy), of which the matrix unit needs 7 % at 64 values a row.  With one query, reading: 142 MB in 33 us.  So a
// maximum is taken of products, not scores, the scale goes into the exponent's factor, and sums are only raised to a new
// maximum when a wave has one.  mx_finish: some eight steps that each wait for the one before, 14 us for one query, 22 for 1024.
#pragma once

#include "mx4.hpp"

namespace hps {

constexpr float kMxLog2e = 1.44269504088896340736f;
constexpr float kMxLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }     // (2^x below 2^-126 is 0)

// What some rows add to a query.  m and the exponents behind l and e are in products (of a biased query: in scores), times
// `unit` they are in powers of two: l = sum 2^((x - m) unit), e = sum 2^((x - m) unit) (x - m) unit.
struct MxPart {
  float m, l, e;
};
constexpr float kMxLowest = -3.402823466e38f;
__device__ __forceinline__ MxPart mx_no_part() { return {kMxLowest, 0.f, 0.f}; }
// The power of two by which sums for m `from` count for a higher m.  (The difference may be beyond float32, and the unit 0.)
__device__ __forceinline__ float mx_drop(float from, float m, float unit) { return fmaxf(from - m, kMxLowest) * unit; }
// Brings a part to a higher m.
__device__ __forceinline__ void mx_raise(MxPart* a, float m, float unit) {
  const float by = mx_drop(a->m, m, unit), f = exp2f(by);
  a->e = f == 0.f ? 0.f : (a->e + a->l * by) * f;       // (`by` may be too large to multiply with)
  a->l *= f;
  a->m = m;
}
__device__ __forceinline__ MxPart mx_join(MxPart a, MxPart b, float unit) {
  const float m = fmaxf(a.m, b.m);
  mx_raise(&a, m, unit);
  mx_raise(&b, m, unit);
  return {m, a.l + b.l, a.e + b.e};
}
// The part of a query that stands for NaN, worked out with another: NaN if it has met a row that is not out.
__device__ __forceinline__ void mx_put_nan(bool nan, MxPart* a) {
  if (nan && a->l > 0.f) a->l = __uint_as_float(0x7FC00000u);
}

// Rows of a part whose sums a wave holds in 32 bits.  (With many queries a part has millions: added up one after the other, their sum is off by 3e-4 at
// 2 M rows, 2e-6 like this.)
constexpr u32 kMxSumRows = 4096;

// The sums of the rows before those, in 64 bits.
struct MxLongPart {
  double l, e;
  float m;
};
__device__ __forceinline__ MxLongPart mx_no_long_part() { return {0.0, 0.0, kMxLowest}; }
// Adds a lane's sums (m of which is the highest so far) and begins new ones.
__device__ __forceinline__ void mx_put_by(MxPart* a, float unit, MxLongPart* to) {
  const float by = mx_drop(to->m, a->m, unit);
  const double f = exp2f(by), e = f == 0.0 ? 0.0 : (to->e + to->l * by) * f;
  *to = {to->l * f + a->l, e + a->e, a->m};
  a->l = a->e = 0.f;
}
__device__ __forceinline__ MxPart mx_shuffle_xor(MxPart a, int distance) {
  return {__shfl_xor(a.m, distance, kWave), __shfl_xor(a.l, distance, kWave), __shfl_xor(a.e, distance, kWave)};
}

// Adds 16 rows' products d to a query's sums.  MASKED: only rows i (of the tile) below `rows` are there.
template <bool BIAS, bool MASKED>
__device__ __forceinline__ void mx_add_rows(const MxTile& d, float scale, const float* bias, u32 rows, float unit, MxPart* sum, float* high) {
  const u32 half = lane_id() / 32;
  float x[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    x[r] = BIAS ? __fmaf_rn(d[r], scale, bias[r]) : d[r];
    if (MASKED && mx_row_of(r, half) >= rows) x[r] = -kMxInf;
  }
  float most[8];
#pragma unroll
  for (int r = 0; r < 5; ++r) most[r] = fmaxf(fmaxf(x[3 * r], x[3 * r + 1]), x[3 * r + 2]);
  most[0] = fmaxf(fmaxf(most[0], most[1]), most[2]);
  most[3] = fmaxf(fmaxf(most[3], most[4]), x[15]);
  most[0] = fmaxf(most[0], most[3]);
  *high = fmaxf(*high, most[0]);
  // (seldom, once a wave has seen some rows)
  if (__any(most[0] > sum->m)) {
    const float m = fmaxf(sum->m, most[0]), by = mx_drop(sum->m, m, unit), f = exp2_fast(by);
    sum->e = f == 0.f ? 0.f : (sum->e + sum->l * by) * f;
    sum->l *= f;
    sum->m = m;
  }
  // Rows that are out: 2^-inf.  A biased exponent may be below all numbers, and is not multiplied with then.
  const float base = -sum->m * unit;
  float l[16], e[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float t = BIAS ? (x[r] - sum->m) * unit : __fmaf_rn(x[r], unit, base);
    if (MASKED && !BIAS && mx_row_of(r, half) >= rows) t = -kMxInf;
    l[r] = exp2_fast(t);
    e[r] = BIAS || MASKED ? fmaxf(t, -1e30f) : t;
  }
  // (added up among themselves first: 16 times fewer additions onto the long sums)
  float e0 = 0.f, e1 = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    e0 = __fmaf_rn(l[r], e[r], e0);
    e1 = __fmaf_rn(l[r + 1], e[r + 1], e1);
  }
  sum->e += e0 + e1;
#pragma unroll
  for (int w = 8; w; w /= 2)
#pragma unroll
    for (int r = 0; r < w; ++r) l[r] += l[r + w];
  sum->l += l[0];
}

// A wave, QT * 32 queries, one part of the rows.
template <typename SHAPE, bool BIAS, int QT>
__global__ void __launch_bounds__(kWave) HPS_MX_WAVES
mx_softmax(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, u32 part_rows, u32 group,
           u32 n_groups, MxPart* __restrict__ parts, float* __restrict__ highest) {
  __shared__ __align__(16) float s_bias[kMxTile];
  __shared__ MxLongPart s_long[QT][kWave];
  const u32 lane = lane_id(), half = lane / 32, part = blockIdx.x;
  const u32 query0 = blockIdx.y * (QT * kMxTile) + lane % 32;
  const u32 first = part * part_rows, end = min(rows.n - first, part_rows) + first;
  // without a bias the maximum is taken of the products themselves: a negative scale goes into the queries' signs
  const float unit = BIAS ? kMxLog2e : fabsf(scale) * kMxLog2e;
  MxRow<SHAPE> q[QT];
  bool nan[QT];
  MxPart sum[QT];
  float high[QT];
#pragma unroll
  for (int k = 0; k < QT; ++k) {
    mx_load_row<SHAPE>(queries, min(query0 + k * kMxTile, queries.n - 1), blocks, &q[k]);
    mx_clear_rest<SHAPE>(blocks, &q[k]);
    if (!BIAS && scale < 0.f) mx_negate<SHAPE>(&q[k]);
    nan[k] = BIAS && mx_take_nan<SHAPE>(blocks, &q[k]);
    sum[k] = mx_no_part();
    s_long[k][lane] = mx_no_long_part();
    high[k] = -kMxInf;
  }
  MxRow<SHAPE> next;
  float next_bias = 0.f;
  if (SHAPE::AHEAD) mx_load_tile<SHAPE>(rows, first, blocks, &next);
  if (BIAS) next_bias = mx_bias(bias, min(first + lane % 32, rows.n - 1));
  u32 in_group = 0;
  for (u32 row0 = first; row0 < end; row0 += kMxTile) {
    MxRow<SHAPE> r;
    if (SHAPE::AHEAD) r = next;
    else mx_load_tile<SHAPE>(rows, row0, blocks, &r);
    const float my_bias = row0 + lane % 32 < end ? next_bias : -kMxInf;
    const u32 ahead = min(row0 + kMxTile + lane % 32, rows.n - 1);
    if (SHAPE::AHEAD) mx_load_tile<SHAPE>(rows, row0 + kMxTile, blocks, &next);
    float b[16] = {};
    if (BIAS) {
      next_bias = mx_bias(bias, ahead);
      // a row that is out has products all the same, but none that are NaN
      if (my_bias == -kMxInf) {
#pragma unroll
        for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) r.scales[w] = 0;
      }
      __builtin_amdgcn_wave_barrier();
      s_bias[lane % 32] = my_bias;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 v = *reinterpret_cast<const float4*>(&s_bias[8 * g + 4 * half]);
        b[4 * g] = v.x; b[4 * g + 1] = v.y; b[4 * g + 2] = v.z; b[4 * g + 3] = v.w;
      }
    }
    MxTile d[QT];
#pragma unroll
    for (int k = 0; k < QT; ++k) d[k] = mx_products<SHAPE>(r, q[k], blocks);
    if (BIAS || row0 + kMxTile <= end) {
#pragma unroll
      for (int k = 0; k < QT; ++k) mx_add_rows<BIAS, false>(d[k], scale, b, 0, unit, &sum[k], &high[k]);
    } else {
#pragma unroll
      for (int k = 0; k < QT; ++k) mx_add_rows<BIAS, true>(d[k], scale, b, end - row0, unit, &sum[k], &high[k]);
    }
    in_group += kMxTile;
    if (highest && (in_group == group || row0 + kMxTile >= end)) {
      in_group = 0;
#pragma unroll
      for (int k = 0; k < QT; ++k) {
        const float h = fmaxf(high[k], __shfl_xor(high[k], 32, kWave));
        const u32 query = query0 + k * kMxTile;
        if (half == 0 && query < queries.n) highest[(u64)query * n_groups + row0 / group] = h;
        high[k] = -kMxInf;
      }
    }
    if ((row0 - first) % kMxSumRows == kMxSumRows - kMxTile) {
#pragma unroll
      for (int k = 0; k < QT; ++k) mx_put_by(&sum[k], unit, &s_long[k][lane]);
    }
  }
#pragma unroll
  for (int k = 0; k < QT; ++k) {
    mx_put_by(&sum[k], unit, &s_long[k][lane]);
    sum[k] = {sum[k].m, (float)s_long[k][lane].l, (float)s_long[k][lane].e};
    sum[k] = mx_join(sum[k], mx_shuffle_xor(sum[k], 32), unit);
    if (BIAS) mx_put_nan(nan[k], &sum[k]);
    const u32 query = query0 + k * kMxTile;
    if (half == 0 && query < queries.n) parts[(u64)query * gridDim.x + part] = sum[k];
  }
}

// Wide rows and more than a few queries: the four waves of a workgroup hold 32 queries each and share the rows' tiles.
template <typename SHAPE, bool BIAS>
__global__ void __launch_bounds__(kMxThreads) HPS_MX_WAVES
mx_softmax_shared(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, u32 part_rows, u32 group,
                  u32 n_groups, MxPart* __restrict__ parts, float* __restrict__ highest) {
  typedef MxShared<SHAPE> Shared;
  __shared__ int4 s_tile[2][Shared::UNITS];
  __shared__ __align__(16) float s_bias[2][kMxTile];
  __shared__ MxLongPart s_long[kMxThreads];
  const u32 lane = lane_id(), half = lane / 32, part = blockIdx.x;
  const u32 query = (blockIdx.y * (kMxThreads / kWave) + threadIdx.x / kWave) * kMxTile + lane % 32;
  const u32 first = part * part_rows, end = min(rows.n - first, part_rows) + first;
  const float unit = BIAS ? kMxLog2e : fabsf(scale) * kMxLog2e;
  MxRow<SHAPE> q;
  mx_load_row<SHAPE>(queries, min(query, queries.n - 1), blocks, &q);
  mx_clear_rest<SHAPE>(blocks, &q);
  if (!BIAS && scale < 0.f) mx_negate<SHAPE>(&q);
  const bool nan = BIAS && mx_take_nan<SHAPE>(blocks, &q);
  MxPart sum = mx_no_part();
  s_long[threadIdx.x] = mx_no_long_part();
  float high = -kMxInf;
  int4 own[Shared::OWN];
  u32 scales[SHAPE::SCALE_WORDS];
  float my_bias = 0.f;
  Shared::load(rows, first, blocks, own);
  mx_load_scales<SHAPE>(rows, min(first + lane % 32, rows.n - 1), blocks, scales);
  if (BIAS) my_bias = mx_bias(bias, min(first + lane % 32, rows.n - 1));
  u32 in_group = 0, buffer = 0;
  for (u32 row0 = first; row0 < end; row0 += kMxTile, buffer ^= 1u) {
    Shared::store(own, blocks, s_tile[buffer]);
    u32 r_scales[SHAPE::SCALE_WORDS];
#pragma unroll
    for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) r_scales[w] = scales[w];
    if (BIAS) {
      const float b = row0 + lane % 32 < end ? my_bias : -kMxInf;
      // a row that is out has products all the same, but none that are NaN
      if (b == -kMxInf) {
#pragma unroll
        for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) r_scales[w] = 0;
      }
      if (threadIdx.x < kMxTile) s_bias[buffer][lane] = b;
    }
    // (a buffer is written two tiles after it was read, and a barrier lies between)
    __syncthreads();
    const u32 ahead = min(row0 + kMxTile + lane % 32, rows.n - 1);
    Shared::load(rows, row0 + kMxTile, blocks, own);
    mx_load_scales<SHAPE>(rows, min(row0 + kMxTile + lane % 32, rows.n - 1), blocks, scales);
    if (BIAS) my_bias = mx_bias(bias, ahead);
    __builtin_amdgcn_sched_barrier(0);          // (the loads above are not to be put off until their results are wanted)
    float b[16] = {};
    if (BIAS) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 v = *reinterpret_cast<const float4*>(&s_bias[buffer][8 * g + 4 * half]);
        b[4 * g] = v.x; b[4 * g + 1] = v.y; b[4 * g + 2] = v.z; b[4 * g + 3] = v.w;
      }
    }
    const MxTile d = mx_products_shared<SHAPE>(s_tile[buffer], r_scales, q, blocks);
    if (BIAS || row0 + kMxTile <= end) mx_add_rows<BIAS, false>(d, scale, b, 0, unit, &sum, &high);
    else mx_add_rows<BIAS, true>(d, scale, b, end - row0, unit, &sum, &high);
    in_group += kMxTile;
    if (highest && (in_group == group || row0 + kMxTile >= end)) {
      in_group = 0;
      const float h = fmaxf(high, __shfl_xor(high, 32, kWave));
      if (half == 0 && query < queries.n) highest[(u64)query * n_groups + row0 / group] = h;
      high = -kMxInf;
    }
    if ((row0 - first) % kMxSumRows == kMxSumRows - kMxTile) mx_put_by(&sum, unit, &s_long[threadIdx.x]);
  }
  mx_put_by(&sum, unit, &s_long[threadIdx.x]);
  sum = {sum.m, (float)s_long[threadIdx.x].l, (float)s_long[threadIdx.x].e};
  sum = mx_join(sum, mx_shuffle_xor(sum, 32), unit);
  if (BIAS) mx_put_nan(nan, &sum);
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

template <int D>
__device__ __forceinline__ u64 mx_exchange(u64 c, bool larger) {
  const u64 o = (u64)mx_lane_xor<D>((u32)(c >> 32)) << 32 | mx_lane_xor<D>((u32)c);
  return (o > c) == larger ? o : c;
}
template <int RUN, int D>
__device__ __forceinline__ u64 mx_sort_run(u64 c) {
  if constexpr (D >= 1) {
    const u32 lane = lane_id();
    c = mx_exchange<D>(c, ((lane & RUN) == 0) == ((lane & D) == 0));
    c = mx_sort_run<RUN, D / 2>(c);
  }
  return c;
}
// Lane i gets the i-th largest of the wave's 64 candidates.
__device__ __forceinline__ u64 mx_sort(u64 c) {
  c = mx_sort_run<2, 1>(c);
  c = mx_sort_run<4, 2>(c);
  c = mx_sort_run<8, 4>(c);
  c = mx_sort_run<16, 8>(c);
  c = mx_sort_run<32, 16>(c);
  return mx_sort_run<64, 32>(c);
}
__device__ __forceinline__ u32 mx_lane_reversed(u32 v) {
  return mx_lane_xor<32>(mx_lane_xor<16>((u32)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true)));
}
// Of two lists in descending order the 64 largest, in descending order.
__device__ __forceinline__ u64 mx_merge(u64 a, u64 b) {
  const u64 r = (u64)mx_lane_reversed((u32)(b >> 32)) << 32 | mx_lane_reversed((u32)b);
  return mx_sort_run<64, 32>(a > r ? a : r);
}
// Adds 64 candidates to a list of which the first `top` count.
__device__ __forceinline__ void mx_offer(u64* list, u64 c, u32 top) {
  const u64 least = wave_lane(*list, (int)top - 1);
  if (__any(c > least)) *list = mx_merge(*list, mx_sort(c));
}
// Joins the lists of a workgroup's first `lists` waves in s_list[0].  (A barrier before the next use of s_list.)
template <int WAVES>
__device__ __forceinline__ void mx_join_lists(u64 (*s_list)[kWave], u64 list, u32 lists) {
  const u32 lane = lane_id(), wave = threadIdx.x / kWave;
  s_list[wave][lane] = list;
#pragma unroll
  for (u32 d = 1; d < WAVES; d *= 2) {
    if (d >= lists) break;
    __syncthreads();
    if (wave % (2 * d) == 0) s_list[wave][lane] = list = mx_merge(list, s_list[wave + d][lane]);
  }
  __syncthreads();
}

// Candidates that a workgroup's threads find and that reach a bound, in any order.  Where they are more than there is room
// for (many equal scores), they are offered to the waves' lists instead, in a second turn.
template <int WAVES>
struct MxFound {
  u64 list[WAVES][kWave];
  u32 count;
  __device__ __forceinline__ void add(u64 c) {
    const u32 at = atomicAdd(&count, 1u);
    if (at < WAVES * kWave) (&list[0][0])[at] = c;
  }
};

// The product of one query with the row each lane names (below n): the rows of the lower lanes and those of the upper ones
// in an instruction each, with the query in all rows of the other operand.
template <int WIDTH>
__device__ __forceinline__ float mx_dots(const MxHeld& queries, u32 query, const MxHeld& rows, u32 row, u32 blocks) {
  const u32 lane = lane_id(), half = lane / 32, other = mx_lane_xor<32>(row);
  const u64 low = (u64)(half ? other : row) * blocks, high = (u64)(half ? row : other) * blocks, one = (u64)query * blocks;
  MxTile a = mx_zero_tile(), b = mx_zero_tile();
#pragma unroll 2
  for (u32 s = 0; s < blocks; s += 2) {
    const u32 block = min(s + half, blocks - 1);
    int4 q = mx_load_block<WIDTH>(queries.codes + (one + block) * WIDTH);
    const int4 l = mx_load_block<WIDTH>(rows.codes + (low + block) * WIDTH), h = mx_load_block<WIDTH>(rows.codes + (high + block) * WIDTH);
    const u32 q_scale = queries.scales[one + block], l_scale = rows.scales[low + block], h_scale = rows.scales[high + block];
    if (s + half >= blocks) q = make_int4(0, 0, 0, 0);
    a = mx_step<0>(q, q_scale, l, l_scale, a);
    b = mx_step<0>(q, q_scale, h, h_scale, b);
  }
  return half ? b[0] : a[0];
}

// The largest value of a group of LANES lanes, in all of them.
template <int LANES, int D = 1>
__device__ __forceinline__ u64 mx_most(u64 c) {
  if constexpr (D < LANES) {
    const u64 o = (u64)mx_lane_xor<D>((u32)(c >> 32)) << 32 | mx_lane_xor<D>((u32)c);
    return mx_most<LANES, 2 * D>(o > c ? o : c);
  }
  return c;
}

// The best groups: every thread takes the best of the groups that fall to it.  `top` or more sets of threads have a best one each;
// the worst of these is a bound that `top` groups reach, and mostly few others (where top is above 16, a wave
// sorts what its threads have and gives its ceil(top / WAVES)-th).  Those that do are collected and sorted.  The rows of the best groups go the
// same way, with the last group's highest score as the bound.
template <int WIDTH, bool BIAS, int WAVES>
__global__ void __launch_bounds__(WAVES * kWave) HPS_MX_WAVES
mx_finish(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, const MxPart* __restrict__ parts,
          u32 n_parts, const float* __restrict__ highest, u32 group, u32 n_groups, const i32* __restrict__ given, u32 n_given,
          u32 top, float* __restrict__ lse_out, float* __restrict__ entropy_out, float* __restrict__ logp_out,
          i32* __restrict__ top_index, float* __restrict__ top_logp) {
  constexpr u32 kThreads = WAVES * kWave, kSets = 16;
  __shared__ MxFound<WAVES> s_groups, s_rows;
  __shared__ float s_m[WAVES], s_l[WAVES], s_e[WAVES];
  __shared__ u64 s_bound[kSets];
  const u32 lane = lane_id(), wave = threadIdx.x / kWave, query = blockIdx.x;
  const float to_score = BIAS ? 1.f : fabsf(scale), unit = to_score * kMxLog2e;
  const float* mine = highest + (u64)query * n_groups;
  const MxPart* my_parts = parts + (u64)query * n_parts;
  // (a group without a number among its scores has -inf, also where the scale is 0)
  auto group_candidate = [&](u32 g) {
    const float h = mine[g];
    return mx_candidate(BIAS || h == -kMxInf ? h : __fmul_rn(h, to_score), g);
  };
  if (threadIdx.x == 0) s_groups.count = s_rows.count = 0;
  if (threadIdx.x < kSets) s_bound[threadIdx.x] = ~0ull;
  float m = kMxLowest;
#pragma unroll 4
  for (u32 i = threadIdx.x; i < n_parts; i += kThreads) m = fmaxf(m, my_parts[i].m);
  u64 best = 0;
  if (top) {
#pragma unroll 8
    for (u32 g = threadIdx.x; g < n_groups; g += kThreads) {
      const u64 c = group_candidate(g);
      best = c > best ? c : best;
    }
  }
  __syncthreads();
  if (top) {
    u64 bound;
    u32 lanes = kWave;
    if (top <= WAVES) bound = mx_most<64>(best);
    else if (top <= 2 * WAVES && 2 * WAVES <= (int)kSets) { bound = mx_most<32>(best); lanes = 32; }
    else if (top <= 4 * WAVES && 4 * WAVES <= (int)kSets) { bound = mx_most<16>(best); lanes = 16; }
    else bound = wave_lane(mx_sort(best), (int)((top + WAVES - 1) / WAVES) - 1);
    if (lane % lanes == 0) s_bound[threadIdx.x / lanes] = bound;
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) m = fmaxf(m, __shfl_xor(m, d, kWave));
  if (lane == 0) s_m[wave] = m;
  __syncthreads();
  if (top) {
    const u64 bound = ~mx_most<16>(~s_bound[lane % kSets]);
    if (best >= bound)
      for (u32 g = threadIdx.x; g < n_groups; g += kThreads) {
        const u64 c = group_candidate(g);
        if (c >= bound) s_groups.add(c);
      }
  }
  // join the parts
  m = s_m[lane % WAVES];
#pragma unroll
  for (int d = 1; d < WAVES; d *= 2) m = fmaxf(m, __shfl_xor(m, d, kWave));
  float l = 0.f, e = 0.f;
  for (u32 i = threadIdx.x; i < n_parts; i += kThreads) {
    MxPart p = my_parts[i];
    mx_raise(&p, m, unit);
    l += p.l;
    e += p.e;
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    l += __shfl_xor(l, d, kWave);
    e += __shfl_xor(e, d, kWave);
  }
  if (lane == 0) { s_l[wave] = l; s_e[wave] = e; }
  __syncthreads();
  l = e = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { l += s_l[w]; e += s_e[w]; }
  const bool empty = l == 0.f;
  const float log2_l = log2f(l), lse = empty ? -kMxInf : __fmaf_rn(log2_l, kMxLn2, m * to_score);
  if (threadIdx.x == 0) {
    lse_out[query] = lse;
    entropy_out[query] = empty ? 0.f : (log2_l - e / l) * kMxLn2;
  }
  // the given rows, by the last waves first
  for (u32 i0 = (WAVES - 1 - wave) * kWave; i0 < n_given; i0 += kThreads) {
    const u32 i = i0 + lane;
    const i32 g = i < n_given ? given[(u64)query * n_given + i] : -1;
    const bool in = g >= 0 && (u32)g < rows.n;
    const u32 at = in ? (u32)g : rows.n - 1;
    const float s = mx_score<BIAS>(mx_dots<WIDTH>(queries, query, rows, at, blocks), scale, BIAS ? mx_bias(bias, at) : 0.f);
    if (i < n_given)
      logp_out[(u64)query * n_given + i] = g < 0 ? 0.f : !in ? __uint_as_float(0x7FC00000u) : s == -kMxInf ? s : s - lse;
  }
  if (top) {
    u32 n = s_groups.count;
    u64 list = 0;
    if (n <= kThreads) {
      if (wave * kWave < n) list = mx_sort(threadIdx.x < n ? s_groups.list[wave][lane] : 0);
    } else {
      n = kThreads;
      __syncthreads();
      for (u32 g0 = wave * kWave; g0 < n_groups; g0 += kThreads) mx_offer(&list, g0 + lane < n_groups ? group_candidate(g0 + lane) : 0, top);
    }
    mx_join_lists<WAVES>(s_groups.list, list, (n + kWave - 1) / kWave);
    const u64 groups = s_groups.list[0][lane];
    // every row that is wanted scores at least as high as the last of `top` groups, each of which has such a row
    const u32 n_best = min(top, n_groups), each = (group + kWave - 1) / kWave;
    const float least = n_best < top ? -kMxInf : mx_candidate_score(wave_lane(groups, (int)n_best - 1));
    // 64 rows, one per lane, of turn i (a NaN and a row taken out are no candidates)
    auto row_candidate = [&](u32 i) -> u64 {
      const u32 g = mx_candidate_number(wave_lane(groups, (int)(i / each)));
      const u32 k = i % each * kWave + lane, row = g * group + k;
      const bool in = k < group && row < rows.n;
      const u32 at = in ? row : rows.n - 1;
      const float s = mx_score<BIAS>(mx_dots<WIDTH>(queries, query, rows, at, blocks), scale, BIAS ? mx_bias(bias, at) : 0.f);
      return in && s >= least && s > -kMxInf ? mx_candidate(s, row) : 0;
    };
    for (u32 i = wave; i < n_best * each; i += WAVES) {
      const u64 c = row_candidate(i);
      if (c) s_rows.add(c);
    }
    __syncthreads();
    n = s_rows.count;
    list = 0;
    if (n <= kThreads) {
      if (wave * kWave < n) list = mx_sort(threadIdx.x < n ? s_rows.list[wave][lane] : 0);
    } else {
      n = kThreads;
      __syncthreads();
      for (u32 i = wave; i < n_best * each; i += WAVES) mx_offer(&list, row_candidate(i), top);
    }
    mx_join_lists<WAVES>(s_rows.list, list, (n + kWave - 1) / kWave);
    if (wave == 0) {
      list = s_rows.list[0][lane];
      if (lane < top) {
        top_index[(u64)query * top + lane] = list ? (i32)mx_candidate_number(list) : -1;
        top_logp[(u64)query * top + lane] = list ? mx_candidate_score(list) - lse : -kMxInf;
      }
    }
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
