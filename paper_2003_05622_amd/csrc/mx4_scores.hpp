// All scores of queries against rows (include/hps_mx4.h: hps_mx4_scores).
//
// What bounds it is writing the scores: 4 (or 2) bytes for 2 dim operations, of which the matrix units do some thousand in
// the time that a byte takes.  So the lanes lie along the rows, and a wave's tiles are dealt out so that a lane has
// neighbouring rows of a query (tile t holds rows RT j + t): a store writes RT neighbouring scores a lane, whole lines a wave.
// A wave holds RT x 32 rows and goes through the query tiles of its part; the rows' operands stay in
// registers, the queries' come out of the caches, those of wide rows out of LDS, where the waves of a workgroup share them.
// 1024 x 262 144 float32 scores (1.07 GB): 204 us at 16 values a row (5.3 TB/s), 210 at 256, 214 at 512, 287 at 1024, where the operands'
// way to the matrix unit takes over (1.9 PFLOP/s).
#pragma once

#include "mx4.hpp"

namespace hps {

// Stores RT neighbouring scores of a query, of which the first `n` are there.  (The GPU stores words of any alignment.)
template <bool PAST_CACHE, typename WORDS>
__device__ __forceinline__ void mx_store_words(WORDS v, WORDS* to) {
  if (PAST_CACHE) __builtin_nontemporal_store(v, to);
  else *to = v;
}
template <int RT, bool BF16, bool PAST_CACHE>
__device__ __forceinline__ void mx_store_scores(char* at, const float* s, u32 n) {
  if (BF16) {
    typedef u32 Pairs __attribute__((ext_vector_type(RT / 2), aligned(2)));
    uint16_t* to = reinterpret_cast<uint16_t*>(at);
    if (n == RT) {
      Pairs v;
#pragma unroll
      for (int t = 0; t < RT / 2; ++t) v[t] = mx_halves(s[2 * t], s[2 * t + 1]);
      mx_store_words<PAST_CACHE>(v, reinterpret_cast<Pairs*>(to));
      return;
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
      if (t < (int)n) to[t] = (uint16_t)mx_halves(s[t], 0.f);
    return;
  }
  typedef float Floats __attribute__((ext_vector_type(RT), aligned(4)));
  float* to = reinterpret_cast<float*>(at);
  if (n == RT) {
    Floats v;
#pragma unroll
    for (int t = 0; t < RT; ++t) v[t] = s[t];
    mx_store_words<PAST_CACHE>(v, reinterpret_cast<Floats*>(to));
    return;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
    if (t < (int)n) to[t] = s[t];
}

// Tiles of rows a wave holds.
template <typename SHAPE>
constexpr int mx_score_tiles() { return SHAPE::STEPS <= 4 ? 4 : 2; }

// WHOLE_LINES: the scores of every query start on a memory line.  They go past the L2 then, which has better things to hold;
// else two waves write a line, and the L2 puts it together.
template <typename SHAPE, bool BIAS, bool BF16, bool WHOLE_LINES>
__global__ void __launch_bounds__(kMxThreads) HPS_MX_WAVES
mx_scores(MxHeld queries, MxHeld rows, u32 blocks, float scale, const float* __restrict__ bias, void* __restrict__ out, u64 stride,
          u32 row_groups, u32 query_parts, u32 part_tiles) {
  constexpr int RT = mx_score_tiles<SHAPE>();
  const u32 lane = lane_id(), half = lane / 32, wave = threadIdx.x / kWave;
  // neighbouring pieces of work, which share rows, to one XCD
  const u32 piece = xcd_piece(blockIdx.x, gridDim.x), row_group = piece / query_parts, query_part = piece - row_group * query_parts;
  const u32 row0 = (row_group * (kMxThreads / kWave) + wave) * (RT * kMxTile), row = row0 + lane % 32 * RT;
  constexpr bool SHARED = SHAPE::STEPS >= 8;
  if (!SHARED && row0 >= rows.n) return;
  MxRow<SHAPE> r[RT];
  float b[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const u32 at = min(row + t, rows.n - 1);
    mx_load_row<SHAPE>(rows, at, blocks, &r[t]);
    mx_clear_rest<SHAPE>(blocks, &r[t]);
    b[t] = BIAS ? mx_bias(bias, at) : 0.f;
  }
  const u32 left = row < rows.n ? min(rows.n - row, (u32)RT) : 0;
  const u32 tiles = (queries.n + kMxTile - 1) / kMxTile, begin = query_part * part_tiles, last = min(begin + part_tiles, tiles);
  const u64 pitch = stride * (BF16 ? 2 : 4);
  char* const mine = static_cast<char*>(out) + half * 4 * pitch + (u64)row * (BF16 ? 2 : 4);
  auto store = [&](const MxTile* d, u32 query0) {
    char* to = mine + query0 * pitch;
    const u32 queries_left = queries.n - query0;
    auto one = [&](int i) {
      float s[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) s[t] = mx_score<BIAS>(d[t][i], scale, b[t]);
      mx_store_scores<RT, BF16, WHOLE_LINES>(to + (8 * (i / 4) + i % 4) * pitch, s, left);
    };
    if (queries_left >= kMxTile) {
#pragma unroll
      for (int i = 0; i < 16; ++i) one(i);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (mx_row_of(i, half) < queries_left) one(i);
    }
  };
  MxTile d[RT];
  if constexpr (SHARED) {
    // (the shared tile is the first operand, and has what lies behind a row's blocks: the rows are without it)
    typedef MxShared<SHAPE> Shared;
    __shared__ int4 s_tile[2][SHARED ? Shared::UNITS : 1];
    int4 own[Shared::OWN];
    u32 scales[SHAPE::SCALE_WORDS], buffer = 0;
    Shared::load(queries, begin * kMxTile, blocks, own);
    mx_load_scales<SHAPE>(queries, min(begin * kMxTile + lane % 32, queries.n - 1), blocks, scales);
    for (u32 tile = begin; tile < last; ++tile, buffer ^= 1u) {
      Shared::store(own, blocks, s_tile[buffer]);
      u32 q_scales[SHAPE::SCALE_WORDS];
#pragma unroll
      for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) q_scales[w] = scales[w];
      __syncthreads();
      Shared::load(queries, (tile + 1) * kMxTile, blocks, own);
      mx_load_scales<SHAPE>(queries, min((tile + 1) * kMxTile + lane % 32, queries.n - 1), blocks, scales);
      __builtin_amdgcn_sched_barrier(0);        // (the loads above are not to be put off until their results are wanted)
#pragma unroll
      for (int t = 0; t < RT; ++t) d[t] = mx_products_shared<SHAPE>(s_tile[buffer], q_scales, r[t], blocks);
      store(d, tile * kMxTile);
    }
  } else {
    MxRow<SHAPE> next;
    mx_load_tile<SHAPE>(queries, begin * kMxTile, blocks, &next);
    for (u32 tile = begin; tile < last; ++tile) {
      const MxRow<SHAPE> q = next;
      mx_load_tile<SHAPE>(queries, (tile + 1) * kMxTile, blocks, &next);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < RT; ++t) d[t] = mx_products<SHAPE>(q, r[t], blocks);
      store(d, tile * kMxTile);
    }
  }
}

}  // namespace hps
