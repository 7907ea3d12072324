// The gradient of log probabilities and entropy with respect to the queries (include/hps_mx4.h: hps_mx4_logprobs_backward).
//
// With p_r = exp(s_r - lse), U the sum of the upstream gradients u_g of the given rows' log probabilities
// and h that of the entropy H:  dL/ds_r = c_r + (u_g where r is given),  c_r = -p_r (U + h (log p_r + H)),
// d query = scale * (sum_r c_r row_r + sum_g u_g row_g).
//
// mx_gradient goes through the rows once: a product of 32 rows and 32 queries leaves a lane with 16 rows' scores for its
// query, c of which is at once the second operand of the product with the rows' values (which rows a step of the
// matrix instruction takes, in which order, is free as long as both operands agree).  The values, exact in
// bfloat16, are unpacked into LDS by the workgroup, in the order the first operand wants them: lane l of a step holds
// column l % 32 of eight rows.  c goes through the matrix instruction in bfloat16 pieces, each the nearest to what the ones before it
// leave: the sum over the rows, together with the given ones, is what little is left of large terms, and eight bits would show.
// Three pieces add up to c's 24 bits exactly; two leave 2^-17 of it at most, 2^-18.7 in the mean square over all fractions.  All
// three are used where p is above 2^-6, which a query has at most 64 rows for.  The others' errors, independent of each other as long
// as the probabilities differ, come to 2^-18.7 sqrt(sum p^2) <= 2^-21.7 of a row, as float32 itself leaves (lse is a float32 number:
// a p is off by 2^-24 |lse| of itself).  Equal probabilities have equal errors, which add up (a query of zeros has nothing else):
// all three are used too where rows of a tile have the same p.  That test takes 1 % of the time.  What no test sees (probabilities of a few sizes that
// take turns) stays below 2^-17 sum |c| |row|.
// Without a gradient of the entropy c is p up to a factor per query, which the end applies.
// mx_gradient_end adds the parts of the rows and the given rows.
//
// What bounds it: vector and matrix instructions, of which the GPU does hardly more than one kind at a time: 74 vector instructions (16
// of them exponentials) and 9 of the matrix unit for 32 x 32 scores at 64 values a row, 166 us one after the other for 1024
// queries and 0.5 M rows, 181 measured and 8 for the end.
#pragma once

#include "mx4_logprobs.hpp"

namespace hps {

constexpr u32 kMxStageTiles = 4;                         // tiles of 32 rows unpacked at a time
constexpr u32 kMxStageRows = kMxStageTiles * kMxTile;
constexpr u32 kMxGradWaves = 4;
// (Of kMxSumRows equal terms the matrix instruction, which cuts off what does not fit, always towards 0, loses 1e-5; of 1 M, added up one
// after the other, 3e-3.  The sums of longer parts go on in the workspace, in 64 bits.)
constexpr float kMxLarge = 0x1p-6f;

typedef __bf16 MxHalves2 __attribute__((ext_vector_type(2)));
typedef __bf16 MxHalves8 __attribute__((ext_vector_type(8)));

// One value of a held row.
__device__ __forceinline__ float mx_value(const MxHeld& m, u32 row, u32 col, u32 row_bytes, u32 blocks) {
  const u32 codes = m.codes[(u64)row * row_bytes + col / 2] >> (4 * (col & 1u)) & 15u;
  return mx_decode(codes, m.scales[(u64)row * blocks + col / kMxBlock]).v[0];
}

// The upstream gradient of a given row, 0 where it has no part in it.  (Loads first: several of these are in flight.)
template <bool BIAS>
__device__ __forceinline__ float mx_upstream(const i32* given, const float* d_logp, u64 at, u32 n_rows, const float* bias) {
  const u32 g = (u32)given[at];                 // (a negative number is beyond the last row)
  const float u = d_logp[at], b = BIAS ? mx_bias(bias, min(g, n_rows - 1)) : 0.f;
  return g >= n_rows || (BIAS && b == -kMxInf) ? 0.f : u;
}

// Where a tile's unpacked values lie, in units of 16 bytes (eight rows of a column): what lane `at` of a step of a block of 32
// columns reads.  The last three bits are mixed with those by which the lanes that write at one time differ, as these
// would otherwise all meet the same few banks.
__device__ __forceinline__ u32 mx_unit(u32 block, u32 step, u32 at) {
  return (block * 2 + step) * kWave + (at ^ (at >> 4 & 1u) ^ (at >> 5 & 1u) << 1 ^ step << 2);
}

// Unpacking: a lane takes eight columns of four neighbouring rows, 8 x COLUMNS / 8 such pieces a tile.
template <int COLUMNS, bool BIAS>
struct MxUnpack {
  static constexpr int PIECES = (COLUMNS + kWave / 8 * 8 - 1) / (kWave / 8 * 8);       // a lane's pieces of a tile
  u32 codes[PIECES][4], scales[PIECES][4];
  float bias[PIECES][4];
  static __device__ __forceinline__ bool place(int piece, u32* quad, u32* word) {
    const u32 at = piece * kWave + lane_id();
    *quad = at % 8;
    *word = at / 8;
    return *word < COLUMNS / 8;
  }
  __device__ __forceinline__ void load(const MxHeld& rows, u32 row0, u32 col0, u32 row_bytes, u32 blocks, const float* of_rows) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      u32 quad, word;
      place(p, &quad, &word);
      // (what is not there is read elsewhere, and left out when it is stored)
      const u32 byte = min((col0 + 8 * word) / 2, row_bytes - 4), block = min((col0 + 8 * word) / kMxBlock, blocks - 1);
      const u32 first = min(row0, rows.n - 1);
      const uint8_t *c = rows.codes + (u64)first * row_bytes, *s = rows.scales + (u64)first * blocks;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32 row = min(4 * quad + i, rows.n - 1 - first);
        codes[p][i] = *reinterpret_cast<const u32*>(c + (__umul24(row, row_bytes) + byte));
        scales[p][i] = s[__umul24(row, blocks) + block];
        if (BIAS) bias[p][i] = mx_bias(of_rows + first, row);
      }
    }
  }
  // to: [COLUMNS / 32][2 steps][64 lanes][8 rows] of a tile
  __device__ __forceinline__ void store(u32 row0, u32 end, u32 col0, u32 row_bytes, uint2* to) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      u32 quad, word;
      if (!place(p, &quad, &word)) continue;
      float s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (a row that is out, or behind the last one, has zeros: also where it stands for NaN)
        const bool in = (col0 + 8 * word) / 2 < row_bytes && row0 + 4 * quad + i < end && !(BIAS && bias[p][i] == -kMxInf);
        if (!in) codes[p][i] = scales[p][i] = 0;
        s[i] = __uint_as_float(scales[p][i] ? scales[p][i] << 23 : 0x00400000u);
      }
      // rows 8 k + 4 half + i of a step (16 rows, k = 0, 1) are elements 4 k + i of lane half
      const u32 step = quad / 4, k = quad / 2 % 2, half = quad % 2;
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        u32 two[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          MxHalves2 v;
          if (c == 0) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[p][i], s[i], 0);
          else if (c == 2) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[p][i], s[i], 1);
          else if (c == 4) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[p][i], s[i], 2);
          else v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[p][i], s[i], 3);
          two[i] = __builtin_bit_cast(u32, v);
        }
        const u32 col = word % 4 * 8 + c;
        to[mx_unit(word / 4, step, half * 32 + col) * 2 + k] =
            make_uint2(__builtin_amdgcn_perm(two[1], two[0], 0x05040100u), __builtin_amdgcn_perm(two[3], two[2], 0x05040100u));
        to[mx_unit(word / 4, step, half * 32 + col + 1) * 2 + k] = make_uint2(__builtin_amdgcn_perm(two[1], two[0], 0x07060302u), __builtin_amdgcn_perm(two[3], two[2], 0x07060302u));
      }
    }
  }
};

// What the exponents of a query are worked out with.
struct MxGradUnit {
  float unit;        // of a product (of a biased query: of a score), to a power of two
  float off;         // the part of it that float32 does not hold, relative
};

// What a lane knows of its query.
template <bool BIAS>
struct MxGradQuery {
  float lse, base, correct, a, b;
  bool none;           // all rows are out
  // log2 p = x unit - base (biased: (x - lse) unit); what base leaves of lse log2 e is a factor of all p, and so, nearly, is
  // what unit leaves: x unit is lse - entropy on average.
  __device__ __forceinline__ void load(u32 query, const MxGradUnit& unit, const float* of_lse, const float* of_entropy) {
    // (any number will do where all rows are out)
    none = of_lse[query] == -kMxInf;
    lse = none ? 0.f : of_lse[query];
    base = lse * kMxLog2e;
    const float rest = __fmaf_rn(lse, kMxLog2e, -base) + lse * 1.92596300e-8f;
    const float x_unit = of_entropy ? base - of_entropy[query] * kMxLog2e : 0.f;
    correct = BIAS ? 1.f : exp2f(__fmaf_rn(unit.off, x_unit, -rest));
    a = 1.f;
    b = 0.f;
  }
  // With a gradient of the entropy: c = p (a + b log2 p).
  __device__ __forceinline__ void load_entropy(u32 query, const float* entropy, const float* d_entropy, const i32* given, const float* d_logp,
                                               u32 n_given, u32 n_rows, const float* bias) {
    double u = 0.0;
#pragma unroll 8
    for (u32 g = lane_id() / 32; g < n_given; g += 2) u += mx_upstream<BIAS>(given, d_logp, (u64)query * n_given + g, n_rows, bias);
    u += __shfl_xor(u, 32, kWave);
    const float h = d_entropy[query];
    a = (float)-((double)h * entropy[query] + u);
    b = -h * kMxLn2;
  }
};

// (-1, 0) and (0, -1) in bfloat16, in registers: the second as a constant of the instruction is not what the GPU takes it for.
struct MxOnes {
  u32 minus_low = 0x0000BF80u, minus_high = 0xBF800000u;
  __device__ __forceinline__ MxOnes() { asm("" : "+v"(minus_low), "+v"(minus_high)); }
};

__device__ __forceinline__ bool mx_same_pair(float a0, float a1, float b0, float b1) {
  return ((u64)__float_as_uint(a1) << 32 | __float_as_uint(a0)) == ((u64)__float_as_uint(b1) << 32 | __float_as_uint(b0));
}

// Adds c row of 32 rows to the sums of 32 queries.  d: their products; values: the rows' unpacked columns.
template <bool BIAS, bool ENTROPY, int BLOCKS>
__device__ __forceinline__ void mx_add_tile(MxTile d, const float* x_bias, float scale, const MxGradQuery<BIAS>& query, float unit,
                                            const uint2* values, const MxOnes& ones, MxTile* sum) {
  const u32 lane = lane_id();
  float p[16], most = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float log2_p = BIAS ? (__fmaf_rn(d[i], scale, x_bias[i]) - query.lse) * unit : __fmaf_rn(d[i], unit, -query.base);
    p[i] = exp2_fast(log2_p);
    most = fmaxf(most, p[i]);
    // (log p of a row far below, or out, is not multiplied with: its p is 0)
    d[i] = ENTROPY ? p[i] * __fmaf_rn(query.b, BIAS ? fmaxf(log2_p, -200.f) : log2_p, query.a) : p[i];
  }
  // Rows of the same p (not of rows that are out): two pairs, as one alone is equal by chance in some tiles of a hundred.
  const bool alike = mx_same_pair(p[0], p[1], p[4], p[5]) && (!BIAS || p[0] > 0.f);
  const bool all_pieces = __any(most > kMxLarge || alike);
#pragma unroll
  for (int step = 0; step < 2; ++step) {
    MxHalves8 value[BLOCKS];
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) value[k] = *reinterpret_cast<const MxHalves8*>(&values[mx_unit(k, step, lane) * 2]);
    auto add = [&](const u32* piece) {
      const uint4 w = make_uint4(piece[0], piece[1], piece[2], piece[3]);
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k)
        sum[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value[k], __builtin_bit_cast(MxHalves8, w), sum[k], 0, 0, 0);
    };
    // pairs of rows: both rounded to the nearest; what that leaves (c - 1 x piece in one instruction, exactly), likewise;
    // and what that leaves
    float c[8];
    u32 piece[4];
    auto nearest = [&] {
#pragma unroll
      for (int i = 0; i < 8; i += 2) piece[i / 2] = mx_halves(c[i], c[i + 1]);
    };
    auto take_off = [&] {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const MxHalves2 both = __builtin_bit_cast(MxHalves2, piece[i / 2]);
        c[i] = __builtin_amdgcn_fdot2_f32_bf16(both, __builtin_bit_cast(MxHalves2, ones.minus_low), c[i], false);
        c[i + 1] = __builtin_amdgcn_fdot2_f32_bf16(both, __builtin_bit_cast(MxHalves2, ones.minus_high), c[i + 1], false);
      }
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = d[8 * step + i];
    nearest();
    add(piece);
    take_off();
    nearest();
    add(piece);
    if (all_pieces) {
      take_off();
      nearest();
      add(piece);
    }
  }
}

// A launch takes up to kMxSumRows rows of each part, from number `done` of the part on.  Where the parts have more (`wide`), a
// workgroup adds its sums to the 64-bit ones that the launches before have left.
struct MxPartRows {
  u32 rows, done;
  bool wide;
  __device__ __forceinline__ u32 first() const { return blockIdx.x * rows + done; }
  __device__ __forceinline__ u32 end(u32 n) const {
    const u32 start = blockIdx.x * rows, all = min(n - start, rows);
    return start + (wide ? min(done + kMxSumRows, all) : all);
  }
};

// Writes a query's sums of COLUMNS columns, at number `at` and following.
template <int BLOCKS>
__device__ __forceinline__ void mx_store_sums(const MxTile* sum, float correct, u32 col0, u32 dim, const MxPartRows& part, void* parts, u64 at) {
  const u32 half = lane_id() / 32;
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32 col = col0 + k * 32 + 8 * g + 4 * half;
      if (col >= dim) continue;
      const float4 v = make_float4(sum[k][4 * g] * correct, sum[k][4 * g + 1] * correct, sum[k][4 * g + 2] * correct, sum[k][4 * g + 3] * correct);
      if (!part.wide) {
        *reinterpret_cast<float4*>(static_cast<float*>(parts) + at + col) = v;
        continue;
      }
      double2* const to = reinterpret_cast<double2*>(static_cast<double*>(parts) + at + col);
      double2 low = make_double2(v.x, v.y), high = make_double2(v.z, v.w);
      if (part.done) {
        const double2 l = to[0], h = to[1];
        low = make_double2(l.x + low.x, l.y + low.y);
        high = make_double2(h.x + high.x, h.y + high.y);
      }
      to[0] = low;
      to[1] = high;
    }
}

// A workgroup: query_groups (1, 2 or 4) x QT x 32 queries, a part of the rows, of which each of 4 / query_groups groups of waves
// takes some tiles of every stage, and COLUMNS columns.  The groups' sums are added up in LDS, so that `parts` holds one for each
// part of the rows: 1 query against 1 M rows, 64 wide, takes 30 us (40 with a part of its own for each group), 8 against 262 144, 16
// wide, 16 us (27), 64 against 65 536, 64 wide, 15.5 us (20.6).
template <typename SHAPE, bool BIAS, bool ENTROPY, int COLUMNS, int QT>
__global__ void __launch_bounds__(kMxGradWaves * kWave) HPS_MX_WAVES
mx_gradient(MxHeld queries, MxHeld rows, u32 dim, u32 blocks, u32 row_bytes, float scale, MxGradUnit unit, const float* __restrict__ bias,
            const float* __restrict__ lse, const float* __restrict__ entropy, const i32* __restrict__ given, const float* __restrict__ d_logp,
            u32 n_given, const float* __restrict__ d_entropy, u32 query_groups, MxPartRows part, void* __restrict__ parts) {
  constexpr int BLOCKS = COLUMNS / 32;
  constexpr u32 kTileWords = BLOCKS * 2 * kWave * 2;           // of 8 bytes, a tile's unpacked values
  __shared__ __align__(16) uint2 s_rows[2][kMxStageTiles][kTileWords];
  __shared__ __align__(16) float s_bias[kMxGradWaves][kMxTile];
  const u32 lane = lane_id(), half = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const u32 splits = kMxGradWaves / query_groups, split = wave / query_groups;
  const u32 query0 = (blockIdx.y * query_groups + wave % query_groups) * (QT * kMxTile) + lane % 32;
  const u32 first = part.first(), end = part.end(rows.n), col0 = blockIdx.z * COLUMNS;
  if (first >= end) return;             // (the last part is shorter)

  MxUnpack<COLUMNS, BIAS> unpack;
  unpack.load(rows, first + wave * kMxTile, col0, row_bytes, blocks, bias);
  MxRow<SHAPE> next;
  float next_bias = 0.f;
  if (SHAPE::AHEAD) mx_load_tile<SHAPE>(rows, first + split * kMxTile, blocks, &next);
  if (BIAS) next_bias = mx_bias(bias, min(first + split * kMxTile + lane % 32, rows.n - 1));

  MxRow<SHAPE> q[QT];
  MxGradQuery<BIAS> query[QT];
  MxTile sum[QT][BLOCKS];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const u32 mine = min(query0 + t * kMxTile, queries.n - 1);
    mx_load_row<SHAPE>(queries, mine, blocks, &q[t]);
    mx_clear_rest<SHAPE>(blocks, &q[t]);
    if (!BIAS && scale < 0.f) mx_negate<SHAPE>(&q[t]);
    query[t].load(mine, unit, lse, entropy);
    if (BIAS && query[t].none) mx_take_out<SHAPE>(&q[t]);
    if (ENTROPY) query[t].load_entropy(mine, entropy, d_entropy, given, d_logp, n_given, rows.n, bias);
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) sum[t][k] = mx_zero_tile();
  }
  const MxOnes ones;

  unpack.store(first + wave * kMxTile, end, col0, row_bytes, s_rows[0][wave]);
  __syncthreads();
  u32 buffer = 0;
  for (u32 stage0 = first; stage0 < end; stage0 += kMxStageRows, buffer ^= 1u) {
    unpack.load(rows, stage0 + kMxStageRows + wave * kMxTile, col0, row_bytes, blocks, bias);
    for (u32 tile = split; tile < kMxStageTiles; tile += splits) {
      const u32 row0 = stage0 + tile * kMxTile;
      if (row0 >= end) continue;
      MxRow<SHAPE> r;
      if (SHAPE::AHEAD) r = next;
      else mx_load_tile<SHAPE>(rows, row0, blocks, &r);
      const float my_bias = row0 + lane % 32 < end ? next_bias : -kMxInf;
      const u32 ahead = tile + splits < kMxStageTiles ? row0 + splits * kMxTile : stage0 + kMxStageRows + split * kMxTile;
      if (SHAPE::AHEAD) mx_load_tile<SHAPE>(rows, ahead, blocks, &next);
      if (BIAS) next_bias = mx_bias(bias, min(ahead + lane % 32, rows.n - 1));
      __builtin_amdgcn_sched_barrier(0);          // (the loads above are not to be put off until their results are wanted)
      float x_bias[16];
      if (BIAS) {
        if (my_bias == -kMxInf) mx_take_out<SHAPE>(&r);
        __builtin_amdgcn_wave_barrier();
        s_bias[wave][lane % 32] = my_bias;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 v = *reinterpret_cast<const float4*>(&s_bias[wave][8 * g + 4 * half]);
          x_bias[4 * g] = v.x; x_bias[4 * g + 1] = v.y; x_bias[4 * g + 2] = v.z; x_bias[4 * g + 3] = v.w;
        }
      }
      MxTile d[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) d[t] = mx_products<SHAPE>(r, q[t], blocks);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        mx_add_tile<BIAS, ENTROPY, BLOCKS>(d[t], x_bias, scale, query[t], unit.unit, s_rows[buffer][tile], ones, sum[t]);
      }
    }
    unpack.store(stage0 + kMxStageRows + wave * kMxTile, end, col0, row_bytes, s_rows[buffer ^ 1u][wave]);
    __syncthreads();
  }
  if (splits > 1) {
    // (one query tile a wave then; the last stage's values are done with)
    float* const of_waves = reinterpret_cast<float*>(&s_rows[0][0][0]);
    static_assert(sizeof(s_rows) >= (kMxGradWaves - 1) * BLOCKS * 16 * kWave * sizeof(float), "");
    if (split > 0) {
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) of_waves[(((wave - query_groups) * BLOCKS + k) * 16 + r) * kWave + lane] = sum[0][k][r];
    }
    __syncthreads();
    if (split > 0) return;
    for (u32 w = wave; w < kMxGradWaves - query_groups; w += query_groups)
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[0][k][r] += of_waves[((w * BLOCKS + k) * 16 + r) * kWave + lane];
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const u32 mine = query0 + t * kMxTile;
    if (mine < queries.n) mx_store_sums<BLOCKS>(sum[t], query[t].correct, col0, dim, part, parts, ((u64)blockIdx.x * queries.n + mine) * dim);
  }
}

// Wide rows and more than a few queries: the four waves hold 32 queries each and go through the rows together, a tile in LDS for the
// products and the next two tiles' columns unpacked (by two waves a tile).
template <typename SHAPE, bool BIAS, bool ENTROPY>
__global__ void __launch_bounds__(kMxThreads) HPS_MX_WAVES
mx_gradient_shared(MxHeld queries, MxHeld rows, u32 dim, u32 blocks, u32 row_bytes, float scale, MxGradUnit unit, const float* __restrict__ bias,
                   const float* __restrict__ lse, const float* __restrict__ entropy, const i32* __restrict__ given,
                   const float* __restrict__ d_logp, u32 n_given, const float* __restrict__ d_entropy, MxPartRows part, void* __restrict__ parts) {
  constexpr u32 COLUMNS = 128, BLOCKS = COLUMNS / 32, kStage = 2;
  constexpr u32 kTileWords = BLOCKS * 2 * kWave * 2;
  typedef MxShared<SHAPE> Shared;
  __shared__ int4 s_tile[2][Shared::UNITS];
  __shared__ __align__(16) uint2 s_rows[2][kStage][kTileWords];
  __shared__ __align__(16) float s_bias[2][kMxTile];
  const u32 lane = lane_id(), half = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const u32 mine = (blockIdx.y * (kMxThreads / kWave) + wave) * kMxTile + lane % 32;
  const u32 first = part.first(), end = part.end(rows.n), col0 = blockIdx.z * COLUMNS;
  if (first >= end) return;             // (the last part is shorter)
  const u32 my_tile = wave / 2 * kMxTile, my_col = col0 + wave % 2 * (COLUMNS / 2), my_words = wave % 2 * (kTileWords / 2);

  MxUnpack<COLUMNS / 2, BIAS> unpack;
  unpack.load(rows, first + my_tile, my_col, row_bytes, blocks, bias);
  int4 own[Shared::OWN];
  u32 scales[SHAPE::SCALE_WORDS];
  float my_bias = 0.f;
  Shared::load(rows, first, blocks, own);
  mx_load_scales<SHAPE>(rows, min(first + lane % 32, rows.n - 1), blocks, scales);
  if (BIAS) my_bias = mx_bias(bias, min(first + lane % 32, rows.n - 1));
  MxRow<SHAPE> q;
  MxGradQuery<BIAS> query;
  MxTile sum[BLOCKS];
  mx_load_row<SHAPE>(queries, min(mine, queries.n - 1), blocks, &q);
  mx_clear_rest<SHAPE>(blocks, &q);
  if (!BIAS && scale < 0.f) mx_negate<SHAPE>(&q);
  query.load(min(mine, queries.n - 1), unit, lse, entropy);
  if (BIAS && query.none) mx_take_out<SHAPE>(&q);
  if (ENTROPY) query.load_entropy(min(mine, queries.n - 1), entropy, d_entropy, given, d_logp, n_given, rows.n, bias);
#pragma unroll
  for (u32 k = 0; k < BLOCKS; ++k) sum[k] = mx_zero_tile();
  const MxOnes ones;

  unpack.store(first + my_tile, end, my_col, row_bytes, s_rows[0][wave / 2] + my_words);
  u32 buffer = 0, tile_buffer = 0;
  for (u32 stage0 = first; stage0 < end; stage0 += kStage * kMxTile, buffer ^= 1u) {
    for (u32 tile = 0; tile < kStage; ++tile, tile_buffer ^= 1u) {
      const u32 row0 = stage0 + tile * kMxTile;
      Shared::store(own, blocks, s_tile[tile_buffer]);
      u32 r_scales[SHAPE::SCALE_WORDS];
#pragma unroll
      for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) r_scales[w] = scales[w];
      if (BIAS) {
        const float b = row0 + lane % 32 < end ? my_bias : -kMxInf;
        if (b == -kMxInf) {
#pragma unroll
          for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) r_scales[w] = 0;
        }
        if (threadIdx.x < kMxTile) s_bias[tile_buffer][lane] = b;
      }
      // (what is written before this barrier was last read before the one before it)
      __syncthreads();
      const u32 ahead = min(row0 + kMxTile + lane % 32, rows.n - 1);
      Shared::load(rows, row0 + kMxTile, blocks, own);
      mx_load_scales<SHAPE>(rows, min(row0 + kMxTile + lane % 32, rows.n - 1), blocks, scales);
      if (BIAS) my_bias = mx_bias(bias, ahead);
      if (tile == 0) unpack.load(rows, stage0 + kStage * kMxTile + my_tile, my_col, row_bytes, blocks, bias);
      __builtin_amdgcn_sched_barrier(0);          // (the loads above are not to be put off until their results are wanted)
      if (row0 >= end) continue;
      float x_bias[16];
      if (BIAS) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 v = *reinterpret_cast<const float4*>(&s_bias[tile_buffer][8 * g + 4 * half]);
          x_bias[4 * g] = v.x; x_bias[4 * g + 1] = v.y; x_bias[4 * g + 2] = v.z; x_bias[4 * g + 3] = v.w;
        }
      }
      const MxTile d = mx_products_shared<SHAPE>(s_tile[tile_buffer], r_scales, q, blocks);
      mx_add_tile<BIAS, ENTROPY, (int)BLOCKS>(d, x_bias, scale, query, unit.unit, s_rows[buffer][tile], ones, sum);
    }
    unpack.store(stage0 + kStage * kMxTile + my_tile, end, my_col, row_bytes, s_rows[buffer ^ 1u][wave / 2] + my_words);
  }
  if (mine < queries.n) mx_store_sums<(int)BLOCKS>(sum, query.correct, col0, dim, part, parts, ((u64)blockIdx.x * queries.n + mine) * dim);
}

// The end: a workgroup takes 64 of the output's values; its waves share the parts and the given rows.  Added up in 64 bits: the two
// may cancel almost entirely.
template <bool BIAS, bool ENTROPY, u32 WAVES>
__global__ void __launch_bounds__(WAVES * kWave)
mx_gradient_end(MxHeld rows, u32 n_queries, u32 dim, u32 blocks, u32 row_bytes, float scale, const float* __restrict__ bias,
                const i32* __restrict__ given, const float* __restrict__ d_logp, u32 n_given, const void* __restrict__ parts,
                u32 n_parts, bool wide, float* __restrict__ out) {
  __shared__ double s_sum[WAVES][kWave], s_given[WAVES][kWave], s_u[WAVES][kWave];
  const u32 lane = lane_id(), wave = threadIdx.x / kWave;
  const u64 total = (u64)n_queries * dim;
  for (u64 i0 = (u64)blockIdx.x * kWave; i0 < total; i0 += (u64)gridDim.x * kWave) {
    const u64 i = i0 + lane;
    if (i < total) {
      const u32 query = (u32)(i / dim), col = (u32)(i - (u64)query * dim);
      double sum = 0.0, of_given = 0.0, u_all = 0.0;
      if (wide) {
        for (u32 p = wave; p < n_parts; p += WAVES) sum += static_cast<const double*>(parts)[p * total + i];
      } else {
#pragma unroll 8
        for (u32 p = wave; p < n_parts; p += WAVES) sum += static_cast<const float*>(parts)[p * total + i];
      }
      for (u32 g = wave; g < n_given; g += WAVES) {
        const u64 at = (u64)query * n_given + g;
        const float u = mx_upstream<BIAS>(given, d_logp, at, rows.n, bias);
        u_all += u;
        if (u != 0.f) of_given += (double)u * mx_value(rows, (u32)given[at], col, row_bytes, blocks);
      }
      s_sum[wave][lane] = sum;
      s_given[wave][lane] = of_given;
      s_u[wave][lane] = u_all;
    }
    __syncthreads();
    if (wave == 0 && i < total) {
      double sum = 0.0, of_given = 0.0, u_all = 0.0;
#pragma unroll
      for (u32 w = 0; w < WAVES; ++w) {
        sum += s_sum[w][lane];
        of_given += s_given[w][lane];
        u_all += s_u[w][lane];
      }
      out[i] = (float)(scale * ((ENTROPY ? sum : -u_all * sum) + of_given));
    }
    __syncthreads();
  }
}

}  // namespace hps
