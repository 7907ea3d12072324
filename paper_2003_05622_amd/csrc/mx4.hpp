// Rows in microscaled 4-bit floating point (include/hps_mx4.h): the form itself, and the kernels that bring
// rows into it (from an array, from the table by key) and read them back.
//
// A block of 32 values x has the scale 2^E, E = floor(log2 max|x|) - 2, so that the largest magnitude
// lies in [4, 8) scales; a value becomes the code nearest to x / 2^E.  E comes from the exponent bits
// of the largest magnitude, compared as whole numbers (a NaN is then the largest of all); the code from the
// GPU's conversion instruction, which divides by the scale exactly, rounds to nearest even and saturates.
#pragma once

#include "common.hpp"
#include "rows.hpp"
#include "table.hpp"

namespace hps {

constexpr u32 kMxBlock = 32;          // values that share a scale
constexpr u32 kMxNoScale = 255;       // the scale byte of a block that stands for NaN

// Bytes of codes a row takes: whole blocks, so that a block is one aligned 16-byte word; rows of a quarter or
// half a block only that (narrow rows are many).
__host__ __device__ constexpr u32 mx_row_bytes(u32 dim) { return dim <= 8 ? 4u : dim <= 16 ? 8u : (dim + kMxBlock - 1) / kMxBlock * 16; }
__host__ __device__ constexpr u32 mx_blocks(u32 dim) { return (dim + kMxBlock - 1) / kMxBlock; }

// The value of lane l ^ D, by moves between lanes (a shuffle goes through the LDS and takes some hundred cycles).
template <int D>
__device__ __forceinline__ u32 mx_lane_xor(u32 v) {
  static_assert(D == 1 || D == 2 || D == 4 || D == 8 || D == 16 || D == 32, "");
  if constexpr (D == 1) return (u32)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
  if constexpr (D == 2) return (u32)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);
  // (the lanes of eight, and then of each four, backwards)
  if constexpr (D == 4) return (u32)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
  if constexpr (D == 8) return (u32)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true);
  if constexpr (D == 16) {
    const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane_id() & 16u ? both[0] : both[1];
  }
  if constexpr (D == 32) {
    const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane_id() & 32u ? both[0] : both[1];
  }
}

// Some of a block's values: a group of lanes with four or eight of them each holds a whole block.
struct MxEight {
  float v[8];
  __device__ __forceinline__ void set(int q, float4 f) { v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w; }
};

// The scale byte of the block whose values GL lanes hold, VALUES each, and the lane's codes.
template <int GL, int VALUES = 8>
__device__ __forceinline__ u32 mx_encode(const MxEight& x, u32* codes) {
  u32 most = 0;
#pragma unroll
  for (int i = 0; i < VALUES; ++i) most = max(most, __float_as_uint(x.v[i]) & 0x7FFFFFFFu);
  if (GL > 1) most = max(most, mx_lane_xor<1>(most));
  if (GL > 2) most = max(most, mx_lane_xor<2>(most));
  if (GL > 4) most = max(most, mx_lane_xor<4>(most));
  const u32 e = most >> 23;
  if (e == 255) {
    *codes = 0;
    return kMxNoScale;
  }
  const u32 scale = e > 2 ? e - 2 : 0;
  // (2^-127 is below the normal numbers)
  const float s = __uint_as_float(scale ? scale << 23 : 0x00400000u);
  u32 c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[0], x.v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[2], x.v[3], s, 1);
  if (VALUES == 8) {
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[4], x.v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x.v[6], x.v[7], s, 3);
  }
  *codes = c;
  return scale;
}

// What eight codes of a block stand for.
__device__ __forceinline__ MxEight mx_decode(u32 codes, u32 scale) {
  const float s = scale == kMxNoScale ? __uint_as_float(0x7FC00000u) : __uint_as_float(scale ? scale << 23 : 0x00400000u);
  MxEight x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const u32 c = codes >> (4 * i) & 15u, m = c & 7u;
    // two exponent bits (bias 1) and a fraction bit; without exponent bits 0 or a half
    const float one = m >= 2 ? __uint_as_float((126u + (m >> 1)) << 23 | (m & 1u) << 22) : 0.5f * (float)m;
    x.v[i] = (c & 8u ? -one : one) * s;
  }
  return x;
}

constexpr int kMxThreads = 256;

template <bool BF16>
__device__ __forceinline__ float4 load_values4(const void* base, u64 at) {
  if (BF16) {
    const uint2 raw = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at);
    return make_float4(bf16_value(raw.x & 0xFFFFu), bf16_value(raw.x >> 16), bf16_value(raw.y & 0xFFFFu), bf16_value(raw.y >> 16));
  }
  return *reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
}

// Eight values a lane, GL lanes a block, flat over all blocks.  Bound by memory: 2^28 float32 values, 64 a row, in 208 us (1.2 GB).
template <bool BF16, int GL>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize(const void* __restrict__ values, u64 n, u32 dim, u64 stride, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const u32 blocks = mx_blocks(dim), row_bytes = mx_row_bytes(dim), sub = threadIdx.x % GL;
  const u64 total = n * blocks;
  for (u64 b = ((u64)blockIdx.x * kMxThreads + threadIdx.x) / GL; b < total; b += (u64)gridDim.x * (kMxThreads / GL)) {
    const u64 row = total < (1ull << 32) ? (u32)b / blocks : b / blocks;
    const u32 block = (u32)(b - row * blocks), col = block * kMxBlock + 8 * sub;
    MxEight x;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      x.set(q, col + 4 * q < dim ? load_values4<BF16>(values, row * stride + col + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f));
    u32 c;
    const u32 scale = mx_encode<GL>(x, &c);
    *reinterpret_cast<u32*>(codes + row * row_bytes + block * 16 + 4 * sub) = c;
    if (sub == 0) scales[b] = (uint8_t)scale;
  }
}

// With the values that the codes stand for: four a lane, LANES (8; narrow rows: 2 or 4) lanes a block, so that a wave stores 1 KB in one piece
// past the L2 (in pieces of 32 bytes a lane that takes 604 us for the 2.3 GB above, through it 399; so 394, and 292 from bfloat16
// instead of 345; without the values the other form is faster, 208 us to 220); kMxInFlight turns are loaded before the first is worked on.
constexpr int kMxInFlight = 4;
template <bool BF16, int LANES>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_round(const void* __restrict__ values, u64 n, u32 dim, u64 stride, uint8_t* __restrict__ codes,
                  uint8_t* __restrict__ scales, float* __restrict__ rounded) {
  constexpr u32 kUnits = kMxThreads / LANES;                           // blocks a turn of the workgroup takes
  const u32 blocks = mx_blocks(dim), row_bytes = mx_row_bytes(dim), sub = threadIdx.x % LANES;
  const u64 total = n * blocks;
  const u32 more_rows = kUnits / blocks, more_blocks = kUnits % blocks;
  for (u64 b0 = (u64)blockIdx.x * (kMxInFlight * kUnits) + threadIdx.x / LANES; b0 < total; b0 += (u64)gridDim.x * (kMxInFlight * kUnits)) {
    u64 row[kMxInFlight];
    u32 col[kMxInFlight];
    float4 v[kMxInFlight];
    u64 at = total < (1ull << 32) ? (u32)b0 / blocks : b0 / blocks;    // (a division of 64 bits takes longer than all the rest)
    u32 block = (u32)(b0 - at * blocks);
#pragma unroll
    for (int q = 0; q < kMxInFlight; ++q) {
      row[q] = at;
      col[q] = block * kMxBlock + 4 * sub;
      v[q] = at < n && col[q] < dim ? load_values4<BF16>(values, at * stride + col[q]) : make_float4(0.f, 0.f, 0.f, 0.f);
      at += more_rows;
      block += more_blocks;
      if (block >= blocks) { block -= blocks; ++at; }
    }
#pragma unroll
    for (int q = 0; q < kMxInFlight; ++q) {
      if (row[q] >= n) break;
      MxEight x = {};
      x.set(0, v[q]);
      u32 c;
      const u32 scale = mx_encode<LANES, 4>(x, &c);
      *reinterpret_cast<uint16_t*>(codes + row[q] * row_bytes + col[q] / 2) = (uint16_t)c;
      if (sub == 0) scales[b0 + q * kUnits] = (uint8_t)scale;
      if (col[q] < dim) {
        const MxEight y = mx_decode(c, scale);
        store_caller4(rounded + row[q] * dim + col[q], true, make_float4(y.v[0], y.v[1], y.v[2], y.v[3]));
      }
    }
  }
}

// Four values a lane, so that a wave stores 1 KB in one piece.
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, u64 n, u32 dim, float* __restrict__ out) {
  const u32 words = dim / 4, row_bytes = mx_row_bytes(dim), blocks = mx_blocks(dim);
  const u64 total = n * words;
  for (u64 i = (u64)blockIdx.x * kMxThreads + threadIdx.x; i < total; i += (u64)gridDim.x * kMxThreads) {
    const u64 row = i / words;
    const u32 word = (u32)(i - row * words);
    const MxEight y = mx_decode(*reinterpret_cast<const uint16_t*>(codes + row * row_bytes + 2 * word), scales[row * blocks + word / 8]);
    store_caller4(out + 4 * i, true, make_float4(y.v[0], y.v[1], y.v[2], y.v[3]));
  }
}

// Rows of the table by key.  As get_rows: a wave finds 64 keys, one per lane, and then goes through their
// blocks, a lane group per block.  2 M keys of 8 M, dim 32: 92 us (get_rows 167, and 52 to quantise what it gives).
template <bool BF16, int GL>
__global__ void __launch_bounds__(kRowThreads)
mx_get(TableView t, const u64* __restrict__ keys, u64 n_keys, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
       uint8_t* __restrict__ found_out) {
  const bool failed = load_error(t.st) != 0;
  const u32 lane = lane_id(), sub = lane % kLookupLanes;
  const u32 blocks = mx_blocks(t.dim), row_bytes = mx_row_bytes(t.dim);
  const u64 n_waves = (u64)gridDim.x * (kRowThreads / kWave);
  for (u64 first = ((u64)blockIdx.x * (kRowThreads / kWave) + threadIdx.x / kWave) * kWave; first < n_keys;
       first += n_waves * kWave) {
    const u64 u = first + lane;
    u64 key = u < n_keys && !failed ? keys[u] : kEmptyKey, line;
    u32 row, free_at;
    search_keys<kLookupLanes>(t, &key, &line, &row, &free_at, sub);
    if (u < n_keys) found_out[u] = row != kNoRow;
    else row = kSkipRow;
    const u32 part = lane % GL;
    for (u32 i = 0; i < blocks * GL; ++i) {            // 64 keys x blocks, 64 / GL blocks a turn
      const u32 at = (i * kWave + lane) / GL, k = at / blocks, block = at - k * blocks, col = block * kMxBlock + 8 * part;
      const u32 r = (u32)__shfl((int)row, (int)k, kWave);
      MxEight x;
#pragma unroll
      for (int q = 0; q < 2; ++q)
        x.set(q, r < kSkipRow && col + 4 * q < t.dim ? load_w4_as<BF16>(t, r, col / 4 + q) : make_float4(0.f, 0.f, 0.f, 0.f));
      u32 c;
      const u32 scale = mx_encode<GL>(x, &c);
      if (r == kSkipRow) continue;
      *reinterpret_cast<u32*>(codes + (first + k) * row_bytes + block * 16 + 4 * part) = c;
      if (part == 0) scales[(first + k) * blocks + block] = (uint8_t)scale;
    }
  }
}

// ---- products of held rows ---------------------------------------------------------------------
// v_mfma_scale_f32_32x32x64: D (32 x 32) += A (32 x 64) B (64 x 32), both in 4 bits with a scale per block.  Lane
// l holds one block (16 bytes) of row l % 32 of either operand, the first or the second of the 64 values by
// l / 32, and that block's scale byte; of D it holds column l % 32 (B's row) and, as element r, row
// mx_row_of(r, l / 32) (A's row).
typedef int MxOperand __attribute__((ext_vector_type(8)));
typedef float MxTile __attribute__((ext_vector_type(16)));
constexpr u32 kMxTile = 32;
constexpr float kMxInf = __builtin_huge_valf();

__device__ __forceinline__ u32 mx_row_of(u32 r, u32 half) { return 8 * (r >> 2) + 4 * half + (r & 3u); }

struct MxHeld {            // rows as a kernel sees them
  const uint8_t* codes;
  const uint8_t* scales;
  u32 n;
};

// For kernels that work on products element by element: with at most 256 registers a lane the compiler has the matrix
// instructions write where other instructions can read, which saves a move each way per element.
#define HPS_MX_WAVES __attribute__((amdgpu_waves_per_eu(2)))

// How a kernel is made for a width: WIDTH bytes of a block (16, or those of a whole narrow row), and STEPS
// instructions of 64 values for a product (1, 2, 4, 8 or 16; where a row has fewer, the last ones are skipped).
template <int WIDTH_, int STEPS_>
struct MxShape {
  static constexpr int WIDTH = WIDTH_, STEPS = STEPS_;
  // whether the next rows are loaded while the present ones are worked on (wide rows fill the registers by themselves)
  static constexpr bool AHEAD = STEPS <= 4;
  // words that hold the scale bytes of a lane's blocks: one each, or of wide rows four to a word
  static constexpr bool PACKED = STEPS > 4;
  static constexpr int SCALE_WORDS = PACKED ? STEPS / 4 : STEPS;
  // (a shape with half the steps would do for up to STEPS blocks: the first STEPS / 2 + 1 steps are always there)
  static constexpr int SURE = STEPS / 2 + 1;
};

// One operand of all steps, as lane l holds it: of its row blocks l / 32, 2 + l / 32, ...
template <typename SHAPE>
struct MxRow {
  int4 codes[SHAPE::STEPS];
  u32 scales[SHAPE::SCALE_WORDS];
};

template <int WIDTH>
__device__ __forceinline__ int4 mx_load_block(const uint8_t* at) {
  if (WIDTH == 16) return *reinterpret_cast<const int4*>(at);
  if (WIDTH == 8) {
    const int2 w = *reinterpret_cast<const int2*>(at);
    return make_int4(w.x, w.y, 0, 0);
  }
  return make_int4(*reinterpret_cast<const int*>(at), 0, 0, 0);
}

// The byte behind the last block of an odd number is another row's, and may stand for NaN.
template <typename SHAPE>
__device__ __forceinline__ void mx_clear_last_scale(u32 blocks, u32* scales) {
  if (!(blocks & 1u)) return;
#pragma unroll
  for (int w = 0; w < SHAPE::SCALE_WORDS; ++w)
    if (lane_id() >= 32 && blocks / 8 == (u32)w) scales[w] &= ~(0xFFu << (8 * (blocks / 2 % 4)));
}

// The scale bytes of a lane's blocks of row `row` (below n).  A block that the row does not have (`blocks` is odd, or below 2 *
// STEPS - 1) has some scale, not that of a NaN unless the row has one.
template <typename SHAPE>
__device__ __forceinline__ void mx_load_scales(const MxHeld& m, u32 row, u32 blocks, u32* to) {
  const u32 half = lane_id() / 32;
  const u64 first = (u64)row * blocks;
  if (!SHAPE::PACKED) {
#pragma unroll
    for (int s = 0; s < SHAPE::STEPS; ++s) to[s] = m.scales[first + min(2 * s + half, blocks - 1)];
    return;
  }
  // Eight scale bytes at a time, those of four steps of both halves; where fewer are left in the array, the last
  // eight of it, shifted.  (A row of such a shape has nine or more.)
  const u64 all = (u64)m.n * blocks;
#pragma unroll
  for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) {
    if (8 * w >= (int)blocks) { to[w] = 0; continue; }
    const u64 at = first + 8 * w, from = min(at, all - 8);
    u64 eight;
    __builtin_memcpy(&eight, m.scales + from, 8);
    eight >>= 8 * (at - from);
    to[w] = __builtin_amdgcn_perm((u32)(eight >> 32), (u32)eight, half ? 0x07050301u : 0x06040200u);
  }
  mx_clear_last_scale<SHAPE>(blocks, to);
}

// Loads a lane's blocks of row `row` (below n).  A block that the row does not have is read as the row's last one: the
// other operand has to be zero there, which mx_clear_rest sees to.
template <typename SHAPE>
__device__ __forceinline__ void mx_load_row(const MxHeld& m, u32 row, u32 blocks, MxRow<SHAPE>* to) {
  const u32 half = lane_id() / 32;
  const u64 first = (u64)row * blocks;
#pragma unroll
  for (int s = 0; s < SHAPE::STEPS; ++s)
    if (s < SHAPE::SURE || 2 * s < (int)blocks) to->codes[s] = mx_load_block<SHAPE::WIDTH>(m.codes + (first + min(2 * s + half, blocks - 1)) * SHAPE::WIDTH);
  mx_load_scales<SHAPE>(m, row, blocks, to->scales);
}

// The same for 32 neighbouring rows, lane l % 32 the row row0 + l % 32 (the last one where there is none), row0 the same in all lanes:
// a scalar base and small offsets (a product of full width takes as long as four other instructions), and no branch, as
// the loads of a loop are only waited for one by one if every turn has the same ones.
struct MxTileRows {
  u32 first, row;        // of the array, and of the lane from there
  __device__ __forceinline__ MxTileRows(u32 n, u32 row0, u32 lane) {
    first = min(row0, n - 1);
    row = min(lane, n - 1 - first);
  }
};
template <typename SHAPE>
__device__ __forceinline__ void mx_load_tile(const MxHeld& m, u32 row0, u32 blocks, MxRow<SHAPE>* to) {
  const u32 half = lane_id() / 32;
  const MxTileRows at(m.n, row0, lane_id() % 32);
  const uint8_t *codes = m.codes + (u64)at.first * blocks * SHAPE::WIDTH, *scales = m.scales + (u64)at.first * blocks;
  const u32 first = __umul24(at.row, blocks);
#pragma unroll
  for (int s = 0; s < SHAPE::STEPS; ++s) {
    const u32 block = first + min(2 * s + half, blocks - 1);
    if (!SHAPE::PACKED || s < SHAPE::SURE || 2 * s < (int)blocks) to->codes[s] = mx_load_block<SHAPE::WIDTH>(codes + block * SHAPE::WIDTH);
    if (!SHAPE::PACKED) to->scales[s] = scales[block];
  }
  if (SHAPE::PACKED) mx_load_scales<SHAPE>(m, at.first + at.row, blocks, to->scales);
}

// Takes out of an operand what mx_load_row has read in place of blocks that the rows do not have.
template <typename SHAPE>
__device__ __forceinline__ void mx_clear_rest(u32 blocks, MxRow<SHAPE>* row) {
  const u32 half = lane_id() / 32;
#pragma unroll
  for (int s = 0; s < SHAPE::STEPS; ++s)
    if (2 * s + half >= blocks) row->codes[s] = make_int4(0, 0, 0, 0);
}

// A row with finite scales, whatever it stands for: its products are numbers, and are not used.
template <typename SHAPE>
__device__ __forceinline__ void mx_take_out(MxRow<SHAPE>* row) {
#pragma unroll
  for (int w = 0; w < SHAPE::SCALE_WORDS; ++w) row->scales[w] = 0;
}

// Whether a row of a lane's operand has a block that stands for NaN; its scales are finite ones then.  (For products whose rows may be
// taken out: such a product is to leave no NaN, and the caller puts it where a row is left.)
template <typename SHAPE>
__device__ __forceinline__ bool mx_take_nan(u32 blocks, MxRow<SHAPE>* row) {
  const u32 half = lane_id() / 32;
  u32 nan = 0;
#pragma unroll
  for (int s = 0; s < SHAPE::STEPS; ++s) {
    const u32 scale = SHAPE::PACKED ? row->scales[s / 4] >> (8 * (s % 4)) & 255u : row->scales[s];
    nan |= 2 * s + half < blocks && scale == kMxNoScale;
  }
  nan |= mx_lane_xor<32>(nan);
  if (nan) mx_take_out<SHAPE>(row);
  return nan != 0;
}

// Changes the signs of all values.
template <typename SHAPE>
__device__ __forceinline__ void mx_negate(MxRow<SHAPE>* row) {
#pragma unroll
  for (int s = 0; s < SHAPE::STEPS; ++s) {
    int4& c = row->codes[s];
    c = make_int4(c.x ^ 0x88888888, c.y ^ 0x88888888, c.z ^ 0x88888888, c.w ^ 0x88888888);
  }
}

template <int BYTE>
__device__ __forceinline__ MxTile mx_step(int4 a, u32 a_scales, int4 b, u32 b_scales, MxTile d) {
  constexpr int kFp4 = 4;
  const MxOperand wa = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, wb = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, wb, d, kFp4, kFp4, BYTE, (int)a_scales, BYTE, (int)b_scales);
}

template <typename SHAPE, int STEP = 0>
__device__ __forceinline__ void mx_steps(const MxRow<SHAPE>& a, const MxRow<SHAPE>& b, u32 blocks, MxTile* d) {
  if constexpr (STEP < SHAPE::STEPS) {
    constexpr int WORD = SHAPE::PACKED ? STEP / 4 : STEP, BYTE = SHAPE::PACKED ? STEP % 4 : 0;
    if (STEP < SHAPE::SURE || 2 * STEP < (int)blocks) *d = mx_step<BYTE>(a.codes[STEP], a.scales[WORD], b.codes[STEP], b.scales[WORD], *d);
    mx_steps<SHAPE, STEP + 1>(a, b, blocks, d);
  }
}

__device__ __forceinline__ MxTile mx_zero_tile() {
  MxTile d;
#pragma unroll
  for (int r = 0; r < 16; ++r) d[r] = 0.f;
  return d;
}

// The products of 32 rows with 32 others; one of the two without what lies behind a row's blocks.
template <typename SHAPE>
__device__ __forceinline__ MxTile mx_products(const MxRow<SHAPE>& a, const MxRow<SHAPE>& b, u32 blocks) {
  MxTile d = mx_zero_tile();
  mx_steps<SHAPE>(a, b, blocks, &d);
  return d;
}

// A tile of 32 rows that the four waves of a workgroup share: wide rows, which would otherwise come out of the caches once for every
// wave and step.  Units of 16 bytes, a block of all rows together; the rows of every other block are swapped eight by
// eight, so that the lanes that store at one time (eight blocks of eight rows) meet all banks.
template <typename SHAPE>
struct MxShared {
  static constexpr int OWN = SHAPE::STEPS / 4;               // units a thread brings: blocks t % 8, 8 + t % 8, ... of row t / 8
  static constexpr int UNITS = SHAPE::STEPS * 2 * kMxTile;
  static __device__ __forceinline__ u32 unit(u32 block, u32 row) { return block * kMxTile + (row ^ (block & 1u) << 3); }
  static __device__ __forceinline__ void load(const MxHeld& m, u32 row0, u32 blocks, int4* own) {
    const u64 first = (u64)min(row0 + threadIdx.x / 8, m.n - 1) * blocks;
#pragma unroll
    for (int j = 0; j < OWN; ++j)
      if (8 * j < (int)blocks) own[j] = mx_load_block<16>(m.codes + (first + min(8 * j + threadIdx.x % 8, blocks - 1)) * 16);
  }
  static __device__ __forceinline__ void store(const int4* own, u32 blocks, int4* tile) {
#pragma unroll
    for (int j = 0; j < OWN; ++j)
      if (8 * j < (int)blocks) tile[unit(8 * j + threadIdx.x % 8, threadIdx.x / 8)] = own[j];
  }
  static __device__ __forceinline__ int4 get(const int4* tile, int step) {
    return tile[unit(2 * step + lane_id() / 32, lane_id() % 32)];
  }
};

// The products of a shared tile's rows (the first operand) with others that have zeros behind their blocks.
template <typename SHAPE, int STEP = 0>
__device__ __forceinline__ void mx_steps_shared(const int4* tile, const u32* scales, const MxRow<SHAPE>& b, u32 blocks, MxTile* d) {
  if constexpr (STEP < SHAPE::STEPS) {
    if (STEP < SHAPE::SURE || 2 * STEP < (int)blocks)
      *d = mx_step<STEP % 4>(MxShared<SHAPE>::get(tile, STEP), scales[STEP / 4], b.codes[STEP], b.scales[STEP / 4], *d);
    mx_steps_shared<SHAPE, STEP + 1>(tile, scales, b, blocks, d);
  }
}
template <typename SHAPE>
__device__ __forceinline__ MxTile mx_products_shared(const int4* tile, const u32* scales, const MxRow<SHAPE>& b, u32 blocks) {
  MxTile d = mx_zero_tile();
  mx_steps_shared<SHAPE>(tile, scales, b, blocks, &d);
  return d;
}

// Two values as bfloat16, rounded to the nearest, ties to even.
__device__ __forceinline__ u32 mx_halves(float low, float high) {
  typedef __bf16 Halves __attribute__((ext_vector_type(2)));
  typedef float Floats __attribute__((ext_vector_type(2)));
  const Floats both = {low, high};
  return __builtin_bit_cast(u32, __builtin_convertvector(both, Halves));
}

// A score; a row whose bias is not finite is out, whatever its codes are.
__device__ __forceinline__ float mx_bias(const float* bias, u32 row) {
  const float b = bias[row];
  return (__float_as_uint(b) & 0x7F800000u) == 0x7F800000u ? -kMxInf : b;
}
template <bool BIAS>
__device__ __forceinline__ float mx_score(float dot, float scale, float bias) {
  if (!BIAS) return __fmul_rn(dot, scale);
  return bias == -kMxInf ? bias : __fmaf_rn(dot, scale, bias);
}

}  // namespace hps
