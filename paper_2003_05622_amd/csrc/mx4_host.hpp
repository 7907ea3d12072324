// Host side of include/hps_mx4.h: argument checks, the division of the work, launches.  Part of hps.hip.
#pragma once

namespace {

constexpr uint64_t kMxMaxQueries = 1ull << 20;
constexpr uint64_t kMxMaxRows = (1ull << 31) - 1;
constexpr uint64_t kMxMaxScores = 1ull << 40;      // scores of a call, more than a GPU has room for
constexpr uint64_t kMxScoreGroups = 2048;          // workgroups of mx_scores that fill the GPU

bool mx_dim_ok(uint32_t dim) { return dim >= 4 && dim <= 1024 && dim % 4 == 0; }
bool mx_aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
size_t mx_code_alignment(uint32_t dim) { return std::min<size_t>(16, mx_row_bytes(dim)); }

bool mx_rows_ok(const hps_mx4_rows* r, uint32_t dim, uint64_t most) {
  if (!r || r->n > most) return false;
  return r->n == 0 || (r->d_codes && r->d_scales && mx_aligned(r->d_codes, mx_code_alignment(dim)));
}
MxHeld mx_held(const hps_mx4_rows* r) { return {r->d_codes, r->d_scales, (u32)r->n}; }

uint64_t mx_ceil(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// How the rows are dealt out over the waves: so many parts that the GPU is full, a multiple of 8, so that all waves of
// a part share an XCD and with it the L2 that holds its rows.
constexpr uint64_t kMxWaves = 4096;
// Up to so many queries the end of the log probabilities takes 16 waves a query, beyond four: 64 x 262 144, 64 wide, best 8: 21 us (25 with four), 256: 33
// (35), 320: 42 (46 with 16), 1024: 75 (95).
constexpr uint64_t kMxFewQueries = 256;
// Workgroups of mx_gradient: as many as run at once (two on a CU, four of the narrow ones with one query tile a wave), so that all end together.
constexpr uint64_t kMxGradGroups = 512;
constexpr uint64_t kMxPartsBytes = 128ull << 20;
struct MxSplit {
  uint64_t query_tiles, part_rows, parts, group, groups;
};
// Query tiles a wave of mx_softmax holds: two share what is read of the rows, unless that leaves much of the last ones empty.  (1024 x 262 144, 64 wide:
// 59 us, 62 with one; 160 x 524 288, five tiles: 28, 31 with two; 64 x 524 288: 16.5, 15.1 with one.)
int mx_wave_tiles(uint64_t n_queries, uint32_t dim) {
  const uint64_t tiles = mx_ceil(n_queries, kMxTile);
  return mx_blocks(dim) <= 8 && (tiles % 2 == 0 || tiles > 8) ? 2 : 1;
}
MxSplit mx_split(uint64_t n_queries, uint64_t n_rows, uint32_t dim, uint32_t top, uint32_t wave_tiles, uint64_t waves) {
  MxSplit s;
  s.query_tiles = mx_ceil(n_queries, kMxTile * wave_tiles);
  // rows of a group: what noting the groups' highest scores costs (4 bytes a group, written and read) against scoring the rows of
  // `top` groups once more
  s.group = kMxTile;
  const double row = mx_row_bytes(dim) + mx_blocks(dim);
  while (top && s.group < 1024 && 8.0 * n_rows / (double)s.group > (double)top * (double)(2 * s.group) * row) s.group *= 2;
  const uint64_t wanted = mx_ceil(std::max<uint64_t>(1, waves / s.query_tiles), kXcds) * kXcds;
  s.part_rows = mx_ceil(mx_ceil(n_rows, wanted), s.group) * s.group;
  s.parts = mx_ceil(n_rows, s.part_rows);
  s.groups = top ? mx_ceil(n_rows, s.group) : 0;
  return s;
}
// Whether the waves of a workgroup share the rows' tiles: rows of more than 256 values, and queries for at least three of its four waves.  (Log
// probabilities, 65 536 rows of 1024: 1024 queries 86 us, 169 without sharing, 96 28 and 35, 64 27 and 28; of 512: 1024 43 and 78, 32 12.8 and 12.5.)
bool mx_shares_rows(uint64_t n_queries, uint32_t dim) { return mx_blocks(dim) > 8 && n_queries > 2 * kMxTile; }
MxSplit mx_softmax_split(uint64_t n_queries, uint64_t n_rows, uint32_t dim, uint32_t top) {
  if (mx_shares_rows(n_queries, dim)) return mx_split(n_queries, n_rows, dim, top, kMxThreads / kWave, kMxWaves / (kMxThreads / kWave));
  return mx_split(n_queries, n_rows, dim, top, (uint32_t)mx_wave_tiles(n_queries, dim), kMxWaves);
}
size_t mx_parts_bytes(const MxSplit& s, uint64_t n_queries) { return align_up(s.parts * n_queries * sizeof(MxPart)); }

template <typename F>
void mx_by_width(uint32_t dim, F f) {
  if (dim <= 8) f(std::integral_constant<int, 4>());
  else if (dim <= 16) f(std::integral_constant<int, 8>());
  else f(std::integral_constant<int, 16>());
}
template <typename F>
void mx_by_shape(uint32_t dim, F f) {
  const uint32_t blocks = mx_blocks(dim);
  if (dim <= 8) f(MxShape<4, 1>());
  else if (dim <= 16) f(MxShape<8, 1>());
  else if (blocks <= 2) f(MxShape<16, 1>());
  else if (blocks <= 4) f(MxShape<16, 2>());
  else if (blocks <= 8) f(MxShape<16, 4>());
  else if (blocks <= 16) f(MxShape<16, 8>());
  else f(MxShape<16, 16>());
}
template <typename F>
void mx_by_flag(bool flag, F f) {
  if (flag) f(std::true_type());
  else f(std::false_type());
}

bool mx_scale_ok(float scale) { return scale >= -0x1p100f && scale <= 0x1p100f; }

}  // namespace

extern "C" {

size_t hps_mx4_row_bytes(uint32_t dim) { return mx_dim_ok(dim) ? mx_row_bytes(dim) : 0; }
size_t hps_mx4_row_scales(uint32_t dim) { return mx_dim_ok(dim) ? mx_blocks(dim) : 0; }

hps_status hps_mx4_quantize(const void* d_values, int32_t type, uint64_t n, uint32_t dim, uint64_t stride,
                            uint8_t* d_codes, uint8_t* d_scales, float* d_rounded, void* stream) {
  if (!mx_dim_ok(dim) || (type != HPS_VALUES_F32 && type != HPS_VALUES_BF16) || stride < dim || stride % 4) return HPS_EINVAL;
  if (n > (1ull << 40) || stride > (1ull << 40) / std::max<uint64_t>(n, 1)) return HPS_EINVAL;
  if (n == 0) return HPS_OK;
  if (!d_values || !d_codes || !d_scales) return HPS_EINVAL;
  if (!mx_aligned(d_values, type == HPS_VALUES_F32 ? 16 : 8) || !mx_aligned(d_codes, mx_code_alignment(dim)) || !mx_aligned(d_rounded, 16))
    return HPS_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  mx_by_width(dim, [&](auto width) {
    constexpr int GL = decltype(width)::value / 4, LANES = 2 * GL;
    const uint64_t all = n * mx_blocks(dim);
    mx_by_flag(type == HPS_VALUES_BF16, [&](auto bf16) {
      constexpr bool BF16 = decltype(bf16)::value;
      if (d_rounded)
        mx_quantize_round<BF16, LANES><<<grid_for(all, kMxThreads / LANES * kMxInFlight, 1u << 20), kMxThreads, 0, s>>>(
            d_values, n, dim, stride, d_codes, d_scales, d_rounded);
      else
        mx_quantize<BF16, GL><<<grid_for(all, kMxThreads / GL, 1u << 20), kMxThreads, 0, s>>>(d_values, n, dim, stride, d_codes, d_scales);
    });
  });
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

hps_status hps_mx4_dequantize(const hps_mx4_rows* rows, uint32_t dim, float* d_out, void* stream) {
  if (!mx_dim_ok(dim) || !mx_rows_ok(rows, dim, (1ull << 40) / dim)) return HPS_EINVAL;
  if (rows->n == 0) return HPS_OK;
  if (!d_out || !mx_aligned(d_out, 16)) return HPS_EINVAL;
  mx_dequantize<<<grid_for(rows->n * (dim / 4), kMxThreads, 1u << 20), kMxThreads, 0, static_cast<hipStream_t>(stream)>>>(
      rows->d_codes, rows->d_scales, rows->n, dim, d_out);
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

hps_status hps_mx4_get(hps_table* t, const uint64_t* d_keys, uint64_t n, uint8_t* d_codes, uint8_t* d_scales,
                       uint8_t* d_found_out, void* stream) {
  if (!t || (n && (!d_keys || !d_codes || !d_scales || !d_found_out || !mx_aligned(d_codes, mx_code_alignment(t->dim))))) return HPS_EINVAL;
  if (n == 0) return HPS_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned blocks = grid_for(n, kRowThreads, kRowMaxBlocks);
  mx_by_width(t->dim, [&](auto width) {
    mx_by_flag(t->view.bf16 != 0, [&](auto bf16) {
      mx_get<decltype(bf16)::value, decltype(width)::value / 4><<<blocks, kRowThreads, 0, s>>>(t->view, d_keys, n, d_codes, d_scales, d_found_out);
    });
  });
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

hps_status hps_mx4_scores(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                          const float* d_bias, void* d_out, int32_t type, uint64_t stride, void* stream) {
  if (!mx_dim_ok(dim) || !mx_rows_ok(queries, dim, kMxMaxQueries) || !mx_rows_ok(rows, dim, kMxMaxRows) || !mx_scale_ok(scale) ||
      (type != HPS_VALUES_F32 && type != HPS_VALUES_BF16) || stride < rows->n || stride > (1ull << 40) ||
      rows->n * queries->n > kMxMaxScores)
    return HPS_EINVAL;
  if (queries->n == 0 || rows->n == 0) return HPS_OK;
  const bool bf16 = type == HPS_VALUES_BF16;
  if (!d_out || !mx_aligned(d_out, bf16 ? 2 : 4) || !mx_aligned(d_bias, 4)) return HPS_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  mx_by_shape(dim, [&](auto shape) {
    typedef decltype(shape) Shape;
    const uint64_t row_groups = mx_ceil(rows->n, mx_score_tiles<Shape>() * kMxTile * (kMxThreads / kWave)), tiles = mx_ceil(queries->n, kMxTile);
    // a part of the queries for every workgroup, as long as that leaves enough of them
    const uint64_t part_tiles = mx_ceil(tiles, std::max<uint64_t>(1, kMxScoreGroups / row_groups)), parts = mx_ceil(tiles, part_tiles);
    // (at most 2^23 workgroups)
    mx_by_flag(d_bias != nullptr, [&](auto biased) {
      mx_by_flag(bf16, [&](auto narrow) {
        // (1024 x 262 144, float32: 203 us past the L2, 300 through it; 333 x 100 003: 49 us past it, 27 through it)
        const bool lines = stride * (bf16 ? 2 : 4) % 128 == 0 && mx_aligned(d_out, 128);
        mx_by_flag(lines, [&](auto whole_lines) {
          mx_scores<Shape, decltype(biased)::value, decltype(narrow)::value, decltype(whole_lines)::value>
              <<<(unsigned)(row_groups * parts), kMxThreads, 0, s>>>(mx_held(queries), mx_held(rows), mx_blocks(dim), scale, d_bias, d_out,
                                                                     stride, (u32)row_groups, (u32)parts, (u32)part_tiles);
        });
      });
    });
  });
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

static bool mx_sizes_ok(uint64_t n_queries, uint64_t n_rows, uint32_t dim) {
  return mx_dim_ok(dim) && n_queries <= kMxMaxQueries && n_rows <= kMxMaxRows;
}

size_t hps_mx4_logprobs_bytes(uint64_t n_queries, uint64_t n_rows, uint32_t dim, uint32_t top) {
  if (!mx_sizes_ok(n_queries, n_rows, dim) || top > HPS_MX4_MAX_TOP) return 0;
  if (n_queries == 0 || n_rows == 0) return kAlign;
  const MxSplit p = mx_softmax_split(n_queries, n_rows, dim, top);
  return mx_parts_bytes(p, n_queries) + align_up(p.groups * n_queries * sizeof(float));
}

hps_status hps_mx4_logprobs(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                            const float* d_bias, const int32_t* d_given, uint32_t n_given, uint32_t top,
                            float* d_lse, float* d_entropy, float* d_logp, int32_t* d_top_index, float* d_top_logp,
                            void* d_workspace, size_t workspace_bytes, void* stream) {
  if (!mx_dim_ok(dim) || !mx_rows_ok(queries, dim, kMxMaxQueries) || !mx_rows_ok(rows, dim, kMxMaxRows) || !mx_scale_ok(scale) ||
      top > HPS_MX4_MAX_TOP || n_given > (1u << 20))
    return HPS_EINVAL;
  const uint64_t m = queries->n;
  if (m == 0) return HPS_OK;
  if (!d_lse || !d_entropy || (n_given && (!d_given || !d_logp)) || (top && (!d_top_index || !d_top_logp))) return HPS_EINVAL;
  if (!mx_aligned(d_bias, 4) || !mx_aligned(d_given, 4) || !mx_aligned(d_lse, 4) || !mx_aligned(d_entropy, 4) || !mx_aligned(d_logp, 4) ||
      !mx_aligned(d_top_index, 4) || !mx_aligned(d_top_logp, 4))
    return HPS_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (rows->n == 0) {
    mx_no_rows<<<grid_for(m * std::max(std::max(n_given, top), 1u), kMxThreads, 1u << 16), kMxThreads, 0, s>>>(
        (u32)m, d_given, n_given, top, d_lse, d_entropy, d_logp, d_top_index, d_top_logp);
    return launch_ok() ? HPS_OK : HPS_EDEVICE;
  }
  if (!d_workspace || !mx_aligned(d_workspace, kAlign)) return HPS_EINVAL;
  if (workspace_bytes < hps_mx4_logprobs_bytes(m, rows->n, dim, top)) return HPS_ENOMEM;
  const MxSplit p = mx_softmax_split(m, rows->n, dim, top);
  MxPart* parts = static_cast<MxPart*>(d_workspace);
  float* highest = top ? reinterpret_cast<float*>(static_cast<char*>(d_workspace) + mx_parts_bytes(p, m)) : nullptr;
  mx_by_flag(d_bias != nullptr, [&](auto biased) {
    constexpr bool B = decltype(biased)::value;
    const dim3 grid((unsigned)p.parts, (unsigned)p.query_tiles);
    mx_by_shape(dim, [&](auto shape) {
      typedef decltype(shape) Shape;
#define HPS_MX_SOFTMAX(QT)                                                                                                   \
  mx_softmax<Shape, B, QT><<<grid, kWave, 0, s>>>(mx_held(queries), mx_held(rows), mx_blocks(dim), scale, d_bias,            \
                                                  (u32)p.part_rows, (u32)p.group, (u32)p.groups, parts, highest)
      if constexpr (Shape::STEPS <= 4) {
        if (mx_wave_tiles(m, dim) == 2) { HPS_MX_SOFTMAX(2); return; }
      } else if (mx_shares_rows(m, dim)) {
        mx_softmax_shared<Shape, B><<<grid, kMxThreads, 0, s>>>(mx_held(queries), mx_held(rows), mx_blocks(dim), scale, d_bias,
                                                                (u32)p.part_rows, (u32)p.group, (u32)p.groups, parts, highest);
        return;
      }
      HPS_MX_SOFTMAX(1);
#undef HPS_MX_SOFTMAX
    });
    mx_by_width(dim, [&](auto width) {
      constexpr int W = decltype(width)::value;
#define HPS_MX_FINISH(WAVES)                                                                                                 \
  mx_finish<W, B, WAVES><<<(unsigned)m, WAVES * kWave, 0, s>>>(                                                              \
      mx_held(queries), mx_held(rows), mx_blocks(dim), scale, d_bias, parts, (u32)p.parts, highest, (u32)p.group,            \
      (u32)p.groups, d_given, n_given, top, d_lse, d_entropy, d_logp, d_top_index, d_top_logp)
      // (few queries leave the GPU idle: then a query's work is spread further)
      if (m <= kMxFewQueries) HPS_MX_FINISH(16);
      else HPS_MX_FINISH(4);
#undef HPS_MX_FINISH
    });
  });
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

// The gradient's division: workgroups of up to four (narrow rows and many queries: eight) query tiles and a part of the rows each;
// where the tiles are fewer than a workgroup's waves, these share the rows instead.
struct MxGradSplit {
  uint64_t wave_tiles, query_groups, grid_queries, columns, grid_columns, part_rows, parts;
  bool wide;                 // parts so long that their sums are held in 64 bits
};
// Whether the waves share the rows' tiles.  (Rows of more than 512 values fill the registers of a wave by themselves: 8 queries against 131 072
// rows of 1024 take 239 us without sharing, 100 queries 211 us with it; 64 queries, 512 wide, 66 us without and 81 with it.)
static bool mx_gradient_shares(uint64_t n_queries, uint32_t dim) { return mx_blocks(dim) > 16 || mx_shares_rows(n_queries, dim); }
static MxGradSplit mx_grad_split(uint64_t n_queries, uint64_t n_rows, uint32_t dim) {
  MxGradSplit s;
  const uint64_t tiles = mx_ceil(n_queries, kMxTile);
  // (two where there are enough of them: 1024 x 524 288, 64 wide, 188 us, 196 with one; 192 x 262 144 41, 43 with two; 224 43.5, 40 with one)
  s.wave_tiles = dim <= 64 && tiles > 6 ? 2 : 1;
  const uint64_t waves = mx_ceil(tiles, s.wave_tiles);
  s.query_groups = waves > 2 || mx_gradient_shares(n_queries, dim) ? 4 : waves;
  s.grid_queries = mx_ceil(waves, s.query_groups);
  s.columns = dim <= 32 ? 32 : dim <= 64 ? 64 : 128;
  s.grid_columns = mx_ceil(dim, s.columns);
  const uint64_t wanted = std::max<uint64_t>(1, kMxGradGroups * (s.columns > 64 || s.wave_tiles == 2 ? 1 : 2) / (s.grid_queries * s.grid_columns));
  s.part_rows = mx_ceil(mx_ceil(n_rows, wanted), kMxStageRows) * kMxStageRows;
  // (waves that share the rows join their sums at the end of the part: each has so many rows at most)
  if (s.query_groups < kMxGradWaves) s.part_rows = std::min<uint64_t>(s.part_rows, kMxSumRows * (kMxGradWaves / s.query_groups));
  // More parts than run at once rather than long ones, as long as their sums lie in the last-level cache.  (1024 x 131 072, 512 / 1024 wide: 516 / 1451 us,
  // 533 / 1494 with long parts.)
  else if (mx_ceil(n_rows, kMxSumRows) * n_queries * dim * sizeof(float) <= kMxPartsBytes) s.part_rows = std::min<uint64_t>(s.part_rows, kMxSumRows);
  s.parts = mx_ceil(n_rows, s.part_rows);
  s.wide = s.query_groups == kMxGradWaves && s.part_rows > kMxSumRows;
  return s;
}

size_t hps_mx4_logprobs_backward_bytes(uint64_t n_queries, uint64_t n_rows, uint32_t dim) {
  if (!mx_sizes_ok(n_queries, n_rows, dim)) return 0;
  if (n_queries == 0 || n_rows == 0) return kAlign;
  const MxGradSplit p = mx_grad_split(n_queries, n_rows, dim);
  return align_up(p.parts * n_queries * dim * (p.wide ? sizeof(double) : sizeof(float)));
}

hps_status hps_mx4_logprobs_backward(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                                     const float* d_bias, const float* d_lse, const float* d_entropy,
                                     const int32_t* d_given, const float* d_dlogp, uint32_t n_given,
                                     const float* d_dentropy, float* d_dqueries, void* d_workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!mx_dim_ok(dim) || !mx_rows_ok(queries, dim, kMxMaxQueries) || !mx_rows_ok(rows, dim, kMxMaxRows) || !mx_scale_ok(scale) ||
      n_given > (1u << 20))
    return HPS_EINVAL;
  const uint64_t m = queries->n;
  if (m == 0) return HPS_OK;
  if (!d_lse || !d_dqueries || (n_given && (!d_given || !d_dlogp)) || (d_dentropy && !d_entropy)) return HPS_EINVAL;
  if (!mx_aligned(d_bias, 4) || !mx_aligned(d_lse, 4) || !mx_aligned(d_entropy, 4) || !mx_aligned(d_given, 4) || !mx_aligned(d_dlogp, 4) ||
      !mx_aligned(d_dentropy, 4) || !mx_aligned(d_dqueries, 16) || !d_workspace || !mx_aligned(d_workspace, kAlign))
    return HPS_EINVAL;
  if (workspace_bytes < hps_mx4_logprobs_backward_bytes(m, rows->n, dim)) return HPS_ENOMEM;
  hipStream_t s = static_cast<hipStream_t>(stream);
  MxGradSplit p = {};
  const u32 blocks = mx_blocks(dim), row_bytes = mx_row_bytes(dim);
  if (rows->n == 0) d_bias = nullptr;                // (there is nothing to read behind it)
  mx_by_flag(d_bias != nullptr, [&](auto biased) {
    mx_by_flag(d_dentropy != nullptr, [&](auto with_entropy) {
      constexpr bool B = decltype(biased)::value, E = decltype(with_entropy)::value;
      if (rows->n) {
        p = mx_grad_split(m, rows->n, dim);
        const double exact = B ? 1.4426950408889634 : std::fabs((double)scale) * 1.4426950408889634;
        const float held = B ? kMxLog2e : std::fabs(scale) * kMxLog2e;
        // (a unit below the normal numbers is off by much, of exponents that are next to nothing)
        const MxGradUnit unit = {held, held > 1e-30f ? (float)(exact / held - 1.0) : 0.f};
        const dim3 grid((unsigned)p.parts, (unsigned)p.grid_queries, (unsigned)p.grid_columns);
        MxPartRows part = {(u32)p.part_rows, 0, p.wide};
        auto launch = [&](auto shape) {
          typedef decltype(shape) Shape;
#define HPS_MX_GRADIENT(COLUMNS, QT)                                                                                         \
  mx_gradient<Shape, B, E, COLUMNS, QT><<<grid, kMxGradWaves * kWave, 0, s>>>(                                               \
      mx_held(queries), mx_held(rows), dim, blocks, row_bytes, scale, unit, d_bias, d_lse, d_entropy, d_given, d_dlogp,      \
      n_given, d_dentropy, (u32)p.query_groups, part, d_workspace)
          if constexpr (Shape::STEPS >= 8) {
            if (mx_gradient_shares(m, dim)) {
              mx_gradient_shared<Shape, B, E><<<grid, kMxThreads, 0, s>>>(
                  mx_held(queries), mx_held(rows), dim, blocks, row_bytes, scale, unit, d_bias, d_lse, d_entropy, d_given, d_dlogp,
                  n_given, d_dentropy, part, d_workspace);
              return;
            }
          }
          if constexpr (Shape::STEPS > 1) {
            if constexpr (Shape::STEPS < 16) HPS_MX_GRADIENT(128, 1);
          } else {
            if (p.columns == 32) { if (p.wave_tiles == 2) HPS_MX_GRADIENT(32, 2); else HPS_MX_GRADIENT(32, 1); }
            else if constexpr (Shape::WIDTH == 16) { if (p.wave_tiles == 2) HPS_MX_GRADIENT(64, 2); else HPS_MX_GRADIENT(64, 1); }
          }
#undef HPS_MX_GRADIENT
        };
        // (part_rows is at most 2^31)
        do {
          mx_by_shape(dim, launch);
          part.done += kMxSumRows;
        } while (p.wide && part.done < p.part_rows);
      }
      const unsigned blocks_end = grid_for(m * dim, kWave, 1u << 20);
#define HPS_MX_END(WAVES)                                                                                                    \
  mx_gradient_end<B, E, WAVES><<<blocks_end, WAVES * kWave, 0, s>>>(mx_held(rows), (u32)m, dim, blocks, row_bytes, scale, d_bias, \
                                                                    d_given, d_dlogp, n_given, d_workspace, (u32)p.parts, p.wide, d_dqueries)
      // (few values: more waves each, 1 x 1 M, 64 wide, 28.6 us, 31.6 with eight; many: as many workgroups at once as there are, 1024 x 524 288 188, 187 with 16)
      if (blocks_end <= 256) HPS_MX_END(16);
      else HPS_MX_END(8);
#undef HPS_MX_END
    });
  });
  return launch_ok() ? HPS_OK : HPS_EDEVICE;
}

}  // extern "C"
