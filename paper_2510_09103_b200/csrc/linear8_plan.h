// The tiles of a product of a linear layer in 8 bits: how the items of a call and its scratch follow from its sizes.  Plain arithmetic,
// the same on the host and on the device.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "op_checks.h"

namespace adapm {
namespace linear8 {

enum : int32_t { FORWARD = ADAPM_LINEAR8_FORWARD, INPUT_GRAD = ADAPM_LINEAR8_INPUT_GRAD, WEIGHT_GRAD = ADAPM_LINEAR8_WEIGHT_GRAD };

constexpr int kTile = 256;                       // rows and columns of a pair's tile of the result
constexpr int kBand = 16;                        // row tiles that share the columns' operand at a time
constexpr int kMostWords = 2048;                 // status words, one per pair of CTAs or per CTA, at the head of the scratch
constexpr int kHeadBytes = 4 * kMostWords;
constexpr int kPlannedPairs = 74;                // what the number of parts goes by: results do not depend on the device's own number
constexpr int kShortStages = 256;                // longest K, in stages of 64, that one accumulator takes for a gradient in bf16

struct Cut { int m0, n0, bn, k0, count, part; };

// A result of `rows` x `cols`, K of `stages` stages, cut into `parts` parts of `each` stages (the last may be shorter).
struct Plan {
  int32_t rows, cols, m_tiles, n_tiles, stages, parts, each, items;
  int64_t part_at, bytes;        // of the scratch: the parts of K (before them: bf16 numbers of a gradient's codes), and all of it

  // Item i; false past the last.  Tiles go down a band of kBand row tiles, column after column.
  __host__ __device__ __forceinline__ bool item(int i, Cut& t) const {
    if (i >= items) return false;
    const int tile = i / parts, per_band = kBand * n_tiles, band = tile / per_band, in = tile - band * per_band;
    const int left = m_tiles - band * kBand, high = left < kBand ? left : kBand, n = in / high;
    t.part = i - tile * parts;
    t.m0 = (band * kBand + in - n * high) * kTile;
    t.n0 = n * kTile;
    t.bn = cols - t.n0 <= kTile / 2 ? kTile / 2 : kTile;
    t.k0 = t.part * each;
    t.count = stages - t.k0 < each ? stages - t.k0 : each;
    return true;
  }
};

// K is cut where there are fewer tiles than pairs of CTAs, so that its parts, summed by one more launch, take less time.  In units of a stage (512
// cycles): an item takes its stages and four more, the sums a launch of about ten and the parts' way to memory and back.
inline Plan plan_of(int64_t rows, int64_t cols, int64_t k, int stage_k, bool grad) {
  Plan p;
  const bool may_cut = grad;
  p.rows = (int32_t)rows; p.cols = (int32_t)cols;
  p.m_tiles = (int32_t)((rows + kTile - 1) / kTile); p.n_tiles = (int32_t)((cols + kTile - 1) / kTile);
  p.stages = (int32_t)((k + stage_k - 1) / stage_k);
  const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
  p.parts = 1; p.each = p.stages;
  double best = 0;
  for (int n = 1; n <= (may_cut && tiles > 0 && tiles < kPlannedPairs ? std::min(64, p.stages / 4) : 0); ++n) {
    const int each = (p.stages + n - 1) / n, parts = (p.stages + each - 1) / each;
    if (parts != n) continue;
    const double rounds = (double)((tiles * parts + kPlannedPairs - 1) / kPlannedPairs);
    const double t = rounds * (each + 4) + (parts > 1 ? 10 + 8.0 * (double)(rows * cols) * parts / 1e6 : 0);
    if (n == 1 || t < best) { best = t; p.parts = parts; p.each = each; }
  }
  p.items = (int32_t)(tiles * p.parts);
  p.part_at = kHeadBytes + (grad ? round_up(k * cols * 2, 256) : 0);
  p.bytes = p.part_at;
  if (p.parts > 1) p.bytes += round_up((int64_t)p.parts * rows * cols * 4, 256);
  return p;
}

inline int check_desc(const adapm_linear8& d, int32_t which) {
  if (which != FORWARD && which != INPUT_GRAD && which != WEIGHT_GRAD) return ADAPM_EINVAL;
  if (d.tokens < 0 || d.out_features <= 0 || d.in_features <= 0) return ADAPM_EINVAL;
  if (d.tokens > (1 << 24) || d.out_features > (1 << 16) || d.in_features > (1 << 16)) return ADAPM_ERANGE;
  if (d.out_features % 8 || d.in_features % 8) return ADAPM_EUNSUPPORTED;
  if (!known_type(d.y_dtype) || !known_type(d.dx_dtype) || !known_type(d.dweight_dtype)) return ADAPM_EINVAL;
  if (d.x_code != ADAPM_CODE_INT8 && d.x_code != ADAPM_CODE_E4M3) return ADAPM_EINVAL;
  if (d.x_group != 0 && d.x_group != 128) return ADAPM_EINVAL;
  if (which == FORWARD && (d.x_code != ADAPM_CODE_INT8 || d.x_group != 0)) return ADAPM_EUNSUPPORTED;
  const bool x8 = which != INPUT_GRAD, w8 = which != WEIGHT_GRAD, dx = which == INPUT_GRAD, dw = which == WEIGHT_GRAD;
  if (d.y_ld < d.out_features || (x8 && d.x8_ld < d.in_features) || (w8 && d.w8_ld < d.in_features) || (dx && d.dx_ld < d.in_features) ||
      (dw && d.dweight_ld < d.in_features)) return ADAPM_EINVAL;
  if (d.y_ld % 8 || (x8 && d.x8_ld % 16) || (w8 && d.w8_ld % 16) || (dx && d.dx_ld % 8) || (dw && d.dweight_ld % 8)) return ADAPM_EALIGN;
  if (std::max(std::max(std::max(x8 ? d.x8_ld : 0, w8 ? d.w8_ld : 0), d.y_ld), std::max(dx ? d.dx_ld : 0, dw ? d.dweight_ld : 0)) >= ((int64_t)1 << 31)) return ADAPM_ERANGE;
  return ADAPM_OK;
}

inline Plan plan_of(const adapm_linear8& d, int32_t which) {
  if (which == FORWARD) return plan_of(d.tokens, d.out_features, d.in_features, 128, false);
  if (which == INPUT_GRAD) return plan_of(d.tokens, d.in_features, d.out_features, 64, true);
  return plan_of(d.out_features, d.in_features, d.tokens, 64, true);
}

// ---- few tokens ----------------------------------------------------------------------------------------------------
// A tile is 128 features x `tn` tokens; the `split` CTAs of a cluster share its K.  The ring has `ring` stages.
struct FewPlan {
  int32_t tn, t_tiles, n_tiles, stages, split, ring, ctas;
  __host__ __device__ int first(int part) const { return (int)((int64_t)stages * part / split); }      // stage of a part of K
};

constexpr int kFewTokens = 256, kFewSmem = 220 * 1024;

inline int few_stage_bytes(int tn) { return 16384 + 128 * tn; }

inline FewPlan few_plan_of(int64_t tokens, int64_t features, int64_t k, int stage_k) {
  FewPlan p;
  p.t_tiles = (int32_t)((tokens + kFewTokens - 1) / kFewTokens);
  p.tn = (int32_t)round_up((tokens + p.t_tiles - 1) / std::max(1, p.t_tiles), 16);
  p.n_tiles = (int32_t)((features + 127) / 128);
  p.stages = (int32_t)((k + stage_k - 1) / stage_k);
  const int64_t tiles = (int64_t)p.t_tiles * p.n_tiles;
  const int bytes = few_stage_bytes(p.tn);
  p.ring = std::min(8, kFewSmem / bytes);
  p.split = 1;
  while (p.split < 8 && 2 * tiles * p.split <= 2 * kPlannedPairs && 4 * p.split <= p.stages) p.split *= 2;
  p.ctas = (int32_t)std::min<int64_t>(tiles * p.split, INT32_MAX);
  return p;
}

// Whether the forward product goes by tiles of few tokens.
inline bool few_is_faster(const FewPlan& few, const Plan& plan) {
  return few.ctas <= kMostWords && plan.m_tiles * plan.n_tiles < kPlannedPairs;
}

}  // namespace linear8
}  // namespace adapm
