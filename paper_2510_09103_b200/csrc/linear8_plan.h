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

constexpr int kTile = 256;                       // rows of a pair's tile of the result, and its columns at most
constexpr int kBand = 16;                        // row tiles that share the columns' operand at a time
constexpr int kMostWords = 2048;                 // status words, one per pair of CTAs or per CTA, at the head of the scratch
constexpr int kScaleWords = 256;                 // behind them, of a gradient in fp32: whether the scales that a CTA saw are powers of two
constexpr int kHeadBytes = 4 * (kMostWords + kScaleWords);
constexpr int kPlanesF32 = 3, kPlanesBf16 = 2;   // bf16 numbers that one times a scale is carried as, where some scale is no power of two
constexpr int kPlannedPairs = 74;                // what the number of parts goes by: results do not depend on the device's own number
// Longest K, in stages of 64, that one accumulator takes for a gradient in bf16: 1024 steps that the tensor cores cut off by up to 2^-23 of what has been summed are
// 2^-13 at most, beside the result's rounding by 2^-9.
constexpr int kShortStages = 256;

// Of the codes' bf16 numbers in the scratch: rows start on 128 bytes (2048 x 4104 x 4104 weight gradient 81 -> 66 us).
inline int64_t decoded_pitch(int64_t cols) { return round_up(cols, 64); }

struct Cut { int m0, n0, bn, k0, count, part; };

// A result of `rows` x `cols`, K of `stages` stages, cut into `parts` parts of `each` stages (the last may be shorter).
struct Plan {
  int32_t rows, cols, m_tiles, n_tiles, width, stages, parts, each, items;
  int64_t part_at, bytes;        // of the scratch: the parts of K (before them: bf16 numbers of a gradient's codes), and all of it

  // Item i; false past the last.  Tiles go down a band of kBand row tiles, column after column.
  __host__ __device__ __forceinline__ bool item(int i, Cut& t) const {
    if (i >= items) return false;
    const int tile = i / parts, per_band = kBand * n_tiles, band = tile / per_band, in = tile - band * per_band;
    const int left = m_tiles - band * kBand, high = left < kBand ? left : kBand, n = in / high;
    t.part = i - tile * parts;
    t.m0 = (band * kBand + in - n * high) * kTile;
    t.n0 = n * width;
    const int there = (cols - t.n0 + 63) / 64 * 64;
    t.bn = there < width ? there : width;
    t.k0 = t.part * each;
    t.count = stages - t.k0 < each ? stages - t.k0 : each;
    return true;
  }
};

// How wide the tiles are, and into how many parts K is cut (summed by one more launch, where there are fewer tiles than pairs of CTAs): what takes
// least.  In units of a stage of 256 columns (512 cycles): an item takes its stages, narrower ones not quite in
// proportion, and four more, the sums a launch of about eight and the
// parts' way to memory and back.  (2048 x 6400 x 1600: 56 tiles of 256 columns for 74 pairs, or 72 of 192.)  K is cut no further than the parts fit
// `room` bytes of scratch.
constexpr int64_t kAnyRoom = INT64_MAX;
inline Plan plan_of(int64_t rows, int64_t cols, int64_t k, int stage_k, bool grad, bool f32, int64_t room = kAnyRoom) {
  Plan p;
  p.rows = (int32_t)rows; p.cols = (int32_t)cols;
  p.part_at = kHeadBytes + (grad ? round_up(k * decoded_pitch(cols) * 2 * (f32 ? kPlanesF32 : 1), 256) : 0);
  auto bytes_of = [&](int64_t parts) { return p.part_at + (parts > 1 ? round_up(parts * rows * cols * 4, 256) : 0); };
  p.m_tiles = (int32_t)((rows + kTile - 1) / kTile);
  p.stages = (int32_t)((k + stage_k - 1) / stage_k);
  double best = -1;
  for (int width = kTile; width >= 128; width -= 64) {
    const int64_t n_tiles = (cols + width - 1) / width, tiles = p.m_tiles * n_tiles;
    const int most = grad && tiles < kPlannedPairs ? std::max(1, std::min(64, p.stages / 4)) : 1;
    for (int n = 1; n <= most; ++n) {
      const int each = (p.stages + n - 1) / n, parts = each ? (p.stages + each - 1) / each : 1;
      if (parts != n || (n > 1 && bytes_of(n) > room)) continue;
      const double rounds = (double)((tiles * parts + kPlannedPairs - 1) / kPlannedPairs);
      const double t = rounds * (each * (0.2 + 0.8 / 256 * width) + 4) + (parts > 1 ? 8 + 2.5 * (double)(rows * cols) * parts / 1e6 : 0);
      if (best >= 0 && t >= best) continue;
      best = t;
      p.width = width; p.n_tiles = (int32_t)n_tiles; p.parts = parts; p.each = each;
      p.items = (int32_t)(tiles * parts);
    }
  }
  p.bytes = bytes_of(p.parts);
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

inline Plan plan_of(const adapm_linear8& d, int32_t which, int64_t room = kAnyRoom) {
  if (which == FORWARD) return plan_of(d.tokens, d.out_features, d.in_features, 128, false, false, room);
  if (which == INPUT_GRAD) return plan_of(d.tokens, d.in_features, d.out_features, 64, true, d.dx_dtype == ADAPM_TYPE_F32, room);
  return plan_of(d.out_features, d.in_features, d.tokens, 64, true, d.dweight_dtype == ADAPM_TYPE_F32, room);
}

// ---- strips -----------------------------------------------------------------------------------------------------------
// A tile is 128 features of the 8-bit operand x `width` columns of the other; the `split` CTAs of a cluster share its K.  The ring has `ring`
// stages of `stage_bytes`, that of a gradient's operands as they lie `raw` of `raw_bytes`.  fold: a gradient's scales go into the other operand,
// whose numbers then take up to `planes` columns of the product each.
struct StripPlan {
  int32_t width, c_tiles, f_tiles, stages, split, ring, stage_bytes, raw, raw_bytes, fold, planes, ctas;
  __host__ __device__ int first(int part) const { return (int)((int64_t)stages * part / split); }      // stage of a part of K
};

constexpr int kLineTokens = 2;                   // up to so many a forward product goes by rows of the weight, end to end
constexpr int kStripWidth = 256, kFoldWidth = 64, kFoldFew = 16, kStripSmem = 224 * 1024, kStripRing = 8;
constexpr int kStripTeams = 4, kStripRawBytes = 64 * 128;        // gradients: stages that are decoded at the same time; bytes of a stage's codes

inline bool f32_gradient(const adapm_linear8& d, int32_t which) {
  return which == INPUT_GRAD ? d.dx_dtype == ADAPM_TYPE_F32 : which == WEIGHT_GRAD && d.dweight_dtype == ADAPM_TYPE_F32;
}

// What strips were measured to take (us): a start and end, longer with their width, stages, and the sums' ways through a cluster.  (Within 6 % of the measured
// times of 240 gradients.)
inline double strips_take(const StripPlan& s, int32_t which) {
  const double width = s.width, each = (s.stages + s.split - 1) / s.split, levels = s.split == 8 ? 3 : s.split == 4 ? 2 : s.split == 2 ? 1 : 0;
  const double rounds = (double)((s.ctas + 2 * kPlannedPairs - 1) / (2 * kPlannedPairs));
  if (which == FORWARD) return 2.0 + rounds * (3.2 + 0.012 * width + each * (0.16 + 0.0006 * width) + levels * (0.3 + 0.0025 * width));
  const double cluster = s.split == 1 ? 0.0 : s.fold ? 1.0 : 0.9 + levels * (0.004 * width - 0.25);
  if (s.fold) return 2.0 + rounds * (2.8 + 0.026 * width + each * (0.39 + 0.0076 * width) + cluster);
  return 2.0 + rounds * (2.5 + 0.011 * width + each * (0.35 + 0.0005 * width) + cluster);
}

inline StripPlan strip_plan_of(const adapm_linear8& d, int32_t which) {
  const int64_t features = which == FORWARD ? d.out_features : d.in_features, columns = which == WEIGHT_GRAD ? d.out_features : d.tokens;
  const int64_t k = which == FORWARD ? d.in_features : which == INPUT_GRAD ? d.out_features : d.tokens;
  const bool f32 = f32_gradient(d, which);
  StripPlan p;
  // (one rounding per term is not averaged out over few columns; with 64 of them folded scales take longer: 64 x 14336 x 4096 51 us for 28, 16 x 14336 x 4096
  // 34 for 28)
  p.fold = which != FORWARD && (f32 || columns <= kFoldFew);
  p.planes = !p.fold ? 1 : f32 ? kPlanesF32 : kPlanesBf16;
  p.f_tiles = (int32_t)((features + 127) / 128);
  const int step = which == FORWARD ? 128 : 64, unit = which == WEIGHT_GRAD ? 64 : 16, widest = p.fold ? kFoldWidth : kStripWidth;
  p.stages = (int32_t)((k + step - 1) / step);
  // How many strips, and how many CTAs to each: what takes least, as long as all run at the same time.  (Clusters have to fit the device's groups of
  // SMs: 1024 x 512 x 14336 in sixteen clusters of eight 29 us, of four 20; 42 x 2176 x 2256 forward in 34 of four 10.8, in 17 6.4.)
  const int64_t fewest = (columns + widest - 1) / widest;
  int64_t split = 1;
  int32_t width = 0, last = -1;
  double best = -1;
  for (int64_t n = fewest; n == fewest || (n * p.f_tiles <= 2 * kPlannedPairs && n < 2 * fewest + 8); ++n) {
    p.width = (int32_t)round_up((columns + n - 1) / std::max<int64_t>(1, n), unit);
    if (p.width == last) continue;
    last = p.width;
    const int64_t tiles = (columns + p.width - 1) / std::max(1, p.width) * p.f_tiles;
    const int64_t most = std::min<int64_t>(p.stages, tiles <= 8 ? 8 : tiles <= 32 ? 4 : tiles <= kPlannedPairs ? 2 : 1);
    for (p.split = 1; p.split == 1 || p.split <= most; p.split *= 2) {
      p.ctas = (int32_t)std::min<int64_t>(tiles * p.split, INT32_MAX);
      const double t = strips_take(p, which);
      if (best >= 0 && t >= best) continue;
      best = t; width = p.width; split = p.split;
    }
  }
  p.width = width; p.split = (int32_t)split;
  p.c_tiles = (int32_t)((columns + width - 1) / std::max(1, width));
  p.ctas = (int32_t)std::min<int64_t>((int64_t)p.c_tiles * p.f_tiles * split, INT32_MAX);
  p.stage_bytes = 16384 + 128 * p.width * p.planes;
  p.raw_bytes = which == FORWARD ? 0 : kStripRawBytes + (p.fold ? 128 * p.width : 0);
  p.ring = std::max(kStripTeams, std::min(kStripRing, (kStripSmem - (p.fold ? kStripTeams : kStripRing) * p.raw_bytes) / p.stage_bytes));
  p.raw = which == FORWARD ? 0 : std::min(kStripRing, (kStripSmem - p.ring * p.stage_bytes) / p.raw_bytes);
  return p;
}

// Whether strips can take a call: a status word for every CTA, and sums no longer than one accumulator takes.
inline bool strips_can(int32_t which, const StripPlan& s) {
  return s.ctas <= kMostWords && (which == FORWARD || s.fold || (s.stages + s.split - 1) / s.split <= kShortStages);
}

// Whether a call goes by strips, by what both forms were measured to take (us): strips as above; a pair's 256 x 256 tiles, for a gradient with the launch that decodes its codes and the
// one that sums the parts of K.
inline bool strips_are_faster(const adapm_linear8& d, int32_t which, const StripPlan& s, const Plan& p) {
  if (!strips_can(which, s)) return false;
  const bool f32 = f32_gradient(d, which);
  if (s.fold && !f32) return true;                    // (for what the call promises)
  const bool grad = which != FORWARD;
  const double strips = strips_take(s, which);
  const double pair_rounds = (double)((p.items + kPlannedPairs - 1) / kPlannedPairs), wide = 0.2 + 0.8 / 256 * p.width, out = (double)p.rows * p.cols * p.parts / 1e6;
  if (!grad) return strips < 6.0 + pair_rounds * (1.0 + 0.31 * p.each * wide);
  const double decoded = 64e-6 * p.stages * p.cols, dy = 1e-6 * d.tokens * d.out_features;
  double pairs;
  if (f32) pairs = 8.0 + pair_rounds * (1.0 + 0.37 * kPlanesF32 * p.each * wide) + 0.14 * dy + 1.5 * decoded + (p.parts > 1 ? 3.5 + 1.7 * out : 0);
  else pairs = 7.0 + pair_rounds * (1.5 + 0.39 * p.each * wide) + 0.1 * dy + 0.5 * decoded + (p.parts > 1 ? 4.5 + 0.25 * out : 0);
  return strips < pairs;
}

// ---- the form of a call ------------------------------------------------------------------------------------------------
enum : int32_t { LINES, STRIPS, PAIRS };
struct Form {
  int32_t form;
  Plan plan;               // of pairs
  StripPlan strip;
  int64_t bytes;           // of the scratch: strips and lines touch nothing but the words at its head
};

inline Form form_within(const adapm_linear8& d, int32_t which, int64_t room) {
  Form f = {};
  f.form = PAIRS;
  f.bytes = kHeadBytes;
  if (d.tokens == 0) return f;
  f.plan = plan_of(d, which, room);
  if (which == FORWARD && d.tokens <= kLineTokens) {
    f.form = LINES;
    return f;
  }
  f.strip = strip_plan_of(d, which);
  if (strips_are_faster(d, which, f.strip, f.plan) || (f.plan.bytes > room && strips_can(which, f.strip))) f.form = STRIPS;
  else f.bytes = f.plan.bytes;
  return f;
}
// What takes least, or, with `room` bytes of scratch that are too few for it, what does with them.  (What another call, with more tokens, asked for may be too few:
// fewer tokens are fewer tiles, whose K is cut into more parts.  K is then cut into as many parts as fit, and where not even the numbers of the
// codes do, which is where that call went by strips, this one does too.)
inline Form form_of(const adapm_linear8& d, int32_t which, int64_t room = kAnyRoom) {
  const Form f = form_within(d, which, kAnyRoom);
  return f.bytes <= room ? f : form_within(d, which, room);
}

}  // namespace linear8
}  // namespace adapm
