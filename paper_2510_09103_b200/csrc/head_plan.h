// The head loss's tiles: how the items of a call follow from its sizes and from the number of tokens with a target, and what of its
// scratch lies where.  Plain arithmetic, the same on the host and on the device.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "op_checks.h"
#ifdef __CUDACC__
#include "tc_common.cuh"
#endif

namespace adapm {
namespace head {

enum : int32_t { CLS_LOGITS = 0, CLS_DH = 1, CLS_DW = 2 };

// head of the scratch: status word, number of tokens with a target, and (forward) a status word of every pair of CTAs
enum : int32_t { HD_STATUS = 0, HD_COUNT = 1, HD_PAIRS = 64 };
constexpr int kMostPairs = 128, kHeadBytes = 4 * (HD_PAIRS + kMostPairs);

constexpr int kTile = 256;
constexpr int kStageK = 64;
constexpr int kGroupM = 16;                  // row tiles that share the head's columns at a time

// `stages` in at most `most` parts of even length: how many, and the stages of each but the last.
__device__ __host__ __forceinline__ void parts_of(int stages, int most, int& n, int& each) {
  each = (stages + most - 1) / most;
  n = (stages + each - 1) / each;
}

// n / d for 0 <= n < 2^31 by a multiplication: with 2^(s-1) < d <= 2^s and m = floor(2^(31+s) / d) + 1 the quotient is
// n m >> (31 + s) (Granlund and Montgomery, PLDI 1994).  Every warp divides a few times per item.
struct Divisor {
  uint32_t d, m;
  int shift;
  __host__ __device__ void set(int x) {
    d = (uint32_t)x;
    int s = 0;
    while ((1ll << s) < x) ++s;
    shift = s - 1;
    m = x > 1 ? (uint32_t)((1ull << (31 + s)) / d + 1) : 0;
  }
  __host__ __device__ __forceinline__ int of(int n) const { return m ? (int)((uint32_t)(((uint64_t)(uint32_t)n * m) >> 32) >> shift) : n; }
};

// One tile of a result: its first row and column, its columns, and its share of K, `count` stages from stage k0 of
// `planes` planes of per_plane stages laid end to end.
struct HeadItem { int cls, m0, n0, bn, k0, count, per_plane, split; };

// bf16 numbers that g is carried as into the product of a gradient, by the gradient's type and the tokens with a target.  Three for
// fp32.  One for bf16, but two where there are few tokens: a token's gradient is mostly its target's element of g, whose rounding
// is averaged out over the tokens only (a norm's error of one token's gradients was up to 2.4 times that of their own rounding, of 64
// tokens 1.4 times).  With so few of them the planes lie 64 rows apart: dw takes them one stage of K after the other, and dh, in
// bf16, as the upper and lower half of one CTA's rows, which are summed like parts of K, so that the weight is multiplied once and not
// twice (100 x 128256 x 4096 with 10 targets: 970 us for 1290; with one plane 940).
constexpr int kFewTokens = 64;
static_assert(kFewTokens == kStageK && 2 * kFewTokens == kTile / 2, "a plane of few tokens is a stage of K of dw and half of a CTA's rows of dh");
__host__ __device__ __forceinline__ int planes_of(bool f32, int with_target) { return f32 ? 3 : with_target <= kFewTokens ? 2 : 1; }

// What the items of a call follow from, beside the number of tokens with a target.
struct Plan {
  int32_t tokens, vocab, hidden, piece, n_pieces, f32_dh, f32_dw, split_dh, split_dw, dh, dw, backward, pairs;
  __host__ __device__ int cols(int i) const {               // of piece i of the vocabulary
    const int left = vocab - i * piece;
    return i < 0 || i >= n_pieces ? 0 : left < piece ? left : piece;
  }
  // Pairs of CTAs of launch i (with every token counted: the host does not know better).
  __host__ __device__ int used(int i) const {
    const int64_t m = (tokens + kTile - 1) / kTile, tiles = (cols(i) + kTile - 1) / kTile, o = backward ? (cols(i - 1) + kTile - 1) / kTile : 0;
    const int64_t items = m * tiles + (o ? (m * split_dh + o * split_dw) * ((hidden + kTile - 1) / kTile) : 0);
    return items < pairs ? (int)items : pairs;
  }
};

// The items of launch i of a call, as every warp of a pair walks through them: in the backward call those of the logits of piece i
// and of the gradients of piece i - 1.  Long items (gradients) first, dealt out in turn; then the short ones (logits) in turn,
// where the pairs that got a long item more join `skip` rounds later.  Made once per call, by the host or by the kernel that
// counts the tokens; a launch that made it anew spent two microseconds on its divisions.
struct Walk {
  int tv, pairs, n_dh, n_long, n_short, extra, skip, rounds;
  int m_tiles, tiles_dw, base_d, more_d, k_logits, k_dh, k_dw, each_dh, each_dw, all_dh, all_dw, last_group;
  int parts_dh, parts_dw;        // of a gradient, as its sum takes them: those of the call's longest piece
  int planes, planes_dw, plane_rows;      // of g as it is made, of those that dw takes along K; rows from one to the next
  int planes_dh, stacked;                 // of those that dh takes along K; 1: it takes two as rows of one tile
  Divisor by_group, by_last, by_d, by_m, by_dw;

  __host__ __device__ void make(const Plan& p, int i, int tv_) {
    tv = tv_;
    pairs = p.used(i);
    m_tiles = (tv + kTile - 1) / kTile;
    const int nt_v = (p.cols(i) + kTile - 1) / kTile, units = (p.hidden + 31) / 32, nt_d = (units + 7) / 8;
    base_d = units / nt_d; more_d = units % nt_d;
    last_group = m_tiles / kGroupM;
    by_group.set(nt_v ? kGroupM * nt_v : 1); by_last.set(m_tiles % kGroupM ? m_tiles % kGroupM : 1);
    by_d.set(nt_d); by_m.set(m_tiles ? m_tiles : 1);
    k_logits = (p.hidden + kStageK - 1) / kStageK;
    n_short = m_tiles * nt_v;
    n_dh = n_long = extra = skip = rounds = k_dh = k_dw = each_dh = each_dw = all_dh = all_dw = tiles_dw = parts_dh = parts_dw = 0;
    planes_dh = p.f32_dh ? 3 : 1;
    planes_dw = planes_of(p.f32_dw, tv);
    planes = planes_of(p.f32_dh || p.f32_dw, tv);
    plane_rows = tv <= kFewTokens ? kFewTokens : m_tiles * kTile;
    stacked = !p.f32_dh && tv <= kFewTokens;
    const int o_cols = p.backward ? p.cols(i - 1) : 0;
    by_dw.set(1);
    if (o_cols == 0) return;
    k_dh = (o_cols + kStageK - 1) / kStageK;
    k_dw = tv > 0 ? (tv + kStageK - 1) / kStageK : 1;
    all_dh = k_dh * planes_dh; all_dw = k_dw * planes_dw;
    // The first piece is as long as any, and the length of its parts is that of every piece's: a shorter piece has as many parts
    // or fewer.  (Cut by itself it can have more, 50 parts of 2045 stages beside 49 of 2052, and nothing would sum the last.)
    parts_of((p.cols(0) + kStageK - 1) / kStageK * planes_dh, p.split_dh, parts_dh, each_dh);
    parts_of(all_dw, p.split_dw, parts_dw, each_dw);
    const int split_dh = (all_dh + each_dh - 1) / each_dh;
    tiles_dw = (o_cols + kTile - 1) / kTile;
    by_dw.set(tiles_dw);
    n_dh = p.dh ? m_tiles * nt_d * split_dh : 0;
    n_long = n_dh + (p.dw ? tiles_dw * nt_d * parts_dw : 0);
    rounds = n_long / pairs;
    extra = n_long % pairs;
    const int surplus = load(0) - load(pairs - 1);
    skip = extra && surplus > 0 ? (surplus + k_logits / 2) / k_logits : 0;
  }
  __host__ __device__ int dealt(int n, int p) const { return n / pairs + (p < n % pairs ? 1 : 0); }
  __host__ __device__ int load(int p) const {
    const int dh = dealt(n_dh, p);
    return dh * each_dh + (dealt(n_long, p) - dh) * each_dw;
  }
  // This pair's item `seq`; false past the last.
  // (Read from shared memory: `uniform` tells the compiler that all lanes have the same.)
#ifdef __CUDACC__
  template <bool BACKWARD>
  __device__ __forceinline__ bool item_uniform(int pair, int seq, HeadItem& t) const {
    using tc::uniform;
    if (!uniform((int)item<BACKWARD>(pair, seq, t))) return false;
    t.cls = uniform(t.cls); t.m0 = uniform(t.m0); t.n0 = uniform(t.n0); t.bn = uniform(t.bn);
    t.k0 = uniform(t.k0); t.count = uniform(t.count); t.per_plane = uniform(t.per_plane);
    return true;
  }
#endif
  template <bool BACKWARD>
  __host__ __device__ __forceinline__ bool item(int pair, int seq, HeadItem& t) const {
    t.split = t.k0 = 0;
    const int mine = BACKWARD ? rounds + (pair < extra ? 1 : 0) : 0;
    if (BACKWARD && seq < mine) {
      int k = pair + seq * pairs;
      const bool dh = k < n_dh;
      t.cls = dh ? CLS_DH : CLS_DW;
      if (!dh) k -= n_dh;
      const int q = by_d.of(k), n = k - q * (int)by_d.d;
      t.split = dh ? by_m.of(q) : by_dw.of(q);
      t.m0 = (q - t.split * (dh ? m_tiles : tiles_dw)) * kTile;
      t.n0 = 32 * (n * base_d + (n < more_d ? n : more_d));      // widths as even as multiples of 32 allow
      t.bn = 32 * (base_d + (n < more_d ? 1 : 0));
      t.per_plane = dh ? k_dh : k_dw;
      t.k0 = t.split * (dh ? each_dh : each_dw);
      const int each = dh ? each_dh : each_dw, left = (dh ? all_dh : all_dw) - t.k0;
      t.count = each < left ? each : left;
      return true;
    }
    const int j = seq - mine;
    int k;
    if (!BACKWARD) k = seq * pairs + pair;
    else if (pair < extra) k = skip * (pairs - extra) + j * pairs + pair;
    else if (j < skip) k = j * (pairs - extra) + pair - extra;
    else k = skip * (pairs - extra) + (j - skip) * pairs + pair;
    if (k >= n_short) return false;
    const int group = by_group.of(k);
    k -= group * (int)by_group.d;
    const int n = group < last_group ? k / kGroupM : by_last.of(k);
    t.cls = CLS_LOGITS;
    t.m0 = (group * kGroupM + k - n * (group < last_group ? kGroupM : (int)by_last.d)) * kTile;
    t.n0 = n * kTile;
    t.bn = kTile;
    t.per_plane = t.count = k_logits;
    return true;
  }
};

struct Layout {
  int64_t t_pad, n_tiles, piece, n_pieces, n_buf, g_rows, split_dh, split_dw;      // g_rows: of one buffer of g
  bool direct;                   // forward over at most a tile of tokens: they are not compacted
  int64_t token, target, compact, lse, dloss, part, part_sum, z_target, g, dh_acc, dw_acc, walks, bytes;      // byte offsets
};

// A piece of the vocabulary: as many columns as make g of one piece and plane about 64 M elements (128 MB: what the two
// gradient products read is then mostly still in L2), of even sizes, and at least 2048 (the sum of dh goes through
// memory once per piece).
constexpr int64_t kPlanPairs = 74;       // what the scratch is planned for (148 SMs)
constexpr int64_t kPieceElems = (int64_t)64 << 20, kPieceMin = 2048;

inline int plan(const adapm_head_loss& d, bool backward, Layout& l) {
  if (d.tokens < 0 || d.vocab <= 0 || d.hidden <= 0) return ADAPM_EINVAL;
  if (d.tokens > (1 << 24) || d.vocab > (1 << 24) || d.hidden > (1 << 16)) return ADAPM_ERANGE;
  if (d.hidden % 8) return ADAPM_EUNSUPPORTED;
  if (d.hidden_ld < d.hidden || d.weight_ld < d.hidden) return ADAPM_EINVAL;
  if (d.hidden_ld % 8 || d.weight_ld % 8) return ADAPM_EALIGN;
  if (d.hidden_ld >= ((int64_t)1 << 32) || d.weight_ld >= ((int64_t)1 << 32)) return ADAPM_ERANGE;      // (sizes in bytes fit 64 bits, pitches a tensor map's 40)
  if (!(d.label_smoothing >= 0.f && d.label_smoothing <= 1.f) || !(d.z_loss >= 0.f) || !std::isfinite(d.z_loss)) return ADAPM_ERANGE;
  if (backward && (!known_type(d.dhidden_dtype) || !known_type(d.dweight_dtype))) return ADAPM_EINVAL;
  l.t_pad = round_up(d.tokens < 1 ? 1 : d.tokens, kTile);
  l.n_tiles = (d.vocab + kTile - 1) / kTile;
  const bool f32_dh = d.dhidden_dtype == ADAPM_TYPE_F32, f32_dw = d.dweight_dtype == ADAPM_TYPE_F32;
  l.g_rows = f32_dh || f32_dw ? 3 * l.t_pad : l.t_pad;      // (two planes of few tokens lie in the rows of one tile)
  const int64_t most = std::max(kPieceMin, kPieceElems / l.t_pad / kTile * kTile);
  l.n_pieces = (d.vocab + most - 1) / most;
  l.piece = round_up((d.vocab + l.n_pieces - 1) / l.n_pieces, kTile);
  l.n_pieces = (d.vocab + l.piece - 1) / l.piece;
  l.n_buf = l.n_pieces > 1 ? 2 : 1;
  if (l.t_pad / kTile * l.n_tiles > (1 << 30) || l.n_buf * l.g_rows >= ((int64_t)1 << 31)) return ADAPM_ERANGE;
  // A gradient's K is cut into parts where an item of it would take more than half of what all items take divided over the
  // pairs: few tokens leave dh a handful of tiles with the whole vocabulary as their K, a small vocabulary does the same to dw.
  // A part is at least 16 stages (5 us), because the parts cost a launch and their way through memory.  512 tokens of 4096 x 256
  // in fp32, both gradients: 78 us without; parts of at least 4 stages 56, of 16 44.
  l.split_dh = l.split_dw = 1;
  if (backward) {
    const int64_t mt = l.t_pad / kTile, nt_d = (d.hidden + kTile - 1) / kTile, tiles = l.piece / kTile;
    const int64_t k_dh = (std::min(l.piece, d.vocab) + kStageK - 1) / kStageK * (f32_dh ? 3 : 1);
    const int64_t k_dw = l.t_pad / kStageK * planes_of(f32_dw, (int)d.tokens);
    const int64_t logits = l.n_pieces > 1 ? mt * tiles * ((d.hidden + kStageK - 1) / kStageK) : 0;
    const int64_t share = std::max<int64_t>(1, (nt_d * (mt * k_dh + tiles * k_dw) + logits) / kPlanPairs);
    auto parts = [&](int64_t k) { return std::max<int64_t>(1, std::min({(2 * k + share - 1) / share, k / 16, (int64_t)256})); };
    l.split_dh = parts(k_dh);
    if (l.n_pieces == 1) l.split_dw = parts(k_dw);
  }
  int64_t at = kHeadBytes;
  auto take = [&](int64_t bytes) { const int64_t o = at; at += round_up(bytes, 256); return o; };
  l.direct = !backward && d.tokens <= kTile;
  l.walks = take(l.direct ? 0 : (backward ? l.n_pieces + 1 : 1) * (int64_t)sizeof(Walk));
  l.token = take(l.t_pad * 4);
  l.target = take(l.t_pad * 4);
  l.compact = take(l.direct ? 0 : l.t_pad * d.hidden * 2);
  l.lse = l.dloss = l.part = l.part_sum = l.z_target = l.g = l.dh_acc = l.dw_acc = 0;
  if (backward) {
    l.lse = take(l.t_pad * 4);
    l.dloss = take(l.t_pad * 4);
    l.g = take(l.n_buf * l.g_rows * l.piece * 2);
    if (l.n_pieces > 1 || l.split_dh > 1) l.dh_acc = take(l.split_dh * l.t_pad * d.hidden * 4);
    else if (!f32_dh) l.dh_acc = take(2 * kFewTokens * d.hidden * 4);
    if (l.split_dw > 1) l.dw_acc = take(l.split_dw * d.vocab * d.hidden * 4);
  } else {
    l.part = take(2 * l.n_tiles * l.t_pad * 8);
    l.part_sum = take(d.label_smoothing != 0.f ? 2 * l.n_tiles * l.t_pad * 4 : 0);
    l.z_target = take(l.t_pad * 4);
  }
  l.bytes = at;
  return ADAPM_OK;
}

inline Plan plan_of(const adapm_head_loss& d, const Layout& l, bool backward, bool dh, bool dw, int pairs) {
  Plan p;
  p.tokens = (int32_t)d.tokens; p.vocab = (int32_t)d.vocab; p.hidden = (int32_t)d.hidden;
  p.piece = (int32_t)(backward ? l.piece : d.vocab); p.n_pieces = (int32_t)(backward ? l.n_pieces : 1);
  p.f32_dh = d.dhidden_dtype == ADAPM_TYPE_F32; p.f32_dw = d.dweight_dtype == ADAPM_TYPE_F32;
  p.split_dh = (int32_t)l.split_dh; p.split_dw = (int32_t)l.split_dw;
  p.dh = dh; p.dw = dw; p.backward = backward; p.pairs = pairs;
  return p;
}

}  // namespace head
}  // namespace adapm
