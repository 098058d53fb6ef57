// Walks through the items of a call of the head loss on the host (head_plan.h), every pair of CTAs in turn, and says what is wrong
// with them: null, or a text.
#include <map>
#include <set>
#include <string>
#include <tuple>
#include <vector>

#include "head_plan.h"

namespace adapm {
void set_error_text(const char*) {}
}  // namespace adapm

using namespace adapm;
using namespace adapm::head;

static std::string wrong(const adapm_head_loss& d, bool backward, bool dh, bool dw, int tv, int pairs) {
  Layout l;
  if (plan(d, backward, l) != ADAPM_OK) return "refused";
  const Plan p = plan_of(d, l, backward, dh, dw, pairs);
  const int launches = backward ? p.n_pieces + 1 : 1, m = (tv + kTile - 1) / kTile;
  Walk first;
  if (backward) first.make(p, 1, tv);
  if (backward && (first.parts_dh < 1 || first.parts_dh > l.split_dh || first.parts_dw < 1 || first.parts_dw > l.split_dw)) return "more parts than the scratch holds";
  // what is written, and what the boxes of a tile's 256 rows reach
  if (backward && (first.plane_rows < tv || first.plane_rows % kStageK || (int64_t)first.planes * first.plane_rows > l.g_rows ||
                   (int64_t)(first.planes_dh - 1) * first.plane_rows + (m > 1 ? m : 1) * kTile > l.g_rows)) return "planes of g that the scratch does not hold";
  for (int i = 0; i < launches; ++i) {
    Walk w;
    w.make(p, i, tv);
    if (p.used(i) < 1 || p.used(i) != w.pairs) return "pairs of CTAs";
    const int cols = p.cols(i), before = backward ? p.cols(i - 1) : 0;
    std::set<std::tuple<int, int, int>> logits;
    std::map<std::tuple<int, int, int>, std::map<int, std::pair<int, int>>> tiles;      // of a gradient: its parts of K
    std::map<std::pair<int, int>, std::map<int, int>> widths;
    std::set<int> parts[2];
    for (int pair = 0; pair < w.pairs; ++pair) {
      HeadItem t;
      for (int seq = 0; backward ? w.item<true>(pair, seq, t) : w.item<false>(pair, seq, t); ++seq) {
        if (t.count < 1 || t.m0 % kTile || t.m0 < 0) return "an item's tile";
        if (t.cls == CLS_LOGITS) {
          if (t.m0 >= m * kTile || t.n0 >= cols || t.n0 % kTile || t.bn != kTile || t.k0 != 0 || t.count != (p.hidden + kStageK - 1) / kStageK) return "logits";
          if (!logits.insert({t.m0, t.n0, 0}).second) return "logits twice";
          continue;
        }
        if (t.bn < 32 || t.bn > kTile || t.bn % 32) return "columns of a gradient";
        if (t.m0 >= (t.cls == CLS_DH ? m * kTile : before)) return "rows of a gradient";
        if (!tiles[{t.cls, t.m0, t.n0}].insert({t.k0, {t.count, t.split}}).second) return "a part twice";
        widths[{t.cls, t.m0}][t.n0] = t.bn;
        parts[t.cls == CLS_DW].insert(t.split);
        if (t.split < 0 || t.split >= (t.cls == CLS_DH ? first.parts_dh : first.parts_dw)) return "a part that is not summed";
      }
    }
    if ((int64_t)logits.size() != (int64_t)m * ((cols + kTile - 1) / kTile)) return "logits left out";
    for (const auto& tile : tiles) {
      const bool is_dh = std::get<0>(tile.first) == CLS_DH;
      int at = 0, split = 0;
      for (const auto& part : tile.second) {
        if (part.first != at || part.second.second != split++) return "parts of K that do not follow one another";
        at += part.second.first;
      }
      const bool f32 = (is_dh ? d.dhidden_dtype : d.dweight_dtype) == ADAPM_TYPE_F32;
      // up to 64 tokens dhidden in bf16 takes two planes as rows of one tile, dweight along K
      const int planes = f32 ? 3 : !is_dh && tv <= 64 ? 2 : 1;
      if (planes > w.planes || (is_dh && w.stacked != (!f32 && tv <= 64)) || (w.stacked && (w.planes < 2 || m > 1))) return "planes of g";
      if (at != planes * (((is_dh ? before : tv > 0 ? tv : 1) + kStageK - 1) / kStageK)) return "K of a gradient";
      if (is_dh && i == 1 && split != first.parts_dh) return "parts of dhidden that the first piece does not write";
      if (!is_dh && split != first.parts_dw) return "parts of dweight";
    }
    for (const auto& row : widths) {
      int at = 0;
      for (const auto& c : row.second) {
        if (c.first != at) return "columns that do not follow one another";
        at += c.second;
      }
      if (at < p.hidden || at - p.hidden >= 32) return "columns of a gradient";
    }
    const int64_t rows = before ? (dh ? m : 0) + (dw ? (before + kTile - 1) / kTile : 0) : 0;
    if ((int64_t)widths.size() != rows) return "rows of a gradient left out";
  }
  return "";
}

extern "C" const char* head_walk_wrong(const adapm_head_loss* d, int backward, int dh, int dw, int tv, int pairs) {
  static std::string what;
  what = wrong(*d, backward != 0, dh != 0, dw != 0, tv, pairs);
  return what.empty() ? nullptr : what.c_str();
}

extern "C" int head_pieces(const adapm_head_loss* d) {
  Layout l;
  return plan(*d, true, l) == ADAPM_OK ? (int)l.n_pieces : 0;
}

extern "C" int head_quotient(int n, int d) {
  Divisor v;
  v.set(d);
  return v.of(n);
}
