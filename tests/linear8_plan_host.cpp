// Walks through the items of a product of a linear layer in 8 bits on the host (linear8_plan.h) and says what is wrong with them: null,
// or a text.
#include <map>
#include <string>
#include <vector>

#include "linear8_plan.h"

namespace adapm {
void set_error_text(const char*) {}
}  // namespace adapm

using namespace adapm;
using namespace adapm::linear8;

static std::string wrong(const adapm_linear8& d, int which) {
  if (check_desc(d, which) != ADAPM_OK) return "refused";
  const Plan p = plan_of(d, which);
  const int64_t k = which == FORWARD ? d.in_features : which == INPUT_GRAD ? d.out_features : d.tokens;
  const int step = which == FORWARD ? 128 : 64;
  if ((int64_t)p.stages * step < k || (int64_t)(p.stages - 1) * step >= k) return "stages";
  if (p.parts > 1 && which == FORWARD) return "a forward product that is cut";
  const bool f32 = which == INPUT_GRAD ? d.dx_dtype == ADAPM_TYPE_F32 : d.dweight_dtype == ADAPM_TYPE_F32;
  const int64_t decoded = which == FORWARD ? 0 : (f32 ? 6 : 2) * k * p.cols, parts = p.parts > 1 ? 4ll * p.parts * p.rows * p.cols : 0;
  if (p.part_at % 256 || p.part_at < kHeadBytes + decoded || p.bytes < p.part_at + parts) return "scratch";
  std::map<std::pair<int, int>, std::vector<Cut>> tiles;
  Cut t;
  int n = 0;
  for (; p.item(n, t); ++n) {
    if (t.m0 < 0 || t.m0 >= p.rows || t.m0 % kTile || t.n0 < 0 || t.n0 >= p.cols || t.n0 % p.width) return "an item's tile";
    if (t.bn % 64 || t.bn < 64 || t.bn > p.width || p.width > kTile) return "an item's columns";
    if (t.n0 + t.bn < p.cols && t.bn != p.width) return "columns left out";
    if (t.count < 1 || t.part < 0 || t.part >= p.parts) return "an item's part";
    auto& of = tiles[{t.m0, t.n0}];
    const int at = of.empty() ? 0 : of.back().k0 + of.back().count;
    if (t.k0 != at || t.part != (int)of.size()) return "parts of K that do not follow one another";
    of.push_back(t);
  }
  if (n != p.items || p.item(n, t)) return "the number of items";
  if ((int64_t)tiles.size() != (int64_t)p.m_tiles * p.n_tiles || (int64_t)p.m_tiles * kTile < p.rows || (int64_t)p.n_tiles * p.width < p.cols) return "tiles left out";
  const StripPlan q = strip_plan_of(d, which);
  const int64_t features = which == FORWARD ? d.out_features : d.in_features, columns = which == WEIGHT_GRAD ? d.out_features : d.tokens;
  if (q.fold && (which == FORWARD || q.width > 64 || q.planes * q.width > 256)) return "folded scales";
  if (!q.fold && q.planes != 1) return "planes";
  if (which != FORWARD && !f32 && columns <= 16 && (!q.fold || !strips_are_faster(d, which, q, p))) return "few columns without 16 bits of a scale";
  if (q.width < 1 || q.width > 256 || q.width % (which == WEIGHT_GRAD ? 64 : 16)) return "a strip's width";
  if ((int64_t)q.c_tiles * q.width < columns || (int64_t)(q.c_tiles - 1) * q.width >= columns) return "strips' columns";
  if ((int64_t)q.f_tiles * 128 < features || (int64_t)(q.f_tiles - 1) * 128 >= features) return "strips' features";
  if ((int64_t)q.stages * step < k || (int64_t)(q.stages - 1) * step >= k) return "a strip's stages";
  if (q.split != 1 && q.split != 2 && q.split != 4 && q.split != 8) return "a cluster";
  if ((int64_t)q.ctas != (int64_t)q.c_tiles * q.f_tiles * q.split && q.ctas <= kMostWords) return "CTAs";
  if (q.first(0) != 0 || q.first(q.split) != q.stages) return "a strip's K";
  for (int i = 0; i < q.split; ++i)
    if (q.first(i + 1) <= q.first(i)) return "a part without a stage";
  if (q.stage_bytes != 16384 + 128 * q.width * q.planes || q.raw_bytes != (which == FORWARD ? 0 : 8192 + (q.fold ? 128 * q.width : 0))) return "bytes of a stage";
  const int64_t ring = (int64_t)q.ring * q.stage_bytes;
  if (q.ring < kStripTeams || q.ring > kStripRing || (which != FORWARD && (q.raw < kStripTeams || q.raw > kStripRing))) return "a ring";
  if (ring + (int64_t)q.raw * q.raw_bytes > kStripSmem || ring < 512 * q.width || kStripSmem + 1024 + 512 > 227 * 1024) return "shared memory";
  for (const auto& of : tiles)
    if (of.second.back().k0 + of.second.back().count != p.stages || (int)of.second.size() != p.parts) return "K";
  return "";
}

extern "C" const char* linear8_plan_wrong(const adapm_linear8* d, int which) {
  static std::string what;
  what = wrong(*d, which);
  return what.empty() ? nullptr : what.c_str();
}

extern "C" int linear8_parts(const adapm_linear8* d, int which) { return plan_of(*d, which).parts; }
