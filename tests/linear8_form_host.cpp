// Which form a product of a linear layer in 8 bits takes (linear8_plan.h), for a host test.
#include "linear8_plan.h"

namespace adapm {
void set_error_text(const char*) {}
}  // namespace adapm

using namespace adapm;
using namespace adapm::linear8;

// "lines", "strips", "folded strips", "pairs", "pairs, K cut" or "pairs, long sums"; null: refused.
extern "C" const char* linear8_form(const adapm_linear8* d, int which) {
  if (check_desc(*d, which) != ADAPM_OK) return nullptr;
  const Form f = form_of(*d, which);
  if (f.form == LINES) return "lines";
  if (f.form == STRIPS) return f.strip.fold ? "folded strips" : "strips";
  if (f.plan.parts > 1) return "pairs, K cut";
  return f.plan.each > kShortStages ? "pairs, long sums" : "pairs";
}
