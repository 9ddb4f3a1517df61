// Attention of a sequence's new tokens over its cached positions and over each other under a rule: causal by blocks, windows, a
// prefix that all see, documents, capped scores, a bias by distance.  What a row sees is at most two ranges of cache positions
// (row_ranges), so that a group of rows walks only the key tiles in which it sees anything, and looks at single keys only in
// those that not all of them see whole.
#include "attend_kernel.hpp"

namespace dinfer {

template <class Rule, int HD> static void launch_ruled_t(bool bf16, const AttendArgs& a, hipStream_t st) {
  if (!bf16) launch_attend_t<float, HD, 1, 1, true, Rule>(a, st);
  else if (most_rows(a.tok.span, a.group) <= TILE) launch_attend_t<bf16_t, HD, 1, 1, true, Rule>(a, st);
  else launch_attend_t<bf16_t, HD, 1, 2, true, Rule>(a, st);
}
template <class Rule> static void launch_ruled_hd(bool bf16, const AttendArgs& a, hipStream_t st) {
  if (a.geom.head_dim == 128) launch_ruled_t<Rule, 128>(bf16, a, st);
  else launch_ruled_t<Rule, 64>(bf16, a, st);
}
void launch_ruled(bool bf16, const AttendArgs& a, hipStream_t st) {
  const bool cap = a.rule.cap > 0.f, bias = a.rule.slope != nullptr;
  if (cap && bias) launch_ruled_hd<RangeRule<true, true>>(bf16, a, st);
  else if (cap) launch_ruled_hd<RangeRule<true, false>>(bf16, a, st);
  else if (bias) launch_ruled_hd<RangeRule<false, true>>(bf16, a, st);
  else launch_ruled_hd<RangeRule<false, false>>(bf16, a, st);
}

template <class Rule, int HD> static bool configure_ruled_t() {
  return configure_attend_t<bf16_t, HD, 1, Rule>() && configure_attend_t<bf16_t, HD, 2, Rule>() && configure_attend_t<float, HD, 1, Rule>();
}
template <class Rule> static bool configure_ruled_hd() { return configure_ruled_t<Rule, 64>() && configure_ruled_t<Rule, 128>(); }
bool configure_ruled() {
  const bool ok = configure_ruled_hd<RangeRule<false, false>>() && configure_ruled_hd<RangeRule<true, false>>() &&
                  configure_ruled_hd<RangeRule<false, true>>() && configure_ruled_hd<RangeRule<true, true>>();
  (void)hipGetLastError();
  return ok;
}

}  // namespace dinfer
