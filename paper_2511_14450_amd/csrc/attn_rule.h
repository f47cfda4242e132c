// What the host makes of a rule of hyp_attn.h.
#pragma once

#include <algorithm>
#include <cmath>
#include <limits>

#include "abi_guard.h"
#include "attn_score.h"
#include "hyp_attn.h"

namespace hyp {
namespace {

inline void check_rule(const hyp_attn_rule_t *r) {
  need(r, HYP_EINVAL, "rule is null");
  need(std::isfinite(r->scale) && r->scale > 0.f, HYP_EINVAL, "rule: scale must be finite and positive");
  need(std::isfinite(r->cap) && r->cap >= 0.f, HYP_EINVAL, "rule: cap must be finite and not negative");
  need(r->cap > 0.f || std::isfinite(r->scale * kLog2e), HYP_EINVAL, "rule: scale must be below 2.3e38 where scores are not capped");
}

// Call: a struct with scale2, to_cap, cap2, cap_c, cap_most and slopes
template <typename Call> void add_rule(Call &p, const hyp_attn_rule_t &rule) {
  p.scale2 = rule.scale * kLog2e;
  if (rule.cap > 0.f) {
    p.to_cap = std::min(rule.scale / rule.cap, std::numeric_limits<float>::max());  // a score of 0 stays one under the smallest caps
    p.cap2 = rule.cap * kLog2e;
    // tanh(x) / x in powers of x^2 up to |x| = 0.4, of least relative error (9.8e-8); up to 0.5 the same error takes a power more, and an
    // instruction more of the thirteen that a score costs
    constexpr double tanh_c[4] = {0.9999999019048974, -0.3333136247072489, 0.13270976813015187, -0.04755360235665809};
    const double k = (double)rule.scale / rule.cap;
    double f = (double)rule.scale * kLog2e;
    for (int i = 0; i < 4; ++i, f *= k * k) p.cap_c[i] = (float)(f * tanh_c[i]);
    p.cap_most = (float)(0.4 / k);
    if (!std::isfinite(p.cap_c[3])) p.cap_most = -1.f;  // a cap so far below the scale that tanh is 0 or 1
  }
  p.slopes = rule.slopes;
}

}  // namespace
}  // namespace hyp
