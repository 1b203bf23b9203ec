// The tiled product of operands along k, with bias, activation and residual:
// x W^T of a dense layer.
#include "product_tile.h"

namespace profk {

bool launch_product_along(ProdArgs g, const ProdPlan& p, float* sums, uint32_t cus, hipStream_t s) {
  if (!granules(g.a, g.as, g.K, g.a_padded) || !granules(g.b, g.bs, g.K, g.b_padded) || !tiles_fit(g)) return false;
  with_act(g.act, [&](auto act) {
    if (g.out_dtype == PROFK_F32) launch_planned<false, false, decltype(act)::value, PROFK_F32, false>(g, p, sums, cus, s);
    else launch_planned<false, false, decltype(act)::value, PROFK_BF16, false>(g, p, sums, cus, s);
  });
  return true;
}

}  // namespace profk
