// The tiled product of operands across k: dz W and dz^T x of a dense layer's
// gradients, without a transposed copy of either.
#include "product_tile.h"

namespace profk {

bool launch_product_grad(ProdArgs g, bool a_across, const ProdPlan& p, float* sums, uint32_t cus, hipStream_t s) {
  if (!granules(g.a, g.as, a_across ? g.I : g.K, g.a_padded) || !granules(g.b, g.bs, g.J, g.b_padded) || !tiles_fit(g) ||
      g.K == 0)
    return false;
  if (a_across) launch_planned<true, true, PROFK_ACT_NONE, PROFK_BF16>(g, p, sums, cus, s);
  else launch_planned<false, true, PROFK_ACT_NONE, PROFK_BF16>(g, p, sums, cus, s);
  return true;
}

}  // namespace profk
