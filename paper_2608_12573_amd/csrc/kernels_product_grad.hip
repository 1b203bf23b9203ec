// The tiled product of operands across k: dz W and dz^T x of a dense layer's
// gradients, without a transposed copy of either.
#include "product_tile.h"

namespace profk {

namespace {

// dx and dW of a size whose tiles the CUs hold all at once, in one launch: the
// first `blocks` workgroups take dx's.
struct PairArgs {
  ProdArgs dx, dw;
  uint32_t ti1, tiles1, ti2, tiles2, blocks;
};
template <bool TWO> __global__ __launch_bounds__(256, 2) void k_prod_pair(PairArgs a) {
  using T = ProdTile<2, 2, 2, 2>;
  __shared__ __align__(16) uint4 s0[T::kGran], s1[T::kGran];
  if (blockIdx.x < a.blocks)
    prod_body<false, true, PROFK_ACT_NONE, PROFK_BF16, 2, 2, 2, 2, false, false, TWO>(a.dx, a.ti1, a.tiles1, blockIdx.x,
                                                                                     a.blocks, s0, s1);
  else
    prod_body<true, true, PROFK_ACT_NONE, PROFK_BF16, 2, 2, 2, 2, false, false, TWO>(
        a.dw, a.ti2, a.tiles2, blockIdx.x - a.blocks, gridDim.x - a.blocks, s0, s1);
}

uint32_t tiles_of(uint32_t n) { return (n + 127) / 128; }

bool grad_granules(const ProdArgs& g, bool a_across) {
  return granules(g.a, g.as, a_across ? g.I : g.K, g.a_padded) && granules(g.b, g.bs, g.J, g.b_padded) &&
         tiles_fit(g) && g.K > 0;
}

}  // namespace

bool launch_product_pair(const ProdArgs& dx, const ProdArgs& dw, hipStream_t s) {
  if (!grad_granules(dx, false) || !grad_granules(dw, true)) return false;
  const uint32_t t1 = tiles_of(dx.I) * tiles_of(dx.J), t2 = tiles_of(dw.I) * tiles_of(dw.J);
  const uint32_t b1 = prod_grid(t1, t1 + kProdXcds), b2 = prod_grid(t2, t2 + kProdXcds);
  const PairArgs a{dx, dw, tiles_of(dx.I), t1, tiles_of(dw.I), t2, b1};
  if (dx.a_low) k_prod_pair<true><<<b1 + b2, 256, 0, s>>>(a);
  else k_prod_pair<false><<<b1 + b2, 256, 0, s>>>(a);
  return true;
}

bool launch_product_grad(ProdArgs g, bool a_across, const ProdPlan& p, float* sums, uint32_t cus, hipStream_t s) {
  if (!grad_granules(g, a_across)) return false;
  const auto launch = [&](auto two) {
    constexpr bool kTwo = decltype(two)::value;
    if (a_across) launch_planned<true, true, PROFK_ACT_NONE, PROFK_BF16, kTwo>(g, p, sums, cus, s);
    else launch_planned<false, true, PROFK_ACT_NONE, PROFK_BF16, kTwo>(g, p, sums, cus, s);
  };
  if (g.a_low) launch(std::true_type{});
  else launch(std::false_type{});
  return true;
}

}  // namespace profk
