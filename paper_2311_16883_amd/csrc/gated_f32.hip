// The matrix products of the gated feed-forward block, binary32.
#include "gated_product.h"

namespace bsr {

int launch_product_f32(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s) {
  return gated ? run_product<float, true>(p, a, s) : run_product<float, false>(p, a, s);
}

}  // namespace bsr
