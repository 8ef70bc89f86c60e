// The matrix products of the gated feed-forward block, binary32.
#include "gated_product.h"

namespace bsr {

int launch_product_f32(const Plan &p, const ProductArgs &a, bool gated, bool loose, hipStream_t s) {
  return gated ? run_product<float, true>(p, a, loose, s) : run_product<float, false>(p, a, loose, s);
}

}  // namespace bsr
