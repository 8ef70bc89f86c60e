// The matrix products of the gated feed-forward block, bfloat16.
#include "gated_product.h"

namespace bsr {

int launch_product_bf16(const Plan &p, const ProductArgs &a, bool gated, hipStream_t s) {
  return gated ? run_product<uint16_t, true>(p, a, s) : run_product<uint16_t, false>(p, a, s);
}

}  // namespace bsr
