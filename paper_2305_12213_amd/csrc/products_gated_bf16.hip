// Gated products in bf16 and the gradients of their rows.
#include "product_epilogues.h"

namespace dynb {

template <> int launch_gated<bf16>(const Product& p, Tiles tiles, const GatedOut<bf16>& ep, Target to) {
  return launch_as<bf16, ROWS_NN, true>(p, tiles, Segs{}, ep, to);
}
template <> int launch_gated_grad<bf16>(const Product& p, Tiles tiles, const GatedGrad<bf16>& ep, Target to) {
  return launch_as<bf16, ROWS_NT, false>(p, tiles, Segs{}, ep, to);
}

}  // namespace dynb
