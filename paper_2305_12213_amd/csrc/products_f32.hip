// Dense and gated products in fp32 and all their gradients.
#include "product_epilogues.h"

namespace dynb {

template <> int launch_linear<float>(const Product& p, Tiles tiles, bool turned, const LinearOut<float>& ep, Target to) {
  return turned ? launch_as<float, ROWS_NT, false>(p, tiles, Segs{}, ep, to)
                : launch_as<float, ROWS_NN, false>(p, tiles, Segs{}, ep, to);
}
template <> int launch_gated<float>(const Product& p, Tiles tiles, const GatedOut<float>& ep, Target to) {
  return launch_as<float, ROWS_NN, true>(p, tiles, Segs{}, ep, to);
}
template <> int launch_gated_grad<float>(const Product& p, Tiles tiles, const GatedGrad<float>& ep, Target to) {
  return launch_as<float, ROWS_NT, false>(p, tiles, Segs{}, ep, to);
}
template <> int launch_weights<float, float>(const Product& p, Tiles tiles, const Segs& s, const WeightOut<float>& ep, Target to) {
  return launch_as<float, WEIGHTS, false>(p, tiles, s, ep, to);
}

}  // namespace dynb
