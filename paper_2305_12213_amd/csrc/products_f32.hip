// Dense and gated products in fp32 and all their gradients.
#include "product_epilogues.h"

namespace dynb {

template <> int launch_linear<float>(const Product& p, Tiles tiles, bool turned, const LinearOut<float>& ep, void* stream) {
  return turned ? launch_as<float, ROWS_NT, false>(p, tiles, Segs{}, ep, stream)
                : launch_as<float, ROWS_NN, false>(p, tiles, Segs{}, ep, stream);
}
template <> int launch_gated<float>(const Product& p, Tiles tiles, const GatedOut<float>& ep, void* stream) {
  return launch_as<float, ROWS_NN, true>(p, tiles, Segs{}, ep, stream);
}
template <> int launch_gated_grad<float>(const Product& p, Tiles tiles, const GatedGrad<float>& ep, void* stream) {
  return launch_as<float, ROWS_NT, false>(p, tiles, Segs{}, ep, stream);
}
template <> int launch_weights<float, float>(const Product& p, Tiles tiles, const Segs& s, const WeightOut<float>& ep, void* stream) {
  return launch_as<float, WEIGHTS, false>(p, tiles, s, ep, stream);
}

}  // namespace dynb
