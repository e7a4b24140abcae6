// Gradients of weights from rows in bf16, in fp32 or bf16.
#include "product_epilogues.h"

namespace dynb {

template <> int launch_weights<bf16, float>(const Product& p, Tiles tiles, const Segs& s, const WeightOut<float>& ep, Target to) {
  return launch_as<bf16, WEIGHTS, false>(p, tiles, s, ep, to);
}
template <> int launch_weights<bf16, bf16>(const Product& p, Tiles tiles, const Segs& s, const WeightOut<bf16>& ep, Target to) {
  return launch_as<bf16, WEIGHTS, false>(p, tiles, s, ep, to);
}

}  // namespace dynb
