// Dense products in bf16 and the gradients of their rows.
#include "product_epilogues.h"

namespace dynb {

template <> int launch_linear<bf16>(const Product& p, Tiles tiles, bool turned, const LinearOut<bf16>& ep, Target to) {
  return turned ? launch_as<bf16, ROWS_NT, false>(p, tiles, Segs{}, ep, to)
                : launch_as<bf16, ROWS_NN, false>(p, tiles, Segs{}, ep, to);
}

}  // namespace dynb
