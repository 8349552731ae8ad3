// The dense layers' products of f32 matrices: dense_product.h.
#include <algorithm>
#include <type_traits>

#include "dense_product.h"

namespace lutnn {

hipError_t launch_product_f32(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s) {
    return product::launch_tile<float>(tile, a_k, b_k, a, s);
}

hipError_t launch_pair_f32(int tile, const PairArgs& p, hipStream_t s) { return product::launch_tiles<float>(tile, p, s); }

}  // namespace lutnn
