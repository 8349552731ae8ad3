// The dense layers' products of bf16 matrices: dense_product.h.
#include <algorithm>
#include <type_traits>

#include "dense_product.h"

namespace lutnn {

hipError_t launch_product_bf16(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s) {
    return product::launch_tile<bf16>(tile, a_k, b_k, a, s);
}

hipError_t launch_pair_bf16(int tile, const PairArgs& p, hipStream_t s) { return product::launch_tiles<bf16>(tile, p, s); }

}  // namespace lutnn
