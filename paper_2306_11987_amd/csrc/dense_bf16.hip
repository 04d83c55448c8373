// The dense products in bf16 (see dense_kernel.h).
#include "dense_kernel.h"

namespace hqlss {

hipError_t run_dense_bf16(hipStream_t s, const DenseArgs& g, int tile, int splits) { return run_dense<kBF16>(s, g, tile, splits); }
hipError_t run_pair_bf16(hipStream_t s, const DenseArgs& dx, int sx, const DenseArgs& dw, int sw, int tile, int cus) { return run_pair<kBF16>(s, dx, sx, dw, sw, tile, cus); }

}  // namespace hqlss
