// The dense products in fp32 (see dense_kernel.h).
#include "dense_kernel.h"

namespace hqlss {

hipError_t run_dense_f32(hipStream_t s, const DenseArgs& g, int tile, int splits) { return run_dense<kF32>(s, g, tile, splits); }

}  // namespace hqlss
