// Products over ragged ranges of rows: the kernels for f32.
#include "nmfmu_ragged_kernels.h"

namespace nmfmu {
namespace ragged {
template hipError_t launch_align<float>(const Align &, hipStream_t);
template hipError_t launch_product<float>(const Product &, hipStream_t);
template hipError_t launch_gradient<float>(const Gradient &, hipStream_t);
template hipError_t launch_factor_gradient<float>(const FactorGradient &, hipStream_t);
}  // namespace ragged
}  // namespace nmfmu
