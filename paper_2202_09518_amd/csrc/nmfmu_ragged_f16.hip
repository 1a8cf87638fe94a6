// Products over ragged ranges of rows: the kernels for f16.
#include "nmfmu_ragged_kernels.h"

namespace nmfmu {
namespace ragged {
template hipError_t launch_align<f16_t>(const Align &, hipStream_t);
template hipError_t launch_product<f16_t>(const Product &, hipStream_t);
template hipError_t launch_gradient<f16_t>(const Gradient &, hipStream_t);
template hipError_t launch_factor_gradient<f16_t>(const FactorGradient &, hipStream_t);
}  // namespace ragged
}  // namespace nmfmu
