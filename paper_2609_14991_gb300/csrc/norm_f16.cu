// tsd_residual_norm's kernels by type of the residual stream and of the block's output.
#include "norm.cuh"

namespace tsd {

template cudaError_t norm_launch<TSD_F16, TSD_F16>(const NormArgs&, NormHow, int, cudaStream_t);

}  // namespace tsd
