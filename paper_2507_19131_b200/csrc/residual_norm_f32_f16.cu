// The norms at a sublayer's border, instances of one pair of types.
#include "residual_norm_bwd.cuh"
#include "residual_norm_fwd.cuh"

namespace mixaq {
template void residual_norm_typed<float, __half>(const ResNormArgs&, int*, cudaStream_t);
template void residual_norm_bwd_typed<float, __half>(BwdParams, cudaStream_t);
}  // namespace mixaq
