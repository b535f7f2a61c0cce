// The norms at a sublayer's border, instances of one pair of types.
#include "residual_norm_bwd.cuh"
#include "residual_norm_fwd.cuh"

namespace mixaq {
template void residual_norm_typed<__nv_bfloat16, __nv_bfloat16>(const ResNormArgs&, int*, cudaStream_t);
template void residual_norm_bwd_typed<__nv_bfloat16, __nv_bfloat16>(BwdParams, cudaStream_t);
}  // namespace mixaq
