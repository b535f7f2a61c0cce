// The forward call of the norms at a sublayer's border: choice of the types (kernel: residual_norm_fwd.cuh).
#include "residual_norm_fwd.cuh"

namespace mixaq {
extern template void residual_norm_typed<float, __nv_bfloat16>(const ResNormArgs&, int*, cudaStream_t);
extern template void residual_norm_typed<float, __half>(const ResNormArgs&, int*, cudaStream_t);
extern template void residual_norm_typed<__nv_bfloat16, __nv_bfloat16>(const ResNormArgs&, int*, cudaStream_t);
extern template void residual_norm_typed<__half, __half>(const ResNormArgs&, int*, cudaStream_t);

void launch_residual_norm(const ResNormArgs& a, int* status, cudaStream_t st) {
  with_types(a.x_dtype, a.y_dtype, [&](auto tx, auto ty) { residual_norm_typed<decltype(tx), decltype(ty)>(a, status, st); });
}

}  // namespace mixaq
