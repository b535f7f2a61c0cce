// Internal interface of the row operators (row_ops.cu and their kernels): e4m3 codes with block scales, their product, norms at a sublayer's
// border.  In a header of its own: the record of the GEMM's DRAM traffic is that of kernels.h and the other sources its kernel is built from.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace mixaq {

enum DType { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };        // values of mixaq_dtype
struct Fp8QuantArgs {
  const void* x; int dtype; long rows, cols, row_stride;
  bool transpose, pow2; int block_rows;
  uint8_t* codes; long code_stride; float* scale; long scale_row_stride, scale_col_stride;
};
void launch_fp8_quantize(const Fp8QuantArgs& a, cudaStream_t st);

struct Fp8Operand { const uint8_t* codes; long rows, stride; int block_rows; const float* scale; long srs, scs; };
struct Fp8MatmulArgs {
  Fp8Operand a, w; long K;
  const float* bias; void* y; int y_dtype; long y_stride;
  int* status;
};
bool launch_fp8_matmul(const Fp8MatmulArgs& g, cudaStream_t st);        // false: set-up failed

struct NormSpec { int kind; const float *gamma, *beta; float eps; };          // kind: values of mixaq_norm_kind
struct ResNormArgs {
  long rows; int dim, x_dtype, y_dtype;
  const void* x; long x_stride; const void* y; long y_stride;                 // y nullable
  const void* gate; long gate_stride, rows_per_gate; bool gate_f32;           // nullable
  float scale;
  NormSpec post, pre;
  void* x_out; long x_out_stride; void* h; long h_stride;                     // h: of the sublayers' type, or
  uint8_t* codes; long code_stride; float* h_scale; long srs, scs; bool pow2;  // codes (h is null then)
};
struct ResNormGradArgs {
  const void* dx_out; long dx_out_stride; const void* dh; long dh_stride;     // nullable
  void* dx; long dx_stride; void* dy; long dy_stride;                         // nullable, as all that follows
  float* dgate; long dgate_stride;
  float* vec[4];                                                              // dpost_gamma, dpost_beta, dpre_gamma, dpre_beta
  float* workspace;
};
void launch_residual_norm(const ResNormArgs& a, int* status, cudaStream_t st);
size_t residual_norm_backward_floats(long rows, int dim, bool gate_per_sequence);   // of the workspace
void launch_residual_norm_backward(const ResNormArgs& a, const ResNormGradArgs& g, int* status, cudaStream_t st);

}  // namespace mixaq
