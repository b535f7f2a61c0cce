// The row operators' kernel launchers of the stand-in: they keep the arguments of the last call and count its launch on its stream.
#include "../../paper_2507_19131_b200/csrc/kernels.h"
#include "fake.h"

extern "C" {
mixaq::Fp8QuantArgs last_quantize;
mixaq::Fp8MatmulArgs last_matmul;
mixaq::ResNormArgs last_norm;
mixaq::ResNormGradArgs last_grads;
int fail_matmul;                                          // the launch's set-up fails while this is set
}

namespace mixaq {
void launch_fp8_quantize(const Fp8QuantArgs& a, cudaStream_t st) { last_quantize = a; ++g_launches; enqueue(st); }
bool launch_fp8_matmul(const Fp8MatmulArgs& g, cudaStream_t st) {
  if (fail_matmul) return false;
  last_matmul = g; ++g_launches; enqueue(st);
  return true;
}
void launch_residual_norm(const ResNormArgs& a, int*, cudaStream_t st) { last_norm = a; ++g_launches; enqueue(st); }
size_t residual_norm_backward_floats(long rows, int dim, bool per_sequence) { return (size_t)(rows > 0 ? 5 * dim : 64) * (per_sequence ? 2 : 1); }
void launch_residual_norm_backward(const ResNormArgs& a, const ResNormGradArgs& g, int*, cudaStream_t st) { last_norm = a; last_grads = g; ++g_launches; enqueue(st); }
}  // namespace mixaq
