// The backward call of the norms at a sublayer's border: launch of the main kernel (residual_norm_bwd.cuh) and the adding up of its sums.
#include "residual_norm_bwd.cuh"

namespace mixaq {
extern template void residual_norm_bwd_typed<float, __nv_bfloat16>(BwdParams, cudaStream_t);
extern template void residual_norm_bwd_typed<float, __half>(BwdParams, cudaStream_t);
extern template void residual_norm_bwd_typed<__nv_bfloat16, __nv_bfloat16>(BwdParams, cudaStream_t);
extern template void residual_norm_bwd_typed<__half, __half>(BwdParams, cudaStream_t);

namespace {

// ---- adding up ------------------------------------------------------------------------------------------------------------
struct JoinParams { const float* sums; int ctas, dim; float* out[SUMS]; };
constexpr int JOIN_COLS = 32, JOIN_PARTS = 16;
// CTA (column group, sum): 16 threads a column take a stretch of the CTAs each, in order, then the stretches are added in order
__global__ void __launch_bounds__(JOIN_COLS * JOIN_PARTS) k_join_sums(const JoinParams p) {
  __shared__ float part[JOIN_PARTS][JOIN_COLS];
  griddep_wait();
  griddep_launch();
  const int s = blockIdx.y, col = blockIdx.x * JOIN_COLS + threadIdx.x % JOIN_COLS, k = threadIdx.x / JOIN_COLS;
  if (!p.out[s]) return;
  const int a = (int)((long)p.ctas * k / JOIN_PARTS), b = (int)((long)p.ctas * (k + 1) / JOIN_PARTS);
  float t = 0.0f;
  if (col < p.dim) {
#pragma unroll 8
    for (int i = a; i < b; ++i) t = __fadd_rn(t, __ldg(p.sums + ((long)i * SUMS + s) * p.dim + col));
  }
  part[k][threadIdx.x % JOIN_COLS] = t;
  __syncthreads();
  if (k == 0 && col < p.dim) {
    for (int i = 1; i < JOIN_PARTS; ++i) t = __fadd_rn(t, part[i][threadIdx.x]);
    p.out[s][col] = t;
  }
}

struct JoinGateParams { const float* parts; long rows, rows_per_gate, per_worker; int dim, col_groups; float* dgate; long stride; };
// sequences whose rows several workers share: their parts in the order of the workers
__global__ void __launch_bounds__(256) k_join_gates(const JoinGateParams p) {
  griddep_wait();
  griddep_launch();
  const long seq = blockIdx.x / (unsigned)p.col_groups;
  const int col = (int)(blockIdx.x - seq * p.col_groups) * 256 + threadIdx.x;
  const long s0 = seq * p.rows_per_gate, s1 = min(s0 + p.rows_per_gate, p.rows);
  const long w0 = s0 / p.per_worker, w1 = (s1 - 1) / p.per_worker;
  if (w0 == w1 || col >= p.dim) return;
  float t = 0.0f;
  for (long w = w0; w <= w1; ++w) t = __fadd_rn(t, __ldg(p.parts + (w * 2 + (s0 > w * p.per_worker ? 1 : 0)) * p.dim + col));
  p.dgate[seq * p.stride + col] = t;
}

size_t sums_floats(const Shape& s, int dim) { return ((size_t)s.ctas * SUMS * dim + 63) / 64 * 64; }

}  // namespace

size_t residual_norm_backward_floats(long rows, int dim, bool gate_per_sequence) {
  if (rows <= 0) return 64;
  const Shape s = shape_for(rows, dim);
  return sums_floats(s, dim) + (gate_per_sequence ? (size_t)s.ctas * s.rows_per_cta * 2 * dim : 0);
}

void launch_residual_norm_backward(const ResNormArgs& a, const ResNormGradArgs& g, int* status, cudaStream_t st) {
  const Shape s = shape_for(a.rows, a.dim);
  BwdParams q;
  q.a = a; q.g = g; q.status = status;
  q.per_worker = s.per_worker;
  q.sums = g.workspace; q.gate_parts = g.workspace + sums_floats(s, a.dim);
  q.gate_mode = !a.gate || !g.dgate ? GATE_NONE : a.rows_per_gate >= a.rows ? GATE_CHANNEL : a.rows_per_gate == 1 ? GATE_TOKEN : GATE_SEQUENCE;
  with_types(a.x_dtype, a.y_dtype, [&](auto tx, auto ty) { residual_norm_bwd_typed<decltype(tx), decltype(ty)>(q, st); });
  JoinParams j;
  j.sums = q.sums; j.ctas = (int)s.ctas; j.dim = a.dim;
  bool any = false;
  for (int i = 0; i < 4; ++i) { j.out[i] = g.vec[i]; any |= g.vec[i] != nullptr; }
  j.out[SUM_GATE] = q.gate_mode == GATE_CHANNEL ? g.dgate : nullptr;
  if (any || j.out[SUM_GATE]) {
    launch_pdl(k_join_sums, dim3((a.dim + JOIN_COLS - 1) / JOIN_COLS, SUMS), JOIN_COLS * JOIN_PARTS, 0, st, j);
    ++g_launches;
  }
  if (q.gate_mode == GATE_SEQUENCE && s.per_worker > 0) {
    const int groups = (a.dim + 255) / 256;
    const long seqs = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate;
    JoinGateParams jg = {q.gate_parts, a.rows, a.rows_per_gate, s.per_worker, a.dim, groups, g.dgate, g.dgate_stride};
    launch_pdl(k_join_gates, dim3((unsigned)(seqs * groups)), 256, 0, st, jg);
    ++g_launches;
  }
}

}  // namespace mixaq
