// Norms at the border of two sublayers, with gate and residual scale (mixaq_residual_norm_forward):
//   x' = x + scale * gate o norm_post(y),   h = norm_pre(x')
// One pass: a row of x and y is read once into registers, x' and h are written; every statistic is a sum over the registers of the
// row's threads, in two passes (mean, then squared deviations), in binary32.  Bound by memory.
#include "residual_norm.cuh"

namespace mixaq {
namespace {

template <int TPR> __host__ __device__ constexpr int cta_threads() { return TPR < 128 ? 128 : TPR; }

struct Vectors { bool x, y, gate, x_out, h, params; };      // rows that are read and written 16 bytes at a time

template <class TX, class TY, int TPR, int VPT>
__global__ void __launch_bounds__(cta_threads<TPR>()) k_residual_norm(const ResNormArgs p, const Vectors vec) {
  __shared__ float2 slots[2][TPR / 32];
  RowReduce<TPR> reduce{slots};
  const int l = threadIdx.x % TPR, C = p.dim;
  const long row = (long)blockIdx.x * (cta_threads<TPR>() / TPR) + threadIdx.x / TPR;
  if (TPR < 128 && row >= p.rows) return;                   // (whole warps)
  griddep_wait();
  griddep_launch();
  const float inv_dim = __fdiv_rn(1.0f, (float)C);
  const bool has_y = p.y != nullptr;

  Vec8<TX> rx[VPT]; Vec8<TY> ry[VPT];
  int n[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + l) * 8;
    n[i] = min(max(C - c, 0), 8);
    if (n[i] > 0) load_row8(static_cast<const TX*>(p.x) + row * p.x_stride + c, vec.x, n[i], rx[i]);
    else load_row8(static_cast<const TX*>(nullptr), false, 0, rx[i]);
    if (has_y && n[i] > 0) load_row8(static_cast<const TY*>(p.y) + row * p.y_stride + c, vec.y, n[i], ry[i]);
    else load_row8(static_cast<const TY*>(nullptr), false, 0, ry[i]);
  }
  float x[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) unpack8(rx[i], x[i]);

  // v[i][j] -> its deviation from the row's mean (LAYER); returns the reciprocal of the standard deviation
  auto normalise = [&](float (&v)[VPT][8], const NormSpec& s) -> float {
    float mean = 0.0f;
    if (s.kind == NORM_LAYER) {
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) t = __fadd_rn(t, v[i][j]);
      mean = __fmul_rn(reduce.sum(t, 0.0f).x, inv_dim);
    }
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = j < n[i] ? __fsub_rn(v[i][j], mean) : 0.0f;
        sq = __fmaf_rn(v[i][j], v[i][j], sq);
      }
    return reciprocal_deviation(reduce.sum(sq, 0.0f).x, inv_dim, s.eps);
  };
  auto scaled = [&](float v, float rstd, float gamma, float beta) { return __fmaf_rn(__fmul_rn(v, rstd), gamma, beta); };

  if (has_y) {
    float y[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) unpack8(ry[i], y[i]);
    const float rstd = p.post.kind != NORM_NONE ? normalise(y, p.post) : 1.0f;
    const long gate_row = p.gate ? row / p.rows_per_gate : 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + l) * 8;
      float g[8];
      load_gate8<TY>(p, gate_row, c, n[i], vec.gate, g);
      if (p.post.kind != NORM_NONE) {
        float gamma[8], beta[8];
        load_params8(p.post.gamma, 1.0f, c, n[i], vec.params, gamma);
        load_params8(p.post.beta, 0.0f, c, n[i], vec.params, beta);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[i][j] = scaled(y[i][j], rstd, gamma[j], beta[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)                           // rounded to the stream's type: what the pre norm sees
        x[i][j] = j < n[i] ? to_f32(from_f32<TX>(__fmaf_rn(__fmul_rn(g[j], p.scale), y[i][j], x[i][j]))) : 0.0f;
      if (n[i] > 0) store8(static_cast<TX*>(p.x_out) + row * p.x_out_stride + c, x[i], vec.x_out && n[i] == 8, n[i]);
    }
  }
  if (p.pre.kind == NORM_NONE) return;
  const float rstd = normalise(x, p.pre);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + l) * 8;
    float gamma[8], beta[8];
    load_params8(p.pre.gamma, 1.0f, c, n[i], vec.params, gamma);
    load_params8(p.pre.beta, 0.0f, c, n[i], vec.params, beta);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] = j < n[i] ? scaled(x[i][j], rstd, gamma[j], beta[j]) : 0.0f;
    if (!p.codes) {
      if (n[i] > 0) store8(static_cast<TY*>(p.h) + row * p.h_stride + c, x[i], vec.h && n[i] == 8, n[i]);
    } else {
      // sixteen neighbouring lanes hold a block of 128 columns
      float m = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max_abs(m, x[i][j]);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
      float s, inv;
      block_scale(m, p.pow2, s, inv);
      if (n[i] > 0) store_codes(p.codes + row * p.code_stride + c, codes8(x[i], inv), n[i]);
      if (n[i] > 0 && l % 16 == 0) p.h_scale[row * p.srs + (long)(c / FP8_BLOCK) * p.scs] = s;
    }
  }
}

template <class TX, class TY, int TPR, int VPT>
void launch_as(const ResNormArgs& a, const Vectors& vec, cudaStream_t st) {
  constexpr int per = cta_threads<TPR>() / TPR;
  launch_pdl(k_residual_norm<TX, TY, TPR, VPT>, dim3((unsigned)((a.rows + per - 1) / per)), cta_threads<TPR>(), 0, st, a, vec);
  ++g_launches;
}

}  // namespace

void launch_residual_norm(const ResNormArgs& a, cudaStream_t st) {
  with_types(a.x_dtype, a.y_dtype, [&](auto tx, auto ty) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    Vectors v;
    v.x = rows_aligned(a.x, a.x_stride, sizeof(TX)); v.y = rows_aligned(a.y, a.y_stride, sizeof(TY));
    v.gate = rows_aligned(a.gate, a.gate_stride, a.gate_f32 ? 4 : sizeof(TY));
    v.x_out = rows_aligned(a.x_out, a.x_out_stride, sizeof(TX)); v.h = rows_aligned(a.h, a.h_stride, sizeof(TY));
    v.params = true;
    for (const float* q : {a.post.gamma, a.post.beta, a.pre.gamma, a.pre.beta}) v.params &= rows_aligned(q, 0, 4);
    // the fewest threads that hold a row at 8 to 32 elements each
    if (a.dim <= 256) launch_as<TX, TY, 32, 1>(a, v, st);
    else if (a.dim <= 1024) launch_as<TX, TY, 32, 4>(a, v, st);
    else if (a.dim <= 2048) launch_as<TX, TY, 128, 2>(a, v, st);
    else if (a.dim <= 4096) launch_as<TX, TY, 256, 2>(a, v, st);
    else if (a.dim <= 8192) launch_as<TX, TY, 512, 2>(a, v, st);
    else launch_as<TX, TY, 1024, 2>(a, v, st);
  });
}

}  // namespace mixaq
