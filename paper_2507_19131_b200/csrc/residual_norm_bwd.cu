// Gradients of the norms at a sublayer's border (mixaq_residual_norm_backward).  With d = dh o gamma_pre, xn the normalised x':
//   dx = dx_out + (d - xn mean(d o xn) [- mean(d)]) / dev(x'),   u = scale * dx,   dgate = sum u o r,   w = u o gate,
//   e = w o gamma_post,   dy = (e - yn mean(e o yn) [- mean(e)]) / dev(y)           (the bracketed means: LayerNorm only)
// and the parameters' gradients are column sums of dh o xn, dh, w o yn, w.
//
// The statistics are computed anew from x' and y, which the gradients need anyway: nothing has to be kept from the forward call.  A row
// is read once into registers; the next row's loads are in flight while a row goes through its four reductions.  Column sums stay in
// registers over the consecutive rows of a worker (a CTA, or a warp for narrow rows), are written out once per CTA and added by a
// second kernel in the order of the CTAs: no atomics, so the result depends on the sizes and the number of SMs only.
#include "residual_norm.cuh"

namespace mixaq {
namespace {

enum { SUM_POST_GAMMA = 0, SUM_POST_BETA, SUM_PRE_GAMMA, SUM_PRE_BETA, SUM_GATE, SUMS };

template <int TPR> __host__ __device__ constexpr int cta_threads() { return TPR < 128 && TPR != 64 ? 128 : TPR; }
// workers (rows at a time) of a CTA
template <int TPR> __host__ __device__ constexpr int cta_rows() { return cta_threads<TPR>() / TPR; }
// resident CTAs per SM that the registers are divided for: 512 threads at 128 registers
template <int TPR> __host__ __device__ constexpr int ctas_per_sm() { return cta_threads<TPR>() >= 512 ? 1 : 512 / cta_threads<TPR>(); }

enum GateMode { GATE_NONE = 0, GATE_CHANNEL, GATE_SEQUENCE, GATE_TOKEN };
struct BwdParams {
  ResNormArgs a; ResNormGradArgs g;
  bool vx, vy, vgate, vdxo, vdh, vdx, vdy, vparams;
  int gate_mode;               // how dgate is summed (GATE_NONE: it is not wanted)
  long per_worker;             // consecutive rows of a worker
  float* sums;                 // [CTA][SUMS][dim]
  float* gate_parts;           // [worker][2][dim]: sums of the first and the last sequence that a worker shares with others
};

template <class TX, class TY, int TPR, int VPT>
__global__ void __launch_bounds__(cta_threads<TPR>(), ctas_per_sm<TPR>()) k_residual_norm_bwd(const BwdParams q) {
  __shared__ float2 slots[2][TPR / 32];
  RowReduce<TPR> reduce{slots};
  const ResNormArgs& p = q.a;
  const ResNormGradArgs& g = q.g;
  const int l = threadIdx.x % TPR, C = p.dim;
  const long worker = (long)blockIdx.x * cta_rows<TPR>() + threadIdx.x / TPR;
  const long first = worker * q.per_worker, end = min(first + q.per_worker, p.rows);
  const float inv_dim = __fdiv_rn(1.0f, (float)C);
  const bool has_y = p.y != nullptr, has_pre = p.pre.kind != NORM_NONE && g.dh != nullptr, has_post = p.post.kind != NORM_NONE;
  griddep_wait();
  griddep_launch();

  int n[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) n[i] = min(max(C - (i * TPR + l) * 8, 0), 8);
  float sums[SUMS][VPT][8];
#pragma unroll
  for (int s = 0; s < SUMS; ++s)
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[s][i][j] = 0.0f;

  struct Raw { Vec8<TX> x[VPT], dxo[VPT]; Vec8<TY> y[VPT], dh[VPT]; } raw;
  auto fetch = [&](long row) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + l) * 8;
      if (has_pre && n[i] > 0) load_row8(static_cast<const TX*>(p.x) + row * p.x_stride + c, q.vx, n[i], raw.x[i]);
      else load_row8(static_cast<const TX*>(nullptr), false, 0, raw.x[i]);
      if (has_y && n[i] > 0) load_row8(static_cast<const TY*>(p.y) + row * p.y_stride + c, q.vy, n[i], raw.y[i]);
      else load_row8(static_cast<const TY*>(nullptr), false, 0, raw.y[i]);
      if (g.dx_out && n[i] > 0) load_row8(static_cast<const TX*>(g.dx_out) + row * g.dx_out_stride + c, q.vdxo, n[i], raw.dxo[i]);
      else load_row8(static_cast<const TX*>(nullptr), false, 0, raw.dxo[i]);
      if (has_pre && n[i] > 0) load_row8(static_cast<const TY*>(g.dh) + row * g.dh_stride + c, q.vdh, n[i], raw.dh[i]);
      else load_row8(static_cast<const TY*>(nullptr), false, 0, raw.dh[i]);
    }
  };
  // the sequence that a row belongs to and the rows until its end
  long seq = 0, left = 0;
  if (p.gate && first < end) { seq = first / p.rows_per_gate; left = (seq + 1) * p.rows_per_gate - first; }

  if (first < end) fetch(first);
  for (long row = first; row < end; ++row) {
    float x[VPT][8], y[VPT][8], dx[VPT][8], dh[VPT][8];
    float sx = 0.0f, sy = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      unpack8(raw.x[i], x[i]); unpack8(raw.y[i], y[i]); unpack8(raw.dxo[i], dx[i]); unpack8(raw.dh[i], dh[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) { sx = __fadd_rn(sx, x[i][j]); sy = __fadd_rn(sy, y[i][j]); }
    }
    if (row + 1 < end) fetch(row + 1);
    float mx = 0.0f, my = 0.0f;
    if (p.pre.kind == NORM_LAYER || p.post.kind == NORM_LAYER) {
      const float2 t = reduce.sum(sx, sy);
      if (p.pre.kind == NORM_LAYER) mx = __fmul_rn(t.x, inv_dim);
      if (p.post.kind == NORM_LAYER) my = __fmul_rn(t.y, inv_dim);
    }
    float qx = 0.0f, qy = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i][j] = j < n[i] ? __fsub_rn(x[i][j], mx) : 0.0f;
        y[i][j] = j < n[i] ? __fsub_rn(y[i][j], my) : 0.0f;
        qx = __fmaf_rn(x[i][j], x[i][j], qx);
        qy = __fmaf_rn(y[i][j], y[i][j], qy);
      }
    float rx = 1.0f, ry = 1.0f;
    {
      const float2 t = reduce.sum(qx, qy);
      if (has_pre) rx = reciprocal_deviation(t.x, inv_dim, p.pre.eps);
      if (has_post) ry = reciprocal_deviation(t.y, inv_dim, p.post.eps);
    }
    if (has_pre) {
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float gamma[8];
        load_params8(p.pre.gamma, 1.0f, (i * TPR + l) * 8, n[i], q.vparams, gamma);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[i][j] = __fmul_rn(x[i][j], rx);
          sums[SUM_PRE_GAMMA][i][j] = __fmaf_rn(dh[i][j], x[i][j], sums[SUM_PRE_GAMMA][i][j]);
          sums[SUM_PRE_BETA][i][j] = __fadd_rn(dh[i][j], sums[SUM_PRE_BETA][i][j]);
          dh[i][j] = __fmul_rn(dh[i][j], gamma[j]);
          a = __fmaf_rn(dh[i][j], x[i][j], a);
          b = __fadd_rn(b, dh[i][j]);
        }
      }
      const float2 t = reduce.sum(a, b);
      const float along = __fmul_rn(t.x, inv_dim), mean = p.pre.kind == NORM_LAYER ? __fmul_rn(t.y, inv_dim) : 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dx[i][j] = __fmaf_rn(__fsub_rn(__fmaf_rn(-along, x[i][j], dh[i][j]), mean), rx, dx[i][j]);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (g.dx && n[i] > 0) store8(static_cast<TX*>(g.dx) + row * g.dx_stride + (i * TPR + l) * 8, dx[i], q.vdx && n[i] == 8, n[i]);
    if (has_y) {
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int c = (i * TPR + l) * 8;
        float gate[8], gamma[8], beta[8], t[8];
        load_gate8<TY>(p, seq, c, n[i], q.vgate, gate);
        if (has_post) {
          load_params8(p.post.gamma, 1.0f, c, n[i], q.vparams, gamma);
          load_params8(p.post.beta, 0.0f, c, n[i], q.vparams, beta);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float u = j < n[i] ? __fmul_rn(dx[i][j], p.scale) : 0.0f;
          y[i][j] = __fmul_rn(y[i][j], ry);
          const float r = has_post ? __fmaf_rn(y[i][j], gamma[j], beta[j]) : y[i][j];
          t[j] = __fmul_rn(u, r);
          sums[SUM_GATE][i][j] = __fadd_rn(sums[SUM_GATE][i][j], t[j]);
          const float w = __fmul_rn(u, gate[j]);
          sums[SUM_POST_GAMMA][i][j] = __fmaf_rn(w, y[i][j], sums[SUM_POST_GAMMA][i][j]);
          sums[SUM_POST_BETA][i][j] = __fadd_rn(w, sums[SUM_POST_BETA][i][j]);
          dx[i][j] = has_post ? __fmul_rn(w, gamma[j]) : w;
          a = __fmaf_rn(dx[i][j], y[i][j], a);
          b = __fadd_rn(b, dx[i][j]);
        }
        if (q.gate_mode == GATE_TOKEN && n[i] > 0) store8(g.dgate + row * g.dgate_stride + c, t, false, n[i]);
      }
      if (has_post) {
        const float2 t = reduce.sum(a, b);
        const float along = __fmul_rn(t.x, inv_dim), mean = p.post.kind == NORM_LAYER ? __fmul_rn(t.y, inv_dim) : 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) dx[i][j] = __fmul_rn(__fsub_rn(__fmaf_rn(-along, y[i][j], dx[i][j]), mean), ry);
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i)
        if (g.dy && n[i] > 0) store8(static_cast<TY*>(g.dy) + row * g.dy_stride + (i * TPR + l) * 8, dx[i], q.vdy && n[i] == 8, n[i]);
    }
    if (p.gate && --left == 0 || row + 1 == end) {
      // a sequence ends, or the worker's rows do: a sequence whose rows are all the worker's own is complete
      if (q.gate_mode == GATE_SEQUENCE) {
        const long s0 = seq * p.rows_per_gate, s1 = min(s0 + p.rows_per_gate, p.rows);
        float* dst = s0 >= first && s1 <= end ? g.dgate + seq * g.dgate_stride : q.gate_parts + (worker * 2 + (s0 > first ? 1 : 0)) * C;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (n[i] > 0) store8(dst + (i * TPR + l) * 8, sums[SUM_GATE][i], false, n[i]);
#pragma unroll
          for (int j = 0; j < 8; ++j) sums[SUM_GATE][i][j] = 0.0f;
        }
      }
      ++seq; left = p.rows_per_gate;
    }
  }

  // the CTA's column sums; several workers add theirs one after the other
  const bool wanted[SUMS] = {g.vec[0] != nullptr, g.vec[1] != nullptr, g.vec[2] != nullptr, g.vec[3] != nullptr, q.gate_mode == GATE_CHANNEL};
  float* out = q.sums + (long)blockIdx.x * SUMS * C;
  if constexpr (cta_rows<TPR>() > 1) {
    __shared__ float joined[SUMS][TPR * VPT * 8];
    for (int w = 0; w < cta_rows<TPR>(); ++w) {
      if ((int)threadIdx.x / TPR == w)
#pragma unroll
        for (int s = 0; s < SUMS; ++s)
#pragma unroll
          for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float* at = &joined[s][(i * 8 + j) * TPR + l];
              sums[s][i][j] = w > 0 ? __fadd_rn(*at, sums[s][i][j]) : sums[s][i][j];
              *at = sums[s][i][j];
            }
      __syncthreads();
    }
    if ((int)threadIdx.x / TPR != cta_rows<TPR>() - 1) return;
  }
#pragma unroll
  for (int s = 0; s < SUMS; ++s)
    if (wanted[s])
#pragma unroll
      for (int i = 0; i < VPT; ++i)
        if (n[i] > 0) store8(out + (long)s * C + (i * TPR + l) * 8, sums[s][i], false, n[i]);
}

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

// ---- host side -------------------------------------------------------------------------------------------------------------
struct Shape { int rows_per_cta; long ctas, per_worker; };
template <int TPR> Shape shape_of(long rows) {
  const long most = (long)sm_count() * ctas_per_sm<TPR>() * cta_rows<TPR>();
  Shape s;
  s.rows_per_cta = cta_rows<TPR>();
  const long workers = rows < most ? rows : most;
  s.per_worker = (rows + workers - 1) / workers;
  s.ctas = ((rows + s.per_worker - 1) / s.per_worker + s.rows_per_cta - 1) / s.rows_per_cta;
  return s;
}
// f(threads of a row, vectors of a thread), as constants
template <class F> auto with_shape(int dim, F f) {
  using std::integral_constant;
  if (dim <= 256) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (dim <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (dim <= 1024) return f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (dim <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (dim <= 4096) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (dim <= 8192) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
Shape shape_for(long rows, int dim) {
  return with_shape(dim, [&](auto tpr, auto) { return shape_of<decltype(tpr)::value>(rows); });
}
size_t sums_floats(const Shape& s, int dim) { return ((size_t)s.ctas * SUMS * dim + 63) / 64 * 64; }

}  // namespace

size_t residual_norm_backward_floats(long rows, int dim, bool gate_per_sequence) {
  if (rows <= 0) return 64;
  const Shape s = shape_for(rows, dim);
  return sums_floats(s, dim) + (gate_per_sequence ? (size_t)s.ctas * s.rows_per_cta * 2 * dim : 0);
}

void launch_residual_norm_backward(const ResNormArgs& a, const ResNormGradArgs& g, cudaStream_t st) {
  const Shape s = shape_for(a.rows, a.dim);
  BwdParams q;
  q.a = a; q.g = g;
  q.per_worker = s.per_worker;
  q.sums = g.workspace; q.gate_parts = g.workspace + sums_floats(s, a.dim);
  q.gate_mode = !a.gate || !g.dgate ? GATE_NONE : a.rows_per_gate >= a.rows ? GATE_CHANNEL : a.rows_per_gate == 1 ? GATE_TOKEN : GATE_SEQUENCE;
  with_types(a.x_dtype, a.y_dtype, [&](auto tx, auto ty) {
    using TX = decltype(tx);
    using TY = decltype(ty);
    q.vx = rows_aligned(a.x, a.x_stride, sizeof(TX)); q.vy = rows_aligned(a.y, a.y_stride, sizeof(TY));
    q.vgate = rows_aligned(a.gate, a.gate_stride, a.gate_f32 ? 4 : sizeof(TY));
    q.vdxo = rows_aligned(g.dx_out, g.dx_out_stride, sizeof(TX)); q.vdh = rows_aligned(g.dh, g.dh_stride, sizeof(TY));
    q.vdx = rows_aligned(g.dx, g.dx_stride, sizeof(TX)); q.vdy = rows_aligned(g.dy, g.dy_stride, sizeof(TY));
    q.vparams = true;
    for (const float* v : {a.post.gamma, a.post.beta, a.pre.gamma}) q.vparams &= rows_aligned(v, 0, 4);
    with_shape(a.dim, [&](auto tpr, auto vpt) {
      constexpr int TPR = decltype(tpr)::value, VPT = decltype(vpt)::value;
      launch_pdl(k_residual_norm_bwd<TX, TY, TPR, VPT>, dim3((unsigned)s.ctas), cta_threads<TPR>(), 0, st, q);
      ++g_launches;
    });
  });
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
