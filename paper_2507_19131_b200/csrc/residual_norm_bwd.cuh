// Gradients of the norms at a sublayer's border (mixaq_residual_norm_backward).  With d = dh o gamma_pre, xn the normalised x':
//   dx = dx_out + (d - xn mean(d o xn) [- mean(d)]) / dev(x'),   u = scale * dx,   dgate = sum u o r,   w = u o gate,
//   e = w o gamma_post,   dy = (e - yn mean(e o yn) [- mean(e)]) / dev(y)           (the bracketed means: LayerNorm only)
// and the parameters' gradients are column sums of dh o xn, dh, w o yn, w.
//
// The statistics are computed anew from x' and y, which the gradients need anyway: nothing has to be kept from the forward call.  Rows
// are read once: they pass through a ring of stages in shared memory, so that copies are under way during a row's four reductions, and
// a worker takes ROWS rows through them together.  Column sums stay in registers over the consecutive rows of a worker, are written
// out once per CTA and added by a second kernel in the order of the CTAs: no atomics, so the result depends on the sizes and the number
// of SMs only.
#pragma once
#include "residual_norm.cuh"

namespace mixaq {

enum { SUM_POST_GAMMA = 0, SUM_POST_BETA, SUM_PRE_GAMMA, SUM_PRE_BETA, SUM_GATE, SUMS };

enum GateMode { GATE_NONE = 0, GATE_CHANNEL, GATE_SEQUENCE, GATE_TOKEN };
struct BwdParams {
  ResNormArgs a; ResNormGradArgs g;
  int gate_mode;               // how dgate is summed (GATE_NONE: it is not wanted)
  int stages; uint32_t x_bytes, y_bytes, stage_bytes;       // of the ring: a row of the stream's type, of the sublayers', ROWS rows of all
  int* status;
  long per_worker;             // consecutive rows of a worker
  float* sums;                 // [CTA][SUMS][dim]
  float* gate_parts;           // [worker][2][dim]: sums of the first and the last sequence that a worker shares with others
};

namespace {

// resident CTAs per SM that the registers are divided for: 512 threads at 128 registers
template <int TPR> __host__ __device__ constexpr int ctas_per_sm() { return cta_threads<TPR>() >= 512 ? 1 : 512 / cta_threads<TPR>(); }

// eight binary32 values of a row at any address
template <int TPR, bool VEC>
__device__ __forceinline__ void store_floats(float* row, int i, int l, int dim, const F8& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) if (present<TPR, VEC>(i, j, l, dim)) row[column<TPR, VEC>(i, j, l)] = element(f, j);
}

template <class TX, class TY, int TPR, int VPT, int ROWS, bool VEC, bool RING>
__global__ void __launch_bounds__(cta_threads<TPR>(), ctas_per_sm<TPR>()) k_residual_norm_bwd(const BwdParams q) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float slots[2][2 * ROWS][TPR / 32];
  __shared__ __align__(8) uint64_t bars[cta_workers<TPR>()][MAX_STAGES];
  RowReduce<TPR, 2 * ROWS> reduce{slots};
  const ResNormArgs& p = q.a;
  const ResNormGradArgs& g = q.g;
  const int l = threadIdx.x % TPR, C = p.dim, in_cta = threadIdx.x / TPR;
  const long worker = (long)blockIdx.x * cta_workers<TPR>() + in_cta;
  const long first = worker * q.per_worker, end = min(first + q.per_worker, p.rows);
  const float inv_dim = __fdiv_rn(1.0f, (float)C);
  const bool has_y = p.y != nullptr, has_pre = p.pre.kind != NORM_NONE && g.dh != nullptr, has_post = p.post.kind != NORM_NONE, has_dxo = g.dx_out != nullptr;
  const RowSource src_x = row_source<TX>(p.x, p.x_stride, p.rows, C), src_dxo = row_source<TX>(g.dx_out, g.dx_out_stride, p.rows, C);
  const RowSource src_y = row_source<TY>(p.y, p.y_stride, p.rows, C), src_dh = row_source<TY>(g.dh, g.dh_stride, p.rows, C);
  // a stage: x, dx_out, y, dh of each of its rows
  const uint32_t off_dxo = q.x_bytes, off_y = 2 * q.x_bytes, off_dh = 2 * q.x_bytes + q.y_bytes, row_bytes = 2 * q.x_bytes + 2 * q.y_bytes;
  uint8_t* const ring = smem + (size_t)in_cta * q.stages * q.stage_bytes;
  const uint32_t ring_at = smem_u32(ring), bar = smem_u32(bars[in_cta]);
  long fetched = 0;
  auto fetch = [&](long row, int stage) {
    const uint32_t full = bar + 8u * (uint32_t)stage;
    uint32_t bytes = 0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (row + r < end)
        bytes += (has_pre ? span_bytes<VEC>(src_x, row + r) + span_bytes<VEC>(src_dh, row + r) : 0u) +
                 (has_dxo ? span_bytes<VEC>(src_dxo, row + r) : 0u) + (has_y ? span_bytes<VEC>(src_y, row + r) : 0u);
    mbar_arrive_expect_tx(full, bytes);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (row + r >= end) break;
      const uint32_t dst = ring_at + (uint32_t)stage * q.stage_bytes + (uint32_t)r * row_bytes;
      if (has_pre) { fetch_row<VEC>(src_x, row + r, dst, full); fetch_row<VEC>(src_dh, row + r, dst + off_dh, full); }
      if (has_dxo) fetch_row<VEC>(src_dxo, row + r, dst + off_dxo, full);
      if (has_y) fetch_row<VEC>(src_y, row + r, dst + off_y, full);
    }
    ++fetched;
  };
  if (RING) {
    if (l == 0) {
      for (int i = 0; i < q.stages; ++i) mbar_init(bar + 8u * (uint32_t)i, 1u);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
  }
  griddep_wait();
  griddep_launch();
  if (RING && l == 0)
    for (int i = 0; i < q.stages && first + i * ROWS < end; ++i) fetch(first + i * ROWS, i);

  const bool full = C == TPR * VPT * 8;
  F8 sums[SUMS][VPT];
#pragma unroll
  for (int s = 0; s < SUMS; ++s)
#pragma unroll
    for (int i = 0; i < VPT; ++i) sums[s][i] = fill8(0.0f);
  // the sequence that a row belongs to and the rows until its end
  long seq = 0, left = 0;
  if (p.gate && first < end) { seq = (uint32_t)first / (uint32_t)p.rows_per_gate; left = (seq + 1) * p.rows_per_gate - first; }

  int stage = 0; uint32_t pass = 0;
  bool ok = true;
  for (long row0 = first; row0 < end; row0 += ROWS) {
    if (RING) {
      ok = worker_and<TPR>(wait_stage(bar + 8u * (uint32_t)stage, pass));
      if (!ok) break;
    }
    // A row that is not there (the second one at a worker's end) counts as zeros; its part of the stage is not looked at.
    const uint8_t* const at = ring + (size_t)stage * q.stage_bytes;
    F8 x[ROWS][VPT], y[ROWS][VPT], dx[ROWS][VPT];
    float t[2 * ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const long row = min(row0 + r, end - 1);
      const bool here = row0 + r < end;
      const StagedRow<TX> rx = staged_row<VEC, RING, TX>(src_x, row, at + r * row_bytes);
      const StagedRow<TY> ry = staged_row<VEC, RING, TY>(src_y, row, at + r * row_bytes + off_y);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        x[r][i] = has_pre && here ? load_staged<TPR, VEC, RING>(rx, i, l, C) : fill8(0.0f);
        y[r][i] = has_y && here ? load_staged<TPR, VEC, RING>(ry, i, l, C) : fill8(0.0f);
      }
    }
    if (p.pre.kind == NORM_LAYER || p.post.kind == NORM_LAYER) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        t[2 * r] = t[2 * r + 1] = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) { t[2 * r] = sum8(x[r][i], make_float2(t[2 * r], 0.0f)); t[2 * r + 1] = sum8(y[r][i], make_float2(t[2 * r + 1], 0.0f)); }
      }
      reduce.sum(t);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float2 mx = f2(p.pre.kind == NORM_LAYER ? __fmul_rn(t[2 * r], inv_dim) : 0.0f), my = f2(p.post.kind == NORM_LAYER ? __fmul_rn(t[2 * r + 1], inv_dim) : 0.0f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) { x[r][i].v[j] = sub2(x[r][i].v[j], mx); y[r][i].v[j] = sub2(y[r][i].v[j], my); }
          if (!full) { mask_cols<TPR, VEC>(x[r][i], i, l, C); mask_cols<TPR, VEC>(y[r][i], i, l, C); }
        }
      }
    }
    float rx[ROWS], ry[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float2 qx = f2(0.0f), qy = f2(0.0f);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) { qx = __ffma2_rn(x[r][i].v[j], x[r][i].v[j], qx); qy = __ffma2_rn(y[r][i].v[j], y[r][i].v[j], qy); }
      t[2 * r] = __fadd_rn(qx.x, qx.y); t[2 * r + 1] = __fadd_rn(qy.x, qy.y);
    }
    reduce.sum(t);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      rx[r] = has_pre ? reciprocal_deviation(t[2 * r], inv_dim, p.pre.eps) : 1.0f;
      ry[r] = has_post ? reciprocal_deviation(t[2 * r + 1], inv_dim, p.post.eps) : 1.0f;
    }
    // `dx` holds d = dh o gamma first.  (Columns that are not there have dh = 0, and below u = 0.)
    if (has_pre) {
      float2 ta[ROWS], tb[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) ta[r] = tb[r] = f2(0.0f);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const F8 gamma = load_params<TPR, VEC>(p.pre.gamma, 1.0f, i, l, C);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          const StagedRow<TY> rdh = staged_row<VEC, RING, TY>(src_dh, min(row0 + r, end - 1), at + r * row_bytes + off_dh);
          const F8 dh = row0 + r < end ? load_staged<TPR, VEC, RING>(rdh, i, l, C) : fill8(0.0f);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[r][i].v[j] = __fmul2_rn(x[r][i].v[j], f2(rx[r]));
            sums[SUM_PRE_GAMMA][i].v[j] = __ffma2_rn(dh.v[j], x[r][i].v[j], sums[SUM_PRE_GAMMA][i].v[j]);
            sums[SUM_PRE_BETA][i].v[j] = __fadd2_rn(dh.v[j], sums[SUM_PRE_BETA][i].v[j]);
            dx[r][i].v[j] = __fmul2_rn(dh.v[j], gamma.v[j]);
            ta[r] = __ffma2_rn(dx[r][i].v[j], x[r][i].v[j], ta[r]);
            tb[r] = __fadd2_rn(tb[r], dx[r][i].v[j]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) { t[2 * r] = __fadd_rn(ta[r].x, ta[r].y); t[2 * r + 1] = __fadd_rn(tb[r].x, tb[r].y); }
      reduce.sum(t);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const long row = min(row0 + r, end - 1);
      const bool here = row0 + r < end;
      const StagedRow<TX> rdxo = staged_row<VEC, RING, TX>(src_dxo, row, at + r * row_bytes + off_dxo);
      const float2 along = f2(-__fmul_rn(t[2 * r], inv_dim)), mean = f2(p.pre.kind == NORM_LAYER ? __fmul_rn(t[2 * r + 1], inv_dim) : 0.0f), dev = f2(rx[r]);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const F8 dxo = has_dxo && here ? load_staged<TPR, VEC, RING>(rdxo, i, l, C) : fill8(0.0f);
        if (has_pre) {
#pragma unroll
          for (int j = 0; j < 4; ++j) dx[r][i].v[j] = __ffma2_rn(sub2(__ffma2_rn(along, x[r][i].v[j], dx[r][i].v[j]), mean), dev, dxo.v[j]);
        } else {
          dx[r][i] = dxo;
        }
        if (g.dx && here) store_cols<TPR, VEC>(static_cast<TX*>(g.dx) + row * g.dx_stride, i, l, C, dx[r][i]);
      }
    }
    if (RING) {
      // the stage is used up: y is in registers
      if constexpr (TPR > 32) __syncthreads();
      else __syncwarp();
      if (l == 0 && row0 + (long)q.stages * ROWS < end) fetch(row0 + (long)q.stages * ROWS, stage);
      if (++stage == q.stages) { stage = 0; pass ^= 1u; }
    }
    if (!has_y) continue;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const long row = row0 + r;
      const bool here = row < end;
      float2 ta = f2(0.0f), tb = f2(0.0f);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        F8 u = dx[r][i], part;
        const F8 gate = load_gate<TPR, VEC, TY>(p, seq, i, l);
        if (!full && p.pre.kind == NORM_LAYER) mask_cols<TPR, VEC>(u, i, l, C);      // (the mean was taken from all columns)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u.v[j] = __fmul2_rn(u.v[j], f2(p.scale));
          y[r][i].v[j] = __fmul2_rn(y[r][i].v[j], f2(ry[r]));
        }
        if (has_post) {
          const F8 gamma = load_params<TPR, VEC>(p.post.gamma, 1.0f, i, l, C), beta = load_params<TPR, VEC>(p.post.beta, 0.0f, i, l, C);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            part.v[j] = __fmul2_rn(u.v[j], __ffma2_rn(y[r][i].v[j], gamma.v[j], beta.v[j]));
            const float2 w = __fmul2_rn(u.v[j], gate.v[j]);
            sums[SUM_POST_GAMMA][i].v[j] = __ffma2_rn(w, y[r][i].v[j], sums[SUM_POST_GAMMA][i].v[j]);
            sums[SUM_POST_BETA][i].v[j] = __fadd2_rn(w, sums[SUM_POST_BETA][i].v[j]);
            dx[r][i].v[j] = __fmul2_rn(w, gamma.v[j]);
            ta = __ffma2_rn(dx[r][i].v[j], y[r][i].v[j], ta);
            tb = __fadd2_rn(tb, dx[r][i].v[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            part.v[j] = __fmul2_rn(u.v[j], y[r][i].v[j]);
            dx[r][i].v[j] = __fmul2_rn(u.v[j], gate.v[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[SUM_GATE][i].v[j] = __fadd2_rn(sums[SUM_GATE][i].v[j], part.v[j]);
        if (q.gate_mode == GATE_TOKEN && here) store_floats<TPR, VEC>(g.dgate + row * g.dgate_stride, i, l, C, part);
      }
      t[2 * r] = __fadd_rn(ta.x, ta.y); t[2 * r + 1] = __fadd_rn(tb.x, tb.y);
      if (p.gate && here && (--left == 0 || row + 1 == end)) {
        // a sequence ends, or the worker's rows do: a sequence whose rows are all the worker's own is complete
        if (q.gate_mode == GATE_SEQUENCE) {
          const long s0 = seq * p.rows_per_gate, s1 = min(s0 + p.rows_per_gate, p.rows);
          float* const dst = s0 >= first && s1 <= end ? g.dgate + seq * g.dgate_stride : q.gate_parts + (worker * 2 + (s0 > first ? 1 : 0)) * C;
#pragma unroll
          for (int i = 0; i < VPT; ++i) {
            store_floats<TPR, VEC>(dst, i, l, C, sums[SUM_GATE][i]);
            sums[SUM_GATE][i] = fill8(0.0f);
          }
        }
        if (row + 1 < end) { ++seq; left = p.rows_per_gate; }
      }
    }
    if (has_post) {
      reduce.sum(t);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float2 along = f2(-__fmul_rn(t[2 * r], inv_dim)), mean = f2(p.post.kind == NORM_LAYER ? __fmul_rn(t[2 * r + 1], inv_dim) : 0.0f), dev = f2(ry[r]);
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) dx[r][i].v[j] = __fmul2_rn(sub2(__ffma2_rn(along, y[r][i].v[j], dx[r][i].v[j]), mean), dev);
      }
    }
    if (g.dy) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
          if (row0 + r < end) store_cols<TPR, VEC>(static_cast<TY*>(g.dy) + (row0 + r) * g.dy_stride, i, l, C, dx[r][i]);
    }
  }
  if (RING && !ok && l == 0) drain_stages(bar, q.stages, fetched, q.status);

  // the CTA's column sums; several workers add theirs one after the other
  const bool wanted[SUMS] = {g.vec[0] != nullptr, g.vec[1] != nullptr, g.vec[2] != nullptr, g.vec[3] != nullptr, q.gate_mode == GATE_CHANNEL};
  float* const out = q.sums + (long)blockIdx.x * SUMS * C;
  if constexpr (cta_workers<TPR>() > 1) {
    __shared__ float2 joined[SUMS][TPR * VPT * 4];
    for (int w = 0; w < cta_workers<TPR>(); ++w) {
      if (in_cta == w)
#pragma unroll
        for (int s = 0; s < SUMS; ++s)
#pragma unroll
          for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float2* const cell = &joined[s][(i * 4 + j) * TPR + l];
              if (w > 0) sums[s][i].v[j] = __fadd2_rn(*cell, sums[s][i].v[j]);
              *cell = sums[s][i].v[j];
            }
      __syncthreads();
    }
    if (in_cta != cta_workers<TPR>() - 1) return;
  }
#pragma unroll
  for (int s = 0; s < SUMS; ++s)
    if (wanted[s])
#pragma unroll
      for (int i = 0; i < VPT; ++i) store_floats<TPR, VEC>(out + (long)s * C, i, l, C, sums[s][i]);
}

// A ring for rows of which two do not fit into RING_BYTES_PER_SM, for CTAs that have their SM to themselves.  (Not for the others: what
// the ring takes is lost to the L1, which has the parameters.  16384 x 4096 takes 364 us with it and 324 without, but 8000 x 8192 with a
// binary32 stream, which has no ring otherwise, 412 instead of 705.)
constexpr int WIDE_RING_BYTES = 200 * 1024;

// ---- shapes ----------------------------------------------------------------------------------------------------------------
struct Shape { int rows_per_cta; long ctas, per_worker; };
template <int TPR> Shape shape_of(long rows) {
  const long most = (long)sm_count() * ctas_per_sm<TPR>() * cta_workers<TPR>();
  Shape s;
  s.rows_per_cta = cta_workers<TPR>();
  const long workers = rows < most ? rows : most;
  s.per_worker = (rows + workers - 1) / workers;
  s.ctas = ((rows + s.per_worker - 1) / s.per_worker + s.rows_per_cta - 1) / s.rows_per_cta;
  return s;
}
// f(threads of a row, vectors of a thread, rows taken together), as constants.  Two rows at a time (WIDE_ROWS) where their registers fit and
// two stages of them the ring: 16-bit rows in vector order (16384 x 4096 bfloat16: 324 us, one row at a time 339).  Others lose by it:
// 16384 x 4096 with a binary32 stream 647 us by two, without a ring, and 405 by one; 10000 x 3001 bfloat16, element by element, 332 by two
// and 239 by one.
template <int WIDE_ROWS, class F> auto with_shape(int dim, F f) {
  using std::integral_constant;
  if (dim <= 256) return f(integral_constant<int, 32>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (dim <= 512) return f(integral_constant<int, 64>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (dim <= 1024) return f(integral_constant<int, 128>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (dim <= 2048) return f(integral_constant<int, 256>{}, integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (dim <= 4096) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{}, integral_constant<int, WIDE_ROWS>{});
  if (dim <= 8192) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
}
Shape shape_for(long rows, int dim) {
  return with_shape<1>(dim, [&](auto tpr, auto, auto) { return shape_of<decltype(tpr)::value>(rows); });
}
}  // namespace

// The main kernel with one pair of types; each pair is instantiated in one source file, so that they compile side by side.
template <class TX, class TY> void residual_norm_bwd_typed(BwdParams q, cudaStream_t st) {
  const ResNormArgs& a = q.a;
  const ResNormGradArgs& g = q.g;
  const Shape s = shape_for(a.rows, a.dim);
  bool vec = a.dim % 8 == 0 && rows_aligned(a.x, a.x_stride, sizeof(TX)) && rows_aligned(a.y, a.y_stride, sizeof(TY)) &&
             rows_aligned(a.gate, a.gate_stride, a.gate_f32 ? 4 : sizeof(TY)) && rows_aligned(g.dx_out, g.dx_out_stride, sizeof(TX)) &&
             rows_aligned(g.dh, g.dh_stride, sizeof(TY)) && rows_aligned(g.dx, g.dx_stride, sizeof(TX)) && rows_aligned(g.dy, g.dy_stride, sizeof(TY));
  for (const float* v : {a.post.gamma, a.post.beta, a.pre.gamma}) vec &= rows_aligned(v, 0, 4);
  auto run_shape = [&](auto tpr, auto vpt, auto rows) {
    constexpr int TPR = decltype(tpr)::value, VPT = decltype(vpt)::value, ROWS = decltype(rows)::value;
    const uint32_t x = (uint32_t)(a.dim * sizeof(TX)), y = (uint32_t)(a.dim * sizeof(TY));
    q.x_bytes = vec ? staged_bytes<true>(x) : staged_bytes<false>(x);
    q.y_bytes = vec ? staged_bytes<true>(y) : staged_bytes<false>(y);
    q.stage_bytes = ROWS * 2 * (q.x_bytes + q.y_bytes);
    int ctas = ctas_per_sm<TPR>(), ring_bytes = RING_BYTES_PER_SM;
    const int most = ctas;
    q.stages = ring_stages(q.stage_bytes, cta_workers<TPR>(), ctas, ring_bytes);
    if (ctas < most) q.stages = 0;                        // (the grid is sized for all)
    if (TPR >= 512 && !q.stages) q.stages = ring_stages(q.stage_bytes, 1, ctas, ring_bytes = WIDE_RING_BYTES);
    auto run = [&](auto kernel, std::atomic<uint64_t>* done) {
      if (done) allow_ring(kernel, *done, TPR >= 512 ? WIDE_RING_BYTES : RING_BYTES_PER_SM);
      launch_pdl(kernel, dim3((unsigned)s.ctas), cta_threads<TPR>(), (size_t)q.stages * q.stage_bytes * cta_workers<TPR>(), st, q);
      ++g_launches;
    };
    // Rows of up to 2048 elements always have room for two stages, and pairs of rows in 16 bits; longer ones may not.
    constexpr long widest = ROWS * 2L * (TPR * VPT * 8) * (sizeof(TX) + sizeof(TY)) + ROWS * 4 * 32;
    constexpr bool always = TPR < 512 || ROWS > 1;
    static_assert(!always || RING_BYTES_PER_SM / ctas_per_sm<TPR>() / cta_workers<TPR>() / widest >= 2, "a ring for every short row");
    if (ROWS == 1 && !always && !q.stages) {
      run(k_residual_norm_bwd<TX, TY, TPR, VPT, 1, false, always>, nullptr);
    } else if (ROWS > 1 || vec) {
      static std::atomic<uint64_t> done{0};
      run(k_residual_norm_bwd<TX, TY, TPR, VPT, ROWS, true, true>, &done);
    } else {
      static std::atomic<uint64_t> done{0};
      run(k_residual_norm_bwd<TX, TY, TPR, VPT, 1, false, true>, &done);
    }
  };
  if constexpr (sizeof(TX) == 2) {
    if (vec) { with_shape<2>(a.dim, run_shape); return; }
  }
  with_shape<1>(a.dim, run_shape);
}

}  // namespace mixaq
