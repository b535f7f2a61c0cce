// Norms at the border of two sublayers, with gate and residual scale (mixaq_residual_norm_forward):
//   x' = x + scale * gate o norm_post(y),   h = norm_pre(x')
// One pass: a row of x and y is read once into registers, x' and h are written; every statistic is a sum over the registers of the
// row's threads, in two passes (mean, then squared deviations), in binary32.
//
// Bound by memory where a row has one reduction (32768 rows of 4096, binary32 stream, RMS pre norm: 257 us, 6.2 TB/s), and by the chain of
// a row's reductions and parameter loads with a post norm on top (357 us, 4.1 TB/s; without the parameter loads 310, without the
// reductions 328).  So workers stay on consecutive rows, have the next ones copied to shared memory meanwhile and compute on pairs of
// values; three CTAs of eight warps, with the registers for loads in flight, hide more than four with fewer (435).
#pragma once
#include "residual_norm.cuh"

namespace mixaq {
namespace {

struct FwdParams { ResNormArgs a; int stages; uint32_t x_bytes, row_bytes, stage_bytes; long per_worker; int* status; };      // bytes in the ring

// resident CTAs per SM that the registers are divided for: 768 threads at 80 each.  (32768 rows of 4096, binary32 stream: 360 us so; two
// CTAs of 512 threads with half the elements 421, four of 128 with twice as many 424, two rows at a time by 512 threads 388.)
template <int TPR> __host__ __device__ constexpr int fwd_ctas_per_sm() { return cta_threads<TPR>() >= 512 ? 1 : 768 / cta_threads<TPR>(); }

template <class TX, class TY, int TPR, int VPT, int ROWS, bool VEC, bool RING>
__global__ void __launch_bounds__(cta_threads<TPR>(), fwd_ctas_per_sm<TPR>()) k_residual_norm(const FwdParams q) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float slots[2][ROWS][TPR / 32];
  __shared__ float block_max[VEC ? 1 : ROWS][VEC ? 1 : VPT * 8][VEC ? 1 : TPR / 32];
  __shared__ __align__(8) uint64_t bars[cta_workers<TPR>()][MAX_STAGES];
  RowReduce<TPR, ROWS> reduce{slots};
  const ResNormArgs& p = q.a;
  const int l = threadIdx.x % TPR, C = p.dim, in_cta = threadIdx.x / TPR;
  const long worker = (long)blockIdx.x * cta_workers<TPR>() + in_cta;
  const long first = worker * q.per_worker, end = min(first + q.per_worker, p.rows);
  const float inv_dim = __fdiv_rn(1.0f, (float)C);
  const bool has_y = p.y != nullptr, has_post = p.post.kind != NORM_NONE;
  const RowSource src_x = row_source<TX>(p.x, p.x_stride, p.rows, C), src_y = row_source<TY>(p.y, p.y_stride, p.rows, C);
  uint8_t* const ring = smem + (size_t)in_cta * q.stages * q.stage_bytes;
  const uint32_t ring_at = smem_u32(ring), bar = smem_u32(bars[in_cta]);
  long fetched = 0;
  auto fetch = [&](long row, int stage) {
    const uint32_t full = bar + 8u * (uint32_t)stage;
    uint32_t bytes = 0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (row + r < end) bytes += span_bytes<VEC>(src_x, row + r) + (has_y ? span_bytes<VEC>(src_y, row + r) : 0u);
    mbar_arrive_expect_tx(full, bytes);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (row + r >= end) break;
      const uint32_t dst = ring_at + (uint32_t)stage * q.stage_bytes + (uint32_t)r * q.row_bytes;
      fetch_row<VEC>(src_x, row + r, dst, full);
      if (has_y) fetch_row<VEC>(src_y, row + r, dst + q.x_bytes, full);
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
  if (first >= end) return;                    // (all of a worker's threads; nothing below spans workers)
  if (RING && l == 0)
    for (int i = 0; i < q.stages && first + i * ROWS < end; ++i) fetch(first + i * ROWS, i);

  // the gate's row and the rows until the next one
  long gate_row = p.gate ? (uint32_t)first / (uint32_t)p.rows_per_gate : 0, left = p.gate ? (gate_row + 1) * p.rows_per_gate - first : p.rows;
  constexpr bool KEEP = VEC && VPT <= 2;       // the gate's values stay in registers
  F8 kept[VPT];
  auto read_gate = [&]() {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      kept[i] = load_gate<TPR, VEC, TY>(p, gate_row, i, l);
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[i].v[j] = __fmul2_rn(kept[i].v[j], f2(p.scale));
    }
  };
  if (KEEP && has_y) read_gate();

  const bool full = C == TPR * VPT * 8;
  // v -> its deviation from the row's mean (LAYER); returns the reciprocals of the standard deviations
  auto normalise = [&](F8 (&v)[ROWS][VPT], const NormSpec& s, float (&t)[ROWS]) {
    if (s.kind == NORM_LAYER) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        t[r] = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) t[r] = sum8(v[r][i], make_float2(t[r], 0.0f));
      }
      reduce.sum(t);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float2 mean = f2(__fmul_rn(t[r], inv_dim));
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[r][i].v[j] = sub2(v[r][i].v[j], mean);
          if (!full) mask_cols<TPR, VEC>(v[r][i], i, l, C);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float2 sq = f2(0.0f);
#pragma unroll
      for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sq = __ffma2_rn(v[r][i].v[j], v[r][i].v[j], sq);
      t[r] = __fadd_rn(sq.x, sq.y);
    }
    reduce.sum(t);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) t[r] = reciprocal_deviation(t[r], inv_dim, s.eps);
  };
  // deviation -> gamma * deviation * rstd + beta (columns that are not there stay zero: so are their parameters, or the deviation is)
  auto scaled = [&](F8& v, float rstd, const F8& gamma, const F8& beta) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v.v[j] = __ffma2_rn(__fmul2_rn(v.v[j], f2(rstd)), gamma.v[j], beta.v[j]);
  };

  int stage = 0; uint32_t pass = 0;
  bool ok = true;
  for (long row0 = first; row0 < end; row0 += ROWS) {
    F8 x[ROWS][VPT], y[ROWS][VPT];
    if (RING) {
      ok = wait_stage(bar + 8u * (uint32_t)stage, pass);
    }
    const uint8_t* const at = ring + (size_t)stage * q.stage_bytes;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      // a row that is not there (the second one at a worker's end) is computed as zeros and not stored
      const bool here = row0 + r < end;
      const StagedRow<TX> rx = staged_row<VEC, RING, TX>(src_x, min(row0 + r, end - 1), at + r * q.row_bytes);
      const StagedRow<TY> ry = staged_row<VEC, RING, TY>(src_y, min(row0 + r, end - 1), at + r * q.row_bytes + q.x_bytes);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        x[r][i] = here && ok ? load_staged<TPR, VEC, RING>(rx, i, l, C) : fill8(0.0f);
        y[r][i] = here && ok && has_y ? load_staged<TPR, VEC, RING>(ry, i, l, C) : fill8(0.0f);
      }
    }
    if (RING) {
      ok = worker_and<TPR>(ok);                             // the stage is used up
      if (!ok) break;
      if (l == 0 && row0 + (long)q.stages * ROWS < end) fetch(row0 + (long)q.stages * ROWS, stage);
      if (++stage == q.stages) { stage = 0; pass ^= 1u; }
    }
    float rstd[ROWS];
    if (has_y) {
      if (has_post) {
        normalise(y, p.post, rstd);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const F8 gamma = load_params<TPR, VEC>(p.post.gamma, 1.0f, i, l, C);
          const F8 beta = load_params<TPR, VEC>(p.post.beta, 0.0f, i, l, C);
#pragma unroll
          for (int r = 0; r < ROWS; ++r) scaled(y[r][i], rstd[r], gamma, beta);
        }
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const bool here = row0 + r < end;
        TX* const out = static_cast<TX*>(p.x_out) + (row0 + r) * p.x_out_stride;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const F8 gate = KEEP ? kept[i] : load_gate<TPR, VEC, TY>(p, gate_row, i, l);
#pragma unroll
          for (int j = 0; j < 4; ++j)                       // rounded to the stream's type: what the pre norm sees
            x[r][i].v[j] = round2<TX>(__ffma2_rn(KEEP ? gate.v[j] : __fmul2_rn(gate.v[j], f2(p.scale)), y[r][i].v[j], x[r][i].v[j]));
          if (here) store_cols<TPR, VEC>(out, i, l, C, x[r][i]);
        }
        if (--left == 0 && row0 + r + 1 < end) {
          ++gate_row; left = p.rows_per_gate;
          if (KEEP) read_gate();
        }
      }
    }
    if (p.pre.kind == NORM_NONE) continue;
    normalise(x, p.pre, rstd);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const F8 gamma = load_params<TPR, VEC>(p.pre.gamma, 1.0f, i, l, C);
      const F8 beta = load_params<TPR, VEC>(p.pre.beta, 0.0f, i, l, C);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        scaled(x[r][i], rstd[r], gamma, beta);
        if (!p.codes && row0 + r < end) store_cols<TPR, VEC>(static_cast<TY*>(p.h) + (row0 + r) * p.h_stride, i, l, C, x[r][i]);
      }
    }
    if (!p.codes) continue;
    if constexpr (VEC) {
      // sixteen neighbouring lanes hold a block of 128 columns
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        uint8_t* const codes = p.codes + (row0 + r) * p.code_stride;
        float* const scales = p.h_scale + (row0 + r) * p.srs;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          float m = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) m = max_abs(max_abs(m, x[r][i].v[j].x), x[r][i].v[j].y);
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
          float s, inv;
          block_scale(m, p.pow2, s, inv);
          const int c = column<TPR, VEC>(i, 0, l);
          if (c < C && row0 + r < end) {
            *reinterpret_cast<uint2*>(codes + c) = codes8(x[r][i].v, inv);
            if (l % 16 == 0) scales[(long)(c / FP8_BLOCK) * p.scs] = s;
          }
        }
      }
    } else {
      // A block's elements: one element of each thread of four warps, of two warps two, of a single warp four.
      constexpr int W = TPR / 32, OF_WARP = TPR < 128 ? 128 / TPR : 1, WARPS = TPR < 128 ? W : 4, BLOCKS = VPT * 8 / OF_WARP;
      const int warp = l / 32, lane = threadIdx.x & 31;
      float m[ROWS][BLOCKS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
          m[r][k] = 0.0f;
#pragma unroll
          for (int j = 0; j < OF_WARP; ++j) m[r][k] = max_abs(m[r][k], element(x[r][(k * OF_WARP + j) / 8], (k * OF_WARP + j) % 8));
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) m[r][k] = max_abs(m[r][k], __shfl_xor_sync(0xffffffffu, m[r][k], o));
          if (TPR > 32 && lane == 0) block_max[r][k][warp] = m[r][k];
        }
      if (TPR > 32) __syncthreads();
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        uint8_t* const codes = p.codes + (row0 + r) * p.code_stride;
        float* const scales = p.h_scale + (row0 + r) * p.srs;
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
          if (TPR > 32) {
#pragma unroll
            for (int w = 0; w < WARPS; ++w) m[r][k] = max_abs(m[r][k], block_max[r][k][warp / WARPS * WARPS + w]);
          }
          float s, inv;
          block_scale(m[r][k], p.pow2, s, inv);
#pragma unroll
          for (int j = 0; j < OF_WARP; ++j) {
            const int e = k * OF_WARP + j, c = column<TPR, VEC>(e / 8, e % 8, l);
            if (c < C && row0 + r < end) {
              codes[c] = (uint8_t)codes4(__fmul_rn(element(x[r][e / 8], e % 8), inv), 0.0f, 0.0f, 0.0f);
              if (c % FP8_BLOCK == 0) scales[(long)(c / FP8_BLOCK) * p.scs] = s;
            }
          }
        }
      }
      if (TPR > 32) __syncthreads();                        // (block_max is written again for the next rows)
    }
  }
  if (RING && !ok && l == 0) drain_stages(bar, q.stages, fetched, q.status);
}

template <class TX, class TY, int TPR, int VPT, int ROWS, bool VEC, bool RING>
void launch_fwd(const FwdParams& q, long workers, cudaStream_t st) {
  const auto kernel = k_residual_norm<TX, TY, TPR, VPT, ROWS, VEC, RING>;
  if (RING) {
    static std::atomic<uint64_t> done{0};
    allow_ring(kernel, done);
  }
  launch_pdl(kernel, dim3((unsigned)((workers + cta_workers<TPR>() - 1) / cta_workers<TPR>())), cta_threads<TPR>(),
             RING ? (size_t)q.stages * q.stage_bytes * cta_workers<TPR>() : 0, st, q);
  ++g_launches;
}
template <class TX, class TY, int TPR, int VPT, int ROWS>
void launch_fwd_shape(FwdParams q, bool vec, cudaStream_t st) {
  const uint32_t x = (uint32_t)(q.a.dim * sizeof(TX)), y = q.a.y ? (uint32_t)(q.a.dim * sizeof(TY)) : 0;
  q.x_bytes = vec ? staged_bytes<true>(x) : staged_bytes<false>(x);
  q.row_bytes = q.x_bytes + (vec ? staged_bytes<true>(y) : staged_bytes<false>(y));
  q.stage_bytes = ROWS * q.row_bytes;
  int ctas = fwd_ctas_per_sm<TPR>();
  q.stages = ring_stages(q.stage_bytes, cta_workers<TPR>(), ctas);
  if (!q.stages) ctas = fwd_ctas_per_sm<TPR>();
  const long resident = (long)sm_count() * ctas * cta_workers<TPR>(), most = q.a.rows < resident ? q.a.rows : resident;
  q.per_worker = (q.a.rows + most - 1) / most;
  const long workers = (q.a.rows + q.per_worker - 1) / q.per_worker;
  // a ring pays from the third step on; rows too long for two stages have none
  const bool ring = q.stages && q.per_worker > 2 * ROWS;
  if (ring) vec ? launch_fwd<TX, TY, TPR, VPT, ROWS, true, true>(q, workers, st) : launch_fwd<TX, TY, TPR, VPT, ROWS, false, true>(q, workers, st);
  else vec ? launch_fwd<TX, TY, TPR, VPT, ROWS, true, false>(q, workers, st) : launch_fwd<TX, TY, TPR, VPT, ROWS, false, false>(q, workers, st);
}

}  // namespace

// The call with one pair of types; each pair is instantiated in one source file, so that they compile side by side.
template <class TX, class TY> void residual_norm_typed(const ResNormArgs& a, int* status, cudaStream_t st) {
  FwdParams q;
  q.a = a; q.status = status;
  bool vec = a.dim % 8 == 0 && rows_aligned(a.x, a.x_stride, sizeof(TX)) && rows_aligned(a.y, a.y_stride, sizeof(TY)) &&
             rows_aligned(a.gate, a.gate_stride, a.gate_f32 ? 4 : sizeof(TY)) && rows_aligned(a.x_out, a.x_out_stride, sizeof(TX)) &&
             rows_aligned(a.h, a.h_stride, sizeof(TY));
  for (const float* v : {a.post.gamma, a.post.beta, a.pre.gamma, a.pre.beta}) vec &= rows_aligned(v, 0, 4);
  // the fewest threads that hold a row at 16 elements each; the narrowest rows go by twos
  if (a.dim <= 256) launch_fwd_shape<TX, TY, 32, 1, 2>(q, vec, st);
  else if (a.dim <= 512) launch_fwd_shape<TX, TY, 32, 2, 1>(q, vec, st);
  else if (a.dim <= 1024) launch_fwd_shape<TX, TY, 64, 2, 1>(q, vec, st);
  else if (a.dim <= 2048) launch_fwd_shape<TX, TY, 128, 2, 1>(q, vec, st);
  else if (a.dim <= 4096) launch_fwd_shape<TX, TY, 256, 2, 1>(q, vec, st);
  else if (a.dim <= 8192) launch_fwd_shape<TX, TY, 512, 2, 1>(q, vec, st);
  else launch_fwd_shape<TX, TY, 1024, 2, 1>(q, vec, st);
}

}  // namespace mixaq
