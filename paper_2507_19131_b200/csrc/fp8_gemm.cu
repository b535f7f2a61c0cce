// Product of two e4m3 matrices with block scales (mixaq_fp8_matmul) on the 5th-generation tensor cores (tcgen05.mma kind::f8f6f4).
//
//   y(m, n) = sum_b sa(m, b) sw(n, b) d_b(m, n) + bias(n),   d_b(m, n) = sum of the 128 products of k-block b
//
// The scales change from k-block to k-block, so the tensor memory holds one k-block's sums d_b at a time and the epilogue warps keep the
// running sums in registers: per k-block they read d_b (tcgen05.ld) and add scale * d_b with packed fused multiply-adds, while the tensor
// core fills the next accumulator.  A k-block of a 128 x BN tile takes the tensor core BN cycles (8 192 multiply-adds a cycle and SM) and
// the FMA pipe BN / 2 (128 packed lanes a cycle).  What bounds it is neither, but the way of an accumulator: full, read, summed, free, next
// MMA.  A pair's k-block takes 730 cycles where its MMAs are 512 (2048 x 4096 x 16384: 131 us, 2.1 PFLOP/s; 8192^3: 474 us, 2.3).
//
// One CTA per SM walks over 128 x BN output tiles: warp 0 feeds a ring of 128-byte-swizzled stages by TMA (no multicast), warp 1 issues
// the MMAs, warp 2 brings a k-block's column scales to shared memory where weights have a scale per row, warp 3 looks for ones far from
// one among them, warps 4-11 are the epilogue (warp w has rows 32 (w % 4) ... of the tile and half of its columns).  Where there are few
// tiles, a cluster of up to 8 CTAs divides the k-blocks of a tile and adds its parts through distributed shared memory, in the order of
// the ranks.
// Every wait on an mbarrier is bounded, as in gemm_tc.cu.
#include "kernels.h"
#include "fp8.cuh"
#include "tc_ptx.cuh"
#include <atomic>
#include <cstring>

namespace mixaq {
namespace {

constexpr int BM = 128, BK = 128, UMMA_K = 32;
constexpr int A_BYTES = BM * BK;
constexpr int EPI_WARPS = 8, FIRST_EPI = 4, THREADS = 32 * (FIRST_EPI + EPI_WARPS);
constexpr int STAGING = 2048;                  // bytes of an epilogue warp's store buffer: 32 rows of 64
constexpr int MAX_SPLIT = 8;
constexpr int MAX_SLOTS = 4, MAX_RING = 8;
// Tiles of 256 columns belong to pairs of CTAs (cta_group::2): 256 rows x 256 columns, 128 rows a CTA, each CTA loading its own rows of a
// and half of the weights' rows.  The others are a CTA's own.
__host__ __device__ constexpr bool paired(int bn) { return bn == 256; }
// Accumulators ("slots") in tensor memory: a pair's tile is multiplied in two halves of 128 columns that are committed one by one, so
// that four slots take turns and the sums of one half are read while the other one is multiplied.
__host__ __device__ constexpr int halves(int bn) { return paired(bn) ? 2 : 1; }
__host__ __device__ constexpr int slot_cols(int bn) { return bn / halves(bn); }
__host__ __device__ constexpr int tmem_cols(int bn) { return MAX_SLOTS * slot_cols(bn); }
__host__ __device__ constexpr int w_rows(int bn) { return paired(bn) ? bn / 2 : bn; }          // rows of the weights that a CTA loads
__host__ __device__ constexpr int stage_bytes(int bn) { return A_BYTES + w_rows(bn) * BK; }
__host__ __device__ constexpr int ring_stages(int bn) { return bn >= 128 ? 6 : MAX_RING; }
// Pairs keep 128 sums a thread: the side warpgroup gives up registers for them (4 x 72 + 8 x 216 of 12 x 168).
constexpr int SIDE_REGS = 72, EPI_REGS = 216;
// Scales come long before their k-block: a latency of 800 cycles out of the L2 and 1 500 out of memory stands against 256 to 512 cycles of a
// k-block (read two k-blocks ahead, every tile width took 750 cycles a k-block).  AHEAD k-blocks of the columns' scales are under way to
// shared memory; of the rows' scales, and of weights' with 128 rows, AHEAD_REGS (4, below) are under way to registers.  Four do not cover
// the latency where tiles are few and k-blocks many: 1536 x 384 x 66800 takes 121 us, and 90 with one scale for all of a's rows.
constexpr int AHEAD = 8;
// stage full, empty; slot full, empty; column scales full, looked at, empty; drain
constexpr int NUM_BARS = 2 * MAX_RING + 2 * MAX_SLOTS + 3 * AHEAD + 1;

__host__ __device__ constexpr int smem_total(int bn, bool cols) {
  return ring_stages(bn) * stage_bytes(bn) + EPI_WARPS * STAGING + (cols ? AHEAD * (bn * 4 + 4) : 0) + NUM_BARS * 8 + 16;
}

struct Params {
  Fp8MatmulArgs g;
  int M, N, k_blocks;
  int m_tiles, n_tiles, tiles;                 // (rows of a pair's tile: 256)
  int split;                                   // CTAs of a cluster that share a tile's k-blocks (1: none)
};

template <bool PAIR>
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// arrival, when the MMAs issued so far are done, on a barrier of this CTA (of a pair: on that of both)
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    mma_commit(bar);
}
// the same place in the shared memory of CTA `rank` of the cluster
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
// a TMA load into this CTA's shared memory that counts on a barrier of the pair's first CTA
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// An arrival on another CTA's barrier that hands over tensor memory only (tcgen05 fences order that): a release at cluster scope would wait
// for all memory operations of the thread, the scales in flight among them, and doubled the time of a k-block.
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t holder, uint32_t cols) {
  if constexpr (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(holder), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(holder), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t cols) {
  if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols) : "memory");
}
// N columns (8, 16 or 32) of the warp's 32 rows, one row per thread; valid after tmem_wait
template <int N>
__device__ __forceinline__ void tmem_ld_rows(uint32_t taddr, float (&r)[N]) {
  if constexpr (N == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(taddr));
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 16)
      asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
          : "=f"(r[i]), "=f"(r[i + 1]), "=f"(r[i + 2]), "=f"(r[i + 3]), "=f"(r[i + 4]), "=f"(r[i + 5]), "=f"(r[i + 6]), "=f"(r[i + 7]),
            "=f"(r[i + 8]), "=f"(r[i + 9]), "=f"(r[i + 10]), "=f"(r[i + 11]), "=f"(r[i + 12]), "=f"(r[i + 13]), "=f"(r[i + 14]), "=f"(r[i + 15])
          : "r"(taddr + (uint32_t)i));
  }
}
// waits for all loads; the registers pass through so that no use of them is scheduled ahead of it
template <int N>
__device__ __forceinline__ void tmem_wait(float (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+f"(r[i]), "+f"(r[i + 1]), "+f"(r[i + 2]), "+f"(r[i + 3]), "+f"(r[i + 4]), "+f"(r[i + 5]), "+f"(r[i + 6]), "+f"(r[i + 7]));
}

// eight columns of the warp's 32 rows, and the wait for all stores
__device__ __forceinline__ void tmem_st_rows(uint32_t taddr, const float (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
      ::"f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster(uint32_t addr, uint32_t rank) {
  const uint32_t a = cluster_addr(addr, rank);
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

// A block's sum is 0 or 2^-18 to 2^25 in magnitude (128 products of codes), so its product with a factor between 2^-100 and 2^100 is a normal
// number.  With a factor beyond, zeros apart, two scales' product, or a sum's with one of them, may leave binary32 where the result does
// not: k-blocks that have such a factor take a way of their own, on which rows and columns without one get the same bits as otherwise.  (NaN
// stays with the ordinary operations, which carry it on.)  The branch costs more than the question: 8192^3 takes 474 us with it and 466
// without, 2048 x 4096 x 4096 with a scale per row of the weights 55.1 and 50.6.  (8192^3 with the branch in front of the first load of tensor
// memory 482; with the question put a k-block ahead 499 to 505.  The latter, asked by the epilogue instead of a warp of its own, 58.9.)
__device__ __forceinline__ bool far_factor(float f, bool zero) {
  const float m = fabsf(f);
  return m > 0x1p100f || (m < 0x1p-100f && !zero);
}
// a w as two factors of about the same exponent: neither is infinite, and a sum times the first is normal if the result is.  (Exponents
// beyond +-250 end in infinity or zero all the same.)
__device__ __forceinline__ void split_factor(float a, float w, float& first, float& second) {
  const double p = __dmul_rn((double)a, (double)w);
  const int e = (int)((uint64_t)__double_as_longlong(p) >> 52 & 2047) - 1023;
  if (e > 1023) { first = (float)p; second = 1.0f; return; }                // an infinite scale
  const int c = max(min(e, 250), -250), h = c / 2;
  first = (float)__dmul_rn(p, __longlong_as_double((long long)(1023 + h - e) << 52));
  second = __int_as_float((127 + c - h) << 23);
}
// acc + d a w, rounded to binary32 once
__device__ __forceinline__ float add_far(float acc, float d, float a, float w) {
  return (float)__fma_rn((double)d, __dmul_rn((double)a, (double)w), (double)acc);
}

// c ? a : b, without a branch (which the compiler makes of it otherwise, and spills 300 bytes around 128 of them)
__device__ __forceinline__ float choose(bool c, float a, float b) {
  float r;
  asm("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tselp.f32 %0, %1, %2, p;\n\t}" : "=f"(r) : "f"(a), "f"(b), "r"((uint32_t)c));
  return r;
}

// n (<= E) elements of a row to memory, as one piece where all are there and the address allows it
template <class T, int E>
__device__ __forceinline__ void store_piece(T* p, const T (&v)[E], bool vec, int n) {
  if (vec && n >= E) {
    if constexpr (sizeof(T) * E == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(v);
    else *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(v);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) if (i < n) p[i] = v[i];
  }
}

// The warp's 32 rows x COLS columns, through its staging buffer: rows of P 16-byte pieces, piece p of row r at p ^ (r / 2), so that
// eight lanes with a row each and four lanes a row both spread over all banks; memory is written in 64-byte runs.
template <class T, int COLS>
__device__ __forceinline__ void store_tile(const float2 (&acc)[COLS / 2], uint8_t* staging, const Params& p, int row0, int col0, int lane) {
  constexpr int E = 16 / (int)sizeof(T), P = COLS / E < 4 ? COLS / E : 4, CHUNK = P * E, PER = 32 / P;
  T* const y = static_cast<T*>(p.g.y);
  const bool vec = reinterpret_cast<uintptr_t>(y) % 16 == 0 && p.g.y_stride * (long)sizeof(T) % 16 == 0;
  const float* bias = p.g.bias;
#pragma unroll
  for (int ch = 0; ch < COLS / CHUNK; ++ch) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
      T v[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int c = ch * CHUNK + q * E + i;
        float f = c & 1 ? acc[c / 2].y : acc[c / 2].x;
        if (bias) f = __fadd_rn(f, __ldg(bias + min(col0 + c, p.N - 1)));
        v[i] = from_f32<T>(f);
      }
      *reinterpret_cast<uint4*>(staging + lane * 64 + ((q ^ (lane >> 1)) & (P - 1)) * 16) = *reinterpret_cast<const uint4*>(v);
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int r = i * PER + lane / P, q = lane % P, col = col0 + ch * CHUNK + q * E;
      const uint4 w = *reinterpret_cast<const uint4*>(staging + r * 64 + ((q ^ (r >> 1)) & (P - 1)) * 16);
      T v[E];
      *reinterpret_cast<uint4*>(v) = w;
      if (row0 + r < p.M) store_piece<T, E>(y + (long)(row0 + r) * p.g.y_stride + col, v, vec, p.N - col);
    }
    __syncwarp();
  }
}

// Sum of the cluster's parts of a tile, 128 x BN binary32 in every CTA's shared memory at `part` (four-column piece q of row r at
// q ^ (r % 8)); this CTA adds and stores its share of the rows.
template <class T, int BN>
__device__ __forceinline__ void join_parts(uint32_t part, const Params& p, int rank, int m0, int n0, int tid) {
  T* const y = static_cast<T*>(p.g.y);
  const bool vec = reinterpret_cast<uintptr_t>(y) % 16 == 0 && p.g.y_stride * (long)sizeof(T) % 16 == 0;
  const int rows = BM / p.split;
  const float* bias = p.g.bias;
  for (int i = tid; i < rows * (BN / 4); i += EPI_WARPS * 32) {
    const int r = rank * rows + i / (BN / 4), q = i % (BN / 4), col = n0 + q * 4;
    if (m0 + r >= p.M || col >= p.N) continue;
    const uint32_t at = part + (uint32_t)((r * (BN / 4) + (q ^ (r & 7))) * 16);
    float4 s = ld_cluster(at, 0);
    for (int j = 1; j < p.split; ++j) {
      const float4 v = ld_cluster(at, j);
      s.x = __fadd_rn(s.x, v.x); s.y = __fadd_rn(s.y, v.y); s.z = __fadd_rn(s.z, v.z); s.w = __fadd_rn(s.w, v.w);
    }
    float f[4] = {s.x, s.y, s.z, s.w};
    T v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (bias) f[c] = __fadd_rn(f[c], __ldg(bias + min(col + c, p.N - 1)));
      v[c] = from_f32<T>(f[c]);
    }
    store_piece<T, 4>(y + (long)(m0 + r) * p.g.y_stride + col, v, vec, p.N - col);
  }
}

struct Ring {
  int slot = 0; uint32_t pass = 0;
  __device__ __forceinline__ void next(int n) { if (++slot == n) { slot = 0; pass ^= 1u; } }
};

// Tiles are walked in bands of 8 row tiles, so that the CTAs at work share rows of both operands in the L2.
constexpr int BAND = 8;
__device__ __forceinline__ void tile_at(const Params& p, int t, int& mt, int& nt) {
  const int per = BAND * p.n_tiles, band = t / per, in = t - band * per;
  const int height = min(BAND, p.m_tiles - band * BAND);
  nt = in / height;
  mt = band * BAND + in - nt * height;
}

// COLSCALE: the weights have a scale per row, so every column of a tile has one of its own
template <int BN, bool COLSCALE>
__global__ void __launch_bounds__(THREADS, 1)
k_fp8_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ Params p) {
  constexpr bool PAIR = paired(BN);
  constexpr int HALVES = halves(BN), SLOT_COLS = slot_cols(BN), RING = ring_stages(BN), STAGE = stage_bytes(BN), COLS = BN / 2;
  constexpr int SLOT_WARPS = EPI_WARPS / HALVES;              // epilogue warps that read a slot
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;     // swizzled tiles need 1024-byte alignment
  uint8_t* const smem = smem_raw + (base - raw);
  uint8_t* const staging = smem + RING * STAGE;
  float* const col_scales = reinterpret_cast<float*>(staging + EPI_WARPS * STAGING);      // [AHEAD][BN]
  uint64_t* const bars = reinterpret_cast<uint64_t*>(col_scales + (COLSCALE ? AHEAD * BN : 0));
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8u * MAX_RING, bar_tfull = bar_empty + 8u * MAX_RING;
  const uint32_t bar_tempty = bar_tfull + 8u * MAX_SLOTS, bar_cfull = bar_tempty + 8u * MAX_SLOTS, bar_cempty = bar_cfull + 8u * AHEAD;
  const uint32_t bar_clooked = bar_cempty + 8u * AHEAD, bar_drain = bar_clooked + 8u * AHEAD;
  uint32_t* const tmem_holder = reinterpret_cast<uint32_t*>(bars + NUM_BARS);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  int* const cols_far = reinterpret_cast<int*>(tmem_holder + 2);        // [AHEAD]: whether a k-block's column scales have a far one
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  uint32_t fills = 0;                          // TMA warp: fills of ring stages so far

  if (tid == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmA) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmW) : "memory");
  }
  if (tid == 0) {
    for (int s = 0; s < RING; ++s) { mbar_init(bar_full + 8u * s, 1u); mbar_init(bar_empty + 8u * s, 1u); }
    for (int a = 0; a < MAX_SLOTS; ++a) {
      mbar_init(bar_tfull + 8u * a, 1u); mbar_init(bar_tempty + 8u * a, SLOT_WARPS * (PAIR ? 2u : 1u));
    }
    for (int a = 0; a < AHEAD; ++a) { mbar_init(bar_cfull + 8u * a, 32u); mbar_init(bar_clooked + 8u * a, 1u); mbar_init(bar_cempty + 8u * a, EPI_WARPS); }
    mbar_init(bar_drain, 1u);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tmem_alloc<PAIR>(smem_u32(tmem_holder), (uint32_t)tmem_cols(BN));
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (PAIR) cluster_sync();                    // the other CTA's barriers are ready, too
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_holder;
  griddep_wait();                              // operands, scales and y may belong to earlier kernels
  griddep_launch();
  if (PAIR && warp < FIRST_EPI) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(SIDE_REGS));

  // this CTA's tiles and, where a cluster divides them, its share of the k-blocks
  const int per_cluster = PAIR ? 2 : p.split, rank = (int)(blockIdx.x % (unsigned)per_cluster);
  const int first = (int)(blockIdx.x / (unsigned)per_cluster), step = (int)(gridDim.x / (unsigned)per_cluster);
  const int kb0 = PAIR ? 0 : (int)((long)p.k_blocks * rank / p.split), kb1 = PAIR ? p.k_blocks : (int)((long)p.k_blocks * (rank + 1) / p.split);
  const int row_off = PAIR ? rank * BM : 0;    // of this CTA's rows in a tile
  constexpr int TILE_M = PAIR ? 2 * BM : BM;

  if (warp == 0) {
    // ---- TMA ----
    const bool leader = elect_one();
    Ring rp;
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += step) {
      int mt, nt;
      tile_at(p, t, mt, nt);
      for (int kb = kb0; kb < kb1; ++kb, rp.next(RING)) {
        const uint32_t o = 8u * (uint32_t)rp.slot, sa = base + (uint32_t)(rp.slot * STAGE);
        if (!mbar_wait_warp(bar_empty + o, rp.pass ^ 1u, abort_flag)) { ok = false; break; }
        ++fills;
        if (leader) {
          if constexpr (PAIR) {
            // both CTAs' bytes count on the first one's barrier; of each half of the columns a CTA has 64 rows
            const uint32_t full = cluster_addr(bar_full + o, 0);
            if (rank == 0) mbar_arrive_expect_tx(bar_full + o, 2u * (uint32_t)STAGE);
            tma_load_pair(sa, &tmA, kb * BK, mt * TILE_M + row_off, full);
            tma_load_pair(sa + A_BYTES, &tmW, kb * BK, nt * BN + rank * 64, full);
            tma_load_pair(sa + A_BYTES + 64 * BK, &tmW, kb * BK, nt * BN + 128 + rank * 64, full);
          } else {
            mbar_arrive_expect_tx(bar_full + o, (uint32_t)STAGE);
            tma_load_2d(sa, &tmA, kb * BK, mt * BM, bar_full + o);
            tma_load_2d(sa + A_BYTES, &tmW, kb * BK, nt * BN, bar_full + o);
          }
        }
        __syncwarp();
      }
    }
  } else if (warp == 1 && (!PAIR || rank == 0)) {
    // ---- MMA ----
    const bool leader = elect_one();
    // D binary32 (1 at bit 4), A and B e4m3 (0 at bits 7 and 10), N / 8, M / 16
    const uint32_t idesc = (1u << 4) | ((uint32_t)(SLOT_COLS >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
    const uint64_t adesc0 = smem_desc_sw128(base), bdesc0 = smem_desc_sw128(base + A_BYTES);
    // A half waits for its own slot only, so that the halves' readers take turns at the FMA pipe.
    Ring rp, ap;
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += step) {
      for (int kb = kb0; kb < kb1 && ok; ++kb, rp.next(RING)) {
        const uint32_t o = 8u * (uint32_t)rp.slot;
        const uint64_t so = (uint64_t)((uint32_t)(rp.slot * STAGE) >> 4);
#pragma unroll
        for (int h = 0; h < HALVES; ++h, ap.next(MAX_SLOTS)) {
          ok = mbar_wait_warp<true>(bar_tempty + 8u * (uint32_t)ap.slot, ap.pass ^ 1u, abort_flag) &&
               (h > 0 || mbar_wait_warp<true>(bar_full + o, rp.pass, abort_flag));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t d = tmem_base + (uint32_t)(ap.slot * SLOT_COLS);
          const uint64_t ad = adesc0 + so, bd = bdesc0 + so + (uint64_t)(h * 64 * BK >> 4);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < BK / UMMA_K; ++kk)
              mma_f8<PAIR>(d, ad + (uint64_t)(kk * (UMMA_K >> 4)), bd + (uint64_t)(kk * (UMMA_K >> 4)), idesc, kk > 0 ? 1u : 0u);
            if (h == HALVES - 1) commit<PAIR>(bar_empty + o);
            commit<PAIR>(bar_tfull + 8u * (uint32_t)ap.slot);
          }
          __syncwarp();
        }
      }
    }
  } else if (COLSCALE && warp == 2) {
    // ---- column scales of a tile's k-blocks ----
    Ring cp;
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += step) {
      int mt, nt;
      tile_at(p, t, mt, nt);
      const float* at[BN / 32];
#pragma unroll
      for (int i = 0; i < BN / 32; ++i) at[i] = p.g.w.scale + (long)min(nt * BN + i * 32 + lane, p.N - 1) * p.g.w.srs;
      for (int kb = kb0; kb < kb1; ++kb, cp.next(AHEAD)) {
        if (!mbar_wait_warp(bar_cempty + 8u * (uint32_t)cp.slot, cp.pass ^ 1u, abort_flag)) { ok = false; break; }
#pragma unroll
        for (int i = 0; i < BN / 32; ++i) cp_async4(smem_u32(col_scales + cp.slot * BN + i * 32 + lane), at[i] + (long)kb * p.g.w.scs);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar_cfull + 8u * (uint32_t)cp.slot) : "memory");
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (COLSCALE && warp == 3) {
    // ---- are there far ones among them? ----
    Ring cp;
    bool ok = true;
    for (int t = first; t < p.tiles && ok; t += step)
      for (int kb = kb0; kb < kb1; ++kb, cp.next(AHEAD)) {
        if (!mbar_wait_warp(bar_cfull + 8u * (uint32_t)cp.slot, cp.pass, abort_flag)) { ok = false; break; }
        bool far = false;
#pragma unroll
        for (int i = 0; i < BN / 32; ++i) {
          const float w = col_scales[cp.slot * BN + i * 32 + lane];
          far |= far_factor(w, w == 0.0f);
        }
        far = __any_sync(0xffffffffu, far);
        if (lane == 0) { cols_far[cp.slot] = far; mbar_arrive(bar_clooked + 8u * (uint32_t)cp.slot); }
        __syncwarp();
      }
  } else if (warp >= FIRST_EPI) {
    // ---- sums in registers, output ----
    if (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(EPI_REGS));
    const int q = warp & 3, half = (warp - FIRST_EPI) >> 2;
    // a pair's warps have whole slots (every second one), the others half the columns of every slot
    const int slot_step = HALVES, col_in_slot = HALVES == 2 ? 0 : half * COLS;
    const uint32_t tmem_q = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)col_in_slot;
    uint8_t* const my_staging = staging + (warp - FIRST_EPI) * STAGING;
    int slot = HALVES == 2 ? half : 0;
    uint32_t pass = 0;
    auto next_slot = [&]() { slot += slot_step; if (slot >= MAX_SLOTS) { slot -= MAX_SLOTS; pass ^= 1u; } };
    const int k_count = kb1 - kb0;
    auto place = [&](int t, int& row0, int& col0) {
      int mt, nt;
      tile_at(p, t, mt, nt);
      row0 = mt * TILE_M + row_off + q * 32; col0 = nt * BN + half * COLS;
    };
    // The scales of AHEAD_REGS k-blocks are in flight to registers, across tiles; they are multiplied when they are used (a product here
    // would wait for the loads).
    constexpr int AHEAD_REGS = 4;
    float a_next[AHEAD_REGS], w_next[AHEAD_REGS];
    int ahead_t = first, ahead_k = 0;
    const float *a_at = nullptr, *w_at = nullptr;
    auto fetch = [&](int i) {
      if (ahead_t >= p.tiles) return;
      if (ahead_k == 0) {
        int row0, col0;
        place(ahead_t, row0, col0);
        a_at = p.g.a.scale + (long)(min(row0 + lane, p.M - 1) / p.g.a.block_rows) * p.g.a.srs + (long)kb0 * p.g.a.scs;
        w_at = p.g.w.scale + (long)(min(col0, p.N - 1) / p.g.w.block_rows) * p.g.w.srs + (long)kb0 * p.g.w.scs;
      }
      a_next[i] = __ldg(a_at);
      if (!COLSCALE) w_next[i] = __ldg(w_at);
      a_at += p.g.a.scs; w_at += p.g.w.scs;
      if (++ahead_k == k_count) { ahead_k = 0; ahead_t += step; }
    };
#pragma unroll
    for (int i = 0; i < AHEAD_REGS; ++i) { a_next[i] = 0.0f; w_next[i] = 1.0f; fetch(i); }
    const uint32_t tempty_at = PAIR ? cluster_addr(bar_tempty, 0) : bar_tempty;
    int col_slot = 0; uint32_t col_pass = 0;
    bool ok = true;
    constexpr int LD = COLS < 32 ? COLS : 32;                 // columns of a load; the next one is in flight during the sums
    for (int t = first; t < p.tiles; t += step) {
      float2 acc[COLS / 2];
#pragma unroll
      for (int i = 0; i < COLS / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
      for (int k = 0; k < k_count; ++k, next_slot()) {
        const float a0 = a_next[0], w0 = w_next[0];
#pragma unroll
        for (int i = 0; i + 1 < AHEAD_REGS; ++i) { a_next[i] = a_next[i + 1]; w_next[i] = w_next[i + 1]; }
        fetch(AHEAD_REGS - 1);
        if (COLSCALE && !mbar_wait_warp<true>(bar_clooked + 8u * (uint32_t)col_slot, col_pass, abort_flag)) { ok = false; break; }
        const float* const cw = col_scales + col_slot * BN + half * COLS;
        // the factor of the row's sums; columns with scales of their own have theirs in front of it
        float s0 = COLSCALE ? a0 : __fmul_rn(a0, w0);
        const bool far = COLSCALE ? cols_far[col_slot] : far_factor(s0, a0 == 0.0f || w0 == 0.0f);
        const bool any_far = COLSCALE ? far : __any_sync(0xffffffffu, far);
        if (!mbar_wait_warp<true>(bar_tfull + 8u * (uint32_t)slot, pass, abort_flag)) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem_q + (uint32_t)(slot * SLOT_COLS);
        auto give_back = [&]() {                              // all is read: the tensor core may have the slot back
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if constexpr (PAIR) arrive_cluster(tempty_at + 8u * (uint32_t)slot);
            else mbar_arrive(bar_tempty + 8u * (uint32_t)slot);
          }
        };
        float r[2][LD];
        tmem_ld_rows(d, r[0]);
        if (!COLSCALE && any_far) {
          tmem_wait(r[0]);
          // a far row's sums are multiplied by the first of two factors where they lie; the others' by one
          float s1 = 1.0f;
          if (far) split_factor(a0, w0, s1, s0);
          __syncwarp();
#pragma unroll 1
          for (int c = 0; c < COLS; c += 8) {
            float v[8];
            tmem_ld_rows(d + (uint32_t)c, v);
            tmem_wait(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s1);
            tmem_st_rows(d + (uint32_t)c, v);
          }
          tmem_st_wait();
          tmem_ld_rows(d, r[0]);
        }
        if (!COLSCALE || !any_far) {
          const float4* const cs = reinterpret_cast<const float4*>(cw);
          const float2 s = f2(s0);
#pragma unroll
          for (int c = 0; c < COLS; c += LD) {
            float (&v)[LD] = r[(c / LD) & 1];
            tmem_wait(v);
            if (c + LD < COLS) tmem_ld_rows(d + (uint32_t)(c + LD), r[(c / LD + 1) & 1]);
            else give_back();
#pragma unroll
            for (int i = 0; i < LD; i += 4) {
              float2 d0 = make_float2(v[i], v[i + 1]), d1 = make_float2(v[i + 2], v[i + 3]);
              if (COLSCALE) {
                const float4 w = cs[(c + i) / 4];
                d0 = __fmul2_rn(d0, make_float2(w.x, w.y)); d1 = __fmul2_rn(d1, make_float2(w.z, w.w));
              }
              acc[(c + i) / 2] = __ffma2_rn(d0, s, acc[(c + i) / 2]);
              acc[(c + i) / 2 + 1] = __ffma2_rn(d1, s, acc[(c + i) / 2 + 1]);
            }
          }
        } else {
          // columns without such a factor get the same bits as above
          tmem_wait(r[0]);
#pragma unroll
          for (int c = 0; c < COLS; c += 8) {
            float v[8];
            tmem_ld_rows(d + (uint32_t)c, v);
            tmem_wait(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float& t = i & 1 ? acc[(c + i) / 2].y : acc[(c + i) / 2].x;
              const float w = cw[c + i], near = __fmaf_rn(__fmul_rn(v[i], w), a0, t);
              t = choose(far_factor(w, w == 0.0f), add_far(t, v[i], a0, w), near);
            }
          }
          give_back();
        }
        if (COLSCALE) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_cempty + 8u * (uint32_t)col_slot);
          if (++col_slot == AHEAD) { col_slot = 0; col_pass ^= 1u; }
        }
      }
      if (!ok) break;
      int out_row, out_col;
      place(t, out_row, out_col);
      if (p.split == 1) {
        if (p.g.y_dtype == DT_F32) store_tile<float, COLS>(acc, my_staging, p, out_row, out_col, lane);
        else if (p.g.y_dtype == DT_BF16) store_tile<__nv_bfloat16, COLS>(acc, my_staging, p, out_row, out_col, lane);
        else store_tile<__half, COLS>(acc, my_staging, p, out_row, out_col, lane);
      } else if (!PAIR) {
        // the part goes where the ring was: every stage has been multiplied when the last slot is full
        const int r = q * 32 + lane;
#pragma unroll
        for (int i = 0; i < COLS / 4; ++i) {
          const int piece = half * (COLS / 4) + i;
          *reinterpret_cast<float4*>(smem + (r * (BN / 4) + (piece ^ (r & 7))) * 16) =
              make_float4(acc[2 * i].x, acc[2 * i].y, acc[2 * i + 1].x, acc[2 * i + 1].y);
        }
      }
    }
  }

  __syncwarp();
  if (!PAIR && p.split > 1) {
    cluster_sync();
    if (warp >= FIRST_EPI) {
      int mt, nt;
      tile_at(p, first, mt, nt);
      const int e = tid - FIRST_EPI * 32;
      if (p.g.y_dtype == DT_F32) join_parts<float, BN>(base, p, rank, mt * BM, nt * BN, e);
      else if (p.g.y_dtype == DT_BF16) join_parts<__nv_bfloat16, BN>(base, p, rank, mt * BM, nt * BN, e);
      else join_parts<__half, BN>(base, p, rank, mt * BM, nt * BN, e);
    }
    cluster_sync();                            // nobody leaves while its part is being read
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (*abort_flag) {
    // A wait ran out: the copies issued must have landed and the MMAs issued must have retired before the CTA may exit (bounded).  The
    // copies of a pair count on the first CTA's barriers, which that CTA waits for; if it did not give up, all have been multiplied.
    const bool issuer = !PAIR || rank == 0;
    if (issuer && warp == 1 && elect_one()) commit<PAIR>(bar_drain);
    __syncthreads();
    if (tid == 0) {
      atomicExch(p.g.status, 1);
      auto drain = [](uint32_t bar, uint32_t parity) {
        for (uint32_t it = 0; it < (1u << 20); ++it) if (mbar_try_wait(bar, parity)) return;
      };
      if (issuer) {
        for (uint32_t s = 0; s < (uint32_t)RING; ++s)
          if (fills > s) drain(bar_full + 8u * s, (fills - 1u - s) / (uint32_t)RING & 1u);
        drain(bar_drain, 0u);
      }
    }
    __syncthreads();
  }
  if (PAIR) {
    cluster_sync();                            // the MMAs read and write both CTAs' memory
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  }
  if (warp == 2) tmem_dealloc<PAIR>(tmem_base, (uint32_t)tmem_cols(BN));
}

// ---- host side -------------------------------------------------------------------------------------------------------------
// rows of `cols` bytes, `stride` bytes apart; boxes of box_rows x 128 bytes with 128-byte swizzle, zeros outside
bool make_rows_map(CUtensorMap* m, const uint8_t* ptr, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
  cuuint32_t box[2] = {BK, box_rows}, estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Per device, once: opt in to the shared memory, check that the register shares fit into what the block is launched with, and count the
// CTAs or pairs that run at once.  0 on failure.
template <int BN, bool COLSCALE>
int set_up(int sms) {
  static_assert(smem_total(BN, COLSCALE) + 1024 <= 227 * 1024, "shared memory");
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev > 63) return 0;
  int at_once = known[dev].load(std::memory_order_acquire);
  if (at_once) return at_once;
  cudaFuncAttributes at;
  const auto kernel = k_fp8_gemm<BN, COLSCALE>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_total(BN, COLSCALE) + 1024) != cudaSuccess ||
      cudaFuncGetAttributes(&at, kernel) != cudaSuccess)
    return 0;
  if (paired(BN) && FIRST_EPI * SIDE_REGS + EPI_WARPS * EPI_REGS > (FIRST_EPI + EPI_WARPS) * at.numRegs) return 0;
  at_once = sms;
  if (paired(BN)) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(sms / 2 * 2)); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = smem_total(BN, COLSCALE) + 1024;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&at_once, kernel, &cfg) != cudaSuccess || at_once < 1) return 0;
  }
  known[dev].store(at_once, std::memory_order_release);
  return at_once;
}

// Tile width and split, from the product's sizes alone: the split is the order in which k-blocks are added, and the same call gives the same
// bits on every device.  A CTA (or pair) takes `block` microseconds a k-block and `store` a tile; a split adds its join.  The constants
// were fitted to the times of all widths and splits at 17 shapes from 1 x 1024 x 8192 to 2048 x 4096 x 16384: the choice is the fastest measured
// at 15 of them and within 6 % at the others.  (us: 1 x 4096 x 4096 by 128 columns in 4 parts 9.2, in 2 parts 10.1, whole 12.6, 32 columns
// whole 16.4; 1024 x 4096 x 4096 by pairs 22, 128 columns 30; 300 x 1000 x 1000 by 32 columns 5.6, 128 columns 7.7.)  A split is
// one round of clusters: where one too many waits for another to end the time doubles (16 clusters of 8 took 14.5 us where 8 took 7.2).  A
// GPC's SMs are no multiple of a cluster, and chips differ in how many each GPC has, so that AT_ONCE counts what the chip with the fewest had:
// 1536 x 384 x 66800 takes 134 us in two parts by 64 columns everywhere, where a chip with room for 36 clusters of 4 takes 131 by 128 columns in
// four, and one with room for 33 takes 161.
constexpr int AT_ONCE[4] = {148, 74, 33, 15};     // clusters of 1, 2, 4 and 8 CTAs
struct Plan { int bn, split; };
Plan pick_plan(int M, int N, int k_blocks) {
  Plan best = {0, 0};
  double best_cost = 0.0;
  for (int bn = 32; bn <= 256; bn *= 2) {
    const int rows = paired(bn) ? 2 * BM : BM, at_once = AT_ONCE[paired(bn) ? 1 : 0];
    const long tiles = (long)((M + rows - 1) / rows) * ((N + bn - 1) / bn);
    const double block = bn == 256 ? 0.52 : bn == 128 ? 0.32 : bn == 64 ? 0.29 : 0.26, store = bn == 256 ? 3.0 : bn == 128 ? 1.7 : bn == 64 ? 1.0 : 0.7;
    for (int split = 1, log2 = 0; split <= MAX_SPLIT; split *= 2, ++log2) {
      if (split > 1 && (paired(bn) || split > k_blocks || tiles > AT_ONCE[log2])) break;
      const long rounds = split > 1 ? 1 : (tiles + at_once - 1) / at_once;
      const double cost = rounds * ((k_blocks + split - 1) / split * block + store) + (split > 1 ? 1.5 + 0.07 * split : 0.0);
      if (!best.bn || cost <= best_cost) { best = {bn, split}; best_cost = cost; }
    }
  }
  return best;
}

template <int BN, bool COLSCALE>
bool launch_as(const Params& p, cudaStream_t st, int sms) {
  const int at_once = set_up<BN, COLSCALE>(sms);
  if (!at_once) return false;
  CUtensorMap mA, mW;
  if (!make_rows_map(&mA, p.g.a.codes, p.M, p.g.K, p.g.a.stride, BM) ||
      !make_rows_map(&mW, p.g.w.codes, p.N, p.g.K, p.g.w.stride, paired(BN) ? 64 : BN))
    return false;
  const int cluster = paired(BN) ? 2 : p.split;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(cluster * (p.split > 1 || p.tiles < at_once ? p.tiles : at_once)));
  cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = smem_total(BN, COLSCALE) + 1024; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, k_fp8_gemm<BN, COLSCALE>, mA, mW, p);
  ++g_launches;
  return true;
}

}  // namespace

bool launch_fp8_matmul(const Fp8MatmulArgs& g, cudaStream_t st) {
  Params p;
  p.g = g; p.M = (int)g.a.rows; p.N = (int)g.w.rows;
  p.k_blocks = (int)((g.K + BK - 1) / BK);
  const int sms = sm_count();
  const Plan plan = pick_plan(p.M, p.N, p.k_blocks);
  p.m_tiles = (p.M + (paired(plan.bn) ? 2 * BM : BM) - 1) / (paired(plan.bn) ? 2 * BM : BM);
  p.n_tiles = (p.N + plan.bn - 1) / plan.bn;
  if ((long)p.m_tiles * p.n_tiles >= (1L << 31) - sms) return false;
  p.tiles = p.m_tiles * p.n_tiles; p.split = plan.split;
  const bool cols = g.w.block_rows == 1;
  switch (plan.bn) {
    case 32:  return cols ? launch_as<32, true>(p, st, sms) : launch_as<32, false>(p, st, sms);
    case 64:  return cols ? launch_as<64, true>(p, st, sms) : launch_as<64, false>(p, st, sms);
    case 128: return cols ? launch_as<128, true>(p, st, sms) : launch_as<128, false>(p, st, sms);
    case 256: return cols ? launch_as<256, true>(p, st, sms) : launch_as<256, false>(p, st, sms);
  }
  return false;
}

}  // namespace mixaq
