// What the forward and the backward kernel of the norms at a sublayer's border share.
#pragma once
#include "fp8.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"
#include <atomic>

namespace mixaq {

enum NormKind { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };

// A row is held by TPR threads ("worker": a CTA, or each of a CTA's four warps), 8 VPT elements a thread, in one of two orders:
//   VEC    thread l has the eight-element vectors l, l + TPR, ...: rows that start on 16-byte boundaries and are a multiple of eight
//          elements long, read and written 16 bytes at a time;
//   else   thread l has the elements l, l + TPR, ...: any row, read and written an element at a time, neighbours by neighbouring lanes.
// RING: rows come by bulk copies into a ring of stages in shared memory, several rows ahead.  The copies start and end on 16-byte
// boundaries: of a row that does not, the pieces that it shares with its neighbours come along, as far as they lie inside the matrix;
// what is left at the matrix's two ends is read from memory.  Without RING (rows too long for two stages) every element is.
template <int TPR> __host__ __device__ constexpr int cta_threads() { return TPR < 64 ? 128 : TPR; }
template <int TPR> __host__ __device__ constexpr int cta_workers() { return cta_threads<TPR>() / TPR; }
template <int TPR, bool VEC> __device__ __forceinline__ int column(int i, int j, int l) { return VEC ? (i * TPR + l) * 8 + j : (i * 8 + j) * TPR + l; }
// (rows in vector order are whole vectors)
template <int TPR, bool VEC> __device__ __forceinline__ bool present(int i, int j, int l, int dim) { return column<TPR, VEC>(i, VEC ? 0 : j, l) < dim; }

// Eight elements of a row, as pairs: the arithmetic works on two values at once.
struct F8 { float2 v[4]; };
__device__ __forceinline__ F8 fill8(float x) { return {{f2(x), f2(x), f2(x), f2(x)}}; }
__device__ __forceinline__ float2 unpack2(const float* p) { return make_float2(p[0], p[1]); }
__device__ __forceinline__ float2 unpack2(const __nv_bfloat16* p) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p)); }
__device__ __forceinline__ float2 unpack2(const __half* p) { return __half22float2(*reinterpret_cast<const __half2*>(p)); }
__device__ __forceinline__ void pack2(float* p, float2 f) { p[0] = f.x; p[1] = f.y; }
__device__ __forceinline__ void pack2(__nv_bfloat16* p, float2 f) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(f.x, f.y); }
__device__ __forceinline__ void pack2(__half* p, float2 f) { *reinterpret_cast<__half2*>(p) = __floats2half2_rn(f.x, f.y); }
// rounded to T and back
template <class T> __device__ __forceinline__ float2 round2(float2 f) {
  if constexpr (sizeof(T) == 4) return f;
  else { __align__(4) T t[2]; pack2(t, f); return unpack2(t); }
}
__device__ __forceinline__ float element(const F8& f, int j) { return j & 1 ? f.v[j / 2].y : f.v[j / 2].x; }

// eight elements (i, 0 ... 7) of a row; zeros where the row has none
template <int TPR, bool VEC, class T>
__device__ __forceinline__ F8 load_cols(const T* row, int i, int l, int dim) {
  F8 f = fill8(0.0f);
  if constexpr (VEC) {
    if (present<TPR, VEC>(i, 0, l, dim)) {
      Vec8<T> r;
      load_row8(row + column<TPR, VEC>(i, 0, l), r);
#pragma unroll
      for (int j = 0; j < 4; ++j) f.v[j] = unpack2(r.v + 2 * j);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      f.v[j] = make_float2(present<TPR, VEC>(i, 2 * j, l, dim) ? to_f32(row[column<TPR, VEC>(i, 2 * j, l)]) : 0.0f,
                           present<TPR, VEC>(i, 2 * j + 1, l, dim) ? to_f32(row[column<TPR, VEC>(i, 2 * j + 1, l)]) : 0.0f);
  }
  return f;
}
template <int TPR, bool VEC, class T>
__device__ __forceinline__ void store_cols(T* row, int i, int l, int dim, const F8& f) {
  if constexpr (VEC) {
    if (present<TPR, VEC>(i, 0, l, dim)) {
      Vec8<T> r;
#pragma unroll
      for (int j = 0; j < 4; ++j) pack2(r.v + 2 * j, f.v[j]);
      const uint4* from = reinterpret_cast<const uint4*>(&r);
      uint4* to = reinterpret_cast<uint4*>(row + column<TPR, VEC>(i, 0, l));
#pragma unroll
      for (int j = 0; j < (int)sizeof(Vec8<T>) / 16; ++j) to[j] = from[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (present<TPR, VEC>(i, j, l, dim)) row[column<TPR, VEC>(i, j, l)] = from_f32<T>(element(f, j));
  }
}
// zeros where the row has no elements
template <int TPR, bool VEC> __device__ __forceinline__ void mask_cols(F8& f, int i, int l, int dim) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (!present<TPR, VEC>(i, 2 * j, l, dim)) f.v[j].x = 0.0f;
    if (!present<TPR, VEC>(i, 2 * j + 1, l, dim)) f.v[j].y = 0.0f;
  }
}
__device__ __forceinline__ float sum8(const F8& f, float2 t) {
#pragma unroll
  for (int j = 0; j < 4; ++j) t = __fadd2_rn(t, f.v[j]);
  return __fadd_rn(t.x, t.y);
}

// One matrix whose rows pass through the ring
struct RowSource { const uint8_t* base; const uint8_t* end; long stride; uint32_t bytes; };      // bytes: of a row, stride and end too
template <class T> __host__ __device__ __forceinline__ RowSource row_source(const void* p, long stride, long rows, int dim) {
  const uint8_t* b = static_cast<const uint8_t*>(p);
  const uint32_t bytes = (uint32_t)(dim * sizeof(T));
  return {b, b + ((rows - 1) * stride * (long)sizeof(T) + bytes), stride * (long)sizeof(T), bytes};
}
// bytes that a row takes in a stage
template <bool VEC> __host__ __device__ __forceinline__ uint32_t staged_bytes(uint32_t row_bytes) { return VEC ? row_bytes : (row_bytes + 15) / 16 * 16 + 16; }
// what is copied of a row
struct RowSpan { const uint8_t *start, *lo, *hi; };
template <bool VEC> __host__ __device__ __forceinline__ RowSpan row_span(const RowSource& s, long row) {
  RowSpan r;
  r.start = s.base + row * s.stride;
  if (VEC) { r.lo = r.start; r.hi = r.start + s.bytes; return r; }
  r.lo = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(r.start) & ~(uintptr_t)15);
  r.hi = reinterpret_cast<const uint8_t*>((reinterpret_cast<uintptr_t>(r.start) + s.bytes + 15) & ~(uintptr_t)15);
  if (r.lo < s.base) r.lo += 16;
  if (r.hi > s.end) r.hi -= 16;
  if (r.hi < r.lo) r.hi = r.lo;
  return r;
}
// a row of this kind as a worker reads it
template <class T> struct StagedRow { const T *global, *staged; int lo, hi; };      // columns lo ... hi - 1 are staged
template <bool VEC, bool RING, class T>
__device__ __forceinline__ StagedRow<T> staged_row(const RowSource& s, long row, const uint8_t* at) {
  if (!RING) return {reinterpret_cast<const T*>(s.base + row * s.stride), nullptr, 0, 0};
  if (VEC) return {nullptr, reinterpret_cast<const T*>(at), 0, 0};
  const RowSpan r = row_span<VEC>(s, row);
  const int lo = (int)(r.lo - r.start) / (int)sizeof(T), hi = (int)(r.hi - r.start) / (int)sizeof(T);
  return {reinterpret_cast<const T*>(r.start), reinterpret_cast<const T*>(at) - lo, lo, hi};
}
template <int TPR, bool VEC, bool RING, class T>
__device__ __forceinline__ F8 load_staged(const StagedRow<T>& r, int i, int l, int dim) {
  if (!RING) return load_cols<TPR, VEC>(r.global, i, l, dim);
  if (VEC || (r.lo <= 0 && r.hi >= dim)) return load_cols<TPR, VEC>(r.staged, i, l, dim);
  auto at = [&](int j) {
    const int c = column<TPR, VEC>(i, j, l);
    return c >= dim ? 0.0f : to_f32(c >= r.lo && c < r.hi ? r.staged[c] : r.global[c]);
  };
  F8 f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f.v[j] = make_float2(at(2 * j), at(2 * j + 1));
  return f;
}
// parameters of the columns; `other` where there are none
template <int TPR, bool VEC>
__device__ __forceinline__ F8 load_params(const float* p, float other, int i, int l, int dim) { return p ? load_cols<TPR, VEC>(p, i, l, dim) : fill8(other); }
// gate values of a row, ones without a gate
template <int TPR, bool VEC, class TY>
__device__ __forceinline__ F8 load_gate(const ResNormArgs& p, long gate_row, int i, int l) {
  if (!p.gate) return fill8(1.0f);
  if (p.gate_f32) return load_cols<TPR, VEC>(static_cast<const float*>(p.gate) + gate_row * p.gate_stride, i, l, p.dim);
  return load_cols<TPR, VEC>(static_cast<const TY*>(p.gate) + gate_row * p.gate_stride, i, l, p.dim);
}

// Sums over a row, N (1, 2 or 4) values at a time.  In a warp the first steps exchange halves of the values instead of adding all of
// them everywhere: N - 1 shuffles for that, log2 P more (P = 32 / N) until lane P k has value k, N to hand them out; 5, 7 and 10 for one,
// two and four values.  More than a warp: one exchange through shared memory, and again.  The buffers alternate: a warp that is at the
// reduction after the next has passed the barrier of the next one, which every warp reaches after it has read this one's sums.
template <int TPR, int N>
struct RowReduce {
  float (*slots)[N][TPR / 32];                 // [2][N][warps of the row]
  int turn = 0;
  __device__ __forceinline__ void sum(float (&v)[N]) {
    constexpr unsigned ALL = 0xffffffffu;
    constexpr int P = 32 / N, W = TPR / 32;
    const int lane = threadIdx.x & 31;
    float a;
    if constexpr (N == 4) {
      const bool h = lane & 16, q = lane & 8;
      const float a0 = __fadd_rn(h ? v[2] : v[0], __shfl_xor_sync(ALL, h ? v[0] : v[2], 16));
      const float a1 = __fadd_rn(h ? v[3] : v[1], __shfl_xor_sync(ALL, h ? v[1] : v[3], 16));
      a = __fadd_rn(q ? a1 : a0, __shfl_xor_sync(ALL, q ? a0 : a1, 8));
    } else if constexpr (N == 2) {
      const bool h = lane & 16;
      a = __fadd_rn(h ? v[1] : v[0], __shfl_xor_sync(ALL, h ? v[0] : v[1], 16));
    } else {
      a = v[0];
    }
#pragma unroll
    for (int o = P / 2; o > 0; o >>= 1) a = __fadd_rn(a, __shfl_xor_sync(ALL, a, o));
    if constexpr (TPR > 32) {
      if ((lane & (P - 1)) == 0) slots[turn][lane / P][threadIdx.x >> 5] = a;
      __syncthreads();
      const float* from = slots[turn][lane / P];
      turn ^= 1;
      if constexpr (W > P) {
        a = from[lane & (P - 1)];
#pragma unroll
        for (int i = P; i < W; i += P) a = __fadd_rn(a, from[(lane & (P - 1)) + i]);
      } else {
        a = from[lane & (W - 1)];
      }
#pragma unroll
      for (int o = (W > P ? P : W) / 2; o > 0; o >>= 1) a = __fadd_rn(a, __shfl_xor_sync(ALL, a, o));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = N == 1 && TPR == 32 ? a : __shfl_sync(ALL, a, i * P);
  }
};

__device__ __forceinline__ float reciprocal_deviation(float squares, float inv_dim, float eps) {
  return __frsqrt_rn(__fmaf_rn(squares, inv_dim, eps));
}

// A worker's ring of stages: `stages` times `stage_bytes`, one full barrier each; all of a worker's threads use a stage up before the
// first of them refills it.
constexpr int MAX_STAGES = 4;
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
      ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// the copies of a row; the bytes that were asked for
template <bool VEC> __device__ __forceinline__ uint32_t span_bytes(const RowSource& s, long row) {
  if (VEC) return s.bytes;
  const RowSpan r = row_span<VEC>(s, row);
  return (uint32_t)(r.hi - r.lo);
}
template <bool VEC> __device__ __forceinline__ void fetch_row(const RowSource& s, long row, uint32_t dst, uint32_t bar) {
  const RowSpan r = row_span<VEC>(s, row);
  if (r.hi > r.lo) bulk_load(dst, r.lo, (uint32_t)(r.hi - r.lo), bar);
}
// bounded; false when the limit ran out
__device__ __forceinline__ bool wait_stage(uint32_t bar, uint32_t parity) {
  for (uint32_t it = 0; it < MAX_POLLS; ++it) if (mbar_try_wait(bar, parity)) return true;
  return false;
}
// When a wait ran out: the copies under way must have landed before the CTA may exit.  `used`: the stages filled so far.
__device__ __forceinline__ void drain_stages(uint32_t bar, int stages, long used, int* status) {
  atomicExch(status, 1);
  for (int i = 0; i < stages; ++i) {
    if (used <= i) continue;
    const uint32_t parity = (uint32_t)((used - 1 - i) / stages & 1);       // of the stage's last fill
    for (uint32_t it = 0; it < (1u << 20); ++it) if (mbar_try_wait(bar + 8u * (uint32_t)i, parity)) break;
  }
}
// one decision of all of a worker's threads, which have all arrived here then
template <int TPR> __device__ __forceinline__ bool worker_and(bool ok) {
  if constexpr (TPR > 32) return __syncthreads_and(ok) != 0;
  else return __all_sync(0xffffffffu, ok) != 0;
}

// host: whether a matrix (element size `size`) may be read and written 16 bytes at a time; no matrix may
inline bool rows_aligned(const void* p, long stride, size_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (long)size % 16 == 0;
}
// Stages of `stage_bytes` for the workers of a CTA, of which `ctas` at most share an SM: fewer CTAs where not even two stages fit, and
// no ring (0) where a single CTA has no room for them.
constexpr int RING_BYTES_PER_SM = 150 * 1024;
inline int ring_stages(long stage_bytes, int workers, int& ctas, long bytes_per_sm = RING_BYTES_PER_SM) {
  for (; ctas > 0; --ctas) {
    const long n = bytes_per_sm / ctas / workers / stage_bytes;
    if (n >= 2) return n > MAX_STAGES ? MAX_STAGES : (int)n;
  }
  ctas = 1;
  return 0;
}
// per device, once: the kernel may have a ring's shared memory
template <class K> inline void allow_ring(K* kernel, std::atomic<uint64_t>& done, int bytes = RING_BYTES_PER_SM) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (done.load(std::memory_order_acquire) >> (dev & 63) & 1) return;
  cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  done.fetch_or(1ull << (dev & 63), std::memory_order_release);
}

// calls f with tags of the types of the residual stream and of the sublayers
template <class F> void with_types(int x_dtype, int y_dtype, F f) {
  if (x_dtype == DT_F32) {
    if (y_dtype == DT_F32) f(float{}, float{});
    else if (y_dtype == DT_BF16) f(float{}, __nv_bfloat16{});
    else f(float{}, __half{});
  } else if (x_dtype == DT_BF16) f(__nv_bfloat16{}, __nv_bfloat16{});
  else f(__half{}, __half{});
}

}  // namespace mixaq
