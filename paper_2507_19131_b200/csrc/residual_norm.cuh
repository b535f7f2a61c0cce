// What the forward and the backward kernel of the norms at a sublayer's border share.
#pragma once
#include "fp8.cuh"
#include "kernels.h"

namespace mixaq {

enum NormKind { NORM_NONE = 0, NORM_LAYER = 1, NORM_RMS = 2 };

// A row is held by TPR threads: thread l has the eight-element vectors l, l + TPR, ...  Sums over the row, two at a time: shuffles,
// and for more than a warp one exchange through shared memory.  The buffers alternate: a warp that is at the reduction after the next
// has passed the barrier of the next one, which every warp reaches after it has read this one's sums.
template <int TPR>
struct RowReduce {
  float2 (*slots)[TPR / 32];                   // [2][warps of the row]
  int turn = 0;
  __device__ __forceinline__ float2 sum(float a, float b) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      a = __fadd_rn(a, __shfl_xor_sync(0xffffffffu, a, o));
      b = __fadd_rn(b, __shfl_xor_sync(0xffffffffu, b, o));
    }
    if constexpr (TPR > 32) {
      constexpr int W = TPR / 32;
      const int lane = threadIdx.x & 31;
      if (lane == 0) slots[turn][threadIdx.x >> 5] = make_float2(a, b);
      __syncthreads();
      const float2 v = slots[turn][lane & (W - 1)];
      turn ^= 1;
      a = v.x; b = v.y;
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1) {
        a = __fadd_rn(a, __shfl_xor_sync(0xffffffffu, a, o));
        b = __fadd_rn(b, __shfl_xor_sync(0xffffffffu, b, o));
      }
    }
    return make_float2(a, b);
  }
};

__device__ __forceinline__ float reciprocal_deviation(float squares, float inv_dim, float eps) {
  return __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(squares, inv_dim, eps)));
}

// eight entries of a vector of parameters; `other` where there is none
__device__ __forceinline__ void load_params8(const float* p, float other, int c, int n, bool vec, float (&f)[8]) {
  if (p && n > 0) {
    Vec8<float> r;
    if (vec && n >= 8) load_vec8(p + c, r);
    else load_some8(p + c, n, r);
    unpack8(r, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = other;
  }
}

// gate values of a row, ones without a gate
template <class TY>
__device__ __forceinline__ void load_gate8(const ResNormArgs& p, long gate_row, int c, int n, bool vec, float (&f)[8]) {
  if (p.gate && n > 0) {
    const long at = gate_row * p.gate_stride + c;
    if (p.gate_f32) {
      Vec8<float> r;
      const float* g = static_cast<const float*>(p.gate) + at;
      if (vec && n >= 8) load_vec8(g, r);
      else load_some8(g, n, r);
      unpack8(r, f);
    } else {
      Vec8<TY> r;
      const TY* g = static_cast<const TY*>(p.gate) + at;
      if (vec && n >= 8) load_vec8(g, r);
      else load_some8(g, n, r);
      unpack8(r, f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.0f;
  }
}

// host: whether every row of a matrix (element size `size`) starts on a 16-byte boundary
inline bool rows_aligned(const void* p, long stride, size_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (long)size % 16 == 0;
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
