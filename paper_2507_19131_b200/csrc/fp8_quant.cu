// Quantizer to e4m3 codes with a scale per block (mixaq_fp8_quantize): one read of x, one write of the codes.
//
// Both kernels are bound by memory: an element takes 2 or 4 bytes in, 1 byte out, and about ten instructions.  What they need is loads in
// flight all the time, so CTAs stay and load their next tile into registers while they work on the present one.
#include "kernels.h"
#include "fp8.cuh"
#include <atomic>
#include <type_traits>

namespace mixaq {
namespace {

// Eight consecutive elements as the 32-bit words they lie in.  Held as 16-bit elements across an iteration the compiler gives each a
// register of its own (158 of them in the kernel of rows, and 42 us for 66800 x 384 instead of 21, eight rows a lane).
template <class T> struct Words8 {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* p, bool vec, int n) {                        // zeros from element `n` on (n may be 0 or less)
    if (vec && n == 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(w)[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = i < n ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
    } else {
      const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? __ldg(q + 2 * i) : 0u) | (2 * i + 1 < n ? (uint32_t)__ldg(q + 2 * i + 1) << 16 : 0u);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu)));
  }
};

// ---- a scale per row and 128 columns ----------------------------------------------------------------------------------------
// Sixteen lanes take a block, eight neighbouring elements each: the row is read in 256- or 512-byte runs, the codes leave in 128-byte
// runs, and the maximum is four shuffles.  A CTA has 64 rows (binary32: 32) of one column block at a time,
// so that its scales are neighbours in the order that products read fastest: 64 bytes of a lane in flight.  66800 x 384: bfloat16 16.4 us
// with four rows a lane (17.3 with two, 20.9 with eight; 24.8 when every tile had a CTA of its own), binary32 22.4 us with two (23.7 with
// four).  Copy bandwidth would take 11.9 and 19.7.
constexpr int ROW_THREADS = 256, ROW_GROUPS = ROW_THREADS / 16;
template <class T> __host__ __device__ constexpr int row_unroll() { return 8 / sizeof(T); }
template <class T> __host__ __device__ constexpr int row_tile() { return ROW_GROUPS * row_unroll<T>(); }

template <class T>
__global__ void __launch_bounds__(ROW_THREADS) k_fp8_rows(const T* x, long row_stride, long rows, int cols, int kb_count, unsigned tiles, bool vec, bool pow2,
                                                          uint8_t* codes, long code_stride, float* scale, long srs, long scs) {
  constexpr int ROW_UNROLL = row_unroll<T>(), ROW_TILE = row_tile<T>();
  const int l16 = threadIdx.x & 15, group = threadIdx.x >> 4;
  struct Tile { long row0; unsigned kb; int c, n; Words8<T> raw[ROW_UNROLL]; };
  auto fetch = [&](unsigned t, Tile& d) {
    const unsigned rt = t / (unsigned)kb_count;
    d.kb = t - rt * (unsigned)kb_count;
    d.row0 = (long)rt * ROW_TILE + group;
    d.c = (int)d.kb * FP8_BLOCK + l16 * 8;
    d.n = max(min(cols - d.c, 8), 0);
#pragma unroll
    for (int u = 0; u < ROW_UNROLL; ++u) {
      const long row = d.row0 + u * ROW_GROUPS;
      d.raw[u].load(x + row * row_stride + d.c, vec, row < rows ? d.n : 0);
    }
  };
  Tile now;
  fetch(blockIdx.x, now);
  for (unsigned t = blockIdx.x; t < tiles; t += gridDim.x) {
    Tile next;
    if (t + gridDim.x < tiles) fetch(t + gridDim.x, next);
#pragma unroll
    for (int u = 0; u < ROW_UNROLL; ++u) {
      const long row = now.row0 + u * ROW_GROUPS;
      float f[8];
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_abs(m, f[i] = now.raw[u].at(i));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
      float s, inv;
      block_scale(m, pow2, s, inv);
      if (row < rows) {
        store_codes(codes + row * code_stride + now.c, codes8(f, inv), now.n);
        if (l16 == 0) scale[row * srs + (long)now.kb * scs] = s;
      }
    }
    now = next;
  }
}

// ---- 128 x 128 tiles: a scale per tile, or the transposed matrix (or both) -----------------------------------------------------
// Thread (group g of 16, lane l of 16) holds rows 8 g ... 8 g + 7 and columns 8 l ... 8 l + 7 of the tile in registers.  Transposed, its
// eight codes of a column are one 8-byte piece of an output row, exchanged through shared memory: piece g of output row c lies at
// g ^ (c / 8), which spreads both the writes (one g, sixteen c) and the reads (one c, sixteen g) of a half warp over all banks.
// 66801 x 1000 bfloat16 transposed: 53 us (79 when every tile had a CTA of its own; copy bandwidth 31); 8192 x 8192 with 128 x 128 scales
// 35 us from bfloat16 and 57 us from binary32 (31 and 51).
constexpr int TILE = 128, TILE_THREADS = 256;

template <class T, bool TRANSPOSE, bool TILE_SCALE>
__global__ void __launch_bounds__(TILE_THREADS) k_fp8_tiles(const T* x, long row_stride, long rows, long cols, long col_tiles, unsigned tiles, bool vec, bool pow2,
                                                            uint8_t* codes, long code_stride, float* scale, long srs, long scs) {
  __shared__ __align__(16) uint8_t exchange[TRANSPOSE ? TILE * TILE : 16];
  __shared__ float part[8][TILE];
  const int tid = threadIdx.x, l = tid & 15, g = tid >> 4, warp = tid >> 5;
  auto fetch = [&](unsigned t, Words8<T> (&d)[8]) {
    const long rt = t / (unsigned)col_tiles, ct = t - rt * col_tiles, r0 = rt * TILE + g * 8, c0 = ct * TILE + l * 8;
    const int n = (int)max(min(cols - c0, 8L), 0L);
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i].load(x + (r0 + i) * row_stride + c0, vec, r0 + i < rows ? n : 0);
  };
  Words8<T> raw[8], next[8];
  fetch(blockIdx.x, raw);
  for (unsigned t = blockIdx.x; t < tiles; t += gridDim.x) {
    if (t + gridDim.x < tiles) fetch(t + gridDim.x, next);
    const long rt = t / (unsigned)col_tiles, ct = t - rt * col_tiles;
    const long r0 = rt * TILE + g * 8, c0 = ct * TILE + l * 8;
    const int n = (int)max(min(cols - c0, 8L), 0L);
    if (TILE_SCALE) {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_abs(m, raw[i].at(j));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
      if ((tid & 31) == 0) part[warp][0] = m;
      __syncthreads();
      m = 0.0f;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = max_abs(m, part[w][0]);
      float s, inv;
      block_scale(m, pow2, s, inv);
      if (tid == 0) scale[(TRANSPOSE ? ct : rt) * srs + (TRANSPOSE ? rt : ct) * scs] = s;
      if constexpr (!TRANSPOSE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = raw[i].at(j);
          if (r0 + i < rows) store_codes(codes + (r0 + i) * code_stride + c0, codes8(f, inv), n);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float f[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = raw[i].at(j);
          const int c = l * 8 + j;
          *reinterpret_cast<uint2*>(exchange + c * TILE + ((g ^ l) << 3)) = codes8(f, inv);
        }
      }
    } else {
      // maxima of the eight columns over the thread's rows, over the warp's two groups, over the warps
      float m[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m[j] = max_abs(m[j], raw[i].at(j));
        m[j] = max_abs(m[j], __shfl_xor_sync(0xffffffffu, m[j], 16));
      }
      if ((tid & 16) == 0) {
        reinterpret_cast<float4*>(&part[warp][l * 8])[0] = make_float4(m[0], m[1], m[2], m[3]);
        reinterpret_cast<float4*>(&part[warp][l * 8])[1] = make_float4(m[4], m[5], m[6], m[7]);
      }
      __syncthreads();
      if (tid < TILE) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v = max_abs(v, part[w][tid]);
        float s, inv;
        block_scale(v, pow2, s, inv);
        part[0][tid] = inv;
        const long c = ct * TILE + tid;
        if (c < cols) scale[c * srs + rt * scs] = s;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = raw[i].at(j);
        const int c = l * 8 + j;
        *reinterpret_cast<uint2*>(exchange + c * TILE + ((g ^ l) << 3)) = codes8(f, part[0][c]);
      }
    }
    if constexpr (TRANSPOSE) {
      __syncthreads();
      // output rows (the tile's columns) 16 at a time, sixteen lanes a row
      const int left = (int)max(min(rows - rt * TILE - l * 8, 8L), 0L);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = i * 16 + g;
        if (ct * TILE + c < cols)
          store_codes(codes + (ct * TILE + c) * code_stride + rt * TILE + l * 8, *reinterpret_cast<uint2*>(exchange + c * TILE + ((l ^ (c >> 3)) << 3)), left);
      }
    }
    __syncthreads();                             // (shared memory is used again for the next tile)
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = next[i];
  }
}

// resident CTAs of a kernel on the device (asked once per kernel and device)
template <auto kernel> unsigned resident(int threads) {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev > 63) dev = 0;
  n = known[dev].load(std::memory_order_relaxed);
  if (!n) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0) != cudaSuccess || n < 1) n = 1;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return (unsigned)(n * sm_count());
}

template <class T>
void launch_typed(const Fp8QuantArgs& a, cudaStream_t st) {
  const T* x = static_cast<const T*>(a.x);
  const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && a.row_stride * sizeof(T) % 16 == 0;
  if (!a.transpose && a.block_rows == 1) {
    const long kb = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const unsigned tiles = (unsigned)((a.rows + row_tile<T>() - 1) / row_tile<T>() * kb), most = resident<k_fp8_rows<T>>(ROW_THREADS);
    k_fp8_rows<T><<<tiles < most ? tiles : most, ROW_THREADS, 0, st>>>(x, a.row_stride, a.rows, (int)a.cols, (int)kb, tiles, vec, a.pow2, a.codes, a.code_stride,
                                                                       a.scale, a.scale_row_stride, a.scale_col_stride);
  } else {
    const long ct = (a.cols + TILE - 1) / TILE;
    const unsigned tiles = (unsigned)(ct * ((a.rows + TILE - 1) / TILE));
    auto run = [&](auto kernel, unsigned most) {
      kernel<<<tiles < most ? tiles : most, TILE_THREADS, 0, st>>>(x, a.row_stride, a.rows, a.cols, ct, tiles, vec, a.pow2, a.codes, a.code_stride, a.scale,
                                                                   a.scale_row_stride, a.scale_col_stride);
    };
    if (!a.transpose) run(k_fp8_tiles<T, false, true>, resident<k_fp8_tiles<T, false, true>>(TILE_THREADS));
    else if (a.block_rows == 1) run(k_fp8_tiles<T, true, false>, resident<k_fp8_tiles<T, true, false>>(TILE_THREADS));
    else run(k_fp8_tiles<T, true, true>, resident<k_fp8_tiles<T, true, true>>(TILE_THREADS));
  }
  ++g_launches;
}

}  // namespace

void launch_fp8_quantize(const Fp8QuantArgs& a, cudaStream_t st) {
  if (a.dtype == DT_F32) launch_typed<float>(a, st);
  else if (a.dtype == DT_BF16) launch_typed<__nv_bfloat16>(a, st);
  else launch_typed<__half>(a, st);
}

}  // namespace mixaq
