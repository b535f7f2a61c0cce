// Quantizer to e4m3 codes with a scale per block (mixaq_fp8_quantize): one read of x, one write of the codes.
//
// Both kernels are bound by memory: an element takes 2 or 4 bytes in, 1 byte out, and about ten instructions.
#include "kernels.h"
#include "fp8.cuh"

namespace mixaq {
namespace {

// ---- a scale per row and 128 columns ----------------------------------------------------------------------------------------
// Sixteen lanes take a block, eight neighbouring elements each: the row is read in 256- or 512-byte runs, the codes leave in 128-byte
// runs, and the maximum is four shuffles.  A CTA has 64 rows of one column block, four of them in flight per lane: it needs no division,
// and its scales are neighbours in the order that products read fastest.
constexpr int ROW_THREADS = 256, ROW_UNROLL = 4, ROW_GROUPS = ROW_THREADS / 16, ROW_TILE = ROW_GROUPS * ROW_UNROLL;

template <class T>
__global__ void __launch_bounds__(ROW_THREADS) k_fp8_rows(const T* x, long row_stride, long rows, int cols, int kb_count, bool vec, bool pow2,
                                                          uint8_t* codes, long code_stride, float* scale, long srs, long scs) {
  const int l16 = threadIdx.x & 15, group = threadIdx.x >> 4;
  const unsigned rt = blockIdx.x / (unsigned)kb_count, kb = blockIdx.x - rt * (unsigned)kb_count;
  const long row0 = (long)rt * ROW_TILE + group;
  const int c = (int)kb * FP8_BLOCK + l16 * 8, n = max(min(cols - c, 8), 0);
  Vec8<T> raw[ROW_UNROLL];
#pragma unroll
  for (int u = 0; u < ROW_UNROLL; ++u) {
    const long row = row0 + u * ROW_GROUPS;
    if (vec && n == 8 && row < rows) load_vec8(x + row * row_stride + c, raw[u]);
    else load_some8(x + row * row_stride + c, row < rows ? n : 0, raw[u]);
  }
#pragma unroll
  for (int u = 0; u < ROW_UNROLL; ++u) {
    const long row = row0 + u * ROW_GROUPS;
    float f[8];
    unpack8(raw[u], f);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max_abs(m, f[i]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s, inv;
    block_scale(m, pow2, s, inv);
    if (row < rows) {
      store_codes(codes + row * code_stride + c, codes8(f, inv), n);
      if (l16 == 0) scale[row * srs + (long)kb * scs] = s;
    }
  }
}

// ---- 128 x 128 tiles: a scale per tile, or the transposed matrix (or both) -----------------------------------------------------
// Thread (group g of 16, lane l of 16) holds rows 8 g ... 8 g + 7 and columns 8 l ... 8 l + 7 of the tile in registers.  Transposed, its
// eight codes of a column are one 8-byte piece of an output row, exchanged through shared memory: piece g of output row c lies at
// g ^ (c / 8), which spreads both the writes (one g, sixteen c) and the reads (one c, sixteen g) of a half warp over all banks.
constexpr int TILE = 128, TILE_THREADS = 256;

template <class T, bool TRANSPOSE, bool TILE_SCALE>
__global__ void __launch_bounds__(TILE_THREADS) k_fp8_tiles(const T* x, long row_stride, long rows, long cols, long col_tiles, bool vec, bool pow2,
                                                            uint8_t* codes, long code_stride, float* scale, long srs, long scs) {
  __shared__ __align__(16) uint8_t exchange[TRANSPOSE ? TILE * TILE : 16];
  __shared__ float part[8][TILE];
  const int tid = threadIdx.x, l = tid & 15, g = tid >> 4, warp = tid >> 5;
  const long rt = blockIdx.x / col_tiles, ct = blockIdx.x - rt * col_tiles;
  const long r0 = rt * TILE + g * 8, c0 = ct * TILE + l * 8;
  const int n = (int)max(min(cols - c0, 8L), 0L);
  Vec8<T> raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const T* p = x + (r0 + i) * row_stride + c0;
    if (r0 + i < rows && n > 0) {
      if (vec && n == 8) load_vec8(p, raw[i]);
      else load_some8(p, n, raw[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) raw[i].v[j] = from_f32<T>(0.0f);
    }
  }
  if (TILE_SCALE) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max_abs(m, to_f32(raw[i].v[j]));
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
        unpack8(raw[i], f);
        if (r0 + i < rows) store_codes(codes + (r0 + i) * code_stride + c0, codes8(f, inv), n);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_f32(raw[i].v[j]);
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
      for (int i = 0; i < 8; ++i) m[j] = max_abs(m[j], to_f32(raw[i].v[j]));
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
      for (int i = 0; i < 8; ++i) f[i] = to_f32(raw[i].v[j]);
      const int c = l * 8 + j;
      *reinterpret_cast<uint2*>(exchange + c * TILE + ((g ^ l) << 3)) = codes8(f, part[0][c]);
    }
  }
  if constexpr (!TRANSPOSE) return;
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

template <class T>
void launch_typed(const Fp8QuantArgs& a, cudaStream_t st) {
  const T* x = static_cast<const T*>(a.x);
  const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && a.row_stride * sizeof(T) % 16 == 0;
  if (!a.transpose && a.block_rows == 1) {
    const long kb = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK, tiles = (a.rows + ROW_TILE - 1) / ROW_TILE * kb;
    k_fp8_rows<T><<<(unsigned)tiles, ROW_THREADS, 0, st>>>(x, a.row_stride, a.rows, (int)a.cols, (int)kb, vec, a.pow2, a.codes, a.code_stride, a.scale,
                                                           a.scale_row_stride, a.scale_col_stride);
  } else {
    const long ct = (a.cols + TILE - 1) / TILE, tiles = ct * ((a.rows + TILE - 1) / TILE);
    auto run = [&](auto kernel) {
      kernel<<<(unsigned)tiles, TILE_THREADS, 0, st>>>(x, a.row_stride, a.rows, a.cols, ct, vec, a.pow2, a.codes, a.code_stride, a.scale,
                                                       a.scale_row_stride, a.scale_col_stride);
    };
    if (!a.transpose) run(k_fp8_tiles<T, false, true>);
    else if (a.block_rows == 1) run(k_fp8_tiles<T, true, false>);
    else run(k_fp8_tiles<T, true, true>);
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
