// Host side of the row operators declared in include/mixaq.h (mixaq_fp8_quantize, mixaq_fp8_matmul, mixaq_residual_norm_*):
// checks of the arguments and launches.  Nothing here computes.
#include "context.h"
#include <cstdint>

using namespace mixaq;

namespace {

constexpr int64_t MAX_EXTENT = (1LL << 31) - 256;        // rows and columns: tile and TMA coordinates are 32-bit
constexpr int64_t MAX_STRIDE = 1LL << 40;                // of the TMA unit

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool dtype_ok(int t) { return t == MIXAQ_F32 || t == MIXAQ_BF16 || t == MIXAQ_F16; }
size_t dtype_size(int t) { return t == MIXAQ_F32 ? 4 : 2; }

// the kernels run on the current device; the context's status word and the caller's buffers belong to the context's
mixaq_status check_device(mixaq_ctx* ctx) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return fail(ctx, MIXAQ_CUDA_ERROR, "no current device"); }
  if (dev != ctx->device) return fail(ctx, MIXAQ_INVALID_ARG, "the current device is not the context's device");
  return MIXAQ_OK;
}

mixaq_status check_matrix(mixaq_ctx* ctx, const mixaq_fp8_matrix* m, bool output) {
  if (!m) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix is NULL");
  if (m->rows < 0 || m->cols < 1) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: rows must not be negative, cols at least 1");
  if (m->rows > MAX_EXTENT || m->cols > MAX_EXTENT || m->row_stride >= MAX_STRIDE)
    return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8 matrix: too many rows or columns, or too long a stride");
  if (m->block_rows != 1 && m->block_rows != 128) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: block_rows must be 1 or 128");
  if (m->row_stride < m->cols || m->row_stride % 16) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: row_stride must be a multiple of 16 and at least cols");
  if (m->scale_row_stride < 0 || m->scale_col_stride < 0) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: negative scale stride");
  if (m->scale_row_stride >= MAX_STRIDE || m->scale_col_stride >= MAX_STRIDE) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8 matrix: too long a scale stride");
  if (output) {
    const int64_t rb = ceil_div(m->rows, m->block_rows), cb = ceil_div(m->cols, 128), sr = m->scale_row_stride, sc = m->scale_col_stride;
    const bool apart = (rb <= 1 || sr >= 1) && (cb <= 1 || sc >= 1) && (rb <= 1 || cb <= 1 || sr > (cb - 1) * sc || sc > (rb - 1) * sr);
    if (!apart) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: scales of the output share places");
  }
  if (m->rows == 0) return MIXAQ_OK;
  if (!m->codes || !m->scale) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: codes or scale is NULL");
  if (!aligned_to(m->codes, 16) || !aligned_to(m->scale, 4)) return fail(ctx, MIXAQ_INVALID_ARG, "fp8 matrix: codes must be 16-byte aligned, scale 4-byte");
  return MIXAQ_OK;
}

Fp8Operand operand(const mixaq_fp8_matrix& m) {
  return {m.codes, (long)m.rows, (long)m.row_stride, m.block_rows, m.scale, (long)m.scale_row_stride, (long)m.scale_col_stride};
}

}  // namespace

extern "C" {

mixaq_status mixaq_fp8_quantize(mixaq_ctx* ctx, const void* x, mixaq_dtype dtype, int64_t rows, int64_t cols, int64_t row_stride,
                                int transpose, int pow2, const mixaq_fp8_matrix* out, void* cuda_stream) {
  if (!ctx) return MIXAQ_INVALID_ARG;
  ctx->launches = 0;
  if (!dtype_ok(dtype)) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: unknown dtype");
  if (rows < 0 || cols < 0) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: rows and cols must not be negative");
  if (rows > MAX_EXTENT || cols > MAX_EXTENT || row_stride >= MAX_STRIDE) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8_quantize: too many rows or columns, or too long a stride");
  if (row_stride < cols) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: row_stride is below cols");
  if (!out) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: out is NULL");
  if (out->rows != (transpose ? cols : rows) || out->cols != (transpose ? rows : cols)) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: out has another shape than x");
  if (rows == 0 || cols == 0) return MIXAQ_OK;
  if (mixaq_status s = check_matrix(ctx, out, true)) return s;
  if (!x || !aligned_to(x, dtype_size(dtype))) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_quantize: x is NULL or not aligned to its elements");
  if (rows * ceil_div(cols, 128) >= MAX_EXTENT) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8_quantize: too many blocks");
  if (mixaq_status s = check_device(ctx)) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  Fp8QuantArgs a;
  a.x = x; a.dtype = dtype; a.rows = rows; a.cols = cols; a.row_stride = row_stride;
  a.transpose = transpose != 0; a.pow2 = pow2 != 0; a.block_rows = out->block_rows;
  a.codes = out->codes; a.code_stride = out->row_stride; a.scale = out->scale;
  a.scale_row_stride = out->scale_row_stride; a.scale_col_stride = out->scale_col_stride;
  g_launches = 0;
  try {
    ProfScope scope(ctx, PC_FP8_QUANT, st);
    launch_fp8_quantize(a, st);
  } catch (...) { return fail(ctx, MIXAQ_INTERNAL, "fp8_quantize: out of host memory"); }
  ctx->launches = g_launches;
  return check_cuda(ctx, "fp8_quantize");
}

mixaq_status mixaq_fp8_matmul(mixaq_ctx* ctx, const mixaq_fp8_matrix* a, const mixaq_fp8_matrix* w, const float* bias,
                              void* y, mixaq_dtype y_dtype, int64_t y_row_stride, void* cuda_stream) {
  if (!ctx) return MIXAQ_INVALID_ARG;
  ctx->launches = 0;
  if (mixaq_status s = check_matrix(ctx, a, false)) return s;
  if (mixaq_status s = check_matrix(ctx, w, false)) return s;
  if (!dtype_ok(y_dtype)) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_matmul: unknown y_dtype");
  if (a->cols != w->cols) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_matmul: a and w differ in columns");
  if (y_row_stride < w->rows) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_matmul: y_row_stride is below the columns of y");
  if (y_row_stride >= MAX_STRIDE) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8_matmul: too long a stride");
  if (a->rows == 0 || w->rows == 0) return MIXAQ_OK;
  if (!y || !aligned_to(y, dtype_size(y_dtype)) || !aligned_to(bias, 4)) return fail(ctx, MIXAQ_INVALID_ARG, "fp8_matmul: y is NULL, or y or bias not aligned to its elements");
  if (ceil_div(a->rows, 128) * ceil_div(w->rows, 32) >= MAX_EXTENT) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "fp8_matmul: too many tiles");
  if (mixaq_status s = check_device(ctx)) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  Fp8MatmulArgs g;
  g.a = operand(*a); g.w = operand(*w); g.K = a->cols;
  g.bias = bias; g.y = y; g.y_dtype = y_dtype; g.y_stride = y_row_stride; g.status = ctx->d_status;
  g_launches = 0;
  bool ok = false;
  try {
    ProfScope scope(ctx, PC_FP8_MATMUL, st);
    ok = launch_fp8_matmul(g, st);
  } catch (...) { return fail(ctx, MIXAQ_INTERNAL, "fp8_matmul: out of host memory"); }
  ctx->launches = g_launches;
  if (!ok) { cudaGetLastError(); return fail(ctx, MIXAQ_INTERNAL, "fp8_matmul: launch set-up failed (tensor map, shared memory or registers)"); }
  return check_cuda(ctx, "fp8_matmul");
}

}  // extern "C"
