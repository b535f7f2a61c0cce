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

// ---- norms ----
bool norm_ok(const mixaq_norm& n) {
  if (n.kind == MIXAQ_NORM_NONE) return true;
  return (n.kind == MIXAQ_NORM_LAYER || n.kind == MIXAQ_NORM_RMS) && n.eps > 0.f && n.eps <= 3.402823466e38f && aligned_to(n.gamma, 4) && aligned_to(n.beta, 4);
}
NormSpec norm_spec(const mixaq_norm& n) { return {(int)n.kind, n.gamma, n.beta, n.eps}; }

// a matrix of `size`-byte elements that has to be there: aligned, rows that do not overlap
bool rows_ok(const void* p, int64_t stride, int64_t dim, size_t size) { return p && aligned_to(p, size) && stride >= dim && stride < MAX_STRIDE; }

// what the forward and the backward call have in common
mixaq_status check_residual_norm(mixaq_ctx* ctx, const mixaq_residual_norm_params* p) {
  if (!p) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: params are NULL");
  if (p->rows < 0 || p->dim < 1) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: rows must not be negative, dim at least 1");
  if (p->rows > MAX_EXTENT || p->dim > MIXAQ_NORM_MAX_DIM) return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "residual_norm: too many rows, or dim beyond MIXAQ_NORM_MAX_DIM");
  if (!dtype_ok(p->x_dtype) || !dtype_ok(p->y_dtype)) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: unknown dtype");
  if (p->x_dtype != MIXAQ_F32 && p->x_dtype != p->y_dtype) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: a 16-bit x needs y of its own type");
  if (!norm_ok(p->post) || !norm_ok(p->pre)) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: norm kind unknown, eps not positive, or gamma or beta not 4-byte aligned");
  if (p->rows > 0 && !p->y && (p->gate || p->post.kind != MIXAQ_NORM_NONE)) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: gate or post norm without y");
  if (p->gate) {
    if (p->gate_dtype != p->y_dtype && p->gate_dtype != MIXAQ_F32) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: gate_dtype must be y_dtype or MIXAQ_F32");
    if (p->rows_per_gate < 1) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: rows_per_gate must be at least 1");
    if (p->gate_stride < 0 || p->gate_stride >= MAX_STRIDE || !aligned_to(p->gate, dtype_size(p->gate_dtype)))
      return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: gate stride out of range, or gate not aligned to its elements");
  }
  return MIXAQ_OK;
}

ResNormArgs norm_args(const mixaq_residual_norm_params& p) {
  ResNormArgs a = {};
  a.rows = p.rows; a.dim = p.dim; a.x_dtype = p.x_dtype; a.y_dtype = p.y_dtype;
  a.x = p.x; a.x_stride = p.x_stride; a.y = p.y; a.y_stride = p.y_stride;
  a.gate = p.gate; a.gate_stride = p.gate_stride; a.gate_f32 = p.gate_dtype == MIXAQ_F32;
  a.rows_per_gate = !p.gate || p.rows_per_gate > p.rows ? p.rows : p.rows_per_gate;       // (rows > 0 here)
  a.scale = p.scale; a.post = norm_spec(p.post); a.pre = norm_spec(p.pre);
  return a;
}
bool gate_per_sequence(const mixaq_residual_norm_params& p) { return p.gate && p.rows_per_gate > 1 && p.rows_per_gate < p.rows; }

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

mixaq_status mixaq_residual_norm_forward(mixaq_ctx* ctx, const mixaq_residual_norm_params* p, const mixaq_fp8_matrix* h_fp8, void* cuda_stream) {
  if (!ctx) return MIXAQ_INVALID_ARG;
  ctx->launches = 0;
  if (mixaq_status s = check_residual_norm(ctx, p)) return s;
  const bool pre = p->pre.kind != MIXAQ_NORM_NONE;
  if (pre ? (p->h && h_fp8) || (p->rows > 0 && !p->h && !h_fp8) : p->h || h_fp8) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: a pre norm needs h or h_fp8, one of them; none takes neither");
  if (p->rows > 0 && !pre && !p->y) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: neither y nor a pre norm");
  if (p->rows > 0 && !p->y && p->x_out) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: x_out without y");
  if (h_fp8) {
    if (h_fp8->rows != p->rows || h_fp8->cols != p->dim || h_fp8->block_rows != 1) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: h_fp8 has another shape than x, or block_rows other than 1");
    if (mixaq_status s = check_matrix(ctx, h_fp8, true)) return s;
  }
  if (p->rows == 0) return MIXAQ_OK;
  const size_t xs = dtype_size(p->x_dtype), ys = dtype_size(p->y_dtype);
  if (!rows_ok(p->x, p->x_stride, p->dim, xs) || (p->y && (!rows_ok(p->y, p->y_stride, p->dim, ys) || !rows_ok(p->x_out, p->x_out_stride, p->dim, xs))) ||
      (p->h && !rows_ok(p->h, p->h_stride, p->dim, ys)))
    return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: x, y, x_out or h missing, not aligned to its elements, or with a stride below dim");
  if ((p->x_out == p->x && p->x_out_stride != p->x_stride) || (p->h && p->h == p->y && p->h_stride != p->y_stride) ||
      (p->h && (p->h == p->x || p->h == p->x_out)) || (p->y && p->x_out == p->y))
    return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm: outputs overlap");
  if (mixaq_status s = check_device(ctx)) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  ResNormArgs a = norm_args(*p);
  a.x_out = p->x_out; a.x_out_stride = p->x_out_stride; a.h = p->h; a.h_stride = p->h_stride;
  if (h_fp8) {
    a.codes = h_fp8->codes; a.code_stride = h_fp8->row_stride; a.h_scale = h_fp8->scale;
    a.srs = h_fp8->scale_row_stride; a.scs = h_fp8->scale_col_stride; a.pow2 = p->pow2 != 0;
  }
  g_launches = 0;
  try {
    ProfScope scope(ctx, PC_RES_NORM, st);
    launch_residual_norm(a, ctx->d_status, st);
  } catch (...) { return fail(ctx, MIXAQ_INTERNAL, "residual_norm_forward: out of host memory"); }
  ctx->launches = g_launches;
  return check_cuda(ctx, "residual_norm_forward");
}

size_t mixaq_residual_norm_backward_workspace_bytes(const mixaq_residual_norm_params* p) {
  if (!p || p->rows < 0 || p->rows > MAX_EXTENT || p->dim < 1 || p->dim > MIXAQ_NORM_MAX_DIM) return 0;
  return residual_norm_backward_floats(p->rows, p->dim, gate_per_sequence(*p)) * sizeof(float);
}

mixaq_status mixaq_residual_norm_backward(mixaq_ctx* ctx, const mixaq_residual_norm_params* p, const mixaq_residual_norm_grads* g,
                                          void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!ctx) return MIXAQ_INVALID_ARG;
  ctx->launches = 0;
  if (mixaq_status s = check_residual_norm(ctx, p)) return s;
  if (!g) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: grads are NULL");
  const bool pre = p->pre.kind != MIXAQ_NORM_NONE, post = p->post.kind != MIXAQ_NORM_NONE;
  float* const vec[4] = {g->dpost_gamma, g->dpost_beta, g->dpre_gamma, g->dpre_beta};
  if ((!pre && (g->dh || vec[2] || vec[3])) || (!post && (vec[0] || vec[1])) || (p->rows > 0 && ((!p->y && g->dy) || (!p->gate && g->dgate))))
    return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: a gradient of something that is missing");
  for (const float* v : vec) if (!aligned_to(v, 4)) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: parameter gradients must be 4-byte aligned");
  if (p->rows > 0) {
    if (!g->dx_out && !g->dh) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: neither dx_out nor dh");
    const size_t xs = dtype_size(p->x_dtype), ys = dtype_size(p->y_dtype);
    if ((g->dh && !rows_ok(p->x, p->x_stride, p->dim, xs)) || (p->y && !rows_ok(p->y, p->y_stride, p->dim, ys)) ||
        (g->dx_out && !rows_ok(g->dx_out, g->dx_out_stride, p->dim, xs)) || (g->dh && !rows_ok(g->dh, g->dh_stride, p->dim, ys)) ||
        (g->dx && !rows_ok(g->dx, g->dx_stride, p->dim, xs)) || (g->dy && !rows_ok(g->dy, g->dy_stride, p->dim, ys)) ||
        (g->dgate && !rows_ok(g->dgate, g->dgate_stride, p->dim, 4)))
      return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: a matrix is missing, not aligned to its elements, or has a stride below dim");
    if ((g->dx && g->dx == g->dx_out && g->dx_stride != g->dx_out_stride) || (g->dy && g->dy == g->dh && g->dy_stride != g->dh_stride) ||
        (g->dy && g->dy == p->y && g->dy_stride != p->y_stride) ||
        (g->dx && (g->dx == p->x || g->dx == p->y || g->dx == g->dh || g->dx == g->dy)) || (g->dy && (g->dy == p->x || g->dy == g->dx_out)))
      return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: outputs overlap");
    if (gate_per_sequence(*p) && ceil_div(p->rows, p->rows_per_gate) * ceil_div(p->dim, 256) > MAX_EXTENT)
      return fail(ctx, MIXAQ_UNSUPPORTED_SHAPE, "residual_norm_backward: too many gates");
    if (!workspace || !aligned_to(workspace, 256)) return fail(ctx, MIXAQ_INVALID_ARG, "residual_norm_backward: workspace is NULL or not 256-byte aligned");
    if (mixaq_residual_norm_backward_workspace_bytes(p) > workspace_bytes) return fail(ctx, MIXAQ_WORKSPACE_TOO_SMALL, "residual_norm_backward: workspace too small");
  }
  if (mixaq_status s = check_device(ctx)) return s;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  g_launches = 0;
  if (p->rows == 0) {
    for (float* v : vec) if (v) cudaMemsetAsync(v, 0, (size_t)p->dim * sizeof(float), st);
    return check_cuda(ctx, "residual_norm_backward");
  }
  ResNormGradArgs a;
  a.dx_out = g->dx_out; a.dx_out_stride = g->dx_out_stride; a.dh = g->dh; a.dh_stride = g->dh_stride;
  a.dx = g->dx; a.dx_stride = g->dx_stride; a.dy = g->dy; a.dy_stride = g->dy_stride;
  a.dgate = g->dgate; a.dgate_stride = g->dgate_stride;
  for (int i = 0; i < 4; ++i) a.vec[i] = vec[i];
  a.workspace = static_cast<float*>(workspace);
  try {
    ProfScope scope(ctx, PC_RES_NORM, st);
    launch_residual_norm_backward(norm_args(*p), a, ctx->d_status, st);
  } catch (...) { return fail(ctx, MIXAQ_INTERNAL, "residual_norm_backward: out of host memory"); }
  ctx->launches = g_launches;
  return check_cuda(ctx, "residual_norm_backward");
}

}  // extern "C"
