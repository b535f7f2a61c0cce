// Which bytes the norms' ring copies of a row (csrc/residual_norm.cuh): row_span for matrices of given places and strides, on the host.
#include "../../paper_2507_19131_b200/csrc/residual_norm.cuh"

// first, last byte + 1 of the copy, relative to the row's first byte
extern "C" void row_copy(long address, long stride, long rows, int dim, int size, int vec, long row, long* lo, long* hi) {
  using namespace mixaq;
  const void* at = reinterpret_cast<const void*>(address);
  const RowSource s = size == 4 ? row_source<float>(at, stride, rows, dim) : row_source<__nv_bfloat16>(at, stride, rows, dim);
  const RowSpan r = vec ? row_span<true>(s, row) : row_span<false>(s, row);
  *lo = r.lo - r.start;
  *hi = r.hi - r.start;
}
