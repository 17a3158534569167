// Dropout from a counter-based generator: kernel and C entries.  See include/prsgd.h for the contract.
//
// out = keep * x / (1 - q) (+ residual).  One pass over the arrays, nothing else is read or written; a thread takes eight columns, the
// 128 bits of one generator call: 16 bits decide for an element, so p is realised to 2^-16 and the scale is that of the
// realised q.  (32 bits an element, two calls: 114 us instead of 91 for 256 MB -> 256 MB of bf16, of which 89 with no generator
// at all.)  The counter is the element's place, not a thread's: any launch shape, type or stride draws the same.
#include <cmath>
#include "philox.h"
#include "rows_io.cuh"

using namespace prsgd;

namespace {

struct DropoutArgs {
  RowWalk walk;
  const void* x; int64_t x_row, x_group;
  const void* res; int64_t res_row, res_group;
  void* out; int64_t out_row, out_group;
  uint32_t threshold;        // an element goes when its 16 bits are below
  float scale;
  uint64_t seed;
  uint32_t step, group0;
  const int64_t* d_step;
};

template <int TY, bool VEC, bool RES>
__global__ void __launch_bounds__(kRowThreads) dropout_kernel(const DropoutArgs a) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const T* x = static_cast<const T*>(a.x) + g * a.x_group;
  const T* res = RES ? static_cast<const T*>(a.res) + g * a.res_group : nullptr;
  T* out = static_cast<T*>(a.out) + g * a.out_group;
  const uint32_t step = a.step + (a.d_step ? (uint32_t)*a.d_step : 0u);
  const int64_t first = (int64_t)blockIdx.x * kRowItems;
  const RowStart s = row_start(a.walk, first);
  int64_t row[kRowUnroll];
  uint32_t chunk[kRowUnroll];
  float v[kRowUnroll][8], r[kRowUnroll][8];
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    const uint32_t i = s.chunk + u * kRowThreads + threadIdx.x, over = a.walk.by_chunks.div(i);
    row[u] = s.row + over;
    chunk[u] = i - over * a.walk.chunks;
    if (row[u] >= a.walk.rows) continue;
    const int n = (int)min((int64_t)8, a.walk.cols - (int64_t)chunk[u] * 8);
    load8<TY, VEC>(x + row[u] * a.x_row + (int64_t)chunk[u] * 8, n, v[u]);
    if (RES) load8<TY, VEC>(res + row[u] * a.res_row + (int64_t)chunk[u] * 8, n, r[u]);
  }
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    if (row[u] >= a.walk.rows) break;
    const int n = (int)min((int64_t)8, a.walk.cols - (int64_t)chunk[u] * 8);
    const Words4 w = philox4x32_10({chunk[u], (uint32_t)row[u], a.group0 + (uint32_t)g, step}, a.seed);
    const uint32_t bits[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = i & 1 ? bits[i >> 1] >> 16 : bits[i >> 1] & 0xFFFFu;
      const float kept = b >= a.threshold ? v[u][i] * a.scale : 0.f;
      v[u][i] = RES ? kept + r[u][i] : kept;
    }
    store8<TY, VEC>(out + row[u] * a.out_row + (int64_t)chunk[u] * 8, n, v[u]);
  }
}

// 65536 q, or -1 where p is out of range.
int dropout_threshold(double p) {
  if (!(p >= 0.0 && p < 1.0)) return -1;
  const double t = std::nearbyint(p * 65536.0);
  return t < 65536.0 ? (int)t : -1;
}

}  // namespace

extern "C" {

int prsgd_dropout(const void* d_x, int32_t type, int64_t row_stride, int64_t group_stride,
                  const void* d_residual, int64_t residual_row_stride, int64_t residual_group_stride,
                  void* d_out, int64_t out_row_stride, int64_t out_group_stride,
                  int64_t groups, int64_t rows, int64_t cols, double p, uint64_t seed, int64_t step, const int64_t* d_step,
                  int64_t first_group, void* cuda_stream) {
  if (!type_known(type)) return op_fail(PRSGD_ERR_ARG, "unknown element type");
  if (groups < 0 || rows < 0 || cols < 0) return op_fail(PRSGD_ERR_ARG, "need groups, rows, cols >= 0");
  const int threshold = dropout_threshold(p);
  if (threshold < 0) return op_fail(PRSGD_ERR_ARG, "p must be in [0, 1 - 2^-17]");
  if (groups > 65535 || rows > 0x7fffffffll || cols > 0x7fffffffll) return op_fail(PRSGD_ERR_SIZE, "more than 65535 groups or 2^31 - 1 rows or columns");
  if (groups == 0 || rows == 0 || cols == 0) return PRSGD_OK;
  int rc = check_rows("x", d_x, type, row_stride, group_stride, groups, rows, cols, false);
  if (rc == PRSGD_OK && d_residual) rc = check_rows("residual", d_residual, type, residual_row_stride, residual_group_stride, groups, rows, cols, false);
  if (rc == PRSGD_OK) rc = check_rows("out", d_out, type, out_row_stride, out_group_stride, groups, rows, cols, true);
  if (rc != PRSGD_OK) return rc;
  if ((d_out == d_x && !same_layout(groups, group_stride, out_group_stride, rows, row_stride, out_row_stride)) ||
      (d_out == d_residual && !same_layout(groups, residual_group_stride, out_group_stride, rows, residual_row_stride, out_row_stride)))
    return op_fail(PRSGD_ERR_ARG, "out is an input's memory with other strides");
  if (((uintptr_t)d_step) % 8) return op_fail(PRSGD_ERR_ALIGN, "d_step must be 8-byte aligned");
  DropoutArgs a{};
  a.walk = row_walk(rows, cols);
  a.x = d_x; a.x_row = row_stride; a.x_group = group_stride;
  a.res = d_residual; a.res_row = residual_row_stride; a.res_group = residual_group_stride;
  a.out = d_out; a.out_row = out_row_stride; a.out_group = out_group_stride;
  a.threshold = (uint32_t)threshold;
  a.scale = (float)(65536.0 / (65536.0 - threshold));
  a.seed = seed; a.step = (uint32_t)step; a.group0 = (uint32_t)first_group; a.d_step = d_step;
  const int64_t blocks = (a.walk.items + kRowItems - 1) / kRowItems;
  if (blocks > 0x7fffffffll) return op_fail(PRSGD_ERR_SIZE, "more than 2^44 elements in a group");
  const bool vec = rows_16(d_x, type, row_stride, group_stride) && rows_16(d_out, type, out_row_stride, out_group_stride) &&
                   (!d_residual || rows_16(d_residual, type, residual_row_stride, residual_group_stride));
  const dim3 grid((unsigned)blocks, (unsigned)groups);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  with_type(type, [&](auto ty) {
    constexpr int TY = decltype(ty)::value;
    if (vec && d_residual) launch_pdl(dropout_kernel<TY, true, true>, grid, dim3(kRowThreads), 0, st, a);
    else if (vec) launch_pdl(dropout_kernel<TY, true, false>, grid, dim3(kRowThreads), 0, st, a);
    else if (d_residual) launch_pdl(dropout_kernel<TY, false, true>, grid, dim3(kRowThreads), 0, st, a);
    else launch_pdl(dropout_kernel<TY, false, false>, grid, dim3(kRowThreads), 0, st, a);
  });
  return op_launched("dropout");
}

int prsgd_dropout_keep(uint64_t seed, int64_t group, int64_t row, int64_t col, int64_t step, double p) {
  const int threshold = dropout_threshold(p);
  if (threshold < 0) return op_fail(PRSGD_ERR_ARG, "p must be in [0, 1 - 2^-17]");
  if (col < 0) return op_fail(PRSGD_ERR_ARG, "need col >= 0");
  const Words4 w = philox4x32_10({(uint32_t)(col / 8), (uint32_t)row, (uint32_t)group, (uint32_t)step}, seed);
  const uint32_t words[4] = {w.x, w.y, w.z, w.w}, word = words[(col % 8) / 2];
  return (col & 1 ? word >> 16 : word & 0xFFFFu) >= (uint32_t)threshold ? 1 : 0;
}

}  // extern "C"
