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

__device__ __forceinline__ Words4 dropout_words(const DropoutArgs& a, const RowPiece& at, uint32_t step) {
  return philox4x32_10({at.chunk, (uint32_t)at.row, a.group0 + blockIdx.y, step}, a.seed);
}

// Rows that begin on 16-byte boundaries and end on multiples of eight columns.
template <int TY, bool RES>
__global__ void __launch_bounds__(kRowThreads) dropout_kernel(const DropoutArgs a) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const T* x = static_cast<const T*>(a.x) + g * a.x_group;
  const T* res = RES ? static_cast<const T*>(a.res) + g * a.res_group : nullptr;
  T* out = static_cast<T*>(a.out) + g * a.out_group;
  const uint32_t step = a.step + (a.d_step ? (uint32_t)*a.d_step : 0u);
  const RowStart s = row_start(a.walk, (int64_t)blockIdx.x * kRowItems);
  RowPiece at[kRowUnroll];
  Raw8<TY> v[kRowUnroll], r[kRowUnroll];
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    at[u] = row_piece(a.walk, s, u * kRowThreads + threadIdx.x);
    if (at[u].row >= a.walk.rows) continue;
    v[u] = load_raw<TY>(x + at[u].row * a.x_row + (int64_t)at[u].chunk * 8);
    if (RES) r[u] = load_raw<TY>(res + at[u].row * a.res_row + (int64_t)at[u].chunk * 8);
  }
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    if (at[u].row >= a.walk.rows) break;
    const Words4 w = dropout_words(a, at[u], step);
    const uint32_t bits[4] = {w.x, w.y, w.z, w.w};
    float y[8], more[8];
    unpack8<TY>(v[u], y);
    if (RES) unpack8<TY>(r[u], more);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = i & 1 ? bits[i >> 1] >> 16 : bits[i >> 1] & 0xFFFFu;
      const float kept = b >= a.threshold ? y[i] * a.scale : 0.f;
      y[i] = RES ? kept + more[i] : kept;
    }
    store_raw<TY>(out + at[u].row * a.out_row + (int64_t)at[u].chunk * 8, y);
  }
}

// Any rows: the lanes of a warp draw for 32 pieces, then take neighbouring columns, whose bits they find in shared memory.
template <int TY, bool RES>
__global__ void __launch_bounds__(kRowThreads) dropout_any_kernel(const DropoutArgs a) {
  using T = typename ElemOf<TY>::type;
  __shared__ uint4 drawn[kRowThreads];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const T* x = static_cast<const T*>(a.x) + g * a.x_group;
  const T* res = RES ? static_cast<const T*>(a.res) + g * a.res_group : nullptr;
  T* out = static_cast<T*>(a.out) + g * a.out_group;
  const uint32_t step = a.step + (a.d_step ? (uint32_t)*a.d_step : 0u);
  const RowStart s = row_start(a.walk, (int64_t)blockIdx.x * kRowItems);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint16_t* bits = reinterpret_cast<const uint16_t*>(drawn + warp * 32);
#pragma unroll 1
  for (int u = 0; u < kRowUnroll; ++u) {
    const uint32_t first = u * kRowThreads + warp * 32;
    T v[8], r[8];
    int64_t row[8];
    uint32_t col[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const RowPiece p = row_piece(a.walk, s, first + j * 4 + (lane >> 3));
      row[j] = p.row;
      col[j] = p.chunk * 8 + (lane & 7);
      if (p.row >= a.walk.rows || col[j] >= a.walk.cols) { row[j] = -1; continue; }
      v[j] = x[p.row * a.x_row + col[j]];
      if (RES) r[j] = res[p.row * a.res_row + col[j]];
    }
    const Words4 w = dropout_words(a, row_piece(a.walk, s, first + lane), step);
    __syncwarp();
    drawn[threadIdx.x] = make_uint4(w.x, w.y, w.z, w.w);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (row[j] < 0) continue;
      const float kept = bits[j * 32 + lane] >= a.threshold ? to_f32(v[j]) * a.scale : 0.f;
      out[row[j] * a.out_row + col[j]] = from_f32<T>(RES ? kept + to_f32(r[j]) : kept);
    }
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
  if (threshold < 0) return op_fail(PRSGD_ERR_ARG, "p must be in [0, 1 - 2^-17)");
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
  const bool whole = cols % 8 == 0 && rows_16(d_x, type, row_stride, group_stride) && rows_16(d_out, type, out_row_stride, out_group_stride) &&
                     (!d_residual || rows_16(d_residual, type, residual_row_stride, residual_group_stride));
  const dim3 grid((unsigned)blocks, (unsigned)groups);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  with_type(type, [&](auto ty) {
    constexpr int TY = decltype(ty)::value;
    if (whole && d_residual) launch_pdl(dropout_kernel<TY, true>, grid, dim3(kRowThreads), 0, st, a);
    else if (whole) launch_pdl(dropout_kernel<TY, false>, grid, dim3(kRowThreads), 0, st, a);
    else if (d_residual) launch_pdl(dropout_any_kernel<TY, true>, grid, dim3(kRowThreads), 0, st, a);
    else launch_pdl(dropout_any_kernel<TY, false>, grid, dim3(kRowThreads), 0, st, a);
  });
  return op_launched("dropout");
}

int prsgd_dropout_keep(uint64_t seed, int64_t group, int64_t row, int64_t col, int64_t step, double p) {
  const int threshold = dropout_threshold(p);
  if (threshold < 0) return op_fail(PRSGD_ERR_ARG, "p must be in [0, 1 - 2^-17)");
  if (col < 0) return op_fail(PRSGD_ERR_ARG, "need col >= 0");
  const Words4 w = philox4x32_10({(uint32_t)(col / 8), (uint32_t)row, (uint32_t)group, (uint32_t)step}, seed);
  const uint32_t words[4] = {w.x, w.y, w.z, w.w}, word = words[(col % 8) / 2];
  return (col & 1 ? word >> 16 : word & 0xFFFFu) >= (uint32_t)threshold ? 1 : 0;
}

}  // extern "C"
