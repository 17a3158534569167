// Arrays of rows [groups][rows][columns] walked in pieces of eight columns, the unit of the operators that move rows
// (embedding, dropout): 16 bytes of a 16-bit type, 32 of fp32.
#pragma once
#include "ops_common.cuh"

namespace prsgd {

// Division of 32-bit numbers by a number known on the host: one multiplication (Granlund and Montgomery, 1994).
struct FastDiv {
  uint32_t d = 1, m = 0, s = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    m = (uint32_t)(((1ull << 32) * ((1ull << l) - d)) / d + 1);
    s = l > 0 ? l - 1 : 0;
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const {
    if (d == 1) return n;
#ifdef __CUDA_ARCH__
    const uint32_t t = __umulhi(m, n);
#else
    const uint32_t t = (uint32_t)(((uint64_t)m * n) >> 32);
#endif
    return (t + ((n - t) >> 1)) >> s;
  }
};

// Rows dealt out to blocks in pieces of eight columns: a block takes kRowItems pieces one after another.
constexpr int kRowThreads = 256, kRowUnroll = 4, kRowItems = kRowThreads * kRowUnroll;
struct RowWalk {
  int64_t rows, cols;
  uint32_t chunks;           // pieces of a row
  FastDiv by_chunks;
  int64_t items;             // pieces of a group
};
inline RowWalk row_walk(int64_t rows, int64_t cols) {
  RowWalk w;
  w.rows = rows; w.cols = cols;
  w.chunks = (uint32_t)((cols + 7) / 8);
  w.by_chunks = FastDiv(w.chunks);
  w.items = rows * (int64_t)w.chunks;
  return w;
}
// Row and first column of item `i` of the block that begins with item `first`.
struct RowStart { int64_t row; uint32_t chunk; };
struct RowPiece { int64_t row; uint32_t chunk; };
__device__ __forceinline__ RowPiece row_piece(const RowWalk& w, const RowStart& s, uint32_t i) {
  const uint32_t k = s.chunk + i, over = w.by_chunks.div(k);
  return {s.row + over, k - over * w.chunks};
}
__device__ __forceinline__ RowStart row_start(const RowWalk& w, int64_t first) {
  RowStart s;
  if (first >> 32) {
    s.row = first / w.chunks;
    s.chunk = (uint32_t)(first - s.row * w.chunks);
  } else {
    const uint32_t r = w.by_chunks.div((uint32_t)first);
    s.row = r;
    s.chunk = (uint32_t)first - r * w.chunks;
  }
  return s;
}

inline bool rows_16(const void* p, int type, int64_t row_stride, int64_t group_stride) {
  const int v = 16 / type_bytes(type);
  return (uintptr_t)p % 16 == 0 && row_stride % v == 0 && group_stride % v == 0;
}

// Eight neighbouring elements as they lie in memory, on a 16-byte boundary: loaded apart from their conversion, so that the loads of several
// pieces are in flight together.
template <int TY> struct Raw8 { uint4 q[TY == PRSGD_TYPE_FP32 ? 2 : 1]; };
template <int TY>
__device__ __forceinline__ Raw8<TY> load_raw(const typename ElemOf<TY>::type* p) {
  Raw8<TY> r;
  r.q[0] = reinterpret_cast<const uint4*>(p)[0];
  if constexpr (TY == PRSGD_TYPE_FP32) r.q[1] = reinterpret_cast<const uint4*>(p)[1];
  return r;
}
template <int TY>
__device__ __forceinline__ Raw8<TY> zero_raw() {
  Raw8<TY> r;
  r.q[0] = make_uint4(0, 0, 0, 0);
  if constexpr (TY == PRSGD_TYPE_FP32) r.q[1] = make_uint4(0, 0, 0, 0);
  return r;
}
template <int TY>
__device__ __forceinline__ void unpack8(const Raw8<TY>& r, float (&v)[8]) {
  const typename ElemOf<TY>::type* h = reinterpret_cast<const typename ElemOf<TY>::type*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_f32(h[i]);
}
template <int TY>
__device__ __forceinline__ void store_raw(typename ElemOf<TY>::type* p, const float (&v)[8]) {
  using T = typename ElemOf<TY>::type;
  Raw8<TY> r;
  T* h = reinterpret_cast<T*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = from_f32<T>(v[i]);
  reinterpret_cast<uint4*>(p)[0] = r.q[0];
  if constexpr (TY == PRSGD_TYPE_FP32) reinterpret_cast<uint4*>(p)[1] = r.q[1];
}
// The same with `n` of the eight there, of which the others are not touched; VEC: p lies on a 16-byte boundary.
template <int TY, bool VEC>
__device__ __forceinline__ void load8(const typename ElemOf<TY>::type* p, int n, float (&v)[8]) {
  if (VEC && n >= 8) {
    unpack8<TY>(load_raw<TY>(p), v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <int TY, bool VEC>
__device__ __forceinline__ void store8(typename ElemOf<TY>::type* p, int n, const float (&v)[8]) {
  if (VEC && n >= 8) {
    store_raw<TY>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<typename ElemOf<TY>::type>(v[i]);
  }
}

// Checks of one array of rows; `written` ones may not overlap themselves.
inline int check_rows(const char* name, const void* p, int type, int64_t row, int64_t group, int64_t groups, int64_t rows, int64_t cols, bool written) {
  if (p == nullptr) return op_fail(PRSGD_ERR_ARG, std::string(name) + " is NULL");
  if (((uintptr_t)p) % type_bytes(type)) return op_fail(PRSGD_ERR_ALIGN, std::string(name) + " is not aligned to its element type");
  if (row < cols || group < 0) return op_fail(PRSGD_ERR_ARG, std::string(name) + ": need row stride >= columns, group stride >= 0");
  if (written && !rows_apart(groups, group, rows, row, cols)) return op_fail(PRSGD_ERR_ARG, std::string("the rows of ") + name + " overlap");
  return PRSGD_OK;
}
inline int op_launched(const char* name) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? PRSGD_OK : op_fail(PRSGD_ERR_CUDA, std::string(name) + ": " + cudaGetErrorString(e));
}

}  // namespace prsgd
