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

// Eight neighbouring elements as fp32, `n` of which exist; VEC: p lies on a 16-byte boundary.
template <int TY, bool VEC>
__device__ __forceinline__ void load8(const typename ElemOf<TY>::type* p, int n, float (&v)[8]) {
  using T = typename ElemOf<TY>::type;
  if (VEC && n >= 8) {
    if constexpr (TY == PRSGD_TYPE_FP32) {
      const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 u = *reinterpret_cast<const uint4*>(p);
      const T* h = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = to_f32(h[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <int TY, bool VEC>
__device__ __forceinline__ void store8(typename ElemOf<TY>::type* p, int n, const float (&v)[8]) {
  using T = typename ElemOf<TY>::type;
  if (VEC && n >= 8) {
    if constexpr (TY == PRSGD_TYPE_FP32) {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint4 u;
      T* h = reinterpret_cast<T*>(&u);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = from_f32<T>(v[i]);
      *reinterpret_cast<uint4*>(p) = u;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
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
