// What the stand-alone training operators share: element types, the device status at the head of a
// workspace, and the error text of context-free calls.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <algorithm>
#include <type_traits>
#include "prsgd_common.cuh"

namespace prsgd {

// Records the text prsgd_last_error(NULL) returns and hands the code back (defined in prsgd_api.cu).
int op_fail(int code, const std::string& msg);

// Whether the rows (`width` elements, `row` >= width apart) of `batch` matrices `stride` apart are all different memory: matrix behind
// matrix, or a row of each in turn ([rows][batch][width] seen as [batch][rows][width]).
inline bool rows_apart(int64_t batch, int64_t stride, int64_t rows, int64_t row, int64_t width) {
  if (batch <= 1 || rows < 1 || width < 1) return true;
  return (__int128)stride >= (__int128)(rows - 1) * row + width || (stride >= width && (rows <= 1 || (__int128)row >= (__int128)(batch - 1) * stride + width));
}

// An output that starts where an input does: only as the same array, element for element.
inline bool same_layout(int64_t batch, int64_t stride_a, int64_t stride_b, int64_t rows, int64_t row_a, int64_t row_b) {
  return (batch <= 1 || stride_a == stride_b) && (rows <= 1 || row_a == row_b);
}

// The status words at the head of the workspace of a call that has nothing to compute (a call without a workspace has none).
inline int op_clear_status(void* d_work, size_t bytes, void* stream) {
  if (d_work == nullptr || bytes < sizeof(DeviceStatus)) return PRSGD_OK;
  const cudaError_t e = cudaMemsetAsync(d_work, 0, sizeof(DeviceStatus), static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PRSGD_OK : op_fail(PRSGD_ERR_CUDA, std::string("clearing a workspace's status: ") + cudaGetErrorString(e));
}

template <int T> struct ElemOf;
template <> struct ElemOf<PRSGD_TYPE_FP32> { using type = float; };
template <> struct ElemOf<PRSGD_TYPE_BF16> { using type = __nv_bfloat16; };
template <> struct ElemOf<PRSGD_TYPE_FP16> { using type = __half; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

inline int type_bytes(int t) { return t == PRSGD_TYPE_FP32 ? 4 : 2; }
inline bool type_known(int t) { return t == PRSGD_TYPE_FP32 || t == PRSGD_TYPE_BF16 || t == PRSGD_TYPE_FP16; }

// Calls f with std::integral_constant<int, T> for the element type `t` (already known to be one).
template <typename F> inline auto with_type(int t, F&& f) {
  if (t == PRSGD_TYPE_FP32) return f(std::integral_constant<int, PRSGD_TYPE_FP32>());
  if (t == PRSGD_TYPE_BF16) return f(std::integral_constant<int, PRSGD_TYPE_BF16>());
  return f(std::integral_constant<int, PRSGD_TYPE_FP16>());
}

__device__ __forceinline__ void op_pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void op_pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace prsgd
