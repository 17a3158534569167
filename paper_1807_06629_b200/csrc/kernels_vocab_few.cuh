// The vocabulary loss of few tokens a group: W is read once, where it lies and in any type, by dot products on the CUDA cores.
//
// The bytes of W bound it (22 elements of 16 bits a cycle and SM at the HBM rate); a token costs one product an element, in packed
// pairs, so up to kFewTokens of them fit beside the loads.  A warp takes four rows of W at a time, so that what it reads of H from
// shared memory serves four rows; the largest logit and the sum of exponentials run along in registers, and a second launch joins
// the blocks'.  1 x 1 x 32000 x 1024: bf16 20 us (10 of them W from HBM, 8 two launches and the reading of H), fp32 27 (20).
#pragma once
#include "kernels_vocab.cuh"

namespace prsgd {

constexpr int kFewTokens = 4, kFewRows = 4, kFewWarps = 8;
constexpr int64_t kFewSmem = 96 * 1024;        // H of a group as fp32

struct VocabFew {
  const void* H; int64_t h_row, h_group;
  const void* W; int64_t w_row, w_group;
  const int32_t* labels;
  int64_t V, per;                              // rows of W a block takes
  int T, D, dp;                                // dp: D rounded up to 8
  int blocks;                                  // of a group
  float2* part; float* zy;                     // [groups][T][blocks], [groups][T]
  float* loss; float* stats;
  DeviceStatus* status;
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

template <int TY, bool VEC, int NT>
__global__ void __launch_bounds__(32 * kFewWarps) vocab_few_kernel(const VocabFew a) {
  using T = typename ElemOf<TY>::type;
  extern __shared__ float h[];                 // [NT][dp], zeros for tokens without a label
  __shared__ float2 sums[kFewWarps][NT];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && g == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  int y[NT];
  bool any = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    y[t] = t < a.T ? a.labels[g * a.T + t] : -1;
    if (y[t] >= a.V) y[t] = -1;
    any |= y[t] >= 0;
  }
  if (!any) return;                            // (nobody reads this group's parts)
  const T* H = static_cast<const T*>(a.H) + g * a.h_group;
  for (int i = threadIdx.x; i < NT * a.dp; i += 32 * kFewWarps) {
    const int t = i / a.dp, c = i - t * a.dp;
    bool on = false;
#pragma unroll
    for (int k = 0; k < NT; ++k) on |= k == t && y[k] >= 0;
    h[i] = on && c < a.D ? to_f32(H[t * a.h_row + c]) : 0.f;
  }
  __syncthreads();
  const T* W = static_cast<const T*>(a.W) + g * a.w_group;
  const int64_t end = min(a.V, (blockIdx.x + 1) * a.per);
  float2 run[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) run[t] = make_float2(-INFINITY, 0.f);
  for (int64_t v0 = blockIdx.x * a.per + warp * kFewRows; v0 < end; v0 += kFewWarps * kFewRows) {
    float2 acc[kFewRows][NT];
#pragma unroll
    for (int r = 0; r < kFewRows; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[r][t] = make_float2(0.f, 0.f);
    const int rows = (int)min((int64_t)kFewRows, end - v0);
#pragma unroll 2
    for (int c = lane * 8; c < a.D; c += 256) {
      float w[kFewRows][8];
      if (VEC && c + 8 <= a.D) {
        Raw8<TY> raw[kFewRows];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) raw[r] = r < rows ? load_raw<TY>(W + (v0 + r) * a.w_row + c) : zero_raw<TY>();
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) unpack8<TY>(raw[r], w[r]);
      } else {
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) load8<TY, false>(W + (v0 + r) * a.w_row + c, r < rows ? a.D - c : 0, w[r]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float4 p = *reinterpret_cast<const float4*>(h + t * a.dp + c), q = *reinterpret_cast<const float4*>(h + t * a.dp + c + 4);
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
          acc[r][t] = fma2(make_float2(w[r][0], w[r][1]), make_float2(p.x, p.y), acc[r][t]);
          acc[r][t] = fma2(make_float2(w[r][2], w[r][3]), make_float2(p.z, p.w), acc[r][t]);
          acc[r][t] = fma2(make_float2(w[r][4], w[r][5]), make_float2(q.x, q.y), acc[r][t]);
          acc[r][t] = fma2(make_float2(w[r][6], w[r][7]), make_float2(q.z, q.w), acc[r][t]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
      if (r >= rows) break;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float z = acc[r][t].x + acc[r][t].y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        if (lane == 0 && v0 + r == y[t]) a.zy[g * a.T + t] = z;
        const float m = fmaxf(run[t].x, z);
        run[t] = make_float2(m, run[t].y * vt_exp2((run[t].x - m) * 1.4426950408889634f) + vt_exp2((z - m) * 1.4426950408889634f));
      }
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[warp][t] = run[t];
  }
  __syncthreads();
  if (threadIdx.x < NT && (int)threadIdx.x < a.T) {
    float2 all = sums[0][threadIdx.x];
    for (int w = 1; w < kFewWarps; ++w) all = vocab_merge(all, sums[w][threadIdx.x]);
    a.part[(g * a.T + threadIdx.x) * a.blocks + blockIdx.x] = all;
  }
}

// A warp a token.
__global__ void __launch_bounds__(128) vocab_few_join_kernel(const VocabFew a) {
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.x;
  const int t = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (t >= a.T) return;
  const int64_t o = g * a.T + t;
  const int y = a.labels[o];
  float loss = 0.f, top = 0.f, log_sum = 0.f;
  if (y >= 0 && y < a.V) {
    const float2* part = a.part + o * a.blocks;
    float2 all = make_float2(-INFINITY, 0.f);
    for (int k = lane; k < a.blocks; k += 32 * 8) {
      float2 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = k + j * 32 < a.blocks ? part[k + j * 32] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) all = vocab_merge(all, p[j]);
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) all = vocab_merge(all, make_float2(__shfl_xor_sync(0xffffffffu, all.x, s), __shfl_xor_sync(0xffffffffu, all.y, s)));
    top = all.x;
    log_sum = logf(all.y);
    loss = log_sum + (top - a.zy[o]);
  }
  if (lane == 0) {
    a.loss[o] = loss;
    a.stats[2 * o] = top;
    a.stats[2 * o + 1] = log_sum;
  }
}

}  // namespace prsgd
