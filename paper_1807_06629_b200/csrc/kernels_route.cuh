// Top-k router with its balance loss, and the gradient.
//   p_te  = softmax over the experts of a token's logits;  the k largest logits are its experts (ties: lowest index)
//   c_e   = how often expert e was chosen, P_e = mean of p_te over the T live tokens of the group
//   loss  = coef E sum_e (c_e / (k T)) P_e
//   dlogit_te = p_te (h_te - sum_j p_tj h_tj),  h_te = dloss coef E c_e / (k T) / T + [e chosen] dweight
#pragma once
#include "ops_common.cuh"

namespace prsgd {

constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxK = 32;
constexpr int kRouteBlocks = 64;        // most blocks of a group: rows of its partial sums in the workspace

struct RouteArgs {
  const void* logits; int64_t row_stride, group_stride;
  const uint8_t* live;          // [G][T] or nullptr
  int64_t G, T;
  int E, k, normalize;
  float coef;
  int32_t* experts; float* weights;       // [G][T][k]
  int32_t* counts; float* mean; float* loss;   // [G][E], [G][E], [G]
  float* part_p; int32_t* part_c; int32_t* part_n;   // [G][blocks][E] twice, [G][blocks]
  int blocks;
  // gradient
  const float* dweights; const float* dloss; void* dlogits; int64_t d_row_stride, d_group_stride;
};

// Order of the logits as unsigned integers: larger key = larger logit, -0 = +0, NaN above all.
__device__ __forceinline__ uint32_t route_key(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One warp per token, a lane holds the logits lane, lane + 32, ...
template <int TY, int PER>
__global__ void __launch_bounds__(256) route_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_p[8][PER * 32];
  __shared__ int s_c[PER * 32];
  __shared__ int s_n;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t g = blockIdx.y;
  for (int e = threadIdx.x; e < PER * 32; e += 256) s_c[e] = 0;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  int alive = 0;
  for (int64_t t = (int64_t)blockIdx.x * 8 + warp; t < a.T; t += (int64_t)gridDim.x * 8) {
    const int64_t row = g * a.T + t;
    float x[PER];
    float mx = -INFINITY;
    bool nan = false;
    const bool on = a.live == nullptr || a.live[row] != 0;
    if (on) {
      const T* p = static_cast<const T*>(a.logits) + g * a.group_stride + t * a.row_stride;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int e = lane + 32 * i;
        x[i] = e < a.E ? to_f32(p[e]) : -INFINITY;
        nan |= x[i] != x[i];
        mx = fmaxf(mx, x[i]);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      nan = __any_sync(0xffffffffu, nan);
    }
    if (!on || (mx == -INFINITY && !nan)) {           // a dead token, or one whose every logit is -inf
      if (lane < a.k) { a.experts[row * a.k + lane] = -1; a.weights[row * a.k + lane] = 0.f; }
      continue;
    }
    ++alive;
    float e_[PER], sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      e_[i] = lane + 32 * i < a.E ? expf(x[i] - mx) : 0.f;
      sum += e_[i];
    }
    sum = warp_sum(sum);
    const float inv = 1.f / sum;
    uint32_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      acc[i] += e_[i] * inv;
      key[i] = lane + 32 * i < a.E ? route_key(x[i]) : 0u;
    }
    float mine = 0.f, chosen_sum = 0.f;
    int my_e = 0;
    for (int j = 0; j < a.k; ++j) {
      uint32_t best = 0; int at = -1; float pe = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (key[i] > best) { best = key[i]; at = lane + 32 * i; pe = e_[i]; }
      const uint32_t top = __reduce_max_sync(0xffffffffu, best);
      const uint32_t cand = best == top && at >= 0 ? (uint32_t)at : 0xFFFFFFFFu;
      const uint32_t win = __reduce_min_sync(0xffffffffu, cand);
      const float wv = __shfl_sync(0xffffffffu, pe, win & 31u);
      chosen_sum += wv;
      if (lane == j) { my_e = (int)win; mine = wv; }
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane + 32 * i == (int)win) key[i] = 0u;
    }
    if (lane < a.k) {
      a.experts[row * a.k + lane] = my_e;
      a.weights[row * a.k + lane] = a.normalize ? mine / chosen_sum : mine * inv;
      atomicAdd(&s_c[my_e], 1);
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) s_p[warp][lane + 32 * i] = acc[i];
  if (lane == 0 && alive) atomicAdd(&s_n, alive);
  __syncthreads();
  const int64_t slot = g * a.blocks + blockIdx.x;
  for (int e = threadIdx.x; e < a.E; e += 256) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += s_p[w][e];
    a.part_p[slot * a.E + e] = s;
    a.part_c[slot * a.E + e] = s_c[e];
  }
  if (threadIdx.x == 0) a.part_n[slot] = s_n;
}

// Sums a group's partial results in block order and forms its loss.  One block of 256 threads per group.
__global__ void __launch_bounds__(256) route_finish_kernel(const RouteArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_w[8];
  const int64_t g = blockIdx.x;
  int n = 0;
  for (int b = 0; b < a.blocks; ++b) n += a.part_n[g * a.blocks + b];
  const float live = n > 0 ? (float)n : 1.f;
  float mine = 0.f;
  for (int e = threadIdx.x; e < a.E; e += 256) {
    float p = 0.f; int c = 0;
    for (int b = 0; b < a.blocks; ++b) {
      p += a.part_p[(g * a.blocks + b) * a.E + e];
      c += a.part_c[(g * a.blocks + b) * a.E + e];
    }
    p /= live;
    a.mean[g * a.E + e] = p;
    a.counts[g * a.E + e] = c;
    mine += ((float)c / ((float)a.k * live)) * p;
  }
  mine = warp_sum(mine);
  if ((threadIdx.x & 31) == 0) s_w[threadIdx.x >> 5] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
    for (int w = 0; w < 8; ++w) s += s_w[w];
    a.loss[g] = a.coef * (float)a.E * s;
  }
}

template <int TY, int PER>
__global__ void __launch_bounds__(256) route_grad_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_h[PER * 32];
  __shared__ int s_w[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t g = blockIdx.y;
  int total = 0;                                      // sum of the counts = k T
  for (int e = threadIdx.x; e < a.E; e += 256) total += a.counts[g * a.E + e];
  total = __reduce_add_sync(0xffffffffu, total);
  if (lane == 0) s_w[warp] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < 8; ++w) total += s_w[w];
  const float kt = total > 0 ? (float)total : 1.f;
  const float up = (a.dloss != nullptr ? a.dloss[g] : 0.f) * a.coef * (float)a.E * (float)a.k / kt;   // (T = k T / k)
  for (int e = threadIdx.x; e < PER * 32; e += 256) s_h[e] = e < a.E ? up * ((float)a.counts[g * a.E + e] / kt) : 0.f;
  __syncthreads();
  for (int64_t t = (int64_t)blockIdx.x * 8 + warp; t < a.T; t += (int64_t)gridDim.x * 8) {
    const int64_t row = g * a.T + t;
    const bool on = a.live == nullptr || a.live[row] != 0;
    T* d = static_cast<T*>(a.dlogits) + g * a.d_group_stride + t * a.d_row_stride;
    const T* p = static_cast<const T*>(a.logits) + g * a.group_stride + t * a.row_stride;
    float x[PER], mx = -INFINITY;
    bool nan = false;
    if (on) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int e = lane + 32 * i;
        x[i] = e < a.E ? to_f32(p[e]) : -INFINITY;
        nan |= x[i] != x[i];
        mx = fmaxf(mx, x[i]);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      nan = __any_sync(0xffffffffu, nan);
    }
    if (!on || (mx == -INFINITY && !nan)) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (lane + 32 * i < a.E) d[lane + 32 * i] = from_f32<T>(0.f);
      continue;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      x[i] = lane + 32 * i < a.E ? expf(x[i] - mx) : 0.f;
      sum += x[i];
    }
    sum = warp_sum(sum);
    const float inv = 1.f / sum;
    float h[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) { x[i] *= inv; h[i] = s_h[lane + 32 * i]; }
    if (a.dweights != nullptr) {
      int my_e = -1; float dw = 0.f;
      if (lane < a.k) { my_e = a.experts[row * a.k + lane]; dw = a.dweights[row * a.k + lane]; }
      if ((unsigned)my_e >= (unsigned)a.E) { my_e = -1; dw = 0.f; }
      float pk = 0.f;                                 // probability of this lane's expert
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const float v = __shfl_sync(0xffffffffu, x[i], my_e & 31);
        if (my_e >= 0 && (my_e >> 5) == i) pk = v;
      }
      if (a.normalize) {
        const float s = warp_sum(pk), dot = warp_sum(dw * pk);
        dw = my_e >= 0 && s > 0.f ? (dw - dot / s) / s : (s != s ? s : 0.f);
      }
      for (int j = 0; j < a.k; ++j) {
        const int e = __shfl_sync(0xffffffffu, my_e, j);
        const float w = __shfl_sync(0xffffffffu, dw, j);
        if (e >= 0 && (e & 31) == lane) {
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if ((e >> 5) == i) h[i] += w;
        }
      }
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) dot += x[i] * h[i];
    dot = warp_sum(dot);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (lane + 32 * i < a.E) d[lane + 32 * i] = from_f32<T>(x[i] * (h[i] - dot));
  }
}

}  // namespace prsgd
