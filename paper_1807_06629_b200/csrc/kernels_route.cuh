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
  int vec, vec_out;             // rows can be read / written 16 bytes at a time
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

// Sums a group's partial results in block order and forms its loss; all 256 threads of a block.
__device__ __forceinline__ void route_finish(const RouteArgs& a, int64_t g) {
  __shared__ float s_w[8];
  __shared__ int s_alive;
  if (threadIdx.x < 32) {
    int n = 0;
    for (int b = threadIdx.x; b < a.blocks; b += 32) n += a.part_n[g * a.blocks + b];
    n = __reduce_add_sync(0xffffffffu, n);
    if (threadIdx.x == 0) s_alive = n;
  }
  __syncthreads();
  const float live = s_alive > 0 ? (float)s_alive : 1.f;
  float mine = 0.f;
  for (int e = threadIdx.x; e < a.E; e += 256) {
    float p = 0.f; int c = 0;
    const float* pp = a.part_p + g * a.blocks * a.E + e;
    const int32_t* pc = a.part_c + g * a.blocks * a.E + e;
#pragma unroll 8
    for (int b = 0; b < a.blocks; ++b) { p += pp[(int64_t)b * a.E]; c += pc[(int64_t)b * a.E]; }
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

__global__ void __launch_bounds__(256) route_finish_kernel(const RouteArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  route_finish(a, blockIdx.x);
}

// What a block adds to its group: slot b of the group's partial sums, or, of a group of one block, the group's results.
__device__ __forceinline__ void route_leave(const RouteArgs& a, int64_t g) {
  if (a.blocks == 1) {
    __syncthreads();                                  // (the block's own global writes, visible to its threads)
    route_finish(a, g);
  }
}

// For top_k above 8: one warp per token, a lane holds the logits lane, lane + 32, ..., and the largest is taken k times.
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
  route_leave(a, g);
}

// ---- top_k <= 8: a few lanes per token ------------------------------------------------------------------------
// L lanes share a token, each holds PER of its logits (16-byte chunks sub, sub + L, ... of the row) and keeps the same
// experts for every token, so the sums over tokens stay in registers.  A lane's LS largest come from sorting networks:
// batches of LS elements sorted and merged into a sorted list (70 min / max steps per 8 elements), then the lists of
// the L lanes merged across lanes; taking the maximum k times over a warp, as above, took 380 instructions a token,
// this 95.  Elements are ordered by (key, lowest index): of 16-bit logits one 32-bit word (16 to 19 bits of key, 10 of
// index), so that a step is one min and one max; of fp32 logits 64 bits.
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float route_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <int TY> struct RouteKey {                   // bf16, fp16: their 13 lowest bits as fp32 are zero
  using T = uint32_t;
  static __device__ __forceinline__ T make(float x, int e) { return (route_order(x) & ~0x1FFFu) | (uint32_t)(1023 - e); }
  static __device__ __forceinline__ int expert(T k) { return 1023 - (int)(k & 1023u); }
  static __device__ __forceinline__ float value(T k) { return route_value(k & ~0x1FFFu, 0x1FFFu); }
  static __device__ __forceinline__ bool none(T k) { return (k | 0x1FFFu) <= 0x007FFFFFu; }       // -inf or no element
  static __device__ __forceinline__ T other(T k, int o) { return __shfl_xor_sync(0xffffffffu, k, o); }
  // fp32 bits in order, -0 = +0 and every NaN on top (the addition leaves +0 and the positive NaN)
  static __device__ __forceinline__ uint32_t route_order(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  }
  static __device__ __forceinline__ float route_value(uint32_t k, uint32_t low) {      // `low`: bits that were dropped
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~(k | low));
  }
};
template <> struct RouteKey<PRSGD_TYPE_FP32> {
  using T = unsigned long long;
  using Word = RouteKey<PRSGD_TYPE_BF16>;
  static __device__ __forceinline__ T make(float x, int e) { return ((T)Word::route_order(x) << 32) | (uint32_t)(1023 - e); }
  static __device__ __forceinline__ int expert(T k) { return 1023 - (int)(uint32_t)k; }
  static __device__ __forceinline__ float value(T k) { return Word::route_value((uint32_t)(k >> 32), 0u); }
  static __device__ __forceinline__ bool none(T k) { return (uint32_t)(k >> 32) <= 0x007FFFFFu; }
  static __device__ __forceinline__ T other(T k, int o) { return __shfl_xor_sync(0xffffffffu, k, o); }
};

template <typename T> __device__ __forceinline__ void route_ce(T& a, T& b) {      // larger first
  const T x = a > b ? a : b, y = a > b ? b : a;
  a = x; b = y;
}
template <int LS, typename T> __device__ __forceinline__ void route_sort(T (&v)[LS]) {
  if constexpr (LS == 8) {
    route_ce(v[0], v[2]); route_ce(v[1], v[3]); route_ce(v[4], v[6]); route_ce(v[5], v[7]);
    route_ce(v[0], v[4]); route_ce(v[1], v[5]); route_ce(v[2], v[6]); route_ce(v[3], v[7]);
    route_ce(v[0], v[1]); route_ce(v[2], v[3]); route_ce(v[4], v[5]); route_ce(v[6], v[7]);
    route_ce(v[2], v[4]); route_ce(v[3], v[5]); route_ce(v[1], v[4]); route_ce(v[3], v[6]);
    route_ce(v[1], v[2]); route_ce(v[3], v[4]); route_ce(v[5], v[6]);
  } else {
    route_ce(v[0], v[1]); route_ce(v[2], v[3]); route_ce(v[0], v[2]); route_ce(v[1], v[3]); route_ce(v[1], v[2]);
  }
}
// l: the LS largest of two sorted lists (their larger halves form a bitonic sequence), sorted
template <int LS, typename T> __device__ __forceinline__ void route_merge(T (&l)[LS], const T (&y)[LS]) {
#pragma unroll
  for (int j = 0; j < LS; ++j) l[j] = l[j] > y[LS - 1 - j] ? l[j] : y[LS - 1 - j];
#pragma unroll
  for (int st = LS / 2; st > 0; st >>= 1)
#pragma unroll
    for (int j = 0; j < LS; ++j)
      if ((j & st) == 0) route_ce(l[j], l[j + st]);
}

template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A lane's PER logits of one row; beyond E, and of a dead token, -inf.
template <int TY, int PER, int L>
__device__ __forceinline__ void route_load(const typename ElemOf<TY>::type* p, int E, int sub, bool on, bool vec, float (&x)[PER]) {
  using T = typename ElemOf<TY>::type;
  constexpr int V = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < PER / V; ++i) {
    const int e0 = (sub + L * i) * V;
    if (vec) {
      uint4 u = make_uint4(0, 0, 0, 0);
      const bool in = on && e0 < E;                   // (E is a multiple of V here)
      if (in) u = *reinterpret_cast<const uint4*>(p + e0);
      const T* h = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int j = 0; j < V; ++j) x[i * V + j] = in ? to_f32(h[j]) : -INFINITY;
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) x[i * V + j] = on && e0 + j < E ? to_f32(p[e0 + j]) : -INFINITY;
    }
  }
}

template <int TY, int PER, int L, int LS>
__global__ void __launch_bounds__(256) route_lanes_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  using Key = RouteKey<TY>;
  constexpr int V = 16 / sizeof(T), TOK = 32 / L;     // tokens of a warp at a time
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_p[8][PER * L];
  __shared__ int s_c[PER * L];
  __shared__ int s_n;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (L - 1);
  const int64_t g = blockIdx.y;
  for (int e = threadIdx.x; e < PER * L; e += 256) s_c[e] = 0;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  int alive = 0;
  const T* logits = static_cast<const T*>(a.logits) + g * a.group_stride;
  const int64_t step = (int64_t)gridDim.x * 8 * TOK;
  for (int64_t t0 = ((int64_t)blockIdx.x * 8 + warp) * TOK; t0 < a.T; t0 += step) {
    const int64_t t = t0 + lane / L, row = g * a.T + t;
    const bool in = t < a.T, on = in && (a.live == nullptr || a.live[row] != 0);
    float x[PER];
    route_load<TY, PER, L>(logits + t * a.row_stride, a.E, sub, on, a.vec != 0, x);
    typename Key::T l[LS];
#pragma unroll
    for (int i = 0; i < PER / LS; ++i) {
      typename Key::T y[LS];
#pragma unroll
      for (int j = 0; j < LS; ++j) {
        const int q = i * LS + j, e = (sub + L * (q / V)) * V + q % V;
        y[j] = e < a.E ? Key::make(x[q], e) : 0;
      }
      route_sort<LS>(y);
      if (i == 0) {
#pragma unroll
        for (int j = 0; j < LS; ++j) l[j] = y[j];
      } else {
        route_merge<LS>(l, y);
      }
    }
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      typename Key::T y[LS];
#pragma unroll
      for (int j = 0; j < LS; ++j) y[j] = Key::other(l[j], o);
      route_merge<LS>(l, y);
    }
    const bool dead = Key::none(l[0]);                // a dead token, or one whose every logit is -inf
    const float top = dead ? 0.f : Key::value(l[0]) * kLog2E;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      x[i] = route_exp2(fmaf(x[i], kLog2E, -top));
      sum += x[i];
    }
    sum = lanes_sum<L>(sum);
    const float inv = dead ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = fmaf(x[i], inv, acc[i]);
    alive += !dead && sub == 0 ? 1 : 0;
    // the token's entries j, j + L, ... belong to lane j of it
    float w[(LS + L - 1) / L], chosen = 0.f;
    int expert[(LS + L - 1) / L];
#pragma unroll
    for (int j = 0; j < LS; ++j) {
      if (j % L == sub && j < a.k) {
        const float y = route_exp2(fmaf(Key::value(l[j]), kLog2E, -top));
        w[j / L] = y; expert[j / L] = Key::expert(l[j]);
        chosen += y;
      }
    }
    float f = inv;
    if (a.normalize) f = 1.f / lanes_sum<L>(chosen);
#pragma unroll
    for (int j = 0; j < LS; ++j) {
      if (j % L == sub && j < a.k && in) {
        a.experts[row * a.k + j] = dead ? -1 : expert[j / L];
        a.weights[row * a.k + j] = dead ? 0.f : w[j / L] * f;
        if (!dead) atomicAdd(&s_c[expert[j / L]], 1);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
#pragma unroll
    for (int o = 16; o >= L; o >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    if (lane < L) s_p[warp][(sub + L * (i / V)) * V + i % V] = acc[i];
  }
  alive = __reduce_add_sync(0xffffffffu, alive);
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
  route_leave(a, g);
}

// Gradient, any top_k.  dlogit_e = p_e (h_e - dot) with h the balance loss's part, the same for all tokens of a group, and
// dot = sum_e p_e h_e + sum_j p_j dw_j over the chosen ones, whose own gradient is then p_j (h_j + dw_j - dot): the rows
// pass through shared memory, where the lanes that own the token's choices put those in.
template <int TY, int PER, int L>
__global__ void __launch_bounds__(256) route_grad_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  constexpr int V = 16 / sizeof(T), TOK = 32 / L;
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_h[PER * L];
  __shared__ int s_w[8];
  __shared__ __align__(16) T s_row[8][TOK][PER * L];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (L - 1), tok = lane / L;
  const int64_t g = blockIdx.y;
  int total = 0;                                      // sum of the counts = k T
  for (int e = threadIdx.x; e < a.E; e += 256) total += a.counts[g * a.E + e];
  total = __reduce_add_sync(0xffffffffu, total);
  if (lane == 0) s_w[warp] = total;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) total += s_w[w];
  const float kt = total > 0 ? (float)total : 1.f;
  const float up = (a.dloss != nullptr ? a.dloss[g] : 0.f) * a.coef * (float)a.E * (float)a.k / kt;   // (T = k T / k)
  for (int e = threadIdx.x; e < PER * L; e += 256) s_h[e] = e < a.E ? up * ((float)a.counts[g * a.E + e] / kt) : 0.f;
  __syncthreads();
  float h[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) h[i] = s_h[(sub + L * (i / V)) * V + i % V];
  const T* logits = static_cast<const T*>(a.logits) + g * a.group_stride;
  T* out = static_cast<T*>(a.dlogits) + g * a.d_group_stride;
  const int64_t step = (int64_t)gridDim.x * 8 * TOK;
  for (int64_t t0 = ((int64_t)blockIdx.x * 8 + warp) * TOK; t0 < a.T; t0 += step) {
    const int64_t t = t0 + tok, row = g * a.T + t;
    const bool in = t < a.T, on = in && (a.live == nullptr || a.live[row] != 0);
    const T* p = logits + t * a.row_stride;
    float x[PER], mx = -INFINITY;
    route_load<TY, PER, L>(p, a.E, sub, on, a.vec != 0, x);
    bool nan = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) { mx = fmaxf(mx, x[i]); nan |= x[i] != x[i]; }
    mx = nan ? INFINITY : mx;                         // (a NaN makes the row's probabilities NaN: inf - inf)
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const bool dead = mx == -INFINITY;
    const float top = dead ? 0.f : mx * kLog2E;
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      x[i] = route_exp2(fmaf(x[i], kLog2E, -top));
      sum += x[i];
      dot = fmaf(x[i], h[i], dot);
    }
    sum = lanes_sum<L>(sum);
    if (mx == INFINITY) sum = __int_as_float(0x7fffffff);
    const float inv = dead ? 0.f : 1.f / sum;
    dot = lanes_sum<L>(dot) * inv;
    // choice j of the token belongs to lane j % L
    constexpr int OWN = kRouteMaxK / L;
    float pj[OWN], dw[OWN], pick = 0.f, pull = 0.f;
    int ej[OWN];
    if (a.dweights != nullptr) {
#pragma unroll
      for (int q = 0; q < OWN; ++q) {
        const int j = q * L + sub;
        ej[q] = -1; pj[q] = dw[q] = 0.f;
        if (q * L < a.k && j < a.k && !dead) {
          const int e = a.experts[row * a.k + j];
          if ((unsigned)e < (unsigned)a.E) {
            ej[q] = e; dw[q] = a.dweights[row * a.k + j];
            pj[q] = route_exp2(fmaf(to_f32(p[e]), kLog2E, -top)) * inv;
            pick += pj[q];
            pull = fmaf(pj[q], dw[q], pull);
          }
        }
      }
      if (a.normalize) {                              // w_j = p_j / S: the weights' gradient through S as well; sum_j p_j dw_j becomes 0
        const float s = lanes_sum<L>(pick), m = lanes_sum<L>(pull);
#pragma unroll
        for (int q = 0; q < OWN; ++q) dw[q] = ej[q] >= 0 ? (dw[q] - m / s) / s : 0.f;
        pull = 0.f;
#pragma unroll
        for (int q = 0; q < OWN; ++q) pull = fmaf(pj[q], dw[q], pull);
      }
      dot += lanes_sum<L>(pull);
    }
    T* srow = s_row[warp][tok];
#pragma unroll
    for (int i = 0; i < PER / V; ++i) {
      __align__(16) T y[V];
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = from_f32<T>(x[i * V + j] * inv * (h[i * V + j] - dot));
      *reinterpret_cast<uint4*>(srow + (sub + L * i) * V) = *reinterpret_cast<const uint4*>(y);
    }
    __syncwarp();
    if (a.dweights != nullptr) {
#pragma unroll
      for (int q = 0; q < OWN; ++q)
        if (q * L < a.k && ej[q] >= 0) srow[ej[q]] = from_f32<T>(pj[q] * (s_h[ej[q]] + dw[q] - dot));
      __syncwarp();
    }
    if (in) {
      T* d = out + t * a.d_row_stride;
#pragma unroll
      for (int i = 0; i < PER / V; ++i) {
        const int e0 = (sub + L * i) * V;
        if (e0 >= a.E) continue;
        if (a.vec_out) {
          uint4 u = *reinterpret_cast<const uint4*>(srow + e0);
          if (dead) u = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(d + e0) = u;
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (e0 + j < a.E) d[e0 + j] = dead ? from_f32<T>(0.f) : srow[e0 + j];
        }
      }
    }
    __syncwarp();
  }
}

}  // namespace prsgd
