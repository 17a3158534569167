// Top-k router with its balance loss, and the gradient.
//   p_te  = softmax over the experts of a token's logits;  the k largest logits are its experts (ties: lowest index)
//   c_e   = how often expert e was chosen, P_e = mean of p_te over the T live tokens of the group
//   loss  = coef E sum_e (c_e / (k T)) P_e
//   dlogit_te = p_te (h_te - sum_j p_tj h_tj),  h_te = dloss coef E c_e / (k T) / T + [e chosen] dweight
#pragma once
#include "ops_common.cuh"
#include "tc_ptx.cuh"

namespace prsgd {

constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxK = 32;
constexpr int kRouteCluster = 8;        // most blocks of a group that make a cluster
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
  DeviceStatus* status;         // of the workspace: cleared by the call (the router waits for nothing that could expire)
  int blocks;
  int clustered;                // the blocks of a group are a cluster, whose first finishes the group
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

__device__ __forceinline__ void route_clear_status(const RouteArgs& a) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.status->error = 0u;
}

// Sums a group's partial results in a fixed order and forms its loss: a cluster, of which each block takes a multiple of 32
// experts.  Each warp takes every eighth row of sums, lanes along the experts, so that their loads are in flight together (a
// thread per expert that walked all rows took 16 us for 18 rows of 100 experts; with one block for all experts of a group the
// whole call took 79 us at 4 x 4096 x 1024, now 40, and 52.6 us at 16 x 16384 x 128, now 50.4).
constexpr int kRouteFinish = 8, kRouteFinishExperts = kRouteMaxExperts / kRouteFinish;
__host__ __device__ constexpr int route_finish_blocks(int E) { return E >= 32 * kRouteFinish ? kRouteFinish : (E + 31) / 32; }
__global__ void __launch_bounds__(256) route_finish_kernel(const RouteArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  if (a.blocks == 0) route_clear_status(a);              // (no tokens: the only launch)
  __shared__ float s_p[8][kRouteFinishExperts];
  __shared__ int s_c[8][kRouteFinishExperts];
  __shared__ float s_w[8], s_loss;
  __shared__ int s_alive;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, parts = (int)gridDim.x;
  const int64_t g = blockIdx.y;
  const int width = ((a.E + parts - 1) / parts + 31) / 32 * 32, e0 = (int)blockIdx.x * width;
  if (warp == 0) {
    int n = 0;
    for (int b = lane; b < a.blocks; b += 32) n += a.part_n[g * a.blocks + b];
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) s_alive = n;
  }
  for (int q = lane; q < width && e0 + q < a.E; q += 32) {
    float p = 0.f;
    int c = 0;
#pragma unroll 4
    for (int b = warp; b < a.blocks; b += 8) {
      const int64_t at = (g * a.blocks + b) * a.E + e0 + q;
      p += a.part_p[at];
      c += a.part_c[at];
    }
    s_p[warp][q] = p;
    s_c[warp][q] = c;
  }
  __syncthreads();
  const float live = s_alive > 0 ? (float)s_alive : 1.f;
  const int q = (int)threadIdx.x, e = e0 + q;
  float mine = 0.f;
  if (q < width && e < a.E) {
    float p = 0.f;
    int c = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) { p += s_p[w][q]; c += s_c[w][q]; }
    p /= live;
    a.mean[g * a.E + e] = p;
    a.counts[g * a.E + e] = c;
    mine = ((float)c / ((float)a.k * live)) * p;
  }
  mine = warp_sum(mine);
  if (lane == 0) s_w[warp] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += s_w[w];
    s_loss = s;
  }
  ptx::cluster_arrive_release();
  ptx::cluster_wait_acquire();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    float s = s_loss;
    for (int r = 1; r < parts; ++r) s += ptx::ld_cluster_f32(ptx::cluster_map(ptx::smem_u32(&s_loss), (uint32_t)r));
    a.loss[g] = a.coef * (float)a.E * s;
  }
  ptx::cluster_arrive_release();                         // (nobody ends while its sum may be read)
  ptx::cluster_wait_acquire();
}

// What a block adds to its group (p: its 8 warps' sums over tokens, n tokens): a row of the group's partial sums, or, of a
// group of one block or one cluster, the group's results.
template <int W>
__device__ __forceinline__ void route_leave(const RouteArgs& a, int64_t g, float (&p)[8][W], int* c, int* p_n) {
  __shared__ float s_loss[8];
  const int64_t slot = g * a.blocks + blockIdx.x;
  int n = *p_n;
  if (a.clustered) {                                     // the first block adds the others' sums, in their order, to its own
    for (int e = threadIdx.x; e < a.E; e += 256) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) s += p[w][e];
      p[0][e] = s;
    }
    ptx::cluster_arrive_release();
    ptx::cluster_wait_acquire();
    if (blockIdx.x == 0) {
      const uint32_t at_p = ptx::smem_u32(&p[0][0]), at_c = ptx::smem_u32(c), at_n = ptx::smem_u32(p_n);
      for (int r = 1; r < a.blocks; ++r) n += (int)ptx::ld_cluster_u32(ptx::cluster_map(at_n, (uint32_t)r));
      for (int e = threadIdx.x; e < a.E; e += 256) {
        float s[kRouteCluster];
        int k[kRouteCluster];
#pragma unroll
        for (int r = 1; r < kRouteCluster; ++r)
          if (r < a.blocks) {
            s[r] = ptx::ld_cluster_f32(ptx::cluster_map(at_p, (uint32_t)r) + 4u * (uint32_t)e);
            k[r] = (int)ptx::ld_cluster_u32(ptx::cluster_map(at_c, (uint32_t)r) + 4u * (uint32_t)e);
          }
        float sum = p[0][e];
        int count = c[e];
#pragma unroll
        for (int r = 1; r < kRouteCluster; ++r)
          if (r < a.blocks) { sum += s[r]; count += k[r]; }
        p[0][e] = sum;
        c[e] = count;
      }
    }
    ptx::cluster_arrive_release();                       // (nobody ends while its sums may be read)
    ptx::cluster_wait_acquire();
    if (blockIdx.x != 0) return;
  }
  const bool whole = a.blocks == 1 || a.clustered;
  const float live = n > 0 ? (float)n : 1.f;
  float mine = 0.f;
  for (int e = threadIdx.x; e < a.E; e += 256) {
    float s = 0.f;
    if (a.clustered) {
      s = p[0][e];
    } else {
#pragma unroll
      for (int w = 0; w < 8; ++w) s += p[w][e];
    }
    if (!whole) {
      a.part_p[slot * a.E + e] = s;
      a.part_c[slot * a.E + e] = c[e];
    } else {
      s /= live;
      a.mean[g * a.E + e] = s;
      a.counts[g * a.E + e] = c[e];
      mine += ((float)c[e] / ((float)a.k * live)) * s;
    }
  }
  if (!whole) {
    if (threadIdx.x == 0) a.part_n[slot] = n;
    return;
  }
  mine = warp_sum(mine);
  if ((threadIdx.x & 31) == 0) s_loss[threadIdx.x >> 5] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += s_loss[w];
    a.loss[g] = a.coef * (float)a.E * s;
  }
}

// For top_k above 8: one warp per token, a lane holds the logits lane, lane + 32, ..., and the largest is taken k times
// (16 x 16384 x 128 bf16: top 9 373 us, top 16 556, top 32 958; the kernels below: top 4 41, top 8 50).
template <int TY, int PER>
__global__ void __launch_bounds__(256, 2) route_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  route_clear_status(a);
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
  route_leave(a, g, s_p, s_c, &s_n);
}

// ---- top_k <= 8: a few lanes per token ------------------------------------------------------------------------
// L lanes share a token, each holds PER of its logits (16-byte chunks sub, sub + L, ... of the row) and keeps the same
// experts for every token, so the sums over tokens stay in registers.  A lane's LS largest come from sorting networks:
// batches of LS elements sorted and merged into a sorted list (70 min / max steps per 8 elements), then the lists of
// the L lanes merged across lanes; taking the maximum k times over a warp, as above, took 380 instructions a token,
// this 95.  Elements are ordered by (key, lowest index): of 16-bit logits one 32-bit word (16 bits of order, 16 of
// index), so that a step is one min and one max; of fp32 logits 64 bits.
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float route_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// e^(x - top) for x <= top.  Subtracted before it is scaled: the largest has exponent 0 and nothing overflows, however large the
// logits are.  (As one fma, x log2e - round(top log2e), the rounding of the second term stays in the exponent: hundreds from
// logits of 1e10 on, and infinite at the lowest values of fp32 and bf16.)
__device__ __forceinline__ float route_exp_below(float x, float top) { return route_exp2((x - top) * kLog2E); }
// ... of two logits, an instruction for both (16 x 16384 x 128 top 8: 51.3 us with one each, 50.4 with this)
__device__ __forceinline__ void route_exp_below(float& x, float& y, float top) {
  asm("{\n.reg .b64 v, t, s;\nmov.b64 v, {%0, %1};\nmov.b64 t, {%2, %2};\nmov.b64 s, {%3, %3};\n"
      "add.rn.f32x2 v, v, t;\nmul.rn.f32x2 v, v, s;\nmov.b64 {%0, %1}, v;\n}" : "+f"(x), "+f"(y) : "f"(-top), "f"(kLog2E));
  x = route_exp2(x);
  y = route_exp2(y);
}

template <int TY> struct RouteKey {                   // bf16, fp16: the 16 bits of the logit in order, then the index
  using T = uint32_t;
  using E = typename ElemOf<TY>::type;
  static constexpr uint32_t kNegInf = TY == PRSGD_TYPE_BF16 ? 0x007Fu : 0x03FFu;      // order of -inf
  // Keys of the two elements of a word: adding 0 leaves +0 for -0 and the positive NaN for every NaN; then all bits of a
  // negative number are turned, of a positive one the sign.  Three of these steps run beside the pipe of the sorting.
  static __device__ __forceinline__ void pair(uint32_t word, int e, T& lo, T& hi) {
    uint32_t c;
    if constexpr (TY == PRSGD_TYPE_BF16) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(c) : "r"(word), "r"(0x3F803F80u), "r"(0u));
    else asm("add.rn.f16x2 %0, %1, %2;" : "=r"(c) : "r"(word), "r"(0u));
    const uint32_t order = c ^ ((((c >> 15) & 0x00010001u) * 0x7FFFu) | 0x80008000u);
    lo = order * 65536u + (uint32_t)(1023 - e);
    hi = (order & 0xFFFF0000u) | (uint32_t)(1022 - e);
  }
  static __device__ __forceinline__ int expert(T k) { return 1023 - (int)(k & 0xFFFFu); }
  static __device__ __forceinline__ float value(T k) {
    const uint16_t o = (uint16_t)(k >> 16), u = (o & 0x8000u) ? o ^ 0x8000u : ~o;
    return to_f32(*reinterpret_cast<const E*>(&u));
  }
  static __device__ __forceinline__ bool none(T k) { return (k >> 16) <= kNegInf; }
};
template <> struct RouteKey<PRSGD_TYPE_FP32> {        // the 32 bits in order, then the index
  using T = unsigned long long;
  static __device__ __forceinline__ T make(float x, int e) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return ((T)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32) | (uint32_t)(1023 - e);
  }
  static __device__ __forceinline__ int expert(T k) { return 1023 - (int)(uint32_t)k; }
  static __device__ __forceinline__ float value(T k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
  }
  static __device__ __forceinline__ bool none(T k) { return (uint32_t)(k >> 32) <= 0x007FFFFFu; }
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

// A lane's PER logits of one row as they are stored, requested one turn ahead of their use.  Beyond E, and of a dead
// token, they are -inf: there are always top_k real ones, and of equal keys the lower index wins, so none of those
// beyond E is ever chosen.
template <int TY, int PER, int L> struct RouteRow {
  using T = typename ElemOf<TY>::type;
  static constexpr int V = 16 / sizeof(T);
  static constexpr uint32_t kFill = TY == PRSGD_TYPE_FP32 ? 0xFF800000u : TY == PRSGD_TYPE_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
  uint4 u[PER / V];
  __device__ __forceinline__ void request(const T* p, int E, int sub, bool on, bool vec) {
#pragma unroll
    for (int i = 0; i < PER / V; ++i) {
      const int e0 = (sub + L * i) * V;
      u[i] = make_uint4(kFill, kFill, kFill, kFill);
      if (vec) {
        if (on && e0 < E) u[i] = *reinterpret_cast<const uint4*>(p + e0);      // (E is a multiple of V here)
      } else {
        T* h = reinterpret_cast<T*>(&u[i]);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (on && e0 + j < E) h[j] = p[e0 + j];
      }
    }
  }
  __device__ __forceinline__ void take(float (&x)[PER]) const {
#pragma unroll
    for (int i = 0; i < PER / V; ++i) {
      const T* h = reinterpret_cast<const T*>(&u[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) x[i * V + j] = to_f32(h[j]);
    }
  }
  // element q of the lane is expert (sub + L (q / V)) V + q % V
  template <int LS> __device__ __forceinline__ void keys(int first, int sub, typename RouteKey<TY>::T (&y)[LS]) const {
#pragma unroll
    for (int j = 0; j < LS; j += 2) {
      const int q = first + j, e = (sub + L * (q / V)) * V + q % V;
      const uint4& w = u[q / V];
      if constexpr (TY == PRSGD_TYPE_FP32) {
        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
        y[j] = RouteKey<TY>::make(__uint_as_float(r[q % V]), e);
        y[j + 1] = RouteKey<TY>::make(__uint_as_float(r[q % V + 1]), e + 1);
      } else {
        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
        RouteKey<TY>::pair(r[q % V / 2], e, y[j], y[j + 1]);
      }
    }
  }
};

template <int TY, int PER, int L, int LS>
__global__ void __launch_bounds__(256, 2) route_lanes_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  using Key = RouteKey<TY>;
  constexpr int V = 16 / sizeof(T), TOK = 32 / L;     // tokens of a warp at a time
  op_pdl_wait();
  op_pdl_trigger();
  route_clear_status(a);
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
  RouteRow<TY, PER, L> next;
  auto request = [&](int64_t t) {
    next.request(logits + t * a.row_stride, a.E, sub, t < a.T && (a.live == nullptr || a.live[g * a.T + t] != 0), a.vec != 0);
  };
  const int64_t first = ((int64_t)blockIdx.x * 8 + warp) * TOK;
  request(first + lane / L);
  for (int64_t t0 = first; t0 < a.T; t0 += step) {
    const int64_t t = t0 + lane / L, row = g * a.T + t;
    const bool in = t < a.T;
    float x[PER];
    next.take(x);
    typename Key::T l[LS];
#pragma unroll
    for (int i = 0; i < PER / LS; ++i) {
      typename Key::T y[LS];
      next.template keys<LS>(i * LS, sub, y);
      route_sort<LS>(y);
      if (i == 0) {
#pragma unroll
        for (int j = 0; j < LS; ++j) l[j] = y[j];
      } else {
        route_merge<LS>(l, y);
      }
    }
    request(t + step);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
      typename Key::T y[LS];
#pragma unroll
      for (int j = 0; j < LS; ++j) y[j] = __shfl_xor_sync(0xffffffffu, l[j], o);
      route_merge<LS>(l, y);
    }
    const bool dead = Key::none(l[0]);                // a dead token, or one whose every logit is -inf
    const float top = dead ? 0.f : Key::value(l[0]);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; i += 2) {
      route_exp_below(x[i], x[i + 1], top);
      sum += x[i];
      sum += x[i + 1];
    }
    sum = lanes_sum<L>(sum);
    const float inv = dead ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = fmaf(x[i], inv, acc[i]);
    alive += !dead && sub == 0 ? 1 : 0;
    // lane `sub` of a token writes its entries sub * OWN, sub * OWN + 1, ...
    constexpr int OWN = LS >= L ? LS / L : 1;
    typename Key::T mine[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      mine[i] = l[i];
#pragma unroll
      for (int q = 1; q < LS / OWN; ++q)
        if (sub == q) mine[i] = l[q * OWN + i];
    }
    float w[OWN], chosen = 0.f;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      w[i] = sub * OWN + i < a.k ? route_exp_below(Key::value(mine[i]), top) : 0.f;
      chosen += w[i];
    }
    float f = inv;
    if (a.normalize) f = 1.f / lanes_sum<L>(chosen);
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      const int j = sub * OWN + i;
      if (j < a.k && in) {
        const int expert = Key::expert(mine[i]);
        a.experts[row * a.k + j] = dead ? -1 : expert;
        a.weights[row * a.k + j] = dead ? 0.f : w[i] * f;
        if (!dead) atomicAdd(&s_c[expert], 1);
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
  route_leave(a, g, s_p, s_c, &s_n);
}

// Gradient, any top_k (OWN choices of a token to a lane).  dlogit_e = p_e (h_e - dot) with h the balance loss's part, the same for all tokens of a group, and
// dot = sum_e p_e h_e + sum_j p_j dw_j over the chosen ones, whose own gradient is then p_j (h_j + dw_j - dot): the rows
// pass through shared memory, where the lanes that own the token's choices put those in.
__host__ __device__ constexpr int route_grad_blocks(int per) { return per <= 16 ? 3 : 2; }      // blocks an SM
template <int TY, int PER, int L, int OWN>
__global__ void __launch_bounds__(256, route_grad_blocks(PER)) route_grad_kernel(const RouteArgs a) {
  using T = typename ElemOf<TY>::type;
  constexpr int V = 16 / sizeof(T), TOK = 32 / L;
  op_pdl_wait();
  op_pdl_trigger();
  __shared__ float s_h[PER * L];
  __shared__ int s_w[8];
  __shared__ __align__(16) T s_row[8][TOK][PER * L + 16 / sizeof(T)];      // (a chunk more: tokens side by side on other banks)
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
  RouteRow<TY, PER, L> next;
  int next_e[OWN];
  float next_w[OWN];
  auto request = [&](int64_t t) {
    const bool on = t < a.T && (a.live == nullptr || a.live[g * a.T + t] != 0);
    next.request(logits + t * a.row_stride, a.E, sub, on, a.vec != 0);
#pragma unroll
    for (int q = 0; q < OWN; ++q) {                   // choice j of the token belongs to lane j % L
      const int j = q * L + sub;
      const bool has = on && a.dweights != nullptr && j < a.k;
      next_e[q] = has ? a.experts[(g * a.T + t) * a.k + j] : -1;
      next_w[q] = has ? a.dweights[(g * a.T + t) * a.k + j] : 0.f;
    }
  };
  const int64_t first = ((int64_t)blockIdx.x * 8 + warp) * TOK;
  request(first + tok);
  for (int64_t t0 = first; t0 < a.T; t0 += step) {
    const int64_t t = t0 + tok;
    const bool in = t < a.T;
    const T* p = logits + t * a.row_stride;
    float x[PER], mx = -INFINITY;
    next.take(x);
    int ej[OWN];
    float xj[OWN], dw[OWN];
#pragma unroll
    for (int q = 0; q < OWN; ++q) {
      ej[q] = (unsigned)next_e[q] < (unsigned)a.E ? next_e[q] : -1;
      dw[q] = ej[q] >= 0 ? next_w[q] : 0.f;
      xj[q] = ej[q] >= 0 ? to_f32(p[ej[q]]) : -INFINITY;
    }
    request(t + step);
#pragma unroll
    for (int i = 0; i < PER; ++i) mx = fmaxf(mx, x[i]);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float top = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < PER; i += 2) {
      route_exp_below(x[i], x[i + 1], top);
      sum += x[i];
      sum += x[i + 1];
      dot = fmaf(x[i], h[i], dot);
      dot = fmaf(x[i + 1], h[i + 1], dot);
    }
    sum = lanes_sum<L>(sum);
    const bool dead = sum == 0.f;                     // only of a row of -inf: else the largest adds 1 (a NaN or +inf makes the sum NaN, and the row with it)
    const float inv = dead ? 0.f : 1.f / sum;
    dot = lanes_sum<L>(dot) * inv;
    float pj[OWN];
    if (a.dweights != nullptr) {
      float pick = 0.f, pull = 0.f;
#pragma unroll
      for (int q = 0; q < OWN; ++q) {
        pj[q] = route_exp_below(xj[q], top) * inv;
        pick += pj[q];
        pull = fmaf(pj[q], dw[q], pull);
      }
      if (a.normalize) {                              // w_j = p_j / S: the weights' gradient through S as well
        const float s = lanes_sum<L>(pick), m = lanes_sum<L>(pull);
        pull = 0.f;
#pragma unroll
        for (int q = 0; q < OWN; ++q) {
          dw[q] = ej[q] >= 0 ? (dw[q] - m / s) / s : 0.f;
          pull = fmaf(pj[q], dw[q], pull);
        }
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
        if (ej[q] >= 0) srow[ej[q]] = from_f32<T>(pj[q] * (s_h[ej[q]] + dw[q] - dot));
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
