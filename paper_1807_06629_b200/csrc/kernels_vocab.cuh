// Softmax cross entropy over a vocabulary and its gradient, logits formed in pieces: z = H W^T, G = (dloss + dlse) softmax(z) -
// dloss onehot, dH = G W, dW = G^T H.  Products of 64 x 64 tiles on the CUDA cores.
#pragma once
#include "rows_io.cuh"

namespace prsgd {

constexpr int kVocabTile = 64, kVocabK = 16, kVocabRun = 8;    // tiles of a block's run along the vocabulary

struct VocabArgs {
  const void* H; int64_t h_row, h_group;
  const void* W; int64_t w_row, w_group;
  const int32_t* labels;
  int64_t T, V;
  int D;
  int runs;
  float2* part;              // [groups][T][runs] (max, sum of e^(z - max))
  float* zy;                 // [groups][T]
  float* loss; float* stats;
  const float* in_stats; const float* dloss; const float* dlse;
  float* G;                  // [groups][T][piece]
  float* acc;                // [groups][T][D]
  int64_t piece, v0, pv;     // columns of a piece; first of this one, how many
  void* dH; int64_t dh_row, dh_group;
  void* dW; int64_t dw_row, dw_group;
  int accumulate;
  DeviceStatus* status;
};

// 64 x 64 sums of a(row, k) b(col, k) over k, 4 x 4 a thread of 16 x 16: element (4 ty + i, 4 tx + j)
template <typename FA, typename FB>
__device__ __forceinline__ void vocab_tile(int64_t K, FA&& fa, FB&& fb, float (&acc)[4][4], float (&sa)[kVocabK][kVocabTile + 4], float (&sb)[kVocabK][kVocabTile + 4]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  for (int64_t k0 = 0; k0 < K; k0 += kVocabK) {
    for (int e = threadIdx.x; e < kVocabK * kVocabTile; e += 256) {
      const int k = e & 15, r = e >> 4;
      sa[k][r] = k0 + k < K ? fa(r, k0 + k) : 0.f;
      sb[k][r] = k0 + k < K ? fb(r, k0 + k) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kVocabK; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
}

template <int TY>
__global__ void __launch_bounds__(256) vocab_stats_kernel(const VocabArgs a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float sa[kVocabK][kVocabTile + 4], sb[kVocabK][kVocabTile + 4];
  op_pdl_wait();
  op_pdl_trigger();
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  const int64_t g = blockIdx.z, t0 = (int64_t)blockIdx.x * kVocabTile;
  const T* H = static_cast<const T*>(a.H) + g * a.h_group;
  const T* W = static_cast<const T*>(a.W) + g * a.w_group;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float m[4], s[4];
  int y[4];
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY; s[i] = 0.f;
    y[i] = t0 + ty * 4 + i < a.T ? a.labels[g * a.T + t0 + ty * 4 + i] : -1;
  }
  for (int64_t v0 = (int64_t)blockIdx.y * kVocabRun * kVocabTile, n = 0; n < kVocabRun && v0 < a.V; ++n, v0 += kVocabTile) {
    float z[4][4];
    vocab_tile(a.D, [&](int r, int64_t k) { return t0 + r < a.T ? to_f32(H[(t0 + r) * a.h_row + k]) : 0.f; },
               [&](int r, int64_t k) { return v0 + r < a.V ? to_f32(W[(v0 + r) * a.w_row + k]) : 0.f; }, z, sa, sb);
    for (int i = 0; i < 4; ++i) {
      float most = -INFINITY;
      for (int j = 0; j < 4; ++j)
        if (v0 + tx * 4 + j < a.V) most = z[i][j] != z[i][j] ? z[i][j] : fmaxf(most, z[i][j]);
      for (int o = 1; o < 16; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      most = fmaxf(most, m[i]);
      float sum = 0.f;
      for (int j = 0; j < 4; ++j)
        if (v0 + tx * 4 + j < a.V) sum += expf(z[i][j] - most);
      for (int o = 1; o < 16; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      s[i] = s[i] * expf(m[i] - most) + sum;
      if (m[i] == -INFINITY) s[i] = sum;
      m[i] = most;
      for (int j = 0; j < 4; ++j)
        if (y[i] >= 0 && v0 + tx * 4 + j == y[i] && y[i] < a.V) a.zy[g * a.T + t0 + ty * 4 + i] = z[i][j];
    }
  }
  if (tx == 0)
    for (int i = 0; i < 4; ++i)
      if (t0 + ty * 4 + i < a.T) a.part[(g * a.T + t0 + ty * 4 + i) * a.runs + blockIdx.y] = make_float2(m[i], s[i]);
}

__global__ void __launch_bounds__(256) vocab_join_kernel(const VocabArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, at = blockIdx.y * a.T + t;
  if (t >= a.T) return;
  const int y = a.labels[at];
  float loss = 0.f, m = 0.f, log_sum = 0.f;
  if (y >= 0 && y < a.V) {
    m = -INFINITY;
    for (int r = 0; r < a.runs; ++r) m = fmaxf(m, a.part[at * a.runs + r].x);
    float s = 0.f;
    for (int r = 0; r < a.runs; ++r) {
      const float2 p = a.part[at * a.runs + r];
      s += p.y * expf(p.x - m);
    }
    log_sum = logf(s);
    loss = log_sum + (m - a.zy[at]);
  }
  a.loss[at] = loss;
  a.stats[2 * at] = m;
  a.stats[2 * at + 1] = log_sum;
}

template <int TY>
__global__ void __launch_bounds__(256) vocab_g_kernel(const VocabArgs a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float sa[kVocabK][kVocabTile + 4], sb[kVocabK][kVocabTile + 4];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z, t0 = (int64_t)blockIdx.x * kVocabTile, v0 = a.v0 + (int64_t)blockIdx.y * kVocabTile, vend = a.v0 + a.pv;
  const T* H = static_cast<const T*>(a.H) + g * a.h_group;
  const T* W = static_cast<const T*>(a.W) + g * a.w_group;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float z[4][4];
  vocab_tile(a.D, [&](int r, int64_t k) { return t0 + r < a.T ? to_f32(H[(t0 + r) * a.h_row + k]) : 0.f; },
             [&](int r, int64_t k) { return v0 + r < vend ? to_f32(W[(v0 + r) * a.w_row + k]) : 0.f; }, z, sa, sb);
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + ty * 4 + i, at = g * a.T + t;
    if (t >= a.T) break;
    const int y = a.labels[at];
    const bool live = y >= 0 && y < a.V;
    const float dl = live && a.dloss ? a.dloss[at] : 0.f, both = dl + (live && a.dlse ? a.dlse[at] : 0.f);
    for (int j = 0; j < 4; ++j) {
      const int64_t v = v0 + tx * 4 + j;
      if (v >= vend) break;
      const float p = live ? expf((z[i][j] - a.in_stats[2 * at]) - a.in_stats[2 * at + 1]) : 0.f;
      a.G[at * a.piece + v - a.v0] = live ? both * p - (v == y ? dl : 0.f) : 0.f;
    }
  }
}

template <int TY>
__global__ void __launch_bounds__(256) vocab_dh_kernel(const VocabArgs a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float sa[kVocabK][kVocabTile + 4], sb[kVocabK][kVocabTile + 4];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z, t0 = (int64_t)blockIdx.x * kVocabTile;
  const int d0 = blockIdx.y * kVocabTile;
  const T* W = static_cast<const T*>(a.W) + g * a.w_group;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float z[4][4];
  vocab_tile(a.pv, [&](int r, int64_t k) { return t0 + r < a.T ? a.G[(g * a.T + t0 + r) * a.piece + k] : 0.f; },
             [&](int r, int64_t k) { return d0 + r < a.D ? to_f32(W[(a.v0 + k) * a.w_row + d0 + r]) : 0.f; }, z, sa, sb);
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + ty * 4 + i;
    if (t >= a.T) break;
    const int y = a.labels[g * a.T + t];
    for (int j = 0; j < 4; ++j) {
      const int d = d0 + tx * 4 + j;
      if (d >= a.D) break;
      float* to = a.acc + (g * a.T + t) * a.D + d;
      const float v = y >= 0 && y < a.V ? (a.v0 > 0 ? *to : 0.f) + z[i][j] : 0.f;
      *to = v;
      if (a.v0 + a.pv == a.V) static_cast<T*>(a.dH)[g * a.dh_group + t * a.dh_row + d] = from_f32<T>(v);
    }
  }
}

template <int TY, int OTY>
__global__ void __launch_bounds__(256) vocab_dw_kernel(const VocabArgs a) {
  using T = typename ElemOf<TY>::type;
  using O = typename ElemOf<OTY>::type;
  __shared__ float sa[kVocabK][kVocabTile + 4], sb[kVocabK][kVocabTile + 4];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z, v0 = (int64_t)blockIdx.x * kVocabTile;
  const int d0 = blockIdx.y * kVocabTile;
  const T* H = static_cast<const T*>(a.H) + g * a.h_group;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float z[4][4];
  vocab_tile(a.T, [&](int r, int64_t k) { return v0 + r < a.pv ? a.G[(g * a.T + k) * a.piece + v0 + r] : 0.f; },
             [&](int r, int64_t k) {
               const int y = a.labels[g * a.T + k];
               return d0 + r < a.D && y >= 0 && y < a.V ? to_f32(H[k * a.h_row + d0 + r]) : 0.f;
             }, z, sa, sb);
  for (int i = 0; i < 4; ++i) {
    const int64_t v = v0 + ty * 4 + i;
    if (v >= a.pv) break;
    for (int j = 0; j < 4; ++j) {
      const int d = d0 + tx * 4 + j;
      if (d >= a.D) break;
      O* to = static_cast<O*>(a.dW) + g * a.dw_group + (a.v0 + v) * a.dw_row + d;
      *to = from_f32<O>((a.accumulate ? to_f32(*to) : 0.f) + z[i][j]);
    }
  }
}

}  // namespace prsgd
