// Softmax cross entropy over a vocabulary and its gradient: the passes before and behind the products (kernels_vocab_tc.cuh).
//
// The tokens that have a label are moved together: row c of the operand H' of a group is its c-th live token (index[c] in the
// call's order).  Padding then costs nothing in the products, whatever its rows hold reaches nothing, and the copy (4 D
// bytes a token beside 2 V D operations) brings any stride, alignment and type to one form: rows of 16-bit values on 16-byte
// boundaries.  fp32 operands become pairs of fp16 values (hi, and lo = what hi rounded off) of x 2^e, e per group such that the
// largest finite magnitude lies in [2^14, 2^15): 22 bits, nothing below 2^-39 of that largest.  W is read where it lies unless
// it is fp32 or its rows do not begin on 16-byte boundaries; then it is copied the same way.
#pragma once
#include "rows_io.cuh"

namespace prsgd {

constexpr int kVocabAmaxBlocks = 64;           // partial maxima per group and operand

// Factors of a group, two for each power of two that may lie outside a float's range.
struct VocabScale {
  float z1, z2;              // logit = sum * z1 * z2
  float g;                   // G is held times g
  float dh1, dh2;            // dH = sum * dh1 * dh2
  float dw1, dw2;
  float h, w;                // operands are held times these
  float pad[7];
};

struct VocabPrep {
  const void* H; int64_t h_row, h_group;
  const void* W; int64_t w_row, w_group;
  int h_type;                // element type of the call
  const int32_t* labels;
  const float* stats; const float* dloss; const float* dlse;
  int64_t groups, T, V;
  int D, grad, vec_h, vec_w;
  int64_t Tp;                // rows of H' (T rounded up to 64)
  int pitch;                 // elements of an operand row (D rounded up to 8)
  int w_groups;              // groups of W (1: shared)
  uint16_t* Hc[2]; uint16_t* Wc[2];            // [groups][Tp][pitch], [w_groups][V][pitch] or nullptr
  float4* rowp;              // [groups][Tp]: (max, log sum, dloss + dlse, dloss)
  int* rowy; int* index;     // [groups][Tp]: label; token
  int* live;                 // [groups]
  VocabScale* scale;         // [groups]
  float* amax;               // [groups][2][kVocabAmaxBlocks]
  float* loss; float* out_stats;
  void* dH; int64_t dh_row, dh_group; int vec_dh;
  unsigned int* counters; int n_counters;
  DeviceStatus* status;
  int h_blocks, w_blocks;    // blocks of a group
};

__device__ __forceinline__ float vocab_block_max(float v, float* sm) {
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sm[threadIdx.x & 7];
  for (int o = 4; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ int vocab_block_sum(int v, int* sm) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sm[threadIdx.x & 7];
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) <= 3.402823466e38f ? fabsf(x) : 0.f; }
// e with x 2^e in [2^top, 2^(top + 1)), 0 for x = 0; within a normal float's exponents
__device__ __forceinline__ int vocab_exponent(float x, int top) { return x > 0.f ? max(-126, min(126, top - ilogbf(x))) : 0; }
__device__ __forceinline__ void vocab_halves(int n, float& a, float& b) { a = exp2f((float)(n / 2)); b = exp2f((float)(n - n / 2)); }

// Largest finite magnitudes of the live rows of H and of W (fp32 operands only), a warp a row and four requests of a lane at a time.
__global__ void __launch_bounds__(256) vocab_amax_kernel(const VocabPrep a) {
  __shared__ float sm[8];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool of_w = blockIdx.x >= kVocabAmaxBlocks;
  const int blk = blockIdx.x % kVocabAmaxBlocks;
  const float* x = of_w ? static_cast<const float*>(a.W) + (a.w_groups > 1 ? g : 0) * a.w_group : static_cast<const float*>(a.H) + g * a.h_group;
  const int64_t rows = of_w ? a.V : a.T, pitch = of_w ? a.w_row : a.h_row;
  const bool vec = (of_w ? a.vec_w : a.vec_h) != 0;
  float most = 0.f;
  for (int64_t r = blk * 8 + warp; r < rows; r += kVocabAmaxBlocks * 8) {
    if (!of_w) {
      const int y = a.labels[g * a.T + r];
      if (y < 0 || y >= a.V) continue;
    }
    const float* row = x + r * pitch;
    const int wide = vec ? a.D & ~3 : 0;
    for (int c0 = 0; c0 < wide; c0 += 512) {
      float4 f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = c0 + (j * 32 + lane) * 4;
        f[j] = c < wide ? *reinterpret_cast<const float4*>(row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) most = fmaxf(fmaxf(fmaxf(most, finite_abs(f[j].x)), fmaxf(finite_abs(f[j].y), finite_abs(f[j].z))), finite_abs(f[j].w));
    }
    for (int c0 = wide; c0 < a.D; c0 += 128) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = c0 + j * 32 + lane < a.D ? row[c0 + j * 32 + lane] : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) most = fmaxf(most, finite_abs(f[j]));
    }
  }
  most = vocab_block_max(most, sm);
  if (threadIdx.x == 0) a.amax[(g * 2 + of_w) * kVocabAmaxBlocks + blk] = most;
}

// A row of D elements into operand rows (of one plane or two), a warp's lanes eight elements each, several pieces in flight.
template <int TY, bool VEC>
__device__ __forceinline__ void vocab_copy_row(const typename ElemOf<TY>::type* from, uint16_t* hi, uint16_t* lo, int D, float scale, int lane) {
  using T = typename ElemOf<TY>::type;
  constexpr int kAhead = TY == PRSGD_TYPE_FP32 ? 2 : 4;
  for (int c0 = lane * 8; c0 < D; c0 += 256 * kAhead) {
    Raw8<TY> r[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int c = c0 + j * 256;
      if (VEC && c + 8 <= D) {
        r[j] = load_raw<TY>(from + c);
      } else {
        T* e = reinterpret_cast<T*>(&r[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = c + i < D ? from[c + i] : from_f32<T>(0.f);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int c = c0 + j * 256;
      if (c >= D) break;
      if constexpr (TY == PRSGD_TYPE_FP32) {
        float v[8];
        unpack8<TY>(r[j], v);
        uint4 u, w;
        __half* p = reinterpret_cast<__half*>(&u);
        __half* q = reinterpret_cast<__half*>(&w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = v[i] * scale;
          p[i] = __float2half_rn(x);
          q[i] = __float2half_rn(x - __half2float(p[i]));
        }
        *reinterpret_cast<uint4*>(hi + c) = u;
        *reinterpret_cast<uint4*>(lo + c) = w;
      } else {
        *reinterpret_cast<uint4*>(hi + c) = r[j].q[0];
      }
    }
  }
}

// Blocks x < h_blocks of a group move its live rows together, the others copy W.  A block counts the live tokens before its own; the
// group's first block counts all, finds the scales, and zeroes the rows behind the last live one that a product may read.
template <int TY>
__global__ void __launch_bounds__(256) vocab_prep_kernel(const VocabPrep a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float smf[8];
  __shared__ int smi[8];
  __shared__ int place[256];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int eh = 0, ew = 0;
  if constexpr (TY == PRSGD_TYPE_FP32) {                   // (every warp by itself)
    const float* m = a.amax + g * 2 * kVocabAmaxBlocks;
    float h = fmaxf(m[lane], m[lane + 32]), w = fmaxf(m[lane + 64], m[lane + 96]);
    static_assert(kVocabAmaxBlocks == 64);
    for (int o = 16; o > 0; o >>= 1) {
      h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, o));
      w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, o));
    }
    eh = vocab_exponent(h, 14);
    ew = vocab_exponent(w, 14);
  }
  if ((int)blockIdx.x >= a.h_blocks) {                     // ---- W
    if (g >= a.w_groups) return;
    const float scale = exp2f((float)ew);
    const T* W = static_cast<const T*>(a.W) + g * a.w_group;
    for (int64_t v = (int64_t)(blockIdx.x - a.h_blocks) * 8 + warp; v < a.V; v += (int64_t)a.w_blocks * 8) {
      const int64_t o = (g * a.V + v) * a.pitch;
      uint16_t* lo = TY == PRSGD_TYPE_FP32 ? a.Wc[1] + o : nullptr;
      if (a.vec_w) vocab_copy_row<TY, true>(W + v * a.w_row, a.Wc[0] + o, lo, a.D, scale, lane);
      else vocab_copy_row<TY, false>(W + v * a.w_row, a.Wc[0] + o, lo, a.D, scale, lane);
    }
    return;
  }
  const int32_t* labels = a.labels + g * a.T;
  const int64_t per = (a.T + a.h_blocks - 1) / a.h_blocks, begin = min(a.T, blockIdx.x * per), end = min(a.T, begin + per);
  auto is_live = [&](int y) { return y >= 0 && y < a.V; };
  int before = 0;
  for (int64_t t = threadIdx.x; t < begin; t += 256) before += is_live(labels[t]) ? 1 : 0;
  before = vocab_block_sum(before, smi);
  const float hs = exp2f((float)eh);
  if (blockIdx.x == 0) {
    if (g == 0) {
      if (threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
      for (int i = threadIdx.x; i < a.n_counters; i += 256) a.counters[i] = 0u;
    }
    int all = 0;
    float most = 0.f;
    for (int64_t t = threadIdx.x; t < a.T; t += 256) {
      if (!is_live(labels[t])) continue;
      ++all;
      if (a.grad) most = fmaxf(most, finite_abs((a.dloss ? fabsf(a.dloss[g * a.T + t]) : 0.f) + (a.dlse ? fabsf(a.dlse[g * a.T + t]) : 0.f)));
    }
    all = vocab_block_sum(all, smi);
    most = vocab_block_max(most, smf);
    if (threadIdx.x == 0) {
      a.live[g] = all;
      const int e = vocab_exponent(most, 13);
      VocabScale s{};
      vocab_halves(-(eh + ew), s.z1, s.z2);
      s.g = exp2f((float)e);
      vocab_halves(-(e + ew), s.dh1, s.dh2);
      vocab_halves(-(e + eh), s.dw1, s.dw2);
      s.h = hs; s.w = exp2f((float)ew);
      a.scale[g] = s;
    }
    if (a.grad) {
      const int64_t last = min((int64_t)(all + 63) / 64 * 64, a.T);      // (behind T the tensor maps read zeros)
      for (int64_t r = all + warp; r < last; r += 8)
        for (int c = lane * 8; c < a.pitch; c += 256) {
          const int64_t o = (g * a.Tp + r) * a.pitch + c;
          *reinterpret_cast<uint4*>(a.Hc[0] + o) = make_uint4(0, 0, 0, 0);
          if (TY == PRSGD_TYPE_FP32) *reinterpret_cast<uint4*>(a.Hc[1] + o) = make_uint4(0, 0, 0, 0);
        }
    }
  }
  const T* H = static_cast<const T*>(a.H) + g * a.h_group;
  for (int64_t t0 = begin; t0 < end; t0 += 256) {
    const int64_t t = t0 + threadIdx.x;
    const int y = t < end ? labels[t] : -1;
    const bool on = is_live(y);
    const unsigned int mask = __ballot_sync(0xffffffffu, on);
    __syncthreads();
    if (lane == 0) smi[warp] = __popc(mask);
    __syncthreads();
    int at = before + __popc(mask & ((1u << lane) - 1u));
    for (int w = 0; w < 8; ++w) {
      if (w < warp) at += smi[w];
      before += smi[w];
    }
    place[threadIdx.x] = on ? at : -1;
    if (t < end) {
      const int64_t c = g * a.Tp + at, o = g * a.T + t;
      if (on) {
        a.rowy[c] = y;
        a.index[c] = (int)t;
        if (a.grad) {
          const float dl = a.dloss ? a.dloss[o] : 0.f, both = dl + (a.dlse ? a.dlse[o] : 0.f);
          a.rowp[c] = make_float4(a.stats[2 * o], a.stats[2 * o + 1], both, dl);
        }
      } else if (!a.grad) {
        a.loss[o] = 0.f;
        a.out_stats[2 * o] = 0.f;
        a.out_stats[2 * o + 1] = 0.f;
      }
    }
    __syncthreads();
    const int here = (int)min((int64_t)256, end - t0);
    for (int i = warp; i < here; i += 8) {
      const int c = place[i];
      if (c >= 0) {
        const int64_t o = (g * a.Tp + c) * a.pitch;
        uint16_t* lo = TY == PRSGD_TYPE_FP32 ? a.Hc[1] + o : nullptr;
        if (a.vec_h) vocab_copy_row<TY, true>(H + (t0 + i) * a.h_row, a.Hc[0] + o, lo, a.D, hs, lane);
        else vocab_copy_row<TY, false>(H + (t0 + i) * a.h_row, a.Hc[0] + o, lo, a.D, hs, lane);
      } else if (a.dH != nullptr) {
        const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        T* to = static_cast<T*>(a.dH) + g * a.dh_group + (t0 + i) * a.dh_row;
        for (int q = lane * 8; q < a.D; q += 256) {
          if (a.vec_dh) store8<TY, true>(to + q, min(8, a.D - q), zero);
          else store8<TY, false>(to + q, min(8, a.D - q), zero);
        }
      }
    }
  }
}

// Largest logit and sum of every live token from those of its runs of the vocabulary: a block takes ROWS tokens, 256 / ROWS threads each.
struct VocabJoin {
  const float2* part;        // [groups][runs][Tp]
  const float* zy; const int* index; const int* live;
  int64_t Tp, T;
  int runs;
  float* loss; float* stats;
};
__device__ __forceinline__ float vt_exp2(float x) {        // (to 2 ulp; results below 2^-126 are 0)
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 vocab_merge(float2 p, float2 q) {
  constexpr float kLog2e = 1.4426950408889634f;
  const float m = fmaxf(p.x, q.x);
  if (m == -INFINITY && p.y == 0.f && q.y == 0.f) return make_float2(m, 0.f);      // (runs without columns)
  return make_float2(m, p.y * vt_exp2((p.x - m) * kLog2e) + q.y * vt_exp2((q.x - m) * kLog2e));
}
template <int ROWS>
__global__ void __launch_bounds__(256) vocab_join_kernel(const VocabJoin a) {
  constexpr int LANES = 256 / ROWS, kAhead = 8;
  __shared__ float2 got[LANES][ROWS];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int live = a.live[g], r = threadIdx.x % ROWS, row = blockIdx.x * ROWS + r, share = threadIdx.x / ROWS;
  if ((int)blockIdx.x * ROWS >= live) return;
  float2 sum = make_float2(-INFINITY, 0.f);
  if (row < live) {
    const float2* part = a.part + g * a.runs * a.Tp + row;
    for (int k = share; k < a.runs; k += LANES * kAhead) {
      float2 p[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) p[j] = k + j * LANES < a.runs ? part[(int64_t)(k + j * LANES) * a.Tp] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) sum = vocab_merge(sum, p[j]);
    }
  }
  got[share][r] = sum;
  __syncthreads();
  for (int n = LANES / 2; n > 0; n >>= 1) {
    if (share < n) got[share][r] = vocab_merge(got[share][r], got[share + n][r]);
    __syncthreads();
  }
  if (share != 0 || row >= live) return;
  sum = got[0][r];
  const float log_sum = logf(sum.y);
  const int64_t o = g * a.T + a.index[g * a.Tp + row];
  a.loss[o] = log_sum + (sum.x - a.zy[g * a.Tp + row]);
  a.stats[2 * o] = sum.x;
  a.stats[2 * o + 1] = log_sum;
}

// dH of the live tokens from its parts along the vocabulary, in order.
struct VocabSum {
  const float* acc;          // [groups][parts][Tp][acc_pitch]
  const int* index; const int* live;
  int64_t Tp, groups;
  int parts, acc_pitch, D;
  void* dH; int64_t dh_row, dh_group;
};
// SHARED: the warps of a block take every eighth part of one row, else a row each.
template <int TY, bool VEC, bool SHARED>
__global__ void __launch_bounds__(256) vocab_sum_kernel(const VocabSum a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float sums[SHARED ? 8 : 1][SHARED ? 256 : 1];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = ((int)blockIdx.y * 32 + lane) * 8, live = a.live[g];
  const int64_t step = a.Tp * a.acc_pitch;
  for (int64_t r = SHARED ? blockIdx.x : (int64_t)blockIdx.x * 8 + warp; r < live; r += (int64_t)gridDim.x * (SHARED ? 1 : 8)) {
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8];
    const float* from = a.acc + (g * a.parts * a.Tp + r) * a.acc_pitch + c;
    if (c < a.D) {
#pragma unroll 4
      for (int p = SHARED ? warp : 0; p < a.parts; p += SHARED ? 8 : 1) {
        unpack8<PRSGD_TYPE_FP32>(load_raw<PRSGD_TYPE_FP32>(from + p * step), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
      }
    }
    if constexpr (SHARED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[warp][i * 32 + lane] = sum[i];
      __syncthreads();
      if (warp == 0) {
        for (int w = 1; w < 8; ++w)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum[i] += sums[w][i * 32 + lane];
      }
      __syncthreads();
      if (warp != 0) continue;
    }
    if (c < a.D) store8<TY, VEC>(static_cast<T*>(a.dH) + g * a.dh_group + a.index[g * a.Tp + r] * a.dh_row + c, min(8, a.D - c), sum);
  }
}

}  // namespace prsgd
