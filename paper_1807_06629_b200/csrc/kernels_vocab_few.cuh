// The vocabulary loss of few tokens a group: W is read once, where it lies and in any type, by dot products on the CUDA cores.
//
// The bytes of W bound it (22 bytes a cycle and SM at the HBM rate, 11 elements of 16 bits); a token costs one product an element, in packed
// pairs, so kFewTurn of them fit beside the loads; of more, neighbouring blocks take kFewTurn each and find W in L2.  A warp takes four rows of W at a time, so that what it reads of H from
// shared memory serves four rows; the largest logit and the sum of exponentials run along in registers, and a second launch joins
// the blocks'.  1 x 1 x 32000 x 1024: bf16 20 us (10 of them W from HBM, 8 two launches and the reading of H), fp32 27 (20).
#pragma once
#include "kernels_vocab.cuh"
#include "vocab_plan.h"

namespace prsgd {

constexpr int kFewRows = 4, kFewWarps = 8;

struct VocabFew {
  const void* H; int64_t h_row, h_group;
  const void* W; int64_t w_row, w_group;
  const int32_t* labels;
  int64_t V, per;                              // rows of W a block takes
  int T, D, dp;                                // dp: D rounded up to 8
  int blocks;                                  // of a group, for each kFewTurn of its tokens
  int turns;                                   // kFewTurn tokens each: the blocks of all turns that take the same rows lie side by side and read them at a time
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
  extern __shared__ __align__(16) float h[];                 // [NT][dp], zeros for tokens without a label
  __shared__ float2 sums[kFewWarps][NT];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int blk = (int)(blockIdx.x / (unsigned)a.turns), first = (int)(blockIdx.x - (unsigned)(blk * a.turns)) * kFewTurn, count = min(NT, a.T - first);
  if (blockIdx.x == 0 && g == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  int y[NT];
  bool any = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    y[t] = t < count ? a.labels[g * a.T + first + t] : -1;
    if (y[t] >= a.V) y[t] = -1;
    any |= y[t] >= 0;
  }
  if (!any) return;                            // (nobody reads this group's parts)
  const T* H = static_cast<const T*>(a.H) + g * a.h_group + first * a.h_row;
  for (int i = threadIdx.x; i < NT * a.dp; i += 32 * kFewWarps) {
    const int t = i / a.dp, c = i - t * a.dp;
    bool on = false;
#pragma unroll
    for (int k = 0; k < NT; ++k) on |= k == t && y[k] >= 0;
    h[i] = on && c < a.D ? to_f32(H[t * a.h_row + c]) : 0.f;
  }
  __syncthreads();
  const T* W = static_cast<const T*>(a.W) + g * a.w_group;
  const int64_t end = min(a.V, (blk + 1) * a.per);
  float2 run[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) run[t] = make_float2(-INFINITY, 0.f);
  for (int64_t v0 = blk * a.per + warp * kFewRows; v0 < end; v0 += kFewWarps * kFewRows) {
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
        if (lane == 0 && v0 + r == y[t]) a.zy[g * a.T + first + t] = z;
        const float m = fmaxf(run[t].x, z), base = vocab_base(m);
        run[t] = make_float2(m, run[t].y * vt_exp2((run[t].x - base) * 1.4426950408889634f) + vt_exp2((z - base) * 1.4426950408889634f));
      }
    }
  }
  if (lane == 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[warp][t] = run[t];
  }
  __syncthreads();
  if ((int)threadIdx.x < count) {
    float2 all = sums[0][threadIdx.x];
    for (int w = 1; w < kFewWarps; ++w) all = vocab_merge(all, sums[w][threadIdx.x]);
    a.part[(g * a.T + first + threadIdx.x) * a.blocks + blk] = all;
  }
}

// A warp a token.
__global__ void __launch_bounds__(32 * kFewTokens) vocab_few_join_kernel(const VocabFew a) {
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

// ---- gradient: a token or two a group ---------------------------------------------------------------------------
// One pass over W: a block takes 32 rows at a time; its warps form their logits as above and G from them (in fp32: nothing is rounded on the
// way), then a thread takes eight columns of every row again (from L1), writes dW = sum_t g_t H_t and adds g_t W to its dH_t in
// registers.  The blocks' dH are added up by a second launch.  Bytes bound it: W read, dW written; 1 x 1 x 32000 x 1024 bf16 44 us (20 of them the
// bytes; two blocks an SM that take turns at waiting), 1 x 131072 x 2048 270 us (164).
constexpr int kFewTile = kFewWarps * kFewRows;
static_assert(kFewGradDim == 32 * kFewWarps * 8, "a thread has eight columns");

struct VocabFewGrad {
  VocabFew f;
  const float* in_stats; const float* dloss; const float* dlse;
  void* dW; int64_t dw_row, dw_group; int accumulate;
  void* dH; int64_t dh_row, dh_group;
  float* acc;                                  // [groups][blocks][T][dp], or nullptr: no dH
  int lanes;                                   // threads side by side along a row (a power of two); the others take rows of their own
};

template <int TY, int OTY, bool VEC, int NT>
__global__ void __launch_bounds__(32 * kFewWarps) vocab_few_grad_kernel(const VocabFewGrad b) {
  using T = typename ElemOf<TY>::type;
  using O = typename ElemOf<OTY>::type;
  constexpr float kLog2e = 1.4426950408889634f;
  extern __shared__ __align__(16) float h[];                 // [NT][dp]; at the end [row groups][NT][dp]
  __shared__ float gs[2][kFewTile][NT];
  const VocabFew& a = b.f;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && g == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  int y[NT];
  float top[NT], log_sum[NT], both[NT], hot[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t o = g * a.T + t;
    y[t] = t < a.T ? a.labels[o] : -1;
    if (y[t] >= a.V) y[t] = -1;
    const bool on = y[t] >= 0;
    top[t] = on ? b.in_stats[2 * o] : 0.f;
    log_sum[t] = on ? b.in_stats[2 * o + 1] : 0.f;
    hot[t] = on && b.dloss ? b.dloss[o] : 0.f;
    both[t] = hot[t] + (on && b.dlse ? b.dlse[o] : 0.f);
  }
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
  O* dW = b.dW ? static_cast<O*>(b.dW) + g * b.dw_group : nullptr;
  const int sub = threadIdx.x / b.lanes, groups = 32 * kFewWarps / b.lanes, c0 = (threadIdx.x - sub * b.lanes) * 8, n = max(0, min(8, a.D - c0));
  float mine[NT][8], sum[NT][8];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mine[t][i] = n > 0 ? h[t * a.dp + c0 + i] : 0.f;
      sum[t][i] = 0.f;
    }
  const int64_t end = min(a.V, (blockIdx.x + 1) * a.per);
  int turn = 0;
  for (int64_t v0 = blockIdx.x * a.per; v0 < end; v0 += kFewTile, turn ^= 1) {
    {                                          // logits and G of four rows a warp
      const int64_t r0 = v0 + warp * kFewRows;
      const int rows = (int)max((int64_t)0, min((int64_t)kFewRows, end - r0));
      float2 acc[kFewRows][NT];
#pragma unroll
      for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = make_float2(0.f, 0.f);
#pragma unroll 2
      for (int c = lane * 8; c < a.D; c += 256) {
        float w[kFewRows][8];
        if constexpr (VEC) {
          Raw8<TY> raw[kFewRows];
#pragma unroll
          for (int r = 0; r < kFewRows; ++r) raw[r] = r < rows ? load_raw<TY>(W + (r0 + r) * a.w_row + c) : zero_raw<TY>();
#pragma unroll
          for (int r = 0; r < kFewRows; ++r) unpack8<TY>(raw[r], w[r]);
        } else {
#pragma unroll
          for (int r = 0; r < kFewRows; ++r) load8<TY, false>(W + (r0 + r) * a.w_row + c, r < rows ? a.D - c : 0, w[r]);
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
      for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float z = acc[r][t].x + acc[r][t].y;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
          const float p = both[t] * vt_exp2(((z - top[t]) - log_sum[t]) * kLog2e);
          if (lane == 0) gs[turn][warp * kFewRows + r][t] = y[t] >= 0 && r < rows ? (r0 + r == y[t] ? p - hot[t] : p) : 0.f;
        }
    }
    __syncthreads();                           // (the next turn's go to the other half)
    if (n > 0) {
      const int rows = (int)min((int64_t)kFewTile, end - v0);
      // four rows' loads before the first store (which the compiler has to take for a store to W)
#pragma unroll 1
      for (int r0 = sub; r0 < rows; r0 += 4 * groups) {
        float w[4][8];
        if constexpr (VEC) {
          Raw8<TY> raw[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[j] = r0 + j * groups < rows ? load_raw<TY>(W + (v0 + r0 + j * groups) * a.w_row + c0) : zero_raw<TY>();
#pragma unroll
          for (int j = 0; j < 4; ++j) unpack8<TY>(raw[j], w[j]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) load8<TY, false>(W + (v0 + r0 + j * groups) * a.w_row + c0, r0 + j * groups < rows ? n : 0, w[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = r0 + j * groups;
          if (r >= rows) break;
          float d[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float k = gs[turn][r][t];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              d[i] = fmaf(k, mine[t][i], d[i]);
              sum[t][i] = fmaf(k, w[j][i], sum[t][i]);
            }
          }
          if (dW == nullptr) continue;
          O* to = dW + (v0 + r) * b.dw_row + c0;
          if (b.accumulate) {
            float old[8];
            load8<OTY, VEC>(to, VEC ? 8 : n, old);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] += old[i];
          }
          store8<OTY, VEC>(to, VEC ? 8 : n, d);
        }
      }
    }
  }
  if (b.acc == nullptr) return;
  __syncthreads();                             // (everyone is done with h)
  if (n > 0) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[(sub * NT + t) * a.dp + c0 + i] = sum[t][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * a.dp; i += 32 * kFewWarps) {
    const int t = i / a.dp, c = i - t * a.dp;
    float all = 0.f;
    for (int k = 0; k < groups; ++k) all += h[(k * NT + t) * a.dp + c];
    b.acc[((g * a.blocks + blockIdx.x) * a.T + t) * a.dp + c] = all;
  }
}

// dH from the blocks' sums, in order: a block takes 32 columns of a token, a warp every eighth of the sums.
template <int TY>
__global__ void __launch_bounds__(256) vocab_few_sum_kernel(const VocabFewGrad b) {
  using T = typename ElemOf<TY>::type;
  __shared__ float sums[8][32];
  const VocabFew& a = b.f;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int t = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
  const int y = a.labels[g * a.T + t];
  const bool on = y >= 0 && y < a.V;
  float sum = 0.f;
  if (on && c < a.D) {
    const float* from = b.acc + (g * a.blocks * a.T + t) * a.dp + c;
#pragma unroll 8
    for (int k = warp; k < a.blocks; k += 8) sum += from[(int64_t)k * a.T * a.dp];
  }
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp != 0 || c >= a.D) return;
  for (int w = 1; w < 8; ++w) sum += sums[w][lane];
  static_cast<T*>(b.dH)[g * b.dh_group + t * b.dh_row + c] = from_f32<T>(sum);
}

}  // namespace prsgd
