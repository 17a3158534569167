// Softmax cross entropy over a vocabulary and its gradient: the passes before and behind the products (kernels_vocab_tc.cuh).
//
// The tokens that have a label are moved together: row c of the operand H' of a group is its c-th live token (index[c] in the
// call's order).  Padding then costs nothing in the products, whatever its rows hold reaches nothing, and the copy (4 D
// bytes a token beside 2 V D operations) brings any stride, alignment and type to one form: rows of 16-bit values on 16-byte
// boundaries.  W is read where it lies unless it is fp32 or its rows do not begin on 16-byte boundaries; then it is copied the same way.
//
// fp32 operands become pairs of fp16 values (hi, and lo = what hi rounded off) of x 2^e, e such that the largest finite magnitude lies
// in [2^14, 2^15): 22 bits, nothing below 2^-39 of that largest.  Each operand is scaled along the axis that its product keeps, so
// that a row or column of any size spoils no other: H and W by rows for the logits, and, in copies of their own for the gradient, W by
// columns (dH = G W) and H, its rows times their share of the gradient, by columns (dW = G^T H).  G_t is held times 2^g_t, such that
// |dloss_t| + |dlse_t| lies in [2^13, 2^14); that share is 2^-g_t.
//
// G of 16-bit types is held times one power of two a group, the same with the group's largest |dloss_t| + |dlse_t|.  fp16 then has
// all its bits for p |dloss_t| down to 2^-27 of that largest and none below 2^-38: a token whose gradients are more than 2^kLiftFrom smaller is
// lifted to 2^-kLiftFrom of it, its row of dH brought back by dH's epilogue, and its row of the copy of H that dW reads taken times
// 2^-lift (what that rounds off is below 2^-36 of the largest a unit of H; lifted all the way, a token 2^10 smaller would lose bits of H there).
#pragma once
#include "rows_io.cuh"

namespace prsgd {

// Factors of a group of 16-bit types: G is held times g (and a token's lift), dH and dW are sums * back.
struct VocabScale { float g, back; };

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
  uint16_t* Hc[2]; uint16_t* Wc[2];            // [groups][Tp][pitch], [w_groups][V][pitch] or nullptr (pairs: scaled by rows)
  // fp32 operands only: factors that undo the scales, two powers of two each (their product may lie outside a float's range)
  float2* rowf; float2* colf;                  // [groups][Tp], [w_groups][Vp] of the rows of H' and W
  // and the gradient's
  uint16_t* Hm[2]; uint16_t* Wm[2];            // as Hc and Wc, scaled by columns; nullptr where no product wants them.  fp16: Hm[0] is Hc times 2^-lift
  float2* rowg;                                // [groups][Tp] of the rows of G; fp16: (2^-lift times the group's `back`, 1)
  float2* dhf; float2* dwf;                    // [w_groups][Dp], [groups][Dp] of the columns of Wm and Hm
  unsigned int* most;                          // [2][groups][Dp] largest finite magnitudes (bits) of those columns: W, H
  int64_t Vp; int Dp;                          // V, D rounded up to 256
  int most_h, most_w, most_rows;               // blocks that look for them in H and W, rows of one
  float* largest;            // [groups], fp16 gradients of many tokens: largest |dloss| + |dlse|; nullptr: each block of vocab_prep_kernel looks for it
  float4* rowp;              // [groups][Tp]: (max, log sum, dloss + dlse, dloss)
  int* rowy; int* index;     // [groups][Tp]: label; token
  int* live;                 // [groups]
  VocabScale* scale;         // [groups]
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
// e with x 2^e in [2^top, 2^(top + 1)) for finite x >= 0 by the exponent's bits, 126 at most (zeros and numbers below 2^-126 too)
__device__ __forceinline__ int vocab_exponent(float x, int top) { return min(126, top + 127 - (int)(__float_as_uint(x) >> 23)); }
__device__ __forceinline__ float vocab_power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }       // -126 <= e <= 127
__device__ __forceinline__ float2 vocab_halves(int n) { return make_float2(vocab_power(n / 2), vocab_power(n - n / 2)); }
// Scale of a token's row of G, from what its gradients are, and its row's share of dW (none of a token without a gradient: its zeros must not meet
// values that its scale sent beyond fp16).
__device__ __forceinline__ int vocab_g_exponent(float dloss, float dlse) {
  const float d = finite_abs(fabsf(dloss) + fabsf(dlse));
  return d > 0.f ? vocab_exponent(d, 13) : 0;
}
constexpr int kLiftFrom = 12;
__device__ __forceinline__ int vocab_lift(float dloss, float dlse, int group_exponent) {        // (0 of a token without a gradient)
  const float d = finite_abs(fabsf(dloss) + fabsf(dlse));
  return d > 0.f ? max(0, vocab_exponent(d, 13) - group_exponent - kLiftFrom) : 0;
}
__device__ __forceinline__ float vocab_share(float dloss, float dlse) {
  return dloss == 0.f && dlse == 0.f ? 0.f : vocab_power(-vocab_g_exponent(dloss, dlse));
}

__global__ void __launch_bounds__(256) vocab_zero_kernel(unsigned int* p, int64_t n) {
  op_pdl_wait();
  op_pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0u;
}

// Largest finite magnitudes of the columns of W and of the live rows of H times their share of the gradient (fp32 operands): a block takes
// 128 columns of some rows, a warp every eighth of them, four requests of a lane at a time.
__global__ void __launch_bounds__(256) vocab_columns_kernel(const VocabPrep a) {
  __shared__ float sm[8][128];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (int)blockIdx.y * 128 + lane * 4;
  const bool of_w = (int)blockIdx.x >= a.most_h;
  if (of_w && g >= a.w_groups) return;
  const float* x = of_w ? static_cast<const float*>(a.W) + g * a.w_group : static_cast<const float*>(a.H) + g * a.h_group;
  const int64_t begin = (int64_t)(blockIdx.x - (of_w ? a.most_h : 0)) * a.most_rows, end = min(of_w ? a.V : a.T, begin + a.most_rows);
  const int64_t pitch = of_w ? a.w_row : a.h_row;
  const bool vec = (of_w ? a.vec_w : a.vec_h) != 0 && c + 4 <= a.D;
  float most[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t r0 = begin + warp; r0 < end; r0 += 32) {
    float f[4][4], share[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + 8 * j;
      share[j] = r < end ? 1.f : 0.f;
      if (!of_w && r < end) {
        const int64_t t = g * a.T + r;
        const int y = a.labels[t];
        const float dl = a.dloss ? a.dloss[t] : 0.f, ds = a.dlse ? a.dlse[t] : 0.f;
        share[j] = y >= 0 && y < a.V ? vocab_share(dl, ds) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) f[j][i] = 0.f;
      if (share[j] == 0.f) continue;
      const float* from = x + r * pitch + c;
      if (vec) {
        const float4 q = *reinterpret_cast<const float4*>(from);
        f[j][0] = q.x; f[j][1] = q.y; f[j][2] = q.z; f[j][3] = q.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < a.D) f[j][i] = from[i];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) most[i] = fmaxf(most[i], finite_abs(f[j][i] * share[j]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sm[warp][lane * 4 + i] = most[i];
  __syncthreads();
  if (threadIdx.x >= 128) return;
  float m = sm[0][threadIdx.x];
  for (int w = 1; w < 8; ++w) m = fmaxf(m, sm[w][threadIdx.x]);
  if (m > 0.f) atomicMax(a.most + ((of_w ? 0 : a.groups) + g) * a.Dp + (int64_t)blockIdx.y * 128 + threadIdx.x, __float_as_uint(m));      // (order of no matter)
}

// A row of D elements into an operand row, a warp's lanes eight elements each, several pieces in flight.
constexpr int kVocabAhead = 4, kSplitAhead = 2;
template <int TY, bool VEC, int N>
__device__ __forceinline__ void vocab_load_row(const typename ElemOf<TY>::type* from, int c0, int D, Raw8<TY> (&r)[N]) {
  using T = typename ElemOf<TY>::type;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = c0 + j * 256;
    if (VEC && c + 8 <= D) {
      r[j] = load_raw<TY>(from + c);
    } else {
      T* e = reinterpret_cast<T*>(&r[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = c + i < D ? from[c + i] : from_f32<T>(0.f);
    }
  }
}
// Where `shared`, also times `share`, rounded again where that leaves fp16's normal numbers.
template <int TY, bool VEC>
__device__ __forceinline__ void vocab_copy_row(const typename ElemOf<TY>::type* from, uint16_t* to, int D, int lane, uint16_t* shared = nullptr, float share = 1.f) {
  for (int c0 = lane * 8; c0 < D; c0 += 256 * kVocabAhead) {
    Raw8<TY> r[kVocabAhead];
    vocab_load_row<TY, VEC>(from, c0, D, r);
#pragma unroll
    for (int j = 0; j < kVocabAhead; ++j) {
      if (c0 + j * 256 >= D) break;
      *reinterpret_cast<uint4*>(to + c0 + j * 256) = r[j].q[0];
      if (TY != PRSGD_TYPE_FP16 || shared == nullptr) continue;
      float v[8];
      unpack8<TY>(r[j], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= share;
      store_raw<TY>(reinterpret_cast<typename ElemOf<TY>::type*>(shared + c0 + j * 256), v);
    }
  }
}
// Eight scaled values as pairs.  An infinity goes to lo beside a zero: as hi it would meet the zeros among the other operand's lo.
__device__ __forceinline__ void vocab_pairs(const float (&v)[8], uint16_t* hi, uint16_t* lo) {
  uint4 u, w;
  __half* p = reinterpret_cast<__half*>(&u);
  __half* q = reinterpret_cast<__half*>(&w);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = __float2half_rn(fabsf(v[i]) == INFINITY ? 0.f : v[i]);
    q[i] = __float2half_rn(v[i] - __half2float(p[i]));
  }
  *reinterpret_cast<uint4*>(hi) = u;
  *reinterpret_cast<uint4*>(lo) = w;
}
// A row of fp32 values as pairs, scaled by its largest, whose factors go to `undo`; and, where by_col, times `share` and scaled by columns.  Read
// once up to 512 columns.
template <bool VEC>
__device__ __forceinline__ void vocab_split_row(const float* from, uint16_t* hi, uint16_t* lo, float2* undo, uint16_t* by_col, uint16_t* by_col_lo, float share,
                                                const unsigned int* most, int D, int lane) {
  constexpr int F = PRSGD_TYPE_FP32;
  Raw8<F> r[kSplitAhead];
  float v[8], top = 0.f;
  for (int c0 = lane * 8; c0 < D; c0 += 256 * kSplitAhead) {
    vocab_load_row<F, VEC>(from, c0, D, r);
#pragma unroll
    for (int j = 0; j < kSplitAhead; ++j) {
      unpack8<F>(r[j], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(v[i]));
    }
  }
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int e = vocab_exponent(top, 14);
  const float scale = vocab_power(e);
  if (lane == 0) *undo = vocab_halves(-e);
  for (int c0 = lane * 8; c0 < D; c0 += 256 * kSplitAhead) {
    if (D > 256 * kSplitAhead) vocab_load_row<F, VEC>(from, c0, D, r);
#pragma unroll
    for (int j = 0; j < kSplitAhead; ++j) {
      const int c = c0 + j * 256;
      if (c >= D) break;
      float x[8];
      unpack8<F>(r[j], v);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = v[i] * scale;
      vocab_pairs(x, hi + c, lo + c);
      if (by_col == nullptr) continue;
      const uint4 m[2] = {*reinterpret_cast<const uint4*>(most + c), *reinterpret_cast<const uint4*>(most + c + 4)};
      const unsigned int* bits = reinterpret_cast<const unsigned int*>(m);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = v[i] * share * vocab_power(vocab_exponent(__uint_as_float(bits[i]), 14));
      vocab_pairs(x, by_col + c, by_col_lo + c);
    }
  }
}

// All tokens of a group by THREADS threads: f(token, whether it is live, |dloss| + |dlse|), eight of a thread requested together.
template <int THREADS, typename F>
__device__ __forceinline__ void vocab_tokens(const VocabPrep& a, int64_t g, F&& f) {
  constexpr int kAhead = 8;
  const int32_t* labels = a.labels + g * a.T;
  const float* const dloss = a.grad && a.dloss ? a.dloss + g * a.T : nullptr;
  const float* const dlse = a.grad && a.dlse ? a.dlse + g * a.T : nullptr;
  for (int64_t t0 = threadIdx.x; t0 < a.T; t0 += THREADS * kAhead) {
    int y[kAhead];
    float d[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      y[j] = t0 + j * THREADS < a.T ? labels[t0 + j * THREADS] : -1;
      d[j] = 0.f;
    }
    if (dloss != nullptr) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) d[j] = t0 + j * THREADS < a.T ? fabsf(dloss[t0 + j * THREADS]) : 0.f;
    }
    if (dlse != nullptr) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) d[j] += t0 + j * THREADS < a.T ? fabsf(dlse[t0 + j * THREADS]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) f(t0 + j * THREADS, y[j] >= 0 && y[j] < a.V, d[j]);
  }
}

// Largest |dloss| + |dlse| of a group's live tokens, before vocab_prep_kernel: of many tokens each of its blocks would read them all (16384
// tokens: 150 MB from L2 in all, 15 us).
__global__ void __launch_bounds__(1024) vocab_largest_kernel(const VocabPrep a) {
  __shared__ float sm[32];
  op_pdl_wait();
  op_pdl_trigger();
  float most = 0.f;
  vocab_tokens<1024>(a, blockIdx.x, [&](int64_t, bool on, float d) { most = fmaxf(most, on ? finite_abs(d) : 0.f); });
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  most = sm[threadIdx.x];
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (threadIdx.x == 0) a.largest[blockIdx.x] = most;
}

// Blocks x < h_blocks of a group move its live rows together, the others copy W.  A block counts the live tokens before its own (and, of fp16 and
// up to kLargestApart tokens, looks for the group's largest gradient); the group's first block counts all, finds the scales, and zeroes the rows behind the last live one that a
// product may read.
template <int TY>
__global__ void __launch_bounds__(256, 4) vocab_prep_kernel(const VocabPrep a) {
  using T = typename ElemOf<TY>::type;
  __shared__ float smf[8];
  __shared__ int smi[8];
  __shared__ int place[256];
  __shared__ float shares[256];
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool SPLIT = TY == PRSGD_TYPE_FP32, LIFT = TY == PRSGD_TYPE_FP16;
  const unsigned int* most_w = SPLIT && a.grad ? a.most + g * a.Dp : nullptr;
  const unsigned int* most_h = SPLIT && a.grad ? a.most + (a.groups + g) * a.Dp : nullptr;
  if ((int)blockIdx.x >= a.h_blocks) {                     // ---- W
    if (g >= a.w_groups) return;
    const T* W = static_cast<const T*>(a.W) + g * a.w_group;
    for (int64_t v = (int64_t)(blockIdx.x - a.h_blocks) * 8 + warp; v < a.V; v += (int64_t)a.w_blocks * 8) {
      const int64_t o = (g * a.V + v) * a.pitch;
      const T* from = W + v * a.w_row;
      if constexpr (SPLIT) {
        float2* undo = a.colf + g * a.Vp + v;
        uint16_t* m = a.Wm[0] ? a.Wm[0] + o : nullptr;
        if (a.vec_w) vocab_split_row<true>(from, a.Wc[0] + o, a.Wc[1] + o, undo, m, a.Wm[1] + o, 1.f, most_w, a.D, lane);
        else vocab_split_row<false>(from, a.Wc[0] + o, a.Wc[1] + o, undo, m, a.Wm[1] + o, 1.f, most_w, a.D, lane);
      } else {
        if (a.vec_w) vocab_copy_row<TY, true>(from, a.Wc[0] + o, a.D, lane);
        else vocab_copy_row<TY, false>(from, a.Wc[0] + o, a.D, lane);
      }
    }
    return;
  }
  const int32_t* labels = a.labels + g * a.T;
  const int64_t per = (a.T + a.h_blocks - 1) / a.h_blocks, begin = min(a.T, blockIdx.x * per), end = min(a.T, begin + per);
  auto is_live = [&](int y) { return y >= 0 && y < a.V; };
  const bool whole = blockIdx.x == 0 || (LIFT && a.grad && a.largest == nullptr);          // (looks at all tokens)
  int before = 0, all = 0;
  float most = 0.f;
  if (!whole) {
    for (int64_t t = threadIdx.x; t < begin; t += 256) before += is_live(labels[t]) ? 1 : 0;
  } else {
    vocab_tokens<256>(a, g, [&](int64_t t, bool on, float d) {
      all += on ? 1 : 0;
      before += on && t < begin ? 1 : 0;
      most = fmaxf(most, on ? finite_abs(d) : 0.f);
    });
  }
  before = vocab_block_sum(before, smi);
  if (blockIdx.x == 0) all = vocab_block_sum(all, smi);
  if (whole && a.grad) most = vocab_block_max(most, smf);
  if (LIFT && a.grad && a.largest != nullptr) most = a.largest[g];
  const int e_group = most > 0.f ? vocab_exponent(most, 13) : 0;
  if (blockIdx.x == 0) {
    if (g == 0) {
      if (threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
      for (int i = threadIdx.x; i < a.n_counters; i += 256) a.counters[i] = 0u;
    }
    if (threadIdx.x == 0) {
      a.live[g] = all;
      a.scale[g] = {vocab_power(e_group), vocab_power(-e_group)};
    }
    if (SPLIT && a.grad) {
      for (int c = threadIdx.x; c < a.D; c += 256) {
        a.dwf[g * a.Dp + c] = vocab_halves(-vocab_exponent(__uint_as_float(most_h[c]), 14));
        if (g < a.w_groups) a.dhf[g * a.Dp + c] = vocab_halves(-vocab_exponent(__uint_as_float(most_w[c]), 14));
      }
    }
    if (a.grad && (!SPLIT || a.Hm[0])) {
      const int64_t last = min((int64_t)(all + 63) / 64 * 64, a.T);      // (behind T the tensor maps read zeros)
      for (int64_t r = all + warp; r < last; r += 8)
        for (int c = lane * 8; c < a.pitch; c += 256) {
          const int64_t o = (g * a.Tp + r) * a.pitch + c;
          *reinterpret_cast<uint4*>((a.Hm[0] ? a.Hm[0] : a.Hc[0]) + o) = make_uint4(0, 0, 0, 0);
          if (SPLIT) *reinterpret_cast<uint4*>(a.Hm[1] + o) = make_uint4(0, 0, 0, 0);
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
          const float dl = a.dloss ? a.dloss[o] : 0.f, ds = a.dlse ? a.dlse[o] : 0.f;
          const int e = SPLIT ? vocab_g_exponent(dl, ds) : LIFT ? vocab_lift(dl, ds, e_group) : 0;
          const float2 up = vocab_halves(e);
          a.rowp[c] = make_float4(a.stats[2 * o], a.stats[2 * o + 1], (dl + ds) * up.x * up.y, dl * up.x * up.y);
          if (SPLIT) { a.rowg[c] = vocab_halves(-e); shares[threadIdx.x] = vocab_share(dl, ds); }
          if (LIFT) {                              // (e_group + e is at most the token's own exponent less kLiftFrom)
            a.rowg[c] = make_float2(vocab_power(-(e_group + e)), 1.f);
            shares[threadIdx.x] = e <= 126 ? vocab_power(-e) : 0.f;
          }
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
        const T* from = H + (t0 + i) * a.h_row;
        if constexpr (SPLIT) {
          float2* undo = a.rowf + g * a.Tp + c;
          uint16_t* m = a.Hm[0] ? a.Hm[0] + o : nullptr;
          const float share = a.grad ? shares[i] : 1.f;
          if (a.vec_h) vocab_split_row<true>(from, a.Hc[0] + o, a.Hc[1] + o, undo, m, a.Hm[1] + o, share, most_h, a.D, lane);
          else vocab_split_row<false>(from, a.Hc[0] + o, a.Hc[1] + o, undo, m, a.Hm[1] + o, share, most_h, a.D, lane);
        } else {
          uint16_t* m = LIFT && a.Hm[0] ? a.Hm[0] + o : nullptr;
          const float share = LIFT && a.grad ? shares[i] : 1.f;
          if (a.vec_h) vocab_copy_row<TY, true>(from, a.Hc[0] + o, a.D, lane, m, share);
          else vocab_copy_row<TY, false>(from, a.Hc[0] + o, a.D, lane, m, share);
        }
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
// What differences to a largest logit are taken to: classes may have logits of -infinity, and so many of them that a part has no others.
__device__ __forceinline__ float vocab_base(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float2 vocab_merge(float2 p, float2 q) {
  constexpr float kLog2e = 1.4426950408889634f;
  const float m = fmaxf(p.x, q.x);
  const float base = vocab_base(m);
  return make_float2(m, p.y * vt_exp2((p.x - base) * kLog2e) + q.y * vt_exp2((q.x - base) * kLog2e));
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
