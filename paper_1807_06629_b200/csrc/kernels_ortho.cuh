// Newton-Schulz orthogonalisation of a batch of matrices and the Muon step built on it.
//   X_0 = U / (||U||_F + eps),   per step:  A = X X^T (the short side; X^T X for tall matrices),
//   P = a I + b A + c A^2,   X <- P X (X P),   and at the end  out = beta out + alpha X.
//
// Numbers.  X, A and P are held as fp16 values times 256 (their entries lie within a few units, and 2^8 keeps the
// smallest ones of a wide matrix above fp16's subnormals), products are summed in fp32.  X carries a second fp16
// value `lo` = what `hi` rounded off, 22 bits together.  With 32-bit precision A and P carry one too and a product is
// hi hi + hi lo + lo hi.  With 16-bit precision the products take `hi` alone, but a X_lo is still added to the product
// on every step but the last: the directions that U does not contain (a momentum of low rank has many) grow by a = 3.44
// per step, 485-fold over five, and X's rounding noise would grow with them (4e-2 of the result at rank 8, 6e-4 with lo).
#pragma once
#include "ops_common.cuh"

namespace prsgd {

constexpr float kNsScale = 256.f, kNsUnscale = 1.f / 256.f;
constexpr int kNsChunks = 64;          // most blocks that sum one matrix's squares

// Where U comes from: G alone, V alone (G == nullptr), or V <- mu V + G with U = V or G + mu V.
struct NsSource {
  const void* G; int64_t g_row, g_batch;
  float* V; int64_t v_row, v_batch;
  WTile v_tile; int v_tiled;             // tile-major V (rows of the parameter store)
  float mu; int nesterov;
  const uint8_t* active;                 // [batch] or nullptr: matrices that take part
};
// Where the result goes: out = beta out + alpha X (beta == 0: out is not read), and a bf16 copy of it.
struct NsDest {
  void* out; int type; int64_t row, batch;
  uint16_t* shadow;                      // same offsets as out, or nullptr
  WTile tile; int tiled;
  float alpha, beta;
  const uint8_t* active;
};
struct NsBuffers {
  __half* x[2][2];                       // [buffer][hi, lo]: [batch][rows][xp]
  __half* A[2]; __half* P[2];            // [hi, lo]: [batch][s][sp]
  double* part;                          // [batch][chunks]
  unsigned int* claim;                   // next unclaimed task
  unsigned int* done;                    // [batch][panels] tiles that have been added to a panel
  int panels;
  // A's tiles formed in `parts` parts of the contraction (few tiles of long ones): the parts' sums and, per warp of a tile's
  // epilogue, how many have been left
  int parts, gram_tiles;                 // (gram_tiles: of a matrix)
  float* part_sums;                      // [batch][tiles][parts][16][4096]
  unsigned int* part_count;              // [batch][tiles][16]
  DeviceStatus* status;
  int own_status;                        // the workspace's own: cleared by the call.  0: a context's, an error in it turns the call into a no-op
  int64_t xp, sp;
  int chunks;
};
struct NsShape { int batch, rows, cols; };

// VEC neighbouring elements of a row as fp32
template <int TY, int VEC>
__device__ __forceinline__ void ns_load(const typename ElemOf<TY>::type* p, float (&u)[VEC]) {
  using T = typename ElemOf<TY>::type;
  if constexpr (VEC == 1) {
    u[0] = to_f32(p[0]);
  } else if constexpr (TY == PRSGD_TYPE_FP32) {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      const float4 x = reinterpret_cast<const float4*>(p)[q];
      u[4 * q] = x.x; u[4 * q + 1] = x.y; u[4 * q + 2] = x.z; u[4 * q + 3] = x.w;
    }
  } else {
    static_assert(VEC == 4);
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    const T* h = reinterpret_cast<const T*>(&x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) u[i] = to_f32(h[i]);
  }
}

// How a block of 256 threads walks its rows: `tx` threads side by side along a row, 4 rows of a thread at a time so
// that their loads are in flight together (one at a time both passes waited for latency: 25 + 35 us at 16 x 1024 x 1024).
constexpr int kNsRows = 4;
template <int VEC, typename F>
__device__ __forceinline__ void ns_walk(const NsShape& sh, F&& f) {
  const int per = (sh.rows + (int)gridDim.x - 1) / (int)gridDim.x;
  const int r1 = min(sh.rows, ((int)blockIdx.x + 1) * per);
  int tx = 1;
  while (tx < 256 && tx * VEC < sh.cols) tx <<= 1;
  const int cx = (threadIdx.x & (tx - 1)) * VEC, ry = threadIdx.x / tx, dy = 256 / tx;
  for (int r = (int)blockIdx.x * per + ry; r < r1; r += dy * kNsRows)
    for (int c = cx; c < sh.cols; c += tx * VEC) f(r, dy, r1, c);
}

// MODE 0: G alone, 1: V alone, 2: both.  Squares of one chunk of rows of a matrix; applies the momentum on the way.
// Grid (chunks, batch).
template <int TY, int VEC, int MODE>
__global__ void __launch_bounds__(256) ns_norm_kernel(const NsShape sh, const NsSource src, const NsBuffers buf) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int m = blockIdx.y;
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < buf.panels; i += 256) buf.done[(int64_t)m * buf.panels + i] = 0u;
    if (buf.parts > 1)
      for (int i = threadIdx.x; i < buf.gram_tiles * 16; i += 256) buf.part_count[(int64_t)m * buf.gram_tiles * 16 + i] = 0u;
    if (m == 0 && threadIdx.x == 0) {
      *buf.claim = 0u;
      if (buf.own_status) buf.status->error = 0u;
    }
  }
  if (!buf.own_status && buf.status->error != 0u) return;
  __shared__ double s_part[8];
  double sum = 0.0;
  if (src.active == nullptr || src.active[m] != 0) {
    const T* g = static_cast<const T*>(src.G) + (int64_t)m * src.g_batch;
    float* v = src.V + (int64_t)m * src.v_batch;
    ns_walk<VEC>(sh, [&](int r, int dy, int r1, int c) {
      float u[kNsRows][VEC], w[kNsRows][VEC];
      float* at[kNsRows];
#pragma unroll
      for (int k = 0; k < kNsRows; ++k) {
        const int rr = r + k * dy;
        const bool on = rr < r1;
#pragma unroll
        for (int i = 0; i < VEC; ++i) u[k][i] = w[k][i] = 0.f;
        if (MODE != 1 && on) ns_load<TY, VEC>(g + (int64_t)rr * src.g_row + c, u[k]);
        if (MODE != 0 && on) {
          at[k] = v + (src.v_tiled ? wtile_offset(src.v_tile, rr, c) : (int64_t)rr * src.v_row + c);
          ns_load<PRSGD_TYPE_FP32, VEC>(at[k], w[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kNsRows; ++k) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (MODE == 1) u[k][i] = w[k][i];
          if (MODE == 2) {
            w[k][i] = fmaf(src.mu, w[k][i], u[k][i]);
            u[k][i] = src.nesterov ? fmaf(src.mu, w[k][i], u[k][i]) : w[k][i];
          }
          sum += (double)u[k][i] * (double)u[k][i];
        }
        if (MODE == 2 && r + k * dy < r1) {
          if constexpr (VEC == 4) *reinterpret_cast<float4*>(at[k]) = make_float4(w[k][0], w[k][1], w[k][2], w[k][3]);
          else at[k][0] = w[k][0];
        }
      }
    });
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 8; ++w) t += s_part[w];
    buf.part[(int64_t)m * buf.chunks + blockIdx.x] = t;
  }
}

// hi = fp16(256 x), lo = fp16(256 x - hi)
__device__ __forceinline__ void ns_split(float x256, __half& hi, __half& lo) {
  hi = __float2half_rn(x256);
  lo = __float2half_rn(x256 - __half2float(hi));
}

// 256 / (||U|| + eps) as two factors that neither overflow nor vanish for any norm fp32 matrices have: a power of two
// (exact) and the rest (rounded once).  NaN for a norm that is none.
__device__ __forceinline__ float2 ns_inverse(double norm) {
  if (!(norm < 1e300)) return make_float2(1.f, __int_as_float(0x7fffffff));
  const int e = norm > 0.0 ? ilogb(norm) / 2 : 0;
  const double p = scalbn(1.0, -e);
  return make_float2((float)p, (float)((double)kNsScale / norm / p));
}

// X_0 = U / (||U|| + eps).  Grid (chunks, batch).
template <int TY, int VEC, int MODE>
__global__ void __launch_bounds__(256) ns_pack_kernel(const NsShape sh, const NsSource src, const NsBuffers buf, float eps) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int m = blockIdx.y;
  if (src.active != nullptr && src.active[m] == 0) return;
  __shared__ float2 s_inv;
  if (threadIdx.x < 32) {
    double total = 0.0;
    for (int i = threadIdx.x; i < buf.chunks; i += 32) total += buf.part[(int64_t)m * buf.chunks + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (threadIdx.x == 0) s_inv = ns_inverse(sqrt(total) + (double)eps);
  }
  __syncthreads();
  const float2 inv = s_inv;
  const T* g = static_cast<const T*>(src.G) + (int64_t)m * src.g_batch;
  const float* v = src.V + (int64_t)m * src.v_batch;
  __half* xh = buf.x[0][0] + (int64_t)m * sh.rows * buf.xp;
  __half* xl = buf.x[0][1] + (int64_t)m * sh.rows * buf.xp;
  ns_walk<VEC>(sh, [&](int r, int dy, int r1, int c) {
    float u[kNsRows][VEC], w[kNsRows][VEC];
#pragma unroll
    for (int k = 0; k < kNsRows; ++k) {
      const int rr = r + k * dy;
      const bool on = rr < r1;
#pragma unroll
      for (int i = 0; i < VEC; ++i) u[k][i] = w[k][i] = 0.f;
      if (on && (MODE == 0 || (MODE == 2 && src.nesterov))) ns_load<TY, VEC>(g + (int64_t)rr * src.g_row + c, u[k]);
      if (on && MODE != 0) ns_load<PRSGD_TYPE_FP32, VEC>(v + (src.v_tiled ? wtile_offset(src.v_tile, rr, c) : (int64_t)rr * src.v_row + c), w[k]);
    }
#pragma unroll
    for (int k = 0; k < kNsRows; ++k) {
      if (r + k * dy >= r1) break;
      __align__(8) __half hi[VEC], lo[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float x = MODE == 0 ? u[k][i] : (MODE == 2 && src.nesterov) ? fmaf(src.mu, w[k][i], u[k][i]) : w[k][i];
        ns_split(x * inv.x * inv.y, hi[i], lo[i]);
      }
      const int64_t o = (int64_t)(r + k * dy) * buf.xp + c;
      if constexpr (VEC == 4) {
        *reinterpret_cast<uint2*>(xh + o) = *reinterpret_cast<uint2*>(hi);
        *reinterpret_cast<uint2*>(xl + o) = *reinterpret_cast<uint2*>(lo);
      } else {
        xh[o] = hi[0]; xl[o] = lo[0];
      }
    }
  });
}

__device__ __forceinline__ void ns_store_final(const NsDest& d, int m, int r, int c, float x) {
  const int64_t o = (int64_t)m * d.batch + (d.tiled ? wtile_offset(d.tile, r, c) : (int64_t)r * d.row + c);
  if (d.type == PRSGD_TYPE_FP32) {
    float* p = static_cast<float*>(d.out) + o;
    const float y = d.beta != 0.f ? fmaf(d.alpha, x, d.beta * *p) : d.alpha * x;
    *p = y;
    if (d.shadow != nullptr) d.shadow[o] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
  } else if (d.type == PRSGD_TYPE_BF16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(d.out) + o;
    *p = __float2bfloat16_rn(d.beta != 0.f ? fmaf(d.alpha, x, d.beta * __bfloat162float(*p)) : d.alpha * x);
  } else {
    __half* p = static_cast<__half*>(d.out) + o;
    *p = __float2half_rn(d.beta != 0.f ? fmaf(d.alpha, x, d.beta * __half2float(*p)) : d.alpha * x);
  }
}

}  // namespace prsgd
