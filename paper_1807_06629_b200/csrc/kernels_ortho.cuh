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
  unsigned int* done;                    // [batch] finished tasks
  DeviceStatus* status;
  int64_t xp, sp;
  int chunks;
};
struct NsShape { int batch, rows, cols; };

// Squares of one chunk of rows of a matrix; applies the momentum on the way.  Grid (chunks, batch).
template <int TY, int VEC>
__global__ void __launch_bounds__(256) ns_norm_kernel(const NsShape sh, const NsSource src, const NsBuffers buf) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int m = blockIdx.y;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    buf.done[m] = 0u;
    if (m == 0) { *buf.claim = 0u; buf.status->error = 0u; }
  }
  __shared__ double s_part[8];
  double sum = 0.0;
  if (src.active == nullptr || src.active[m] != 0) {
    const int per = (sh.rows + (int)gridDim.x - 1) / (int)gridDim.x;
    const int r1 = min(sh.rows, ((int)blockIdx.x + 1) * per);
    int tx = 1;
    while (tx < 256 && tx * VEC < sh.cols) tx <<= 1;
    const int cx = (threadIdx.x & (tx - 1)) * VEC, ry = threadIdx.x / tx, dy = 256 / tx;
    const T* g = static_cast<const T*>(src.G) + (int64_t)m * src.g_batch;
    float* v = src.V + (int64_t)m * src.v_batch;
    for (int r = (int)blockIdx.x * per + ry; r < r1; r += dy) {
      for (int c = cx; c < sh.cols; c += tx * VEC) {
        float u[VEC];
        if (src.G != nullptr) {
          if constexpr (VEC == 4) {
            if constexpr (TY == PRSGD_TYPE_FP32) {
              const float4 q = *reinterpret_cast<const float4*>(g + (int64_t)r * src.g_row + c);
              u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
            } else {
              const uint2 q = *reinterpret_cast<const uint2*>(g + (int64_t)r * src.g_row + c);
              const T* h = reinterpret_cast<const T*>(&q);
#pragma unroll
              for (int i = 0; i < VEC; ++i) u[i] = to_f32(h[i]);
            }
          } else {
            u[0] = to_f32(g[(int64_t)r * src.g_row + c]);
          }
        }
        if (src.V != nullptr) {
          float* at = v + (src.v_tiled ? wtile_offset(src.v_tile, r, c) : (int64_t)r * src.v_row + c);
          float w[VEC];
          if constexpr (VEC == 4) {
            const float4 q = *reinterpret_cast<const float4*>(at);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
          } else {
            w[0] = at[0];
          }
          if (src.G != nullptr) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              w[i] = fmaf(src.mu, w[i], u[i]);
              u[i] = src.nesterov ? fmaf(src.mu, w[i], u[i]) : w[i];
            }
            if constexpr (VEC == 4) *reinterpret_cast<float4*>(at) = make_float4(w[0], w[1], w[2], w[3]);
            else at[0] = w[0];
          } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) u[i] = w[i];
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum += (double)u[i] * (double)u[i];
      }
    }
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

// X_0 = U / (||U|| + eps).  Grid (chunks, batch).
template <int TY, int VEC>
__global__ void __launch_bounds__(256) ns_pack_kernel(const NsShape sh, const NsSource src, const NsBuffers buf, float eps) {
  using T = typename ElemOf<TY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int m = blockIdx.y;
  if (src.active != nullptr && src.active[m] == 0) return;
  double total = 0.0;
  for (int i = 0; i < buf.chunks; ++i) total += buf.part[(int64_t)m * buf.chunks + i];
  // (the quotient in 64 bits: a norm beyond fp32's range still divides; 1 / 0 of a zero matrix with eps = 0 gives NaN)
  const double inv = (double)kNsScale / (sqrt(total) + (double)eps);
  const int per = (sh.rows + (int)gridDim.x - 1) / (int)gridDim.x;
  const int r1 = min(sh.rows, ((int)blockIdx.x + 1) * per);
  int tx = 1;
  while (tx < 256 && tx * VEC < sh.cols) tx <<= 1;
  const int cx = (threadIdx.x & (tx - 1)) * VEC, ry = threadIdx.x / tx, dy = 256 / tx;
  const T* g = static_cast<const T*>(src.G) + (int64_t)m * src.g_batch;
  const float* v = src.V + (int64_t)m * src.v_batch;
  __half* xh = buf.x[0][0] + (int64_t)m * sh.rows * buf.xp;
  __half* xl = buf.x[0][1] + (int64_t)m * sh.rows * buf.xp;
  for (int r = (int)blockIdx.x * per + ry; r < r1; r += dy) {
    for (int c = cx; c < sh.cols; c += tx * VEC) {
      __half hi[VEC], lo[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float u = 0.f;
        if (src.G != nullptr) u = to_f32(g[(int64_t)r * src.g_row + c + i]);
        if (src.V != nullptr) {
          const float w = v[src.v_tiled ? wtile_offset(src.v_tile, r, c + i) : (int64_t)r * src.v_row + c + i];
          u = src.G == nullptr || !src.nesterov ? w : fmaf(src.mu, w, u);
        }
        ns_split((float)((double)u * inv), hi[i], lo[i]);
      }
      const int64_t o = (int64_t)r * buf.xp + c;
      if constexpr (VEC == 4) {
        *reinterpret_cast<uint2*>(xh + o) = *reinterpret_cast<uint2*>(hi);
        *reinterpret_cast<uint2*>(xl + o) = *reinterpret_cast<uint2*>(lo);
      } else {
        xh[o] = hi[0]; xl[o] = lo[0];
      }
    }
  }
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

// One product of the chain on the CUDA cores, 64 x 64 tiles.  kind 0: A, 1: P, 2: X.
struct NsGemmArgs {
  NsShape sh; NsBuffers buf; NsDest dst;
  int kind, from, last, split;           // from: buffer that holds X
  float a, b, c;
};

__global__ void __launch_bounds__(256) ns_gemm_kernel(const NsGemmArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  const int m = blockIdx.z;
  if (a.dst.active != nullptr && a.dst.active[m] == 0) return;
  const bool tall = a.sh.rows > a.sh.cols;
  const int s = min(a.sh.rows, a.sh.cols), l = max(a.sh.rows, a.sh.cols);
  const int R = a.kind == 2 ? a.sh.rows : s, C = a.kind == 2 ? a.sh.cols : s, K = a.kind == 0 ? l : s;
  __shared__ float L[16][65], Rr[16][65];
  const __half* xh = a.buf.x[a.from][0] + (int64_t)m * a.sh.rows * a.buf.xp;
  const __half* xl = a.buf.x[a.from][1] + (int64_t)m * a.sh.rows * a.buf.xp;
  const int64_t so = (int64_t)m * s * a.buf.sp;
  auto X = [&](int r, int c) { return __half2float(xh[(int64_t)r * a.buf.xp + c]) + (a.split ? __half2float(xl[(int64_t)r * a.buf.xp + c]) : 0.f); };
  auto S = [&](__half* const* q, int r, int c) {
    return __half2float(q[0][so + (int64_t)r * a.buf.sp + c]) + (a.split ? __half2float(q[1][so + (int64_t)r * a.buf.sp + c]) : 0.f);
  };
  auto left = [&](int i, int k) { return a.kind == 0 ? (tall ? X(k, i) : X(i, k)) : a.kind == 1 ? S(a.buf.A, i, k) : (tall ? X(i, k) : S(a.buf.P, i, k)); };
  auto right = [&](int k, int j) { return a.kind == 0 ? (tall ? X(k, j) : X(j, k)) : a.kind == 1 ? S(a.buf.A, k, j) : (tall ? S(a.buf.P, k, j) : X(k, j)); };
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ti = threadIdx.x / 16, tj = threadIdx.x % 16;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += 16) {
    for (int e = threadIdx.x; e < 1024; e += 256) {
      const int k = e & 15, i = e >> 4;
      L[k][i] = i0 + i < R && k0 + k < K ? left(i0 + i, k0 + k) : 0.f;
      Rr[k][i] = j0 + i < C && k0 + k < K ? right(k0 + k, j0 + i) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(L[k][ti * 4 + p], Rr[k][tj * 4 + q], acc[p][q]);
    __syncthreads();
  }
  for (int p = 0; p < 4; ++p)
    for (int q = 0; q < 4; ++q) {
      const int i = i0 + ti * 4 + p, j = j0 + tj * 4 + q;
      if (i >= R || j >= C) continue;
      float v = acc[p][q] * kNsUnscale;                 // 256 times the product
      if (a.kind < 2) {
        if (a.kind == 1) v = a.c * v + a.b * S(a.buf.A, i, j) + (i == j ? a.a * kNsScale : 0.f);
        __half hi, lo;
        ns_split(v, hi, lo);
        __half* const* o = a.kind == 0 ? a.buf.A : a.buf.P;
        o[0][so + (int64_t)i * a.buf.sp + j] = hi;
        if (a.split) o[1][so + (int64_t)i * a.buf.sp + j] = lo;
        continue;
      }
      const int64_t xo = (int64_t)m * a.sh.rows * a.buf.xp + (int64_t)i * a.buf.xp + j;
      if (!a.split && !a.last) v += a.a * __half2float(a.buf.x[a.from][1][xo]);
      if (a.last) { ns_store_final(a.dst, m, i, j, v * kNsUnscale); continue; }
      __half hi, lo;
      ns_split(v, hi, lo);
      a.buf.x[1 - a.from][0][xo] = hi;
      a.buf.x[1 - a.from][1][xo] = lo;
    }
}

}  // namespace prsgd
