// Newton-Schulz chain of matrices whose short side is at most 128, in one launch: a cluster of CTAs per matrix holds it in
// shared memory from its first reading to the result, so that nothing but the matrix itself is read and written.
//
// CTA r of the cluster keeps `w` columns (of the long side) of X as fp16 pairs.  Per step it forms its share of A = X X^T on
// the tensor cores.  Up to a short side of 32 it sends its share to all (st.async, counted on the receiver's barrier), and every
// CTA sums all of A, in rank order, and forms P = a I + b A + c A^2 in fp32 for itself (16 matrices of 10 x 1024: 37 -> 19.6 us,
// against the form for longer sides); above, each CTA fetches and sums a part of A and hands it to all, and P is formed on the
// tensor cores.  (Shares sent to the CTAs that sum them, a lane to a row: 8 x 64 x 1024 43 -> 55 us; what crosses between CTAs has to
// go from neighbouring lanes to neighbouring places.)  All products but that of P in fp32 are hi hi + hi lo + lo hi whatever
// the precision asked for: with so little work the time is that of the waits between the steps, not of the products.
// (16 matrices of 10 x 1024: about 150 us as three products a step of the chain's tiles.)
#pragma once
#include "kernels_ortho_tc.cuh"

namespace prsgd {

constexpr int kNsSmallThreads = 256, kNsSmallSide = 128, kNsSmallCtas = 8;
// columns of a CTA that fit beside A and its shares: X 256 bytes a column (512 above a short side of 64), A 32 or 64 KB,
// its shares up to 128 KB (short side up to 32), 16 KB (up to 64) or 64 KB
__host__ __device__ constexpr int ns_small_cols(int s) { return s <= 64 ? 256 : 192; }
// The whole of an SM's shared memory, whatever is needed: a second CTA on the SM would wait for the TMEM this one holds,
// and clusters that wait for one another's TMEM would wait for good.
constexpr size_t kNsSmallSmem = 225 * 1024;
__host__ __device__ constexpr int ns_small_share_bytes(int sp, int ctas) { return sp * sp * 4 * (sp <= 32 ? 4 * ctas : 1); }
__host__ __device__ constexpr int ns_small_bytes(int sp, int ctas, int w) {
  return w / 64 * 16384 * (sp <= 64 ? 1 : 2) + 2 * ((sp + 63) / 64) * 16384 + ns_small_share_bytes(sp, ctas) + 1024;
}
static_assert(ns_small_bytes(32, kNsSmallCtas, 256) <= (int)kNsSmallSmem && ns_small_bytes(64, kNsSmallCtas, 256) <= (int)kNsSmallSmem &&
              ns_small_bytes(128, kNsSmallCtas, 192) <= (int)kNsSmallSmem, "shared memory of the small form");
enum { NS_ERR_SMALL = 0x711 };

struct NsSmallArgs {
  NsShape sh; NsSource src; NsDest dst;
  DeviceStatus* status;
  int own_status;
  int steps, tall, s, l, ctas, w, sp;    // w: columns of a CTA (multiple of 64), sp: short side, multiple of 16
  float a, b, c, eps;
  int vec_out;
};

namespace ptx {
// stores into a CTA's shared memory that count their bytes on a barrier there
__device__ __forceinline__ void send_f64(uint32_t to_cluster, uint32_t bar_cluster, double v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];"
               ::"r"(to_cluster), "l"(__double_as_longlong(v)), "r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void send_data_v4(uint32_t to_cluster, uint32_t bar_cluster, float x, float y, float z, float w) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(to_cluster), "f"(x), "f"(y), "f"(z), "f"(w), "r"(bar_cluster) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_v2(uint32_t at, uint32_t x, uint32_t y) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(taddr) : "memory");
  return r;
}
// A bounded wait for what other CTAs of the cluster have sent.
__device__ __forceinline__ bool mbar_wait_sent(uint32_t bar, uint32_t parity, volatile int* abort_flag, DeviceStatus* status, unsigned what) {
  long long t0 = 0;
  for (uint32_t it = 1;; ++it) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
    if ((it & 63u) == 0u) {
      if (*abort_flag) return false;
      const long long now = clock64();
      if (t0 == 0) t0 = now;
      if (now - t0 > kWaitLimitCycles) {
        *abort_flag = 1;
        if (atomicCAS(&status->error, 0u, what) == 0u) status->where = blockIdx.x;
        return false;
      }
    }
  }
}
}  // namespace ptx

__device__ __forceinline__ float ld_shared_f32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// MODE as in ns_norm_kernel; VEC: elements of a row that are read together.
template <int TY, int MODE, int VEC>
__global__ void __launch_bounds__(kNsSmallThreads, 1) ns_small_kernel(const __grid_constant__ NsSmallArgs a) {
  using T = typename ElemOf<TY>::type;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t bars[4];                // products; norms; shares of even and of odd steps
  __shared__ __align__(8) double s_norms[kNsSmallCtas];
  __shared__ double s_part[8];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int m = (int)blockIdx.x / a.ctas, rank = (int)blockIdx.x % a.ctas;
  const uint32_t x_hi = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  // Up to a short side of 64 the 128 rows of an operand block hold X_hi and, from row sp on, X_lo: a product with both has
  // all parts.
  const bool stacked = a.sp <= 64, everyone = a.sp <= 32;
  const uint32_t x_bytes = (uint32_t)(a.w / 64) * 16384u, x_lo = x_hi + (stacked ? (uint32_t)a.sp * 128u : x_bytes);
  const uint32_t s_hi = x_hi + (stacked ? 1u : 2u) * x_bytes, s_bytes = (uint32_t)((a.sp + 63) / 64) * 16384u, s_lo = s_hi + s_bytes;
  // Shares of A, 16-byte chunks: [step & 1][sender][hi or lo rows][all], or this CTA's own: [all]
  const uint32_t shares = s_lo + s_bytes;
  const uint32_t bar = ptx::smem_u32(&bars[0]), bar_norm = bar + 8u, bar_share = bar + 16u;
  ptx::pdl_wait();
  ptx::pdl_trigger();
  if (a.own_status && blockIdx.x == 0 && threadIdx.x == 0) a.status->error = 0u;
  if (a.src.active != nullptr && a.src.active[m] == 0) return;       // (the whole cluster)
  if (threadIdx.x == 0) {
#pragma unroll 1
    for (uint32_t b = 0; b < 4; ++b) ptx::mbar_init(bar + b * 8u, 1);
    abort_flag = 0;
    ptx::fence_mbar_init();
  }
  ptx::cluster_arrive_release();                           // (the barriers are there: waited for before the first is sent to)
  if (warp == 1) ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), 512);
  // X is zeroed: its rows that a product's result depends on (rows of an operand block beyond them reach only rows of the
  // result that nobody reads, and all of A and P is written)
  const uint32_t rows_bytes = (uint32_t)(stacked ? 2 * a.sp : a.sp) * 128u;
#pragma unroll 1
  for (uint32_t block = x_hi; block < s_hi; block += 16384u)
    for (uint32_t o = threadIdx.x * 16u; o < rows_bytes; o += kNsSmallThreads * 16u) st_shared_v4(block + o, 0u, 0u, 0u, 0u);

  // element (i, j) of this CTA's X, i along the short side: G[i][j0 + j], or of a tall matrix G[j0 + j][i]
  const int j0 = rank * a.w, nj = max(0, min(a.w, a.l - j0));
  const int outer = a.tall ? nj : a.s, inner = a.tall ? a.s : nj;
  const T* const g = static_cast<const T*>(a.src.G) + (int64_t)m * a.src.g_batch;
  float* const v = a.src.V + (int64_t)m * a.src.v_batch;
  // 16-byte chunks of 8 along a row of 128 bytes, swizzled over 8 rows; 64 columns to a block of 16 KB
  auto at = [&](int i, int j) { return (uint32_t)(j >> 6) * 16384u + (uint32_t)i * 128u + (uint32_t)((((j & 63) >> 3) ^ (i & 7)) * 16) + (uint32_t)(j & 7) * 2u; };
  // U is read once: its squares are summed, and until the norm is known its fp32 bits stay in the two halves of its place
  // in X.  Warps along rows of G, lanes along columns (VEC of them each), eight rows of a warp requested together.
  auto v_at = [&](int row, int col) { return a.src.v_tiled ? wtile_offset(a.src.v_tile, row, col) : (int64_t)row * a.src.v_row + col; };
  double sum = 0.0;
  constexpr int B = 8, W = kNsSmallThreads / 32;
  __syncthreads();                                         // (X has been zeroed)
#pragma unroll 1
  for (int p = warp; p < outer; p += W * B)
#pragma unroll 1
    for (int q = lane * VEC; q < inner; q += 32 * VEC) {
      float u[B][VEC];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int pb = p + W * b;
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[b][e] = 0.f;
        if (pb >= outer) continue;
        const int row = a.tall ? j0 + pb : pb, col = a.tall ? q : j0 + q;
        if constexpr (MODE != 1) ns_load<TY, VEC>(g + (int64_t)row * a.src.g_row + col, u[b]);
        if constexpr (MODE != 0) {
          float* const o = v + v_at(row, col);
          float w[VEC];
          ns_load<PRSGD_TYPE_FP32, VEC>(o, w);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if constexpr (MODE == 1) {
              u[b][e] = w[e];
            } else {
              w[e] = fmaf(a.src.mu, w[e], u[b][e]);
              u[b][e] = a.src.nesterov ? fmaf(a.src.mu, w[e], u[b][e]) : w[e];
            }
          }
          if constexpr (MODE == 2) {
            if constexpr (VEC == 4) *reinterpret_cast<float4*>(o) = make_float4(w[0], w[1], w[2], w[3]);
            else o[0] = w[0];
          }
        }
      }
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const int pb = p + W * b;
        if (pb >= outer) continue;
        uint32_t top[VEC], low[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          sum += (double)u[b][e] * (double)u[b][e];
          top[e] = __float_as_uint(u[b][e]) >> 16; low[e] = __float_as_uint(u[b][e]) & 0xffffu;
        }
        const uint32_t o = a.tall ? at(q, pb) : at(pb, q);
        if constexpr (VEC == 4) {
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(x_hi + o), "r"(top[0] | (top[1] << 16)), "r"(top[2] | (top[3] << 16)) : "memory");
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(x_lo + o), "r"(low[0] | (low[1] << 16)), "r"(low[2] | (low[3] << 16)) : "memory");
        } else {
          asm volatile("st.shared.b16 [%0], %1;" ::"r"(x_hi + o), "h"((uint16_t)top[0]) : "memory");
          asm volatile("st.shared.b16 [%0], %1;" ::"r"(x_lo + o), "h"((uint16_t)low[0]) : "memory");
        }
      }
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_part[warp] = sum;
  __syncthreads();
  ptx::cluster_wait_acquire();
  if ((int)threadIdx.x < a.ctas) {
    double t = 0.0;
    for (int i = 0; i < 8; ++i) t += s_part[i];
    if (threadIdx.x == 0) ptx::mbar_expect_tx(bar_norm, (uint32_t)a.ctas * 8u);
    ptx::send_f64(ptx::cluster_map(ptx::smem_u32(&s_norms[rank]), threadIdx.x), ptx::cluster_map(bar_norm, threadIdx.x), t);
  }
  (void)ptx::mbar_wait_sent(bar_norm, 0u, &abort_flag, a.status, NS_ERR_SMALL);      // (after an expiry every later wait returns at once)
  double total = lane < a.ctas ? s_norms[lane] : 0.0;
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);      // (lanes 0 to 7 hold the parts)
  total = __shfl_sync(0xffffffffu, total, 0);
  const float2 inv = ns_inverse(sqrt(total) + (double)a.eps);
#pragma unroll 1
  for (int idx = (int)threadIdx.x; idx < a.s * (a.w / 8); idx += kNsSmallThreads) {
    const int row = idx / (a.w / 8);
    const uint32_t o = at(row, (idx - row * (a.w / 8)) * 8);
    const uint4 h = ld_shared_v4(x_hi + o), l = ld_shared_v4(x_lo + o);
    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
    uint32_t ho[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y0 = __uint_as_float((hw[e] << 16) | (lw[e] & 0xffffu)) * inv.x * inv.y, y1 = __uint_as_float((hw[e] & 0xffff0000u) | (lw[e] >> 16)) * inv.x * inv.y;
      ho[e] = pack_half2(y0, y1);
      const float2 f = unpack_half2(ho[e]);
      lo[e] = pack_half2(y0 - f.x, y1 - f.y);
    }
    st_shared_v4(x_hi + o, ho[0], ho[1], ho[2], ho[3]);
    st_shared_v4(x_lo + o, lo[0], lo[1], lo[2], lo[3]);
  }

  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = tmem_slot, d_s = tmem, d_x = tmem + 256u;      // sums of A and P, of X
  const int quarter = warp & 3, half = warp >> 2, i = quarter * 32 + lane;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const bool issuer = warp == 0 && ptx::elect_one();
  uint32_t parity = 0;
  // One product over k16 steps of 16.  (Four steps to a turn, at fixed distances: computing descriptors between the MMAs took
  // longer than the MMAs.)
  const uint64_t k_of = ptx::smem_desc_sw128(0u, 16u, 1024u), mn_of = ptx::smem_desc_sw128(0u, 16384u, 1024u);
  auto product = [&](auto a_is_mn, auto b_is_mn, uint32_t d, uint32_t n, int k16, uint32_t x, uint32_t y, uint32_t more) {
    constexpr bool a_mn = decltype(a_is_mn)::value, b_mn = decltype(b_is_mn)::value;
    constexpr uint64_t a_k = a_mn ? 128u : 2u, b_k = b_mn ? 128u : 2u, a_block = a_mn ? 512u : 1024u, b_block = b_mn ? 512u : 1024u;
    const uint32_t idesc = ptx::idesc_f16(128, (int)n, a_mn, b_mn);
    // (a shared address carries the CTA's rank above its 18 bits)
    uint64_t da = (a_mn ? mn_of : k_of) + ((x & 0x3FFFFu) >> 4), db = (b_mn ? mn_of : k_of) + ((y & 0x3FFFFu) >> 4);
    int k = k16;
#pragma unroll 1
    for (; k >= 4; k -= 4, da += a_block, db += b_block) {
      if (issuer) {
        ptx::mma_bf16(d, da, db, idesc, more);
        ptx::mma_bf16(d, da + a_k, db + b_k, idesc, 1u);
        ptx::mma_bf16(d, da + 2u * a_k, db + 2u * b_k, idesc, 1u);
        ptx::mma_bf16(d, da + 3u * a_k, db + 3u * b_k, idesc, 1u);
      }
      more = 1u;
    }
#pragma unroll 1
    for (; k > 0; --k, da += a_k, db += b_k) {
      if (issuer) ptx::mma_bf16(d, da, db, idesc, more);
      more = 1u;
    }
  };
  // Those that `issue` makes, of what has been written to shared memory before.
  auto products = [&](auto issue) {
    ptx::fence_proxy_async();
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == 0) {
      issue();
      if (issuer) ptx::mma_commit(bar);
      __syncwarp();
    }
    (void)ptx::mbar_wait(bar, parity, &abort_flag, a.status, NS_ERR_SMALL);
    parity ^= 1u;
    ptx::tc_fence_after();
  };
  const std::false_type along_k;
  const std::true_type along_mn;
  const int chunks = a.sp / 4, all = a.sp * chunks;        // 16-byte chunks of fp32 values of a row of A, of A
  const int senders = a.ctas * (a.sp == 16 ? 1 : 2);       // (a short side up to 16: hi and lo rows are added in the warp that has both)
  auto sent_at = [&](int buf, int from, int idx) { return (uint32_t)((buf * senders + from) * all + (idx ^ ((idx >> 3) & 7))) * 16u; };
  auto own_at = [&](int row, int q) { return shares + (uint32_t)(row * chunks + (q ^ (row & 3))) * 16u; };
  const int mine0 = all * rank / a.ctas, mine1 = all * (rank + 1) / a.ctas;            // the part of A that this CTA sums
  const uint32_t gram = s_hi + 8192u;                      // if everyone sums: A in fp32, [sp][sp], below the rows of P

#pragma unroll 1
  for (int step = 0; step < a.steps; ++step) {
    const bool last = step + 1 == a.steps;
    // ---- A = X X^T: this CTA's share, then the sum of all
    products([&] {
      if (everyone) {
        product(along_k, along_k, d_s, 2u * a.sp, a.w / 16, x_hi, x_hi, 0u);           // [hi; lo] [hi; lo]^T
      } else if (stacked) {
        product(along_k, along_k, d_s, 2u * a.sp, a.w / 16, x_hi, x_hi, 0u);           // hi [hi; lo]^T, and lo hi^T added to the right half
        product(along_k, along_k, d_s + a.sp, a.sp, a.w / 16, x_lo, x_hi, 1u);
      } else {
        product(along_k, along_k, d_s, a.sp, a.w / 16, x_lo, x_hi, 0u);
        product(along_k, along_k, d_s, a.sp, a.w / 16, x_hi, x_lo, 1u);
        product(along_k, along_k, d_s, a.sp, a.w / 16, x_hi, x_hi, 1u);
      }
    });
    // (what is sent alternates between two places: a sender may be a step ahead of a receiver)
    const uint32_t got = bar_share + (uint32_t)(step & 1) * 8u;
    if (everyone && threadIdx.x == 0) ptx::mbar_expect_tx(got, (uint32_t)(senders * all) * 16u);
    const int rows = everyone ? 2 * a.sp : a.sp;
    if (quarter * 32 < rows) {
      const int lo = i >= a.sp ? 1 : 0, row = i - lo * a.sp;
#pragma unroll 1
      for (int c = everyone ? 0 : half * 16; c < a.sp; c += everyone ? 16 : 32) {
        uint32_t r[16];
        float y[16];
        ptx::tmem_ld16(d_s + lanes + (uint32_t)c, r);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = __uint_as_float(r[e]);
        if (stacked) {                                     // the small products (lo rows of [hi; lo]: lo hi only)
          ptx::tmem_ld16(d_s + lanes + (uint32_t)(a.sp + c), r);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) y[e] += lo ? 0.f : __uint_as_float(r[e]);
        }
        if (everyone) {                                    // (the two warps of a quarter send to half of the CTAs each)
          if (a.sp == 16) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] += __shfl_down_sync(0xffffffffu, y[e], 16);
          }
          if (i < (a.sp == 16 ? 16 : rows)) {
            const int from = a.sp == 16 ? rank : 2 * rank + lo, idx = row * chunks + c / 4;
#pragma unroll
            for (int r2 = half; r2 < kNsSmallCtas; r2 += 2) {
              if (r2 >= a.ctas) break;
              const uint32_t there = ptx::cluster_map(got, (uint32_t)r2), to = ptx::cluster_map(shares, (uint32_t)r2);
#pragma unroll
              for (int q = 0; q < 4; ++q) ptx::send_data_v4(to + sent_at(step & 1, from, idx + q), there, y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
            }
          }
        } else if (i < rows) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            st_shared_v4(own_at(row, c / 4 + q), __float_as_uint(y[4 * q]), __float_as_uint(y[4 * q + 1]), __float_as_uint(y[4 * q + 2]), __float_as_uint(y[4 * q + 3]));
        }
      }
    }
    if (everyone) {
      (void)ptx::mbar_wait_sent(got, (uint32_t)(step >> 1) & 1u, &abort_flag, a.status, NS_ERR_SMALL);
      if ((int)threadIdx.x < all) {
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int r = 0; r < senders; ++r) {
          const uint4 u = ld_shared_v4(shares + sent_at(step & 1, r, (int)threadIdx.x));
          f.x += __uint_as_float(u.x); f.y += __uint_as_float(u.y); f.z += __uint_as_float(u.z); f.w += __uint_as_float(u.w);
        }
        st_shared_v4(gram + threadIdx.x * 16u, __float_as_uint(f.x * kNsUnscale), __float_as_uint(f.y * kNsUnscale), __float_as_uint(f.z * kNsUnscale),
                     __float_as_uint(f.w * kNsUnscale));
      }
      __syncthreads();
      // ---- P = a I + b A + c A^2 in fp32: a lane to a column (or two warp halves to 16 of them), four rows a warp at most
      const int col = a.sp == 16 ? lane & 15 : lane, row0 = a.sp == 16 ? warp * 2 + (lane >> 4) : warp;
      const uint32_t pitch = (uint32_t)a.sp * 4u;
      float sq[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int k = 0; k < a.sp; k += 4) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ld_shared_f32(gram + (uint32_t)(k + e) * pitch + (uint32_t)col * 4u);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          if (n > 0 && a.sp == 16) break;
          const uint4 u = ld_shared_v4(gram + (uint32_t)(row0 + 8 * n) * pitch + (uint32_t)k * 4u);
          sq[n] = fmaf(__uint_as_float(u.x), x[0], sq[n]); sq[n] = fmaf(__uint_as_float(u.y), x[1], sq[n]);
          sq[n] = fmaf(__uint_as_float(u.z), x[2], sq[n]); sq[n] = fmaf(__uint_as_float(u.w), x[3], sq[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if (n > 0 && a.sp == 16) break;
        const int row = row0 + 8 * n;
        float y = fmaf(kNsUnscale * a.c, sq[n], a.b * ld_shared_f32(gram + (uint32_t)row * pitch + (uint32_t)col * 4u));
        if (row == col && row < a.s) y += a.a * kNsScale;
        const __half h = __float2half_rn(y), l = __float2half_rn(y - __half2float(h));
        asm volatile("st.shared.b16 [%0], %1;" ::"r"(s_hi + at(row, col)), "h"(__half_as_ushort(h)) : "memory");
        asm volatile("st.shared.b16 [%0], %1;" ::"r"(s_lo + at(row, col)), "h"(__half_as_ushort(l)) : "memory");
      }
      // ---- X <- P X as X^T P, whose rows, columns of X, keep all warps busy
      products([&] {
        const uint32_t idesc = ptx::idesc_f16(128, a.sp, 1, 0);
        const uint64_t xh = mn_of + ((x_hi & 0x3FFFFu) >> 4), xl = mn_of + ((x_lo & 0x3FFFFu) >> 4), ph = k_of + ((s_hi & 0x3FFFFu) >> 4), pl = k_of + ((s_lo & 0x3FFFFu) >> 4);
#pragma unroll 1
        for (uint32_t k = 0; k < (uint32_t)a.sp / 16u; ++k) {
          if (issuer) {
#pragma unroll
            for (uint32_t g = 0; g < 2; ++g) {             // 128 columns of X each (of the second, whatever lies behind w <= 128: not read)
              const uint64_t x_at = g * 2048u + k * 128u;
              ptx::mma_bf16(d_x + g * a.sp, xl + x_at, ph + 2u * k, idesc, k != 0u ? 1u : 0u);
              ptx::mma_bf16(d_x + g * a.sp, xh + x_at, pl + 2u * k, idesc, 1u);
              ptx::mma_bf16(d_x + g * a.sp, xh + x_at, ph + 2u * k, idesc, 1u);
            }
          }
        }
      });
      const bool keep = last && !a.own_status && a.status->error != 0u;    // (a context whose device error stands keeps its parameters)
      const int j = warp * 32 + lane;
      if (warp * 32 < a.w) {
        const uint32_t from = d_x + lanes + (uint32_t)(half * a.sp);
        if (!last) {
#pragma unroll 1
          for (int c = 0; c < a.sp; c += 16) {
            uint32_t r[16];
            ptx::tmem_ld16(from + (uint32_t)c, r);
            ptx::tmem_ld_wait();
            const uint32_t o = (uint32_t)(j >> 6) * 16384u + (uint32_t)c * 128u + (uint32_t)(j & 7) * 2u, chunk = (uint32_t)(j & 63) >> 3;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float y = __uint_as_float(r[e]) * kNsUnscale;
              const __half h = __float2half_rn(y), l = __float2half_rn(y - __half2float(h));
              const uint32_t to = x_hi + o + (uint32_t)e * 128u + ((chunk ^ (uint32_t)(e & 7)) * 16u);
              asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(__half_as_ushort(h)) : "memory");
              asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + (x_lo - x_hi)), "h"(__half_as_ushort(l)) : "memory");
            }
          }
        } else if (!keep) {                                // (rolled: what runs once is fetched anew, at about 20 cycles an instruction)
#pragma unroll 1
          for (int c = 0; c < a.s; ++c) {
            const float y = __uint_as_float(ptx::tmem_ld1(from + (uint32_t)c)) * (kNsUnscale * kNsUnscale);
            if (j < nj) ns_store_final(a.dst, m, a.tall ? j0 + j : c, a.tall ? c : j0 + j, y);
          }
        }
      }
      continue;
    }
    ptx::cluster_arrive_release();
    ptx::cluster_wait_acquire();
#pragma unroll 2
    for (int idx = mine0 + (int)threadIdx.x; idx < mine1; idx += kNsSmallThreads) {
      const int row = idx / chunks, q = idx - row * chunks;
      const uint32_t from = own_at(row, q);
      float4 part[kNsSmallCtas], f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < kNsSmallCtas; ++r)
        if (r < a.ctas) part[r] = ptx::ld_cluster_v4(ptx::cluster_map(from, (uint32_t)r));
#pragma unroll
      for (int r = 0; r < kNsSmallCtas; ++r)
        if (r < a.ctas) { f.x += part[r].x; f.y += part[r].y; f.z += part[r].z; f.w += part[r].w; }
      f.x *= kNsUnscale; f.y *= kNsUnscale; f.z *= kNsUnscale; f.w *= kNsUnscale;
      const uint32_t h0 = pack_half2(f.x, f.y), h1 = pack_half2(f.z, f.w);
      const float2 b0 = unpack_half2(h0), b1 = unpack_half2(h1);
      const uint32_t l0 = pack_half2(f.x - b0.x, f.y - b0.y), l1 = pack_half2(f.z - b1.x, f.w - b1.y), o = at(row, q * 4);
#pragma unroll 1
      for (int r = 0; r < a.ctas; ++r) {
        ptx::st_cluster_v2(ptx::cluster_map(s_hi + o, (uint32_t)r), h0, h1);
        ptx::st_cluster_v2(ptx::cluster_map(s_lo + o, (uint32_t)r), l0, l1);
      }
    }
    ptx::cluster_arrive_release();                         // A is whole, and its shares have been read
    ptx::cluster_wait_acquire();
    // ---- P = a I + b A + c A^2, in the place of A
    products([&] {
      product(along_k, along_k, d_s, a.sp, a.sp / 16, s_lo, s_hi, 0u);
      product(along_k, along_k, d_s, a.sp, a.sp / 16, s_hi, s_lo, 1u);
      product(along_k, along_k, d_s, a.sp, a.sp / 16, s_hi, s_hi, 1u);
    });
    if (quarter * 32 < a.sp) {
#pragma unroll 1
      for (int c = half * 16; c < a.sp; c += 32) {
        uint32_t r[16];
        ptx::tmem_ld16(d_s + lanes + (uint32_t)c, r);
        ptx::tmem_ld_wait();
        if (i < a.sp) {
#pragma unroll
          for (int q = 0; q < 2; ++q) {                    // chunks of 8
            const uint32_t o = at(i, c + 8 * q);
            const uint4 h = ld_shared_v4(s_hi + o), l = ld_shared_v4(s_lo + o);
            const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
            uint32_t ho[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 ah = unpack_half2(hw[e]), al = unpack_half2(lw[e]);
              const int col = c + 8 * q + 2 * e;
              float y0 = fmaf(kNsUnscale * a.c, __uint_as_float(r[8 * q + 2 * e]), a.b * ah.x) + a.b * al.x;
              float y1 = fmaf(kNsUnscale * a.c, __uint_as_float(r[8 * q + 2 * e + 1]), a.b * ah.y) + a.b * al.y;
              if (i < a.s) { y0 += col == i ? a.a * kNsScale : 0.f; y1 += col + 1 == i ? a.a * kNsScale : 0.f; }
              ho[e] = pack_half2(y0, y1);
              const float2 b = unpack_half2(ho[e]);
              lo[e] = pack_half2(y0 - b.x, y1 - b.y);
            }
            st_shared_v4(s_hi + o, ho[0], ho[1], ho[2], ho[3]);
            st_shared_v4(s_lo + o, lo[0], lo[1], lo[2], lo[3]);
          }
        }
      }
    }
    // ---- X <- P X, in its place
    products([&] {
      product(along_k, along_mn, d_x, a.w, a.sp / 16, s_lo, x_hi, 0u);
      product(along_k, along_mn, d_x, a.w, a.sp / 16, s_hi, x_lo, 1u);
      product(along_k, along_mn, d_x, a.w, a.sp / 16, s_hi, x_hi, 1u);
    });
    const bool keep = last && !a.own_status && a.status->error != 0u;      // (a context whose device error stands keeps its parameters)
    if (quarter * 32 < a.s) {
      const uint32_t box = s_hi + (uint32_t)(warp & 7) * 4096u;          // (P is not needed any more; 32 KB at least)
#pragma unroll 1
      for (int c = half * 32; c < a.w; c += 64) {
        uint32_t raw[32];
        ptx::tmem_ld32(d_x + lanes + (uint32_t)c, raw);
        ptx::tmem_ld_wait();
        float y[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(raw[e]) * kNsUnscale;
        if (!last) {
          if (i < a.s) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t ho[4], lo[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                ho[e] = pack_half2(y[8 * q + 2 * e], y[8 * q + 2 * e + 1]);
                const float2 b = unpack_half2(ho[e]);
                lo[e] = pack_half2(y[8 * q + 2 * e] - b.x, y[8 * q + 2 * e + 1] - b.y);
              }
              const uint32_t o = at(i, c + 8 * q);
              st_shared_v4(x_hi + o, ho[0], ho[1], ho[2], ho[3]);
              st_shared_v4(x_lo + o, lo[0], lo[1], lo[2], lo[3]);
            }
          }
        } else if (keep) {
        } else if (!a.tall) {
          if (c < nj) ns_finish(a.dst, a.vec_out, m, quarter * 32, j0 + c, a.s, min(a.l, j0 + a.w), box, lane, y);
        } else if (i < a.s) {                              // (lanes hold neighbouring columns of the result)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (c + e < nj) ns_store_final(a.dst, m, j0 + c + e, i, y[e] * kNsUnscale);
        }
      }
    }
  }
  if (abort_flag) {                                        // what others have sent may still be in flight: let it land
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) { }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_arrive_release();                           // (nobody ends while something may be sent to it)
  ptx::cluster_wait_acquire();
  if (warp == 1) { ptx::tmem_relinquish(); ptx::tmem_dealloc(tmem, 512); }
}

}  // namespace prsgd
