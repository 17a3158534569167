// The products of the Newton-Schulz chain on the tensor cores (see kernels_ortho.cuh for the mathematics).
//
// One persistent launch runs all 3 * steps products of all matrices.  A pair of CTAs (cta_group::2) forms a 256 x 256
// tile: each loads half of both operands (128 rows of A, 128 of B, 64 of K per stage) by TMA and keeps 128 rows of
// the sum in its TMEM, two sums of 256 columns so that the epilogue of one tile runs beside the products of the next.
// A and P are symmetric: only tiles on and above the diagonal are formed and stored, and where a product needs one below
// it reads the stored one MN-major.  Nothing is ever transposed in memory.
//
// Tiles are claimed in order from a device counter (matrices in groups, within a group product by product), and a
// tile starts when the panels it reads are counted as done: 256 rows (tall: columns) of X, A or P along the short side,
// one counter per panel that runs through all products.  A tile of A or P reads panels ti and tj whole and belongs to both
// (as its transpose); a tile of X reads one panel of P and adds to one of X.  Reading is always over before the next
// product writes the same place: a panel of X is done only when all tiles of P that read its panel of A are, and a
// panel of P needs every panel of A, hence every tile of X before.  A claimed tile waits only for tiles claimed
// earlier, so the CTAs that run always make progress, whatever share of the grid is resident; and while one matrix's
// last tiles drain, the pairs that are free work on the next matrix instead of waiting for a grid.
#pragma once
#include "kernels_ortho.cuh"
#include "tc_ptx.cuh"

namespace prsgd {

constexpr int kNsStages = 5, kNsRing = 4, kNsEpiWarps = 8, kNsThreads = 32 * (4 + kNsEpiWarps);
constexpr int kNsWarpCols = 1024 / kNsEpiWarps;       // an epilogue warp takes 32 rows of a CTA's 128 x 256 sums and this many columns
constexpr uint32_t kNsStageBytes = 32768, kNsWarpBytes = 8192;      // operand stage of a CTA; staging of an epilogue warp
constexpr size_t kNsSmem = 1024 + (size_t)kNsStages * kNsStageBytes + kNsEpiWarps * kNsWarpBytes;
constexpr int kNsAhead = 8;            // the next tile is claimed when this many blocks of 64 of the current one are left to load
constexpr int kNsPromote = 2;          // 32-bit precision: blocks of 64 whose products are summed in TMEM before they join the sum in registers
enum { NS_ERR_DEP = 0x701, NS_ERR_FULL, NS_ERR_EMPTY, NS_ERR_ACC, NS_ERR_ACC_FREE, NS_ERR_RING, NS_ERR_RING_FREE };

struct NsMaps {
  CUtensorMap x[2][2], A[2], P[2];           // operands read MN-major: [buffer][hi, lo], box {64, 64, 1}
  CUtensorMap xk[2][2], Ak[2], Pk[2];        // ... K-major: box {64, 128, 1}
};

struct NsChainArgs {
  NsShape sh; NsBuffers buf; NsDest dst;
  int steps, split, tall, s, l;
  float a, b, c;
  int ts, tsym, tr, tc;          // tiles along the short side; tiles of A and P on and above the diagonal; tile rows and columns of X
  int parts;                     // parts of the contraction of A's tiles, a task each
  int per_step, per_panel;       // tasks of a matrix and step; tiles of one panel
  int group, total;              // matrices of a group; tasks of the launch
  int vec_out;                   // result rows can be written 16 bytes at a time
};

struct NsTask { int m, step, kind, part, ti, tj; int pi, pj, need; };      // pi, pj: the panels (256 rows or columns along the short side) it takes from and adds to

__device__ __forceinline__ NsTask ns_decode(const NsChainArgs& a, int t) {
  const int per_group = a.group * a.steps * a.per_step;
  const int g = t / per_group;
  int rem = t - g * per_group;
  const int gs = min(a.group, a.sh.batch - g * a.group);
  NsTask k;
  k.step = rem / (gs * a.per_step);
  rem -= k.step * gs * a.per_step;
  k.need = k.step * a.per_panel;
  k.kind = 0;
  if (rem >= gs * a.tsym * a.parts) { rem -= gs * a.tsym * a.parts; k.kind = 1; k.need += a.ts; }
  if (k.kind == 1 && rem >= gs * a.tsym) { rem -= gs * a.tsym; k.kind = 2; k.need += a.ts; }
  const int tiles = k.kind == 2 ? a.tr * a.tc : k.kind == 1 ? a.tsym : a.tsym * a.parts;
  k.m = rem / tiles;
  int q = rem - k.m * tiles;
  k.m += g * a.group;
  k.part = 0;
  if (k.kind == 0) { k.part = q % a.parts; q /= a.parts; }
  if (k.kind == 2) {                                    // panel by panel
    if (a.tall) { k.tj = q / a.tr; k.ti = q - k.tj * a.tr; k.pi = k.pj = k.tj; }
    else        { k.ti = q / a.tc; k.tj = q - k.ti * a.tc; k.pi = k.pj = k.ti; }
  } else {                                              // q = tj (tj + 1) / 2 + ti, ti <= tj
    int j = (int)((sqrtf(8.f * (float)q + 1.f) - 1.f) * 0.5f);
    while (j * (j + 1) / 2 > q) --j;
    while ((j + 1) * (j + 2) / 2 <= q) ++j;
    k.tj = k.pj = j; k.ti = k.pi = q - j * (j + 1) / 2;
  }
  k.need *= 2 * kNsEpiWarps;                            // every epilogue warp of the pair counts a tile
  k.pi += k.m * a.ts; k.pj += k.m * a.ts;
  return k;
}

// The blocks of 64 of a task's contraction: first and number.
__device__ __forceinline__ int ns_blocks(const NsChainArgs& a, const NsTask& k, int& n) {
  const int kb = ((k.kind == 0 ? a.l : a.s) + 63) / 64;
  if (k.kind != 0 || a.parts == 1) { n = kb; return 0; }
  const int first = kb * k.part / a.parts;
  n = kb * (k.part + 1) / a.parts - first;
  return first;
}

namespace ptx {
// loads into this CTA's shared memory, counted on a barrier that may be the pair's other CTA's
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"((uint64_t)map), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_dst, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void mma_f16_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// arrives on the barrier at this offset in both CTAs of the pair once the MMAs issued so far have completed
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Arrives on a barrier of either CTA of the pair.  Relaxed: what is handed on is TMEM (ordered by tcgen05.fence) or a ring
// entry that has been read; a release would wait for all of the thread's stores, microseconds after an epilogue.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory");
}
__device__ __forceinline__ void red_add(unsigned int* p, unsigned int v) {       // (relaxed: after a fence)
  asm volatile("red.relaxed.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// Hands 16 bytes to a CTA of the cluster and counts them on its barrier (which expects 16 bytes and one arrival).
__device__ __forceinline__ void send_v4(uint32_t to_cluster, uint32_t bar_cluster, uint4 v) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], 16;" ::"r"(bar_cluster) : "memory");
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(to_cluster), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "r"(bar_cluster) : "memory");
}
// mbar_wait by all 32 lanes of a warp, which leave it together
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, DeviceStatus* status, unsigned what) {
  long long t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((it & 63u) == 0u) {
      bool stop = *abort_flag != 0;
      const long long now = clock64();
      if (t0 == 0) t0 = now;
      if (!stop && now - t0 > kWaitLimitCycles) {
        stop = true;
        *abort_flag = 1;
        if (atomicCAS(&status->error, 0u, what) == 0u) status->where = blockIdx.x;
      }
      if (__any_sync(0xffffffffu, stop)) return false;
    }
  }
}
// 32 lanes x 32 consecutive fp32 columns, back into TMEM
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
        "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
        "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]),
        "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(p));
  return p != 0;
}
// fp16 operands, fp32 sum
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int a_mn_major, int b_mn_major) {
  return (1u << 4) | ((uint32_t)a_mn_major << 15) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
}  // namespace ptx

__device__ __forceinline__ uint32_t pack_half2(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// fp16 pairs of 32 values
__device__ __forceinline__ void ns_pack(const float (&v)[32], uint32_t (&h)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) h[i] = pack_half2(v[2 * i], v[2 * i + 1]);
}
// ... and, in their place, of what that rounding left
__device__ __forceinline__ void ns_pack_rest(const float (&v)[32], uint32_t (&h)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float2 f = unpack_half2(h[i]);
    h[i] = pack_half2(v[2 * i] - f.x, v[2 * i + 1] - f.y);
  }
}
__device__ __forceinline__ void ns_add(float (&v)[32], const uint32_t (&h)[16], float f) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float2 x = unpack_half2(h[i]);
    v[2 * i] = fmaf(f, x.x, v[2 * i]);
    v[2 * i + 1] = fmaf(f, x.y, v[2 * i + 1]);
  }
}
__device__ __forceinline__ void st_shared_v4(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// A warp's box of 32 rows x 64 halves in shared memory, where values change between one row per lane (as they come from
// TMEM, `half` of its columns at a time) and one 16-byte chunk per lane, eight lanes to a row: a store then touches four
// lines of 128 bytes (with rows of 64 bytes the stores of a tile took twice as long, with a row per lane eight times).
// Chunk c of row r sits at chunk c ^ (r % 8): free of bank conflicts both ways.
__device__ __forceinline__ uint32_t ns_chunk(uint32_t box, int row, int q) { return box + (uint32_t)row * 128u + (uint32_t)((q ^ (row & 7)) * 16); }
__device__ __forceinline__ void ns_put(uint32_t box, int lane, int half, const uint32_t (&h)[16]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) st_shared_v4(ns_chunk(box, lane, half * 4 + q), h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
}
__device__ __forceinline__ void ns_get(uint32_t box, int lane, int half, uint32_t (&h)[16]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint4 u = ld_shared_v4(ns_chunk(box, lane, half * 4 + q));
    h[4 * q] = u.x; h[4 * q + 1] = u.y; h[4 * q + 2] = u.z; h[4 * q + 3] = u.w;
  }
}
// The 32 x 64 block at p (rows `pitch` apart, a multiple of 8), of which `rows` and `cols` exist: chunk lane % 8 of row
// 4 i + lane / 8.  Read past L1, which does not see what other SMs wrote meanwhile.
__device__ __forceinline__ void ns_fetch(const __half* p, int64_t pitch, int rows, int cols, int lane, uint4 (&u)[8]) {
  const int row0 = lane >> 3, c = (lane & 7) * 8;
  const __half* q = p + (int64_t)row0 * pitch + c;
#pragma unroll
  for (int i = 0; i < 8; ++i, q += 4 * pitch) u[i] = row0 + 4 * i < rows && c < cols ? __ldcg(reinterpret_cast<const uint4*>(q)) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void ns_put_fetched(uint32_t box, int lane, const uint4 (&u)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) st_shared_v4(ns_chunk(box, 4 * i + (lane >> 3), lane & 7), u[i].x, u[i].y, u[i].z, u[i].w);
}
__device__ __forceinline__ void ns_store_box(uint32_t box, __half* p, int64_t pitch, int rows, int cols, int lane) {
  const int row0 = lane >> 3, c = (lane & 7) * 8;
  __half* q = p + (int64_t)row0 * pitch + c;
#pragma unroll
  for (int i = 0; i < 8; ++i, q += 4 * pitch) {
    const uint4 u = ld_shared_v4(ns_chunk(box, row0 + 4 * i, lane & 7));
    if (row0 + 4 * i < rows && c < cols) *reinterpret_cast<uint4*>(q) = u;
  }
}

// Columns c .. c + 3 of row r of what is there, where the result is added to it and the whole four can be read together.
__device__ __forceinline__ float4 ns_old4(const NsDest& d, int64_t o) {
  if (d.type == PRSGD_TYPE_FP32) return *reinterpret_cast<const float4*>(static_cast<const float*>(d.out) + o);
  uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(d.out) + o);
  const bool bf = d.type == PRSGD_TYPE_BF16;
  const float2 x = bf ? __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&u.x)) : unpack_half2(u.x);
  const float2 y = bf ? __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&u.y)) : unpack_half2(u.y);
  return make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void ns_write4(const NsDest& d, int64_t o, float4 w) {
  if (d.type == PRSGD_TYPE_FP32) {
    *reinterpret_cast<float4*>(static_cast<float*>(d.out) + o) = w;
    if (d.shadow == nullptr) return;
  }
  uint2 u;
  if (d.type == PRSGD_TYPE_FP16) {
    u = make_uint2(pack_half2(w.x, w.y), pack_half2(w.z, w.w));
  } else {
    const __nv_bfloat162 x = __floats2bfloat162_rn(w.x, w.y), y = __floats2bfloat162_rn(w.z, w.w);
    u = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  }
  *reinterpret_cast<uint2*>((d.type == PRSGD_TYPE_FP32 ? d.shadow : static_cast<uint16_t*>(d.out)) + o) = u;
}

// 32 rows x 32 columns of the result (of `rows` x `cols`), a row per lane, through shared memory so that the lanes of a warp write
// neighbouring columns (with rows per lane every store touches 32 lines).
__device__ __forceinline__ void ns_finish(const NsDest& d, bool vec, int m, int r0, int c0, int rows, int cols, uint32_t box, int lane,
                                          const float (&v)[32]) {
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 8; ++q)
    st_shared_v4(box + (uint32_t)lane * 128u + (uint32_t)((q ^ (lane & 7)) * 16), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                 __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
  __syncwarp();
  const int c = c0 + (lane & 7) * 4, row0 = r0 + (lane >> 3);
  if (vec && c + 4 <= cols) {                              // four rows together, so that what is added to is requested together
    const float al = d.alpha * kNsUnscale;
#pragma unroll 1
    for (int i = 0; i < 8; i += 4) {
      float4 w[4], old[4];
      int64_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rr = row0 + 4 * (i + j);
        o[j] = (int64_t)m * d.batch + (d.tiled ? wtile_offset(d.tile, rr, c) : (int64_t)rr * d.row + c);
        old[j] = d.beta != 0.f && rr < rows ? ns_old4(d, o[j]) : make_float4(0.f, 0.f, 0.f, 0.f);
        const int br = 4 * (i + j) + (lane >> 3);
        const uint4 u = ld_shared_v4(box + (uint32_t)br * 128u + (uint32_t)(((lane & 7) ^ (br & 7)) * 16));
        w[j] = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (row0 + 4 * (i + j) >= rows) continue;
        if (d.beta != 0.f) {
          w[j] = make_float4(fmaf(d.beta, old[j].x, al * w[j].x), fmaf(d.beta, old[j].y, al * w[j].y), fmaf(d.beta, old[j].z, al * w[j].z), fmaf(d.beta, old[j].w, al * w[j].w));
        } else {
          w[j] = make_float4(al * w[j].x, al * w[j].y, al * w[j].z, al * w[j].w);
        }
        ns_write4(d, o[j], w[j]);
      }
    }
    return;
  }
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    const int br = i * 4 + (lane >> 3);
    const uint4 u = ld_shared_v4(box + (uint32_t)br * 128u + (uint32_t)(((lane & 7) ^ (br & 7)) * 16));
    if (r0 + br >= rows) continue;
    const float w[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < cols) ns_store_final(d, m, r0 + br, c + e, w[e] * kNsUnscale);
  }
}

// SPLIT: 32-bit precision, products of fp16 pairs.
template <bool SPLIT>
__global__ void __launch_bounds__(kNsThreads, 1) ns_chain_kernel(const __grid_constant__ NsMaps maps, const __grid_constant__ NsChainArgs a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * kNsStages + 4 + 2 * kNsRing + 1];
  __shared__ __align__(16) uint4 ring[kNsRing];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  const uint32_t stage0 = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1u;                 // clusters of two along x
  DeviceStatus* status = a.buf.status;
  auto bar = [&](int i) { return ptx::smem_u32(&bars[i]); };
  auto full = [&](int s) { return bar(s); };                              // in the leader (rank 0): its stage has both CTAs' operands
  auto empty = [&](int s) { return bar(kNsStages + s); };                 // in each: the MMAs that read the stage are done
  auto tfull = [&](int i) { return bar(2 * kNsStages + i); };             // in each: sum i is complete
  auto tempty = [&](int i) { return bar(2 * kNsStages + 2 + i); };        // in the leader: all epilogue warps have read sum i
  auto sfull = [&](int i) { return bar(2 * kNsStages + 4 + i); };         // in each: ring entry i holds a task
  auto sempty = [&](int i) { return bar(2 * kNsStages + 4 + kNsRing + i); };   // in the leader: everyone has read it
  const uint32_t loaded = bar(2 * kNsStages + 4 + 2 * kNsRing);            // in the leader: all loads of a tile have been issued
  if (threadIdx.x == 0) {
    ptx::mbar_init(loaded, 1);
    for (int s = 0; s < kNsStages; ++s) { ptx::mbar_init(full(s), 1); ptx::mbar_init(empty(s), 1); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(tfull(i), 1); ptx::mbar_init(tempty(i), 2 * kNsEpiWarps); }
    for (int i = 0; i < kNsRing; ++i) { ptx::mbar_init(sfull(i), 1); ptx::mbar_init(sempty(i), 2 * kNsEpiWarps + 5); }
    abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) ptx::tmem_alloc_pair(ptx::smem_u32(&tmem_slot), 512);
  __syncthreads();
  ptx::cluster_arrive_release();
  ptx::cluster_wait_acquire();
  ptx::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  if (warp == 1) ptx::tmem_relinquish_pair();
  ptx::pdl_wait();
  ptx::pdl_trigger();
  volatile int* ab = &abort_flag;

  // The next task from the ring, for a whole warp; kind < 0 at the end or when a wait gave up.  Whoever gets it may read
  // what the task depends on: the scheduler saw it done (acquire) before it sent the task, and it is read where it was
  // made visible, in L2 (TMA behind a proxy fence, ld.cg), never through an L1 that could hold older values.
  auto next_task = [&](int n) -> NsTask {
    const int r = n % kNsRing;
    NsTask k;
    k.kind = -1; k.m = k.step = k.part = k.ti = k.tj = 0;
    if (!ptx::warp_wait(sfull(r), (uint32_t)((n / kNsRing) & 1), ab, status, NS_ERR_RING)) return k;
    const uint4 w = ld_shared_v4(ptx::smem_u32(&ring[r]));
    k.kind = __shfl_sync(0xffffffffu, (int)w.x, 0); k.m = __shfl_sync(0xffffffffu, (int)w.y, 0); 
    const uint32_t sp = __shfl_sync(0xffffffffu, w.z, 0);
    k.step = (int)(sp & 0xffffu); k.part = (int)(sp >> 16);
    const uint32_t t = __shfl_sync(0xffffffffu, w.w, 0);
    k.ti = (int)(t >> 16); k.tj = (int)(t & 0xffffu);
    return k;
  };
  auto free_task = [&](int n) { ptx::mbar_arrive_cluster(ptx::cluster_map(sempty(n % kNsRing), 0)); };

  // The load and product roles are walked by whole warps with one elected lane that issues: in a branch of a single
  // lane the compiler cannot keep descriptors and addresses in uniform registers, and the instructions between two
  // MMAs then take longer than an MMA (720 cycles instead of 512 per block of 64 measured).
  // With 32-bit precision the epilogue's sums take registers from the other warps: 128 * 64 + 256 * 216 of the launch's 384 * 168.
  if (warp < 4) {
    if constexpr (SPLIT) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 0 || warp == 3) {                          // ---- operand loads: warp 0 A, warp 3 B --------------------------
      const bool second = warp == 3, issue = ptx::elect_one();
      uint32_t s = 0, phase = 1;                           // (a fresh barrier passes a wait for the phase before its first)
      for (int n = 0;; ++n) {
        const NsTask k = next_task(n);
        if (k.kind < 0) break;
        if (issue) { free_task(n); ptx::fence_proxy_async_all(); }
        const int from = k.step & 1;
        int kb;
        const int k0 = ns_blocks(a, k, kb), blocks = kb * (SPLIT ? 3 : 1);
        const bool of_x = k.kind == 0 || (k.kind == 2 && second != (a.tall != 0));
        const bool x_mn = k.kind == 0 ? a.tall != 0 : second;                      // (of X)
        const int tile = second ? k.tj : k.ti, at0 = tile * 256 + (int)rank * 128;
        const int ask = max(0, blocks - kNsAhead);
        bool ok = true;
        for (int p = 0, b = 0; p < (SPLIT ? 3 : 1) && ok; ++p) {
          const int part = SPLIT && p == (second ? 1 : 0) ? 1 : 0;       // lo hi, hi lo, hi hi: the small ones first
          const CUtensorMap* map_mn = of_x ? &maps.x[from][part] : k.kind == 1 ? &maps.A[part] : &maps.P[part];
          const CUtensorMap* map_k = of_x ? &maps.xk[from][part] : k.kind == 1 ? &maps.Ak[part] : &maps.Pk[part];
          for (int q = k0; q < k0 + kb; ++q, ++b) {
            const bool mn = of_x ? x_mn : (q >> 2) < tile;               // (symmetric: below the diagonal the transpose is stored)
            if (!ptx::warp_wait(empty((int)s), phase, ab, status, NS_ERR_EMPTY)) { ok = false; break; }
            if (issue) {
              if (rank == 0 && !second) ptx::mbar_expect_tx(full((int)s), 2 * kNsStageBytes);
              const uint32_t fb = ptx::cluster_map(full((int)s), 0), at = stage0 + s * kNsStageBytes + (second ? 16384u : 0u);
              if (mn) {
                ptx::tma_load_3d_pair(at, map_mn, fb, at0, q * 64, k.m);
                ptx::tma_load_3d_pair(at + 8192u, map_mn, fb, at0 + 64, q * 64, k.m);
              } else {
                ptx::tma_load_3d_pair(at, map_k, fb, q * 64, at0, k.m);
              }
              if (b == ask && rank == 0 && !second) ptx::mbar_arrive(loaded);
            }
            __syncwarp();
            if (++s == kNsStages) { s = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
      }
    } else if (warp == 1 && rank == 0) {                   // ---- products (the leader issues for the pair) --------------
      const bool issue = ptx::elect_one();
      uint32_t s = 0, phase = 0, sums = 0;
      for (int n = 0;; ++n) {
        const NsTask k = next_task(n);
        if (k.kind < 0) break;
        if (issue) free_task(n);
        int kb;
        (void)ns_blocks(a, k, kb);
        const int blocks = kb * (SPLIT ? 3 : 1);
        // blocks of 64 below which the operands lie MN-major
        const int a_mn_until = k.kind == 0 ? (a.tall ? kb : 0) : (k.kind == 2 && a.tall) ? 0 : 4 * k.ti;
        const int b_mn_until = k.kind == 0 ? (a.tall ? kb : 0) : (k.kind == 2 && !a.tall) ? kb : 4 * k.tj;
        bool ok = true;
        int next = 0;                                      // block that starts a new sum
        uint32_t acc = 0;
        for (int q = 0, qk = 0; q < blocks; ++q) {
          const bool first = q == next;
          if (first) {
            next = !SPLIT ? blocks : q < 2 * kb ? 2 * kb : q + kNsPromote;
            acc = sums & 1u;
            if (sums >= 2 && !ptx::warp_wait(tempty((int)acc), ((sums >> 1) - 1) & 1, ab, status, NS_ERR_ACC_FREE)) { ok = false; break; }
            ptx::tc_fence_after();
            ++sums;
          }
          if (!ptx::warp_wait(full((int)s), phase, ab, status, NS_ERR_FULL)) { ok = false; break; }
          ptx::tc_fence_after();
          if (issue) {
            const bool a_mn = qk < a_mn_until, b_mn = qk < b_mn_until;
            const uint32_t idesc = ptx::idesc_f16(256, 256, a_mn, b_mn);
            // a step of 16 along the contraction: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major block
            const uint64_t at = s * (kNsStageBytes >> 4), da_k = a_mn ? 128u : 2u, db_k = b_mn ? 128u : 2u;
            const uint64_t da = at + (a_mn ? ptx::smem_desc_sw128(stage0, 8192u, 1024u) : ptx::smem_desc_sw128(stage0, 16u, 1024u));
            const uint64_t db = at + (b_mn ? ptx::smem_desc_sw128(stage0 + 16384u, 8192u, 1024u) : ptx::smem_desc_sw128(stage0 + 16384u, 16u, 1024u));
  #pragma unroll
            for (uint32_t h = 0; h < 4; ++h)
              ptx::mma_f16_pair(tmem + acc * 256u, da + h * da_k, db + h * db_k, idesc, !first || h != 0 ? 1u : 0u);
            ptx::mma_commit_pair(empty((int)s));
            if (q + 1 == blocks || q + 1 == next) ptx::mma_commit_pair(tfull((int)acc));
          }
          __syncwarp();
          if (++s == kNsStages) { s = 0; phase ^= 1u; }
          if (++qk == kb) qk = 0;
        }
        if (!ok) break;
      }
    } else if (warp == 2 && lane == 0 && rank == 0) {      // ---- claims tiles for the pair --------------------------------
      for (int n = 0;; ++n) {
        const int r = n % kNsRing;
        // Not before the last loads of the tile before are being issued: a tile claimed sooner would only keep those that
        // depend on it waiting.  (Claiming, handing on and the panels' counters take about 2 us.)
        if (n > 0 && !ptx::mbar_wait(loaded, (uint32_t)((n - 1) & 1), ab, status, NS_ERR_RING_FREE)) break;
        if (n >= kNsRing && !ptx::mbar_wait(sempty(r), (uint32_t)(((n / kNsRing) - 1) & 1), ab, status, NS_ERR_RING_FREE)) break;
        NsTask k;
        k.kind = -1; k.m = k.step = k.part = k.ti = k.tj = 0;
        for (;;) {
          const int t = (int)atomicAdd(a.buf.claim, 1u);
          if (t >= a.total || (n == 0 && !a.buf.own_status && status->error != 0u)) break;
          const NsTask got = ns_decode(a, t);
          if (a.dst.active != nullptr && a.dst.active[got.m] == 0) continue;
          k = got;
          break;
        }
        if (k.kind >= 0 && k.need > 0 &&
            !(ptx::flag_wait(a.buf.done + k.pi, (unsigned)k.need, ab, status, NS_ERR_DEP) &&
              (k.pj == k.pi || ptx::flag_wait(a.buf.done + k.pj, (unsigned)k.need, ab, status, NS_ERR_DEP))))
          break;
  #pragma unroll
        for (uint32_t c = 0; c < 2; ++c) {
          ptx::send_v4(ptx::cluster_map(ptx::smem_u32(&ring[r]), c), ptx::cluster_map(sfull(r), c),
                       make_uint4((uint32_t)k.kind, (uint32_t)k.m, ((uint32_t)k.part << 16) | (uint32_t)k.step, ((uint32_t)k.ti << 16) | (uint32_t)k.tj));
        }
        if (k.kind < 0) break;
      }
    }
  } else {                                               // ---- epilogue ---------------------------------------------
    if constexpr (SPLIT) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int quarter = warp & 3, share = (warp - 4) >> 2;
    const uint32_t box_hi = stage0 + kNsStages * kNsStageBytes + (uint32_t)(warp - 4) * kNsWarpBytes, box_lo = box_hi + 4096u;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(share * kNsWarpCols);
    uint32_t sums = 0;
    for (int n = 0;; ++n) {
      const NsTask k = next_task(n);
      if (k.kind < 0) break;
      if (lane == 0) free_task(n);
      const int from = k.step & 1;
      const bool last = k.kind == 2 && k.step + 1 == a.steps;
      const int R = k.kind == 2 ? a.sh.rows : a.s, C = k.kind == 2 ? a.sh.cols : a.s;
      const int64_t pitch = k.kind == 2 ? a.buf.xp : a.buf.sp;
      const int r0 = k.ti * 256 + (int)rank * 128 + quarter * 32, c_warp = k.tj * 256 + share * kNsWarpCols;
      const int rows = min(32, R - r0), units = rows > 0 ? min(kNsWarpCols / 64, max(0, (C - c_warp + 63) / 64)) : 0;       // of 64 columns
      const int64_t at = (int64_t)k.m * R * pitch + (int64_t)r0 * pitch + c_warp;
      // 16-bit precision: b A is added to c A^2, a X_lo to P X_hi; requested a unit ahead.  (32-bit: b A_hi and b A_lo.)
      const bool fetch = k.kind == 1 || (!SPLIT && k.kind == 2 && !last);
      const __half* const add_hi = (k.kind == 1 ? a.buf.A[0] : a.buf.x[from][1]) + at;
      const __half* const add_lo = SPLIT ? a.buf.A[1] + at : nullptr;
      uint4 ahead[8];
      if (!SPLIT && fetch) ns_fetch(add_hi, pitch, rows, C - c_warp, lane, ahead);
      uint32_t acc = sums & 1u;
      bool ok = true;
      if constexpr (SPLIT) {
        // The partial sums of the tile are added in registers, where they are rounded, not cut off; the total goes back
        // to TMEM, over the last of them, so that what follows is a loop of few instructions.
        int kb;
        (void)ns_blocks(a, k, kb);
        const int parts = 1 + (kb + kNsPromote - 1) / kNsPromote;
        float total[kNsWarpCols / 32][32];
#pragma unroll
        for (int i = 0; i < kNsWarpCols; ++i) total[i >> 5][i & 31] = 0.f;
        for (int p = 0; p < parts; ++p, ++sums) {
          acc = sums & 1u;
          ok = ptx::warp_wait(tfull((int)acc), (sums >> 1) & 1u, ab, status, NS_ERR_ACC);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int ch = 0; ch < kNsWarpCols / 32; ++ch) {
            uint32_t raw[32];
            ptx::tmem_ld32(lanes + acc * 256u + (uint32_t)(ch * 32), raw);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) total[ch][i] += __uint_as_float(raw[i]);
          }
          if (p + 1 < parts) {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster(ptx::cluster_map(tempty((int)acc), 0));
          }
        }
        if (!ok) break;
#pragma unroll
        for (int ch = 0; ch < kNsWarpCols / 32; ++ch) ptx::tmem_st32(lanes + acc * 256u + (uint32_t)(ch * 32), total[ch]);
        ptx::tmem_st_wait();
      } else {
        ok = ptx::warp_wait(tfull((int)acc), (sums >> 1) & 1u, ab, status, NS_ERR_ACC);
        ++sums;
        if (!ok) break;
        ptx::tc_fence_after();
      }
      // A tile of A in parts: leave this part's sum; whichever warp leaves the last one of its 32 x 128 values adds them up, in
      // the parts' order, and goes on with the total in TMEM.  Nobody waits.
      if (k.kind == 0 && a.parts > 1) {
        const int64_t tile = (int64_t)k.m * a.tsym + k.tj * (k.tj + 1) / 2 + k.ti;
        const int slot = (int)rank * kNsEpiWarps + warp - 4;
        float4* const sums_of = reinterpret_cast<float4*>(a.buf.part_sums) + (tile * a.parts * 16 + slot) * 1024 + lane;
        if (units > 0) {
#pragma unroll 1
          for (int ch = 0; ch < 4; ++ch) {
            uint32_t raw[32];
            ptx::tmem_ld32(lanes + acc * 256u + (uint32_t)(ch * 32), raw);
            ptx::tmem_ld_wait();
            float4* const to = sums_of + (int64_t)k.part * 16384 + ch * 256;
#pragma unroll
            for (int q = 0; q < 8; ++q)
              __stcg(to + q * 32, make_float4(__uint_as_float(raw[4 * q]), __uint_as_float(raw[4 * q + 1]), __uint_as_float(raw[4 * q + 2]), __uint_as_float(raw[4 * q + 3])));
          }
        }
        __syncwarp();
        unsigned int left = 0;
        if (lane == 0) {
          asm volatile("fence.acq_rel.gpu;" ::: "memory");
          left = atomicAdd(a.buf.part_count + tile * 16 + slot, 1u);
          asm volatile("fence.acq_rel.gpu;" ::: "memory");
        }
        left = __shfl_sync(0xffffffffu, left, 0);
        if (left + 1u != (unsigned)a.parts) {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive_cluster(ptx::cluster_map(tempty((int)acc), 0));
          continue;
        }
        if (lane == 0) a.buf.part_count[tile * 16 + slot] = 0u;      // (for the next step, whose tiles wait for this one)
        if (units > 0) {
#pragma unroll 1
          for (int ch = 0; ch < 4; ++ch) {
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
#pragma unroll 1
            for (int p = 0; p < a.parts; ++p) {
              const float4* const from_part = sums_of + (int64_t)p * 16384 + ch * 256;
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                const float4 x = __ldcg(from_part + q * 32);
                v[4 * q] += x.x; v[4 * q + 1] += x.y; v[4 * q + 2] += x.z; v[4 * q + 3] += x.w;
              }
            }
            ptx::tmem_st32(lanes + acc * 256u + (uint32_t)(ch * 32), v);
          }
          ptx::tmem_st_wait();
        }
      }
      // A rolled loop, and short: code that a tile runs through once is fetched anew every time, at about 20 cycles an
      // instruction (unrolled, this took 8 to 10 thousand cycles a tile, longer than the products of K = 1024).
#pragma unroll 1
      for (int u = 0; u < units; ++u) {
        const int cu = c_warp + u * 64;
        const int64_t o = at + u * 64;
        __syncwarp();                                    // (all lanes are done with the boxes)
        if (fetch) {
          if constexpr (SPLIT) {
            ns_fetch(add_lo + u * 64, pitch, rows, C - cu, lane, ahead);
            ns_put_fetched(box_lo, lane, ahead);
            ns_fetch(add_hi + u * 64, pitch, rows, C - cu, lane, ahead);
            ns_put_fetched(box_hi, lane, ahead);
          } else {
            ns_put_fetched(box_hi, lane, ahead);
            if (u + 1 < units) ns_fetch(add_hi + (u + 1) * 64, pitch, rows, C - cu - 64, lane, ahead);
          }
          __syncwarp();
        }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const int c0 = cu + h * 32;
          float v[32];
          {
            uint32_t raw[32];
            ptx::tmem_ld32(lanes + acc * 256u + (uint32_t)(u * 64 + h * 32), raw);
            ptx::tmem_ld_wait();
            const float f = k.kind == 1 ? kNsUnscale * a.c : kNsUnscale;
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(raw[i]) * f;
          }
          if (last) {
            ns_finish(a.dst, a.vec_out != 0, k.m, r0, c0, a.sh.rows, a.sh.cols, h == 0 ? box_hi : box_lo, lane, v);
            continue;
          }
          uint32_t w[16];                                // (a lane reads and writes its own row of the boxes)
          if (fetch) {
#pragma unroll 1
            for (int j = 0; j < (SPLIT ? 2 : 1); ++j) {
              ns_get(j == 0 ? box_hi : box_lo, lane, h, w);
              ns_add(v, w, k.kind == 1 ? a.b : a.a);
            }
          }
          if (k.kind == 1 && c0 == r0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += i == lane ? a.a * kNsScale : 0.f;
          }
          ns_pack(v, w);
          ns_put(box_hi, lane, h, w);
          if (SPLIT || k.kind == 2) {
            ns_pack_rest(v, w);
            ns_put(box_lo, lane, h, w);
          }
        }
        if (last) continue;
        __syncwarp();
        ns_store_box(box_hi, (k.kind == 0 ? a.buf.A[0] : k.kind == 1 ? a.buf.P[0] : a.buf.x[1 - from][0]) + o, pitch, rows, C - cu, lane);
        if (SPLIT || k.kind == 2)
          ns_store_box(box_lo, (k.kind == 0 ? a.buf.A[1] : k.kind == 1 ? a.buf.P[1] : a.buf.x[1 - from][1]) + o, pitch, rows, C - cu, lane);
      }
      ptx::tc_fence_before();                            // the sum has been read: the next product may overwrite it
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::cluster_map(tempty((int)acc), 0));
      if (!last && lane == 0) {                          // count the tile, everything the warp wrote before it
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
        const int pi = k.m * a.ts + (k.kind == 2 && a.tall ? k.tj : k.ti), pj = k.m * a.ts + (k.kind == 2 && !a.tall ? k.ti : k.tj);
        ptx::red_add(a.buf.done + pi, 1u);
        if (pj != pi) ptx::red_add(a.buf.done + pj, 1u);
      }
    }
  }
  __syncwarp();
  __syncthreads();
  if (abort_flag) {                                      // copies and products may still be in flight: let them land
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) { }
  }
  ptx::tc_fence_before();
  ptx::cluster_arrive_release();
  ptx::cluster_wait_acquire();
  if (warp == 1) ptx::tmem_dealloc_pair(tmem, 512);
}

}  // namespace prsgd
