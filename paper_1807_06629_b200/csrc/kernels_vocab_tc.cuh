// The products of the vocabulary loss and of its gradient on the tensor cores, one persistent launch each.
//
// A pair of CTAs (cta_group::2) forms a 256 x 256 tile: each loads half of both operands (128 rows of A, 128 of B, 64 of the
// contraction per stage) by TMA and keeps 128 rows of the sum in its TMEM, two sums of 256 columns so that the epilogue of one
// tile runs beside the products of the next.  Tokens are the rows of a tile of logits, so a thread of the epilogue owns a
// token: maxima and sums of exponentials need no exchange between threads.
//  * Loss: a task is a run of tiles along the vocabulary for one block of 256 tokens; its epilogue keeps each token's running (max, sum of
//    e^(z - max)) in registers and leaves them once per run.  Runs are ordered so that the pairs which work at a time share them: W comes
//    from HBM once, H' stays in L2.
//  * Gradient: the vocabulary is taken in pieces.  Tiles of G of a piece (logits again, then the softmax's gradient in the epilogue, held in
//    16 bits) and tiles of dW = G^T H' and dH += G W that use it are tasks of one list: G of piece k, then the uses of piece k - lag, so
//    that what a task waits for was claimed a phase earlier.  A piece of G takes about 64 MB, the fastest between pieces that stay in L2
//    (126 MB) and few additions to dH (vocab_plan.h).  G^T, W^T and H'^T are read MN-major: nothing is transposed in memory.  dH of several
//    pieces adds up in fp32 in the workspace, each tile in the order of the pieces; a long contraction is cut into parts with sums of their
//    own, added up by a last launch.
// Tasks are claimed in order from a device counter, and a claimed task waits only for tasks claimed earlier, so the CTAs that run
// always make progress, whatever share of the grid is resident.
#pragma once
#include "kernels_vocab.cuh"
#include "tc_pair.cuh"
#include "vocab_plan.h"

namespace prsgd {

constexpr int kVtEpiWarps = 16, kVtThreads = 32 * (4 + kVtEpiWarps), kVtRing = 4;
// Epilogue warps take 32 rows of a CTA's 128 x 256 sums each.  Where sums are added in registers (PROMOTE) all sixteen share a tile, 64 columns each; else
// eight take the tiles of one TMEM sum and eight those of the other, 128 columns each, so that one tile's stores run beside the next one's
// exponentials (gradient, 256 x 256 tiles of G with D = 1024: 10.9 thousand cycles a tile, products 8.2).
constexpr int kVtShares = kVtEpiWarps / 4;
constexpr uint32_t kVtStageBytes = 32768, kVtWarpBytes = 4096;
__host__ __device__ constexpr int vt_stages(bool grad) { return grad ? 5 : 6; }            // (the gradient's epilogue needs shared memory too)
constexpr size_t vt_smem(bool grad) { return 1024 + (size_t)vt_stages(grad) * kVtStageBytes + (grad ? kVtEpiWarps * kVtWarpBytes : 0); }
// A tensor core cuts off what the running sum does not hold, 2^-24 of it a step of 16 on average and always towards zero: what has to be
// exact to fp32 is summed in TMEM over this many blocks of 64 only, and those sums are added in registers, where they are rounded (stats at
// 16384 x 131072 x 2048: off by 1.9e-6 with one sum, by 4.3e-7 with sums of 512 products, for 2 to 5 % of the time).
constexpr int kVtPromote = 8;
// Pairs: what a logit is off by, its softmax is off by relatively, and a learnt token's gradient 1 - p by more: with sums of 512 products dH and dW of few tokens were off
// by up to 2.5e-6 (plain fp32 3e-7), logits by 5.5e-7 of theirs.  One block a sum for the gradient's logits (2.5e-7 of few tokens, logits 1.2e-7), else four:
// 1 x 2048 x 32000 x 1024 gradient 1024 -> 1063 us (everything in sums of one block 1111), loss the same.
constexpr int kVtPromotePairs = 4, kVtPromoteGrad = 1;
// Gradients of 16-bit types are rounded by more, each term of a sum by 2^-9 or 2^-12 of its own: they are one sum while it has at most kVtLongest
// products (cut off by about 2^-15 of it), and sums of 64 blocks beyond (131072 tokens of one sign, fp16: dW was off by 4.6e-4).
constexpr int kVtPromoteLong = 64;
constexpr int kVtAhead = 8;                    // the next task is claimed when this many blocks of 64 of the current one are left to load
enum { VT_ERR_DEP = 0x801, VT_ERR_FULL, VT_ERR_EMPTY, VT_ERR_ACC, VT_ERR_ACC_FREE, VT_ERR_RING, VT_ERR_RING_FREE, VT_ERR_MEET };
enum { VT_STATS = 0, VT_G, VT_DH, VT_DW };

struct VocabMaps {
  CUtensorMap hk[2], wk[2];                    // [hi, lo] H', W read K-major: box {64, 128}
  CUtensorMap hm[2], wm[2], gk[2], gm[2];      // MN-major (box {64, 64}); G both ways
};

struct VocabChain {
  int groups, D;
  int64_t T, V, Tp;
  int w_shared, w_swap;                        // W of all groups is one; W's groups lie row by row in turn: map dimensions (D, groups, V)
  int bf16;                                    // operands are bf16 (else fp16)
  const int* live; const float4* rowp; const int* rowy; const int* index; const VocabScale* scale;
  const float2* rowf; const float2* colf; const float2* rowg; const float2* dhf; const float2* dwf; int64_t Vp; int Dp;      // of pairs, see VocabPrep
  // loss
  int runs, run;                               // runs of the vocabulary, tiles of one
  float2* part; float* zy;
  // gradient
  int pieces, piece, gp;                       // pieces of a group, columns of one (a multiple of 256), columns of a row of G (a multiple of 64)
  int slots, lag, parts, run_w;                // ...; parts of dH's contraction; tiles of dW along the vocabulary of one task
  int tiles, td, kd, kpart, last_tiles, last_blocks;   // tiles along the vocabulary, along D; blocks of 64 of D, of a part; tiles, blocks of a group's last piece
  int h_first;                                 // dH before dW among the uses of a piece
  FastDiv by_td, by_run_w;
  uint16_t* G[2];                              // [slots][Tp][gp]
  float* acc; int acc_pitch;                   // [groups][parts][Tp][acc_pitch] or nullptr: one piece, one part
  void* dH; int64_t dh_row, dh_group; int dh_type, vec_dh;
  void* dW; int64_t dw_row, dw_group; int dw_type, vec_dw, accumulate;
  unsigned int* claim; unsigned int* done_g; unsigned int* done_u;     // [groups * pieces] epilogue warps done with tiles of G, with uses of them
  DeviceStatus* status;
};

// A task as its pair's warps get it: tile (ti, tj) of group g, of piece p of the vocabulary; n tiles or part n; k0, kb: blocks of 64 of its
// contraction; seq = g * pieces + p and the place of that piece's G; live tokens of the group.
struct VTask { int kind, g, ti, tj, n, p, seq, slot, live, k0, kb, pad; };

// Blocks of a sum of a task's tiles (0: all), and sums of a tile: one, or one of the small products of pairs and as many as there are.
template <bool GRAD, bool SPLIT, bool LONG>
__device__ __forceinline__ constexpr int vt_step(int kind) {
  return SPLIT ? (kind == VT_G ? kVtPromoteGrad : kVtPromotePairs) : !GRAD ? kVtPromote : LONG ? kVtPromoteLong : 0;
}
template <bool SPLIT>
__device__ __forceinline__ int vt_sums(int kb, int step) { return step == 0 ? 1 : (SPLIT ? 1 : 0) + (kb + step - 1) / step; }

__device__ __forceinline__ int vt_tiles(int n) { return (n + 255) >> 8; }
__device__ __forceinline__ int vt_piece_tiles(const VocabChain& a, int p) { return p + 1 == a.pieces ? a.last_tiles : a.piece >> 8; }
__device__ __forceinline__ int vt_uses_h(const VocabChain& a, int tm) { return a.dH != nullptr ? tm * a.td * a.parts : 0; }
__device__ __forceinline__ int vt_uses_w(const VocabChain& a, int nv) { return a.dW != nullptr ? (int)a.by_run_w.div((uint32_t)(nv + a.run_w - 1)) * a.td : 0; }

// The list of tasks, walked in order by the thread that claims them, without a division on the way (one thread's divisions were most
// of the 3 to 5 us that a claim took): a phase holds the tiles of G of one piece and the uses of the one `lag` before.
struct VWalk {
  int phase, phases;
  unsigned int base, count;    // tasks before this phase, in it
  int g, p, slot, live;        // piece whose G is in it (loss: its group)
  int gu, pu, slot_u, live_u;  // piece whose uses are
  int n_g, n_w, n_h;           // tiles of G, tasks of dW and of dH
};
template <bool GRAD>
__device__ __forceinline__ void vt_fill(const VocabChain& a, VWalk& w) {
  if constexpr (!GRAD) {
    w.count = (unsigned)(vt_tiles(w.live) * a.runs);
  } else {
    w.n_g = w.g < a.groups ? vt_tiles(w.live) * vt_piece_tiles(a, w.p) : 0;
    w.n_w = w.gu >= 0 ? vt_uses_w(a, vt_piece_tiles(a, w.pu)) : 0;
    w.n_h = w.gu >= 0 ? vt_uses_h(a, vt_tiles(w.live_u)) : 0;
    w.count = (unsigned)(w.n_g + w.n_w + w.n_h);
  }
}
template <bool GRAD>
__device__ __forceinline__ void vt_first(const VocabChain& a, VWalk& w) {
  w.phase = 0; w.phases = GRAD ? a.groups * a.pieces + a.lag : a.groups;
  w.base = 0; w.g = w.p = w.slot = 0; w.live = a.live[0];
  w.gu = -1; w.pu = w.slot_u = w.live_u = 0; w.n_g = w.n_w = w.n_h = 0;
  vt_fill<GRAD>(a, w);
}
template <bool GRAD>
__device__ __forceinline__ bool vt_decode(const VocabChain& a, VWalk& w, unsigned int t, VTask& k) {
  while (t - w.base >= w.count) {
    w.base += w.count;
    if (++w.phase >= w.phases) return false;
    if (!GRAD || ++w.p == a.pieces) {
      w.p = 0;
      if (++w.g < a.groups) w.live = a.live[w.g];
    }
    if (GRAD) {
      if (++w.slot == a.slots) w.slot = 0;
      if (w.phase == a.lag) {
        w.gu = 0; w.live_u = a.live[0];
      } else if (w.phase > a.lag) {
        if (++w.slot_u == a.slots) w.slot_u = 0;
        if (++w.pu == a.pieces) { w.pu = 0; w.live_u = a.live[++w.gu]; }
      }
    }
    vt_fill<GRAD>(a, w);
  }
  unsigned int q = t - w.base;
  k.n = k.k0 = 0;
  k.kb = a.kd;
  if (!GRAD || q < (unsigned)w.n_g) {
    const unsigned int tm = (unsigned)vt_tiles(w.live);
    k.kind = GRAD ? VT_G : VT_STATS;
    k.g = w.g; k.p = w.p; k.seq = w.phase; k.slot = w.slot; k.live = w.live;
    k.tj = (int)(q / tm);
    k.ti = (int)(q - (unsigned)k.tj * tm);
    if (!GRAD) {
      k.p = k.tj;                                // (the run)
      k.tj *= a.run;
      k.n = min(a.run, a.tiles - k.tj);
    }
    return true;
  }
  q -= (unsigned)w.n_g;
  k.g = w.gu; k.p = w.pu; k.seq = w.phase - a.lag; k.slot = w.slot_u; k.live = w.live_u;
  const bool of_h = a.h_first ? q < (unsigned)w.n_h : q >= (unsigned)w.n_w;
  if (!of_h) {
    if (a.h_first) q -= (unsigned)w.n_h;
    k.kind = VT_DW;
    k.ti = (int)a.by_td.div(q);
    k.tj = (int)q - k.ti * a.td;
    k.ti *= a.run_w;
    k.n = min(a.run_w, vt_piece_tiles(a, w.pu) - k.ti);
    k.kb = (w.live_u + 63) >> 6;
    return true;
  }
  if (!a.h_first) q -= (unsigned)w.n_w;
  k.kind = VT_DH;
  const unsigned int tiles = (unsigned)(vt_tiles(w.live_u) * a.td);
  k.n = a.parts > 1 ? (int)(q / tiles) : 0;
  q -= (unsigned)k.n * tiles;
  k.ti = (int)a.by_td.div(q);
  k.tj = (int)q - k.ti * a.td;
  k.k0 = k.n * a.kpart;
  k.kb = max(0, min(a.kpart, (w.pu + 1 == a.pieces ? a.last_blocks : a.piece >> 6) - k.k0));
  return true;
}

namespace ptx {
// Hands 48 bytes to a CTA of the cluster and counts them on its barrier (which expects them and one arrival).
__device__ __forceinline__ void send_48(uint32_t to_cluster, uint32_t bar_cluster, const uint4 (&v)[3]) {
  asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], 48;" ::"r"(bar_cluster) : "memory");
#pragma unroll
  for (uint32_t i = 0; i < 3; ++i)
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(to_cluster + 16u * i), "r"(v[i].x), "r"(v[i].y), "r"(v[i].z), "r"(v[i].w), "r"(bar_cluster) : "memory");
}
}  // namespace ptx

// A warp's box of 32 rows x 128 bytes, where values change between one row per lane (as they come from TMEM) and 16 bytes per
// lane, eight lanes to a row.  Chunk c of row r sits at chunk c ^ (r % 8): free of bank conflicts both ways.
__device__ __forceinline__ uint32_t vt_chunk(uint32_t box, int row, int q) { return box + (uint32_t)row * 128u + (uint32_t)((q ^ (row & 7)) * 16); }

// Two values as 16-bit ones.
__device__ __forceinline__ uint32_t vt_pack(int bf16, float x, float y) {
  if (bf16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  return pack_half2(x, y);
}
__device__ __forceinline__ float2 vt_unpack(int bf16, uint32_t u) {
  return bf16 ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u)) : unpack_half2(u);
}
__device__ __forceinline__ void vt_write1(void* out, int type, int64_t o, float v) {
  if (type == PRSGD_TYPE_FP32) static_cast<float*>(out)[o] = v;
  else if (type == PRSGD_TYPE_BF16) static_cast<__nv_bfloat16*>(out)[o] = __float2bfloat16_rn(v);
  else static_cast<__half*>(out)[o] = __float2half_rn(v);
}
__device__ __forceinline__ float vt_read1(const void* out, int type, int64_t o) {
  if (type == PRSGD_TYPE_FP32) return static_cast<const float*>(out)[o];
  if (type == PRSGD_TYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(out)[o]);
  return __half2float(static_cast<const __half*>(out)[o]);
}

// Where 32 rows of a tile go.
struct VOut {
  void* out; int type; int64_t row;            // first row's place; elements between rows
  const int* index;                            // rows through index, or one after another
  int rows, cols;                              // rows of the 32 that exist; columns of the array
  int add, vec;                                // added to what is there; rows begin on 16-byte boundaries
  int reduce;                                  // the adding is left to L2 (fp32 rows on 16-byte boundaries whose pitch is a multiple of 4)
};
// Element offsets of rows lane / 8 + 4 i, i = 0..7 (-1: not there).
__device__ __forceinline__ void vt_rows(const VOut& d, int lane, int64_t (&o)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 4 * i + (lane >> 3);
    o[i] = r < d.rows ? (d.index ? (int64_t)d.index[r] : (int64_t)r) * d.row : -1;
  }
}

// Adds four floats to memory in L2.  (A sum read, added to and written back by the SM waits for its old values: about 1 us four times
// a tile, as long as the products of a tile of dH.)
__device__ __forceinline__ void vt_red4(float* p, uint4 v) {
  asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};"
               ::"l"(p), "f"(__uint_as_float(v.x)), "f"(__uint_as_float(v.y)), "f"(__uint_as_float(v.z)), "f"(__uint_as_float(v.w)) : "memory");
}

// 32 rows x 32 columns (from column c0) of fp32 values, a row per lane, to where they go, through `box`: a lane writes four columns.
__device__ __forceinline__ void vt_out32(const VOut& d, uint32_t box, int lane, int c0, const float (&v)[32]) {
  __syncwarp();
#pragma unroll
  for (int q = 0; q < 8; ++q)
    st_shared_v4(vt_chunk(box, lane, q), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
  __syncwarp();
  const int c = c0 + (lane & 7) * 4;
  if (c >= d.cols) return;
  if (d.vec && c + 4 <= d.cols && d.type == PRSGD_TYPE_FP32) {
    float* const out = static_cast<float*>(d.out) + c;
    int64_t o[8];
    vt_rows(d, lane, o);
    if (d.reduce) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 u = ld_shared_v4(vt_chunk(box, 4 * i + (lane >> 3), lane & 7));
        if (o[i] >= 0) vt_red4(out + o[i], u);
      }
      return;
    }
    float4 old[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) old[i] = d.add && o[i] >= 0 ? *reinterpret_cast<const float4*>(out + o[i]) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint4 u = ld_shared_v4(vt_chunk(box, 4 * i + (lane >> 3), lane & 7));
      if (o[i] >= 0)
        *reinterpret_cast<float4*>(out + o[i]) = make_float4(__uint_as_float(u.x) + old[i].x, __uint_as_float(u.y) + old[i].y, __uint_as_float(u.z) + old[i].z, __uint_as_float(u.w) + old[i].w);
    }
    return;
  }
  if (d.vec && c + 4 <= d.cols) {                          // 16-bit values that are added to
    uint16_t* const out = static_cast<uint16_t*>(d.out) + c;
    const int bf16 = d.type == PRSGD_TYPE_BF16;
    int64_t o[8];
    vt_rows(d, lane, o);
    uint2 old[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) old[i] = d.add && o[i] >= 0 ? *reinterpret_cast<const uint2*>(out + o[i]) : make_uint2(0u, 0u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint4 u = ld_shared_v4(vt_chunk(box, 4 * i + (lane >> 3), lane & 7));
      const float2 x = vt_unpack(bf16, old[i].x), y = vt_unpack(bf16, old[i].y);
      if (o[i] >= 0)
        *reinterpret_cast<uint2*>(out + o[i]) = make_uint2(vt_pack(bf16, __uint_as_float(u.x) + x.x, __uint_as_float(u.y) + x.y),
                                                           vt_pack(bf16, __uint_as_float(u.z) + y.x, __uint_as_float(u.w) + y.y));
    }
    return;
  }
#pragma unroll 1
  for (int r = lane >> 3; r < d.rows; r += 4) {            // (in few instructions: code is fetched where others' is in use)
    const int64_t o = (d.index ? (int64_t)d.index[r] : (int64_t)r) * d.row + c;
#pragma unroll 1
    for (int k = 0; k < 4 && c + k < d.cols; ++k) {
      float w;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w) : "r"(vt_chunk(box, r, lane & 7) + 4u * (uint32_t)k) : "memory");
      vt_write1(d.out, d.type, o + k, d.add ? w + vt_read1(d.out, d.type, o + k) : w);
    }
  }
}
// 32 rows x 64 columns of 16-bit values, a row per lane, through `box`: 32 columns (half h) into it, and from there eight columns a lane.
__device__ __forceinline__ void vt_put32(int bf16, uint32_t box, int lane, int h, const float (&v)[32]) {
  if (h == 0) __syncwarp();
#pragma unroll
  for (int q = 0; q < 4; ++q)
    st_shared_v4(vt_chunk(box, lane, h * 4 + q), vt_pack(bf16, v[8 * q], v[8 * q + 1]), vt_pack(bf16, v[8 * q + 2], v[8 * q + 3]),
                 vt_pack(bf16, v[8 * q + 4], v[8 * q + 5]), vt_pack(bf16, v[8 * q + 6], v[8 * q + 7]));
}
__device__ __forceinline__ void vt_out64(const VOut& d, uint32_t box, int lane, int c0) {
  __syncwarp();
  const int c = c0 + (lane & 7) * 8;
  if (c >= d.cols) return;
  int64_t o[8];
  vt_rows(d, lane, o);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 u = ld_shared_v4(vt_chunk(box, 4 * i + (lane >> 3), lane & 7));
    if (o[i] < 0) continue;
    uint16_t* to = static_cast<uint16_t*>(d.out) + o[i] + c;
    if (c + 8 <= d.cols) {
      *reinterpret_cast<uint4*>(to) = u;
    } else {
      const uint16_t* e = reinterpret_cast<const uint16_t*>(&u);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < d.cols) to[k] = e[k];
    }
  }
}

// 32 sums of scaled operands: times the factors of the thread's row and of 32 columns.
__device__ __forceinline__ void vt_undo32(float (&v)[32], float2 row, const float2* cols) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const float4 f = *reinterpret_cast<const float4*>(cols + i);
    v[i] = v[i] * (row.x * f.x) * (row.y * f.y);
    v[i + 1] = v[i + 1] * (row.x * f.z) * (row.y * f.w);
  }
}

// SPLIT: fp32 operands, products of fp16 pairs.  LONG: a gradient of 16-bit types with contractions of more than kVtLongest products.
template <bool GRAD, bool SPLIT, bool LONG = false>
__global__ void __launch_bounds__(kVtThreads, 1) vocab_chain_kernel(const __grid_constant__ VocabMaps maps, const __grid_constant__ VocabChain a) {
  constexpr int kStages = vt_stages(GRAD), kPasses = SPLIT ? 3 : 1;
  constexpr bool PROMOTE = SPLIT || !GRAD || LONG;
  constexpr int kGroups = PROMOTE ? 1 : 2, kWarpCols = PROMOTE ? 64 : 128;
  constexpr float kLog2e = 1.4426950408889634f;
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 4 + 2 * kVtRing + 1];
  __shared__ __align__(16) uint4 ring[3 * kVtRing];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float2 shares[GRAD ? 1 : 4][GRAD ? 1 : 128][kVtShares];
  __shared__ __align__(8) uint64_t meet[4][4];
  const uint32_t stage0 = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1u;                 // clusters of two along x
  DeviceStatus* status = a.status;
  auto bar = [&](int i) { return ptx::smem_u32(&bars[i]); };
  auto full = [&](int s) { return bar(s); };                              // in the leader (rank 0): its stage has both CTAs' operands
  auto empty = [&](int s) { return bar(kStages + s); };                   // in each: the MMAs that read the stage are done
  auto tfull = [&](int i) { return bar(2 * kStages + i); };               // in each: sum i is complete
  auto tempty = [&](int i) { return bar(2 * kStages + 2 + i); };          // in the leader: all epilogue warps have read sum i
  auto sfull = [&](int i) { return bar(2 * kStages + 4 + i); };           // in each: ring entry i holds a task
  auto sempty = [&](int i) { return bar(2 * kStages + 4 + kVtRing + i); };     // in the leader: everyone has read it
  const uint32_t loaded = bar(2 * kStages + 4 + 2 * kVtRing);             // in the leader: all loads of a task have been issued
  if (threadIdx.x == 0) {
    ptx::mbar_init(loaded, 1);
    for (int s = 0; s < kStages; ++s) { ptx::mbar_init(full(s), 1); ptx::mbar_init(empty(s), 1); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(tfull(i), 1); ptx::mbar_init(tempty(i), 2 * kVtEpiWarps / kGroups); }
    for (int i = 0; i < kVtRing; ++i) { ptx::mbar_init(sfull(i), 1); ptx::mbar_init(sempty(i), 2 * kVtEpiWarps + 5); }
    for (int i = 0; i < 16; ++i) ptx::mbar_init(ptx::smem_u32(&meet[i >> 2][i & 3]), kVtShares - 1);
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
  // made visible, in L2 (TMA behind a proxy fence, ld.cg).
  auto next_task = [&](int n) -> VTask {
    const int r = n % kVtRing;
    VTask k;
    k.kind = -1;
    if (!ptx::warp_wait(sfull(r), (uint32_t)((n / kVtRing) & 1), ab, status, VT_ERR_RING)) return k;
    const uint32_t at = ptx::smem_u32(&ring[3 * r]);
    const uint4 w = ld_shared_v4(at), x = ld_shared_v4(at + 16u), y = ld_shared_v4(at + 32u);
    auto all = [&](uint32_t v) { return (int)__shfl_sync(0xffffffffu, v, 0); };
    k.kind = all(w.x); k.g = all(w.y); k.ti = all(w.z); k.tj = all(w.w);
    k.n = all(x.x); k.p = all(x.y); k.seq = all(x.z); k.slot = all(x.w);
    k.live = all(y.x); k.k0 = all(y.y); k.kb = all(y.z);
    return k;
  };
  auto free_task = [&](int n) { ptx::mbar_arrive_cluster(ptx::cluster_map(sempty(n % kVtRing), 0)); };

  // The load and product roles are walked by whole warps with one elected lane that issues, so that descriptors and addresses stay
  // in uniform registers.  The epilogue's sums take registers from them: 128 * 64 + 512 * 104 of the launch's 640 * 96.
  // Every load warp of the pair has a part in every stage, rows without tokens included: one that only waited for stages to be free
  // could fall two rounds behind, and would take the barrier's phase for another.
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 0 || warp == 3) {                          // ---- operand loads: warp 0 A, warp 3 B --------------------------
      const bool second = warp == 3, issue = ptx::elect_one();
      uint32_t s = 0, phase = 1;                           // (a fresh barrier passes a wait for the phase before its first)
      for (int n = 0;; ++n) {
        const VTask k = next_task(n);
        if (k.kind < 0) break;
        if (issue) { free_task(n); ptx::fence_proxy_async_all(); }
        const int k0 = k.k0, kb = k.kb, tiles = k.kind == VT_STATS || k.kind == VT_DW ? k.n : 1, blocks = tiles * kb * kPasses, ask = max(0, blocks - kVtAhead);
        const int wg = a.w_shared ? 0 : k.g;
        const bool of_w = second ? k.kind != VT_DW : false, of_g = !second && k.kind >= VT_DH;
        const bool mn = GRAD && (k.kind == VT_DW || (second && k.kind == VT_DH));
        const int z = of_w ? wg : of_g ? k.slot : k.g;
        const bool swap = of_w && a.w_swap;
        if (issue && blocks == 0 && rank == 0 && !second) ptx::mbar_arrive(loaded);
        bool ok = true;
        for (int j = 0, b = 0; j < tiles && ok; ++j) {
          // first row (column) of this CTA's half of the operand, first of the contraction
          int at0 = (second ? k.tj + (k.kind == VT_STATS ? j : 0) : k.ti + (k.kind == VT_DW ? j : 0)) * 256 + (int)rank * 128, q0 = 0;
          if (GRAD && of_w) {
            if (k.kind == VT_G) at0 += k.p * a.piece;
            else q0 = k.p * a.piece;
          }
          for (int p = 0; p < kPasses && ok; ++p) {
            const int plane = SPLIT && p == (second ? 1 : 0) ? 1 : 0;      // lo hi, hi lo, hi hi: the small ones first
            const CUtensorMap* map = of_w ? (mn ? &maps.wm[plane] : &maps.wk[plane]) : of_g ? (mn ? &maps.gm[plane] : &maps.gk[plane])
                                          : (mn ? &maps.hm[plane] : &maps.hk[plane]);
            for (int q = k0; q < k0 + kb; ++q, ++b) {
              if (!ptx::warp_wait(empty((int)s), phase, ab, status, VT_ERR_EMPTY)) { ok = false; break; }
              if (issue) {
                if (rank == 0 && !second) ptx::mbar_expect_tx(full((int)s), 2 * kVtStageBytes);
                const uint32_t fb = ptx::cluster_map(full((int)s), 0), at = stage0 + s * kVtStageBytes + (second ? 16384u : 0u);
                if (mn) {
                  const int y = q0 + q * 64;
                  ptx::tma_load_3d_pair(at, map, fb, at0, swap ? z : y, swap ? y : z);
                  ptx::tma_load_3d_pair(at + 8192u, map, fb, at0 + 64, swap ? z : y, swap ? y : z);
                } else {
                  ptx::tma_load_3d_pair(at, map, fb, q * 64, swap ? z : at0, swap ? at0 : z);
                }
                if (b == ask && rank == 0 && !second) ptx::mbar_arrive(loaded);
              }
              __syncwarp();
              if (++s == kStages) { s = 0; phase ^= 1u; }
            }
          }
        }
        if (!ok) break;
      }
    } else if (warp == 1 && rank == 0) {                   // ---- products (the leader issues for the pair) --------------
      const bool issue = ptx::elect_one();
      const uint32_t format = a.bf16 ? (1u << 7) | (1u << 10) : 0u;
      uint32_t s = 0, phase = 0, sums = 0;
      for (int n = 0;; ++n) {
        const VTask k = next_task(n);
        if (k.kind < 0) break;
        if (issue) free_task(n);
        const int step = vt_step<GRAD, SPLIT, LONG>(k.kind);
        const int kb = k.kb, blocks = kb * kPasses, tiles = blocks > 0 ? (k.kind == VT_STATS || k.kind == VT_DW ? k.n : 1) : 0;
        const bool a_mn = GRAD && k.kind == VT_DW, b_mn = GRAD && k.kind >= VT_DH;
        const uint32_t idesc = ptx::idesc_f16(256, 256, a_mn, b_mn) | format;
        // a step of 16 along the contraction: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major block
        const uint64_t da_k = a_mn ? 128u : 2u, db_k = b_mn ? 128u : 2u;
        const uint64_t da0 = a_mn ? ptx::smem_desc_sw128(stage0, 8192u, 1024u) : ptx::smem_desc_sw128(stage0, 16u, 1024u);
        const uint64_t db0 = b_mn ? ptx::smem_desc_sw128(stage0 + 16384u, 8192u, 1024u) : ptx::smem_desc_sw128(stage0 + 16384u, 16u, 1024u);
        bool ok = true;
        for (int j = 0; j < tiles && ok; ++j) {
          int next = 0;                                    // block that starts a new sum
          uint32_t acc = 0;
          for (int q = 0; q < blocks; ++q) {
            const bool first = q == next;
            if (first) {
              next = !PROMOTE ? blocks : SPLIT && q < 2 * kb ? 2 * kb : min(blocks, q + step);
              acc = sums & 1u;
              if (sums >= 2 && !ptx::warp_wait(tempty((int)acc), ((sums >> 1) - 1) & 1, ab, status, VT_ERR_ACC_FREE)) { ok = false; break; }
              ptx::tc_fence_after();
              ++sums;
            }
            if (!ptx::warp_wait(full((int)s), phase, ab, status, VT_ERR_FULL)) { ok = false; break; }
            ptx::tc_fence_after();
            if (issue) {
              const uint64_t at = s * (kVtStageBytes >> 4);
#pragma unroll
              for (uint32_t h = 0; h < 4; ++h)
                ptx::mma_f16_pair(tmem + acc * 256u, da0 + at + h * da_k, db0 + at + h * db_k, idesc, !first || h != 0 ? 1u : 0u);
              ptx::mma_commit_pair(empty((int)s));
              if (q + 1 == next) ptx::mma_commit_pair(tfull((int)acc));
            }
            __syncwarp();
            if (++s == kStages) { s = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
      }
    } else if (warp == 2 && lane == 0 && rank == 0) {      // ---- claims tasks for the pair --------------------------------
      VWalk w;
      vt_first<GRAD>(a, w);
      int ready_g = -1, ready_u = -1;                      // pieces seen to be done
      for (int n = 0;; ++n) {
        const int r = n % kVtRing;
        // Not before the last loads of the task before are being issued: a task claimed sooner would only keep those that
        // depend on it waiting.
        if (n > 0 && !ptx::mbar_wait(loaded, (uint32_t)((n - 1) & 1), ab, status, VT_ERR_RING_FREE)) break;
        if (n >= kVtRing && !ptx::mbar_wait(sempty(r), (uint32_t)(((n / kVtRing) - 1) & 1), ab, status, VT_ERR_RING_FREE)) break;
        VTask k;
        const unsigned int t = atomicAdd(a.claim, 1u);
        if (!vt_decode<GRAD>(a, w, t, k)) {
          k.kind = -1;
          k.g = k.ti = k.tj = k.n = k.p = k.seq = k.slot = k.live = k.k0 = k.kb = 0;
        }
        if (GRAD && k.kind >= 0) {
          // what it waits for: tiles of G; the uses of the piece whose place it takes; for dH, the piece before of the same group
          int wait_g = -1, wait_u = -1;
          if (k.kind == VT_G) wait_u = k.seq - a.slots;
          else wait_g = k.seq;
          if (k.kind == VT_DH && k.p > 0) wait_u = k.seq - 1;
          if (wait_g > ready_g) {
            const unsigned int need = (unsigned)(vt_tiles(k.live) * vt_piece_tiles(a, k.p)) * 2u * kVtEpiWarps;
            if (need > 0 && !ptx::flag_wait(a.done_g + wait_g, need, ab, status, VT_ERR_DEP)) break;
            ready_g = wait_g;
          }
          if (wait_u >= 0 && wait_u != ready_u) {
            const int g = wait_u / a.pieces, p = wait_u - g * a.pieces;
            const unsigned int need = (unsigned)(vt_uses_h(a, vt_tiles(a.live[g])) + vt_uses_w(a, vt_piece_tiles(a, p))) * 2u * kVtEpiWarps;
            if (need > 0 && !ptx::flag_wait(a.done_u + wait_u, need, ab, status, VT_ERR_DEP)) break;
            ready_u = wait_u;
          }
        }
        const uint4 words[3] = {make_uint4((uint32_t)k.kind, (uint32_t)k.g, (uint32_t)k.ti, (uint32_t)k.tj),
                                make_uint4((uint32_t)k.n, (uint32_t)k.p, (uint32_t)k.seq, (uint32_t)k.slot),
                                make_uint4((uint32_t)k.live, (uint32_t)k.k0, (uint32_t)k.kb, 0u)};
#pragma unroll
        for (uint32_t c = 0; c < 2; ++c) ptx::send_48(ptx::cluster_map(ptx::smem_u32(&ring[3 * r]), c), ptx::cluster_map(sfull(r), c), words);
        if (k.kind < 0) break;
      }
    }
  } else {                                               // ---- epilogue ---------------------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    const int quarter = warp & 3, group = PROMOTE ? 0 : (warp - 4) >> 3, share = ((warp - 4) >> 2) & (kVtShares / kGroups - 1);
    const uint32_t box = stage0 + kStages * kVtStageBytes + (uint32_t)(warp - 4) * kVtWarpBytes;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(share * kWarpCols);
    uint32_t sums = 0;
    for (int n = 0;; ++n) {
      const VTask k = next_task(n);
      if (k.kind < 0) break;
      if (lane == 0) free_task(n);
      const VocabScale* sc = a.scale + k.g;
      const int r0 = k.ti * 256 + (int)rank * 128 + quarter * 32;
      const int kb = k.kb, parts = vt_sums<SPLIT>(kb, vt_step<GRAD, SPLIT, LONG>(k.kind));
      // Waits for the warp's 64 columns of a tile's sum; several sums (PROMOTE) are added in registers and the total goes back to TMEM, over
      // the last of them, so that what follows needs registers for 32 columns only.
      uint32_t acc = 0;
      auto release = [&]() {                             // the sum has been read: the next products may overwrite it
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(ptx::cluster_map(tempty((int)acc), 0));
      };
      auto gather = [&]() -> bool {
        if (!PROMOTE || parts == 1) {
          acc = sums & 1u;                               // (one group: the sum is its own)
          if (!ptx::warp_wait(tfull((int)acc), (sums >> 1) & 1u, ab, status, VT_ERR_ACC)) return false;
          ++sums;
          ptx::tc_fence_after();
          return true;
        }
        float total[2][32];
#pragma unroll
        for (int i = 0; i < 64; ++i) total[i >> 5][i & 31] = 0.f;
#pragma unroll 1
        for (int p = 0; p < parts; ++p, ++sums) {
          acc = sums & 1u;
          if (!ptx::warp_wait(tfull((int)acc), (sums >> 1) & 1u, ab, status, VT_ERR_ACC)) return false;
          ptx::tc_fence_after();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t raw[16];
            ptx::tmem_ld16(lanes + acc * 256u + (uint32_t)(q * 16), raw);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) total[q >> 1][(q & 1) * 16 + i] += __uint_as_float(raw[i]);
          }
          if (p + 1 < parts) release();
        }
        ptx::tmem_st32(lanes + acc * 256u, total[0]);
        ptx::tmem_st32(lanes + acc * 256u + 32u, total[1]);
        ptx::tmem_st_wait();
        return true;
      };
      auto others = [&]() -> bool {                      // a tile of the other group
        if (kGroups == 1 || (sums & 1u) == (uint32_t)group) return false;
        ++sums;
        return true;
      };
      auto half = [&](int h, float (&v)[32]) {
        ptx::tmem_ld32(lanes + acc * 256u + (uint32_t)(h * 32), *reinterpret_cast<uint32_t(*)[32]>(v));
        ptx::tmem_ld_wait();
      };
      bool ok = true;
      if constexpr (!GRAD) {
        const int row = r0 + lane;
        const int y = row < k.live ? a.rowy[(int64_t)k.g * a.Tp + row] : -1;
        float m = -INFINITY, sum = 0.f;
        const float2 rf = SPLIT && row < k.live ? a.rowf[(int64_t)k.g * a.Tp + row] : make_float2(1.f, 1.f);
#pragma unroll 1
        for (int j = 0; j < k.n; ++j) {
          ok = gather();
          if (!ok) break;
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            const int64_t c0 = (int64_t)(k.tj + j) * 256 + share * 64 + h * 32;
            const int cols = (int)min((int64_t)32, a.V - c0), mine = (int)(y - c0);
            if (cols <= 0) break;
            float v[32];
            half(h, v);
            if (SPLIT) vt_undo32(v, rf, a.colf + (a.w_shared ? 0 : k.g) * a.Vp + c0);
            if (cols < 32) {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = i < cols ? v[i] : -INFINITY;
            }
            if (__any_sync(0xffffffffu, y >= 0 && mine >= 0 && mine < 32)) {
              float at = 0.f;
#pragma unroll
              for (int i = 0; i < 32; ++i) at = mine == i ? v[i] : at;
              if (y >= 0 && mine >= 0 && mine < 32) a.zy[(int64_t)k.g * a.Tp + row] = at;
            }
            float most[4] = {m, v[1], v[2], v[3]};
            most[0] = fmaxf(m, v[0]);
#pragma unroll
            for (int i = 4; i < 32; ++i) most[i & 3] = fmaxf(most[i & 3], v[i]);
            const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            const float base = vocab_base(top);
            float part[4] = {sum * vt_exp2((m - base) * kLog2e), 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 32; ++i) part[i & 3] += vt_exp2((v[i] - base) * kLog2e);
            sum = (part[0] + part[1]) + (part[2] + part[3]);
            m = top;
          }
          release();
        }
        if (!ok) break;
        // The four warps that share the rows put theirs together: one pair of numbers a token and run.  Three leave theirs, the first waits
        // for them (bounded).  A warp is at most two runs ahead of the first one, which has to release a run's sums before the products of the run
        // after next are formed, so four places do.
        float2* const at = shares[n & 3][quarter * 32 + lane];
        at[share] = make_float2(m, sum);
        __syncwarp();
        const uint32_t met = ptx::smem_u32(&meet[n & 3][quarter]);
        if (share != 0) {
          if (lane == 0) ptx::mbar_arrive(met);
        } else {
          if (!ptx::warp_wait(met, (uint32_t)((n >> 2) & 1), ab, status, VT_ERR_MEET)) break;
          if (row < k.live) {
            const float2 all = vocab_merge(vocab_merge(at[0], at[1]), vocab_merge(at[2], at[3]));
            a.part[((int64_t)k.g * a.runs + k.p) * a.Tp + row] = all;
          }
        }
      } else {
        if (k.kind == VT_G) {
          if (!others()) {
            const int row = r0 + lane;
            const bool on = row < k.live;
            const int64_t at = (int64_t)k.g * a.Tp + row, piece0 = (int64_t)k.p * a.piece;
            const float4 rp = on ? a.rowp[at] : make_float4(0.f, 0.f, 0.f, 0.f);
            const int64_t y = on ? a.rowy[at] - piece0 : -1;       // its label's column of the piece
            const float2 rf = SPLIT && on ? a.rowf[at] : make_float2(1.f, 1.f);
            const float up = SPLIT ? 1.f : sc->g, both = rp.z * up, hot = rp.w * up;
            // the rows a product reads: up to the next multiple of 64 (behind the call's last token zeros are read in any case), zeros
            // behind the last live one
            VOut d;
            d.type = PRSGD_TYPE_FP16; d.row = a.gp; d.index = nullptr; d.add = 0; d.vec = 1; d.cols = a.gp; d.reduce = 0;
            d.rows = (int)min((int64_t)32, min(a.T, (int64_t)((k.live + 63) & ~63)) - r0);
            const int64_t o = ((int64_t)k.slot * a.Tp + r0) * a.gp, width = a.V - piece0;
            ok = gather();
            if (!ok) break;
            // 64 columns through the box at a time (pairs: what the first rounding left goes in a second round)
            constexpr int kRounds = SPLIT ? 2 : kWarpCols / 64;
#pragma unroll 1
            for (int round = 0; round < kRounds; ++round) {
              const int unit = SPLIT ? 0 : round, cu = k.tj * 256 + share * kWarpCols + unit * 64;
              const bool some = d.rows > 0 && cu < a.gp;
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                const int c0 = cu + h * 32, cols = on ? (int)max((int64_t)0, min((int64_t)32, width - c0)) : 0;
                const int64_t mine = y - c0;
                float v[32];
                half(unit * 2 + h, v);
                if (h == 1 && round == kRounds - 1) release();
                if (!some) continue;
                if (SPLIT) vt_undo32(v, rf, a.colf + (a.w_shared ? 0 : k.g) * a.Vp + piece0 + c0);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = both * vt_exp2(((v[i] - rp.x) - rp.y) * kLog2e);
                if (__any_sync(0xffffffffu, y >= 0 && mine >= 0 && mine < 32)) {
#pragma unroll
                  for (int i = 0; i < 32; ++i) v[i] -= y >= 0 && mine == i ? hot : 0.f;
                }
                if (cols < 32) {
#pragma unroll
                  for (int i = 0; i < 32; ++i) v[i] = i < cols ? v[i] : 0.f;
                }
                if (SPLIT && round == 1) {
#pragma unroll
                  for (int i = 0; i < 32; i += 2) {
                    const float2 f = unpack_half2(pack_half2(v[i], v[i + 1]));
                    v[i] -= f.x; v[i + 1] -= f.y;
                  }
                }
                vt_put32(SPLIT ? 0 : a.bf16, box, lane, h, v);
              }
              d.out = a.G[SPLIT ? round : 0] + o;
              if (some) vt_out64(d, box, lane, cu);
            }
          }
        } else {
          const bool of_w = k.kind == VT_DW;
          const float2 rf = a.rowg != nullptr && !of_w && r0 + lane < k.live ? a.rowg[(int64_t)k.g * a.Tp + r0 + lane] : make_float2(SPLIT ? 1.f : sc->back, 1.f);
          const float back = rf.x;                       // (of 16-bit types)
          const float2* const cf = of_w ? a.dwf + (int64_t)k.g * a.Dp : a.dhf + (int64_t)(a.w_shared ? 0 : k.g) * a.Dp;
          VOut d;
          d.cols = a.D; d.index = nullptr; d.reduce = 0;
#pragma unroll 1
          for (int j = 0; j < (of_w ? k.n : 1); ++j) {
            if (kb > 0 ? others() : kGroups == 2 && (j & 1) != group) continue;
            if (of_w) {
              const int rj = r0 + j * 256;               // first row of this warp's part of the tile
              const int64_t v0 = (int64_t)k.p * a.piece + rj, o = (int64_t)k.g * a.dw_group + v0 * a.dw_row;
              d.rows = (int)max((int64_t)-1, min((int64_t)min(32, a.piece - rj), a.V - v0));
              d.type = a.dw_type; d.row = a.dw_row; d.add = a.accumulate; d.vec = a.vec_dw;
              d.out = static_cast<char*>(a.dW) + o * (a.dw_type == PRSGD_TYPE_FP32 ? 4 : 2);
            } else {
              d.rows = min(32, k.live - r0);
              if (a.acc == nullptr) {
                d.type = a.dh_type; d.row = a.dh_row; d.add = 0; d.vec = a.vec_dh;
                d.index = a.index + (int64_t)k.g * a.Tp + r0;
                d.out = static_cast<char*>(a.dH) + (int64_t)k.g * a.dh_group * (a.dh_type == PRSGD_TYPE_FP32 ? 4 : 2);
              } else {
                d.type = PRSGD_TYPE_FP32; d.row = a.acc_pitch; d.add = d.reduce = k.p > 0; d.vec = 1;
                d.cols = a.acc_pitch;
                d.out = a.acc + (((int64_t)k.g * a.parts + k.n) * a.Tp + r0) * a.acc_pitch;
              }
            }
            if (kb > 0) ok = gather();
            if (!ok) break;
            const bool narrow = d.type != PRSGD_TYPE_FP32 && !d.add && d.vec;
#pragma unroll 1
            for (int unit = 0; unit < kWarpCols / 64; ++unit) {
              const int cu = k.tj * 256 + share * kWarpCols + unit * 64;
              const bool some = cu < a.D && d.rows > 0 && !(kb == 0 && d.add);
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                float v[32];
                if (kb > 0) {
                  half(unit * 2 + h, v);
                  if (h == 1 && unit == kWarpCols / 64 - 1) release();
                  if (!SPLIT) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] *= back;
                  } else if (some) {
                    vt_undo32(v, rf, cf + cu + h * 32);
                  }
                } else {
#pragma unroll
                  for (int i = 0; i < 32; ++i) v[i] = 0.f;
                }
                if (!some) continue;
                if (narrow) vt_put32(d.type == PRSGD_TYPE_BF16, box, lane, h, v);
                else vt_out32(d, box, lane, cu + h * 32, v);
              }
              if (narrow && some) vt_out64(d, box, lane, cu);
            }
          }
          if (!ok) break;
        }
        __syncwarp();
        if (lane == 0) {                                 // count the task, what others read of it before it
          if (k.kind == VT_G || (k.kind == VT_DH && a.pieces > 1)) asm volatile("fence.acq_rel.gpu;" ::: "memory");
          ptx::red_add((k.kind == VT_G ? a.done_g : a.done_u) + k.seq, 1u);
        }
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
