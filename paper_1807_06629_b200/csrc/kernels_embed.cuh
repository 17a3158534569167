// Token embeddings: out_t = scale * table[id_t], and its gradient dtable_v = scale * sum_{t: id_t = v} dout_t.
//
// The lookup moves rows: its floor is the rows read once and written once.  The gradient sorts the tokens of a group by id (stable,
// least significant digits first) and adds the rows of each run of equal ids in the tokens' order, so that no two blocks
// add to one place and the result does not depend on their order.  The sorted tokens are dealt out in units of equal length,
// whatever the runs' lengths (the most frequent token of a text makes up several percent of it): a run inside a unit is
// finished there, one that crosses a border leaves its parts in the workspace for a last launch that adds them in order.
#pragma once
#include "rows_io.cuh"
#include "tc_ptx.cuh"

namespace prsgd {

struct EmbedArgs {
  RowWalk walk;                                  // of a group's tokens
  const void* table; int64_t row, group;
  const int32_t* ids;
  void* out; int64_t out_row, out_group;
  int64_t tokens, vocab;
  float scale;
};

// Rows that begin on 16-byte boundaries and end on multiples of eight columns.
template <int TY, int OTY>
__global__ void __launch_bounds__(kRowThreads) embed_kernel(const EmbedArgs a) {
  using T = typename ElemOf<TY>::type;
  using O = typename ElemOf<OTY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const T* table = static_cast<const T*>(a.table) + g * a.group;
  O* out = static_cast<O*>(a.out) + g * a.out_group;
  const int32_t* ids = a.ids + g * a.tokens;
  const RowStart s = row_start(a.walk, (int64_t)blockIdx.x * kRowItems);
  RowPiece at[kRowUnroll];
  int id[kRowUnroll];
  Raw8<TY> v[kRowUnroll];
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    at[u] = row_piece(a.walk, s, u * kRowThreads + threadIdx.x);
    id[u] = at[u].row < a.walk.rows ? ids[at[u].row] : -1;
  }
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u)
    v[u] = id[u] >= 0 && id[u] < a.vocab ? load_raw<TY>(table + id[u] * a.row + (int64_t)at[u].chunk * 8) : zero_raw<TY>();
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    if (at[u].row >= a.walk.rows) break;
    float y[8];
    unpack8<TY>(v[u], y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= a.scale;
    store_raw<OTY>(out + at[u].row * a.out_row + (int64_t)at[u].chunk * 8, y);
  }
}

// Any rows: the lanes of a warp take neighbouring columns of its 32 pieces.
template <int TY, int OTY>
__global__ void __launch_bounds__(kRowThreads) embed_any_kernel(const EmbedArgs a) {
  using T = typename ElemOf<TY>::type;
  using O = typename ElemOf<OTY>::type;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.y;
  const T* table = static_cast<const T*>(a.table) + g * a.group;
  O* out = static_cast<O*>(a.out) + g * a.out_group;
  const int32_t* ids = a.ids + g * a.tokens;
  const RowStart s = row_start(a.walk, (int64_t)blockIdx.x * kRowItems);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
  for (int u = 0; u < kRowUnroll; ++u) {
    int64_t row[8];
    uint32_t col[8];
    int id[8];
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const RowPiece p = row_piece(a.walk, s, u * kRowThreads + warp * 32 + j * 4 + (lane >> 3));
      col[j] = p.chunk * 8 + (lane & 7);
      row[j] = p.row < a.walk.rows && col[j] < a.walk.cols ? p.row : -1;
      id[j] = row[j] >= 0 ? ids[row[j]] : -1;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = id[j] >= 0 && id[j] < a.vocab ? table[id[j] * a.row + col[j]] : from_f32<T>(0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (row[j] >= 0) out[row[j] * a.out_row + col[j]] = from_f32<O>(to_f32(v[j]) * a.scale);
  }
}

// ---- gradient -------------------------------------------------------------------------------------------------
constexpr int kSortBits = 9, kSortWarps = 32, kSortPitch = (1 << kSortBits) + 1;
constexpr int kSortCtas = 8, kSortTurn = 32 * kSortWarps;            // most blocks that share a group's tokens; tokens of a block's turn
constexpr size_t kSortCounts = ((size_t)kSortWarps * kSortPitch * 4 + 15) / 16 * 16;
constexpr size_t kSortSmem = kSortCounts + (4 << kSortBits);

struct EmbedGradArgs {
  const void* dout; int64_t row, group;
  const int32_t* ids;
  void* dtable; int64_t t_row, t_group;
  int64_t groups, tokens, vocab;
  int dim, chunks;
  float scale;
  int accumulate;
  int passes, bits;                              // digits of an id; bits of a digit
  int ctas, turns;                               // blocks (a cluster) that sort a group; 1024 tokens each they take at a time
  int unit, units;                               // sorted tokens of a unit; units of a group
  int lanes;                                     // threads side by side along a row; kRowThreads / lanes units share a block
  uint2* keys[2];                                // [groups][tokens] (id, token), sorted ones in keys[passes & 1]
  int* live;                                     // [groups]
  float* parts;                                  // [groups][units][2][chunks * 8]: sum of the run that began in an earlier unit; of the one that goes on
  DeviceStatus* status;
};

// Tokens of a group by id, by a cluster of blocks.  A warp takes an equal share of them, counts its digits, and places them behind those of smaller
// digits, of earlier blocks and of earlier warps; within a warp's 32 the order is the lanes'.  Counted without atomics: the many
// equal digits of frequent ids took turns.  Loops are rolled: code that is run through once is fetched anew at every launch, at about 20
// cycles an instruction.  (8192 tokens, two digits: a block alone 18 us, of which 11 thousand cycles a digit went into the ballots of eight turns.)
__device__ void embed_sort(const EmbedGradArgs& a, int64_t g, int cta, uint32_t* counts) {
  __shared__ uint32_t sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, digits = 1 << a.bits, turns = a.turns;
  const int32_t* ids = a.ids + g * a.tokens;
  uint32_t* mine = counts + warp * kSortPitch;
  uint32_t* totals = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(counts) + kSortCounts);    // of this block, read by the others
  int n = (int)a.tokens;
  for (int p = 0; p < a.passes; ++p) {
    const uint2* from = a.keys[p & 1] + g * a.tokens;
    uint2* to = a.keys[(p + 1) & 1] + g * a.tokens;
    const int begin = min(n, (cta * kSortWarps + warp) * turns * 32), end = min(n, begin + turns * 32);
    auto digit = [&](uint2 k) { return (k.x >> (p * a.bits)) & (uint32_t)(digits - 1); };
    auto get = [&](int turn) -> uint2 {          // (id, token), or (-1, ) for none
      const int i = begin + turn * 32 + lane;
      if (i >= end) return make_uint2(0xFFFFFFFFu, 0u);
      if (p > 0) return __ldcg(from + i);        // (written by other blocks meanwhile)
      const int id = ids[i];
      return make_uint2(id >= 0 && id < a.vocab ? (uint32_t)id : 0xFFFFFFFFu, (uint32_t)i);
    };
    for (int d = lane; d < digits; d += 32) mine[d] = 0;
    __syncthreads();
    auto place = [&](uint2 k) -> uint32_t {
      const bool some = k.x != 0xFFFFFFFFu;
      const uint32_t d = digit(k);
      uint32_t same = __ballot_sync(0xffffffffu, some), at = 0;     // lanes of this digit, bit by bit
#pragma unroll
      for (int b = 0; b < kSortBits; ++b) {
        if (b >= a.bits) break;
        const uint32_t bit = (d >> b) & 1u, with = __ballot_sync(0xffffffffu, bit != 0u);
        same &= with ^ (bit - 1u);
      }
      if (some) at = mine[d] + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (some && (same >> lane) == 1u) mine[d] = at + 1u;          // (the last of its digit)
      __syncwarp();
      return at;
    };
    uint2 key = make_uint2(0xFFFFFFFFu, 0u);     // of a single turn: kept, with its number among the warp's of its digit
    uint32_t within = 0;
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
      key = get(turn);
      within = place(key);
    }
    __syncthreads();
    // exclusive sums, digit by digit, within one block by block and warp by warp: a thread takes half the warps of a digit
    const int d = threadIdx.x >> 1, w0 = (threadIdx.x & 1) * (kSortWarps / 2);
    uint32_t part = 0, first_half = 0, before = 0, total = 0;
    if (d < digits) {
#pragma unroll 4
      for (int w = 0; w < kSortWarps / 2; ++w) part += counts[(w0 + w) * kSortPitch + d];
    }
    const uint32_t other = __shfl_xor_sync(0xffffffffu, part, 1);
    if (threadIdx.x & 1) first_half = other;
    if (d < digits && (threadIdx.x & 1) == 0) totals[d] = part + other;
    if (a.ctas == 1) {
      total = part + other;
    } else {
      ptx::cluster_arrive_release();
      ptx::cluster_wait_acquire();
      uint32_t t[kSortCtas];
#pragma unroll
      for (int c = 0; c < kSortCtas; ++c) t[c] = d < digits && c < a.ctas ? ptx::ld_cluster_u32(ptx::cluster_map(ptx::smem_u32(totals + d), (uint32_t)c)) : 0u;
#pragma unroll
      for (int c = 0; c < kSortCtas; ++c) {
        if (c < cta) before += t[c];
        total += t[c];
      }
    }
    uint32_t run = threadIdx.x & 1 ? 0u : total;  // (a digit counted once)
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += up;
    }
    if (lane == 31) sums[warp] = run;
    __syncthreads();
    if (warp == 0) {
      uint32_t s = sums[lane];
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += up;
      }
      sums[lane] = s;
    }
    __syncthreads();
    run += (warp > 0 ? sums[warp - 1] : 0u) - total + before + first_half;
    n = (int)sums[kSortWarps - 1];
    if (d < digits) {
#pragma unroll 4
      for (int w = 0; w < kSortWarps / 2; ++w) {
        uint32_t* c = counts + (w0 + w) * kSortPitch + d;
        const uint32_t here = *c;
        *c = run;
        run += here;
      }
    }
    __syncthreads();
    if (turns == 1) {
      if (key.x != 0xFFFFFFFFu) to[mine[digit(key)] + within] = key;
    } else {
#pragma unroll 1
      for (int turn = 0; turn < turns; ++turn) {
        const uint2 k = get(turn);
        const uint32_t at = place(k);
        if (k.x != 0xFFFFFFFFu) to[at] = k;
      }
    }
    // the next digit reads what all blocks have placed, and writes `totals` that others have read
    if (a.ctas == 1) {
      __syncthreads();
    } else {
      ptx::cluster_arrive_release();
      ptx::cluster_wait_acquire();
    }
  }
  if (cta == 0 && threadIdx.x == 0) a.live[g] = n;
}

// The first groups * ctas blocks sort; the others write zeros meanwhile, rows whose ids occur included (their sums follow).
template <int OTY, bool VEC>
__global__ void __launch_bounds__(1024) embed_sort_kernel(const EmbedGradArgs a) {
  extern __shared__ uint32_t counts[];
  op_pdl_wait();
  op_pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  const int64_t sorters = a.groups * a.ctas;
  if (blockIdx.x < sorters) {                    // (whole clusters)
    const int64_t g = blockIdx.x / a.ctas;
    embed_sort(a, g, (int)(blockIdx.x - g * a.ctas), counts);
    return;
  }
  using O = typename ElemOf<OTY>::type;
  const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int64_t rows = a.groups * a.vocab, blocks = gridDim.x - sorters;
  const int per = 1024 / a.lanes, sub = threadIdx.x / a.lanes, c0 = threadIdx.x - sub * a.lanes;
  if (sub >= per) return;
  for (int64_t r = (blockIdx.x - sorters) * per + sub; r < rows; r += blocks * per) {
    const int64_t g = r / a.vocab;
    O* to = static_cast<O*>(a.dtable) + g * a.t_group + (r - g * a.vocab) * a.t_row;
    for (int c = c0; c < a.chunks; c += a.lanes) store8<OTY, VEC>(to + c * 8, min(8, a.dim - c * 8), zero);
  }
}

// Rows of a run's sum, eight columns a thread (`n` of which exist; VEC: all, on a 16-byte boundary).
template <int OTY, bool VEC>
__device__ __forceinline__ void embed_write(const EmbedGradArgs& a, typename ElemOf<OTY>::type* to, int n, const Raw8<OTY>& old, const float (&sum)[8]) {
  float v[8];
  if (a.accumulate) {
    if (VEC) unpack8<OTY>(old, v);
    else load8<OTY, false>(to, n, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(a.scale, sum[i], v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.scale * sum[i];
  }
  store8<OTY, VEC>(to, n, v);
}

// One unit's sums for one thread's columns.  Rows of dout, and what the sums are added to, are requested two tokens ahead, with four blocks
// an SM (4 x 8192 tokens with an id, 2048 columns, whole call: 92 us; four ahead and two blocks 95, eight ahead 112).
template <int TY, int OTY, bool VEC, bool OVEC>
__device__ __forceinline__ void embed_unit_sum(const EmbedGradArgs& a, int64_t g, int u, int c, int n, int live, int begin, int end) {
  using T = typename ElemOf<TY>::type;
  using O = typename ElemOf<OTY>::type;
  constexpr int kAhead = 2;
  const uint2* keys = a.keys[a.passes & 1] + g * a.tokens;
  const T* dout = static_cast<const T*>(a.dout) + g * a.group + c * 8;
  O* table = static_cast<O*>(a.dtable) + g * a.t_group + c * 8;
  float* parts = a.parts + ((g * a.units + u) * 2) * (int64_t)a.chunks * 8 + c * 8;
  bool inner = begin == 0 || keys[begin - 1].x != keys[begin].x;        // the current run began in this unit
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = begin; i < end; i += kAhead) {
    uint2 k[kAhead + 1];
    Raw8<TY> v[kAhead];
    Raw8<OTY> old[kAhead];
#pragma unroll
    for (int j = 0; j <= kAhead; ++j) k[j] = i + j < live ? keys[i + j] : make_uint2(0xFFFFFFFFu, 0u);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (VEC) v[j] = i + j < end ? load_raw<TY>(dout + (int64_t)k[j].y * a.row) : zero_raw<TY>();
      if (OVEC && a.accumulate && i + j < end && k[j].x != k[j + 1].x) old[j] = load_raw<OTY>(table + k[j].x * a.t_row);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= end) break;
      float x[8];
      if (VEC) unpack8<TY>(v[j], x);
      else load8<TY, false>(dout + (int64_t)k[j].y * a.row, n, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
      if (k[j].x == k[j + 1].x) continue;                // the run goes on
      if (inner) embed_write<OTY, OVEC>(a, table + k[j].x * a.t_row, n, old[j], sum);
      else store_raw<PRSGD_TYPE_FP32>(parts, sum);
      inner = true;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    }
  }
  // a run that the next unit goes on with
  if (end < live && keys[end - 1].x == keys[end].x) store_raw<PRSGD_TYPE_FP32>(inner ? parts + (int64_t)a.chunks * 8 : parts, sum);
}

template <int TY, int OTY, bool VEC, bool OVEC>
__global__ void __launch_bounds__(kRowThreads, 4) embed_sum_kernel(const EmbedGradArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int per = blockDim.x / a.lanes, sub = threadIdx.x / a.lanes;
  const int u = blockIdx.x * per + sub, c = blockIdx.y * a.lanes + threadIdx.x - sub * a.lanes;
  if (sub >= per || u >= a.units || c >= a.chunks) return;
  const int live = a.live[g], begin = u * a.unit, end = min(live, begin + a.unit), n = min(8, a.dim - c * 8);
  if (begin >= end) return;
  if (n == 8) embed_unit_sum<TY, OTY, VEC, OVEC>(a, g, u, c, n, live, begin, end);
  else embed_unit_sum<TY, OTY, false, false>(a, g, u, c, n, live, begin, end);
}

// The runs that cross borders: the unit in which a run begins adds the parts behind it, in order.
template <int OTY, bool OVEC>
__global__ void __launch_bounds__(kRowThreads) embed_join_kernel(const EmbedGradArgs a) {
  using O = typename ElemOf<OTY>::type;
  constexpr int kAhead = 8;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int per = blockDim.x / a.lanes, sub = threadIdx.x / a.lanes;
  const int u = blockIdx.x * per + sub, c = blockIdx.y * a.lanes + threadIdx.x - sub * a.lanes;
  if (sub >= per || u >= a.units || c >= a.chunks) return;
  const int live = a.live[g], begin = u * a.unit, end = min(live, begin + a.unit);
  if (begin >= end || end >= live) return;
  const uint2* keys = a.keys[a.passes & 1] + g * a.tokens;
  const uint32_t id = keys[end - 1].x, next = keys[end].x, first = keys[begin].x, before = begin > 0 ? keys[begin - 1].x : 0xFFFFFFFFu;
  if (next != id || (first == id && before == id)) return;              // ends here, or began earlier
  const int64_t pitch = (int64_t)a.chunks * 8;
  const float* parts = a.parts + g * a.units * 2 * pitch + c * 8;
  float sum[8];
  unpack8<PRSGD_TYPE_FP32>(load_raw<PRSGD_TYPE_FP32>(parts + ((int64_t)u * 2 + 1) * pitch), sum);
  const int n = min(8, a.dim - c * 8);
  O* to = static_cast<O*>(a.dtable) + g * a.t_group + id * a.t_row + c * 8;
  Raw8<OTY> old = zero_raw<OTY>();
  if (OVEC && n == 8 && a.accumulate) old = load_raw<OTY>(to);
  for (int w = u + 1; (int64_t)w * a.unit < live; w += kAhead) {
    bool in[kAhead];
    Raw8<PRSGD_TYPE_FP32> more[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {                   // (parts are requested before it is known whether they are this run's)
      const int64_t at = (int64_t)(w + j) * a.unit;
      in[j] = at < live;
      if (in[j]) more[j] = load_raw<PRSGD_TYPE_FP32>(parts + (int64_t)(w + j) * 2 * pitch);
      if (in[j]) in[j] = keys[at].x == id;
    }
    if (!in[0]) break;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (!in[j]) break;
      float x[8];
      unpack8<PRSGD_TYPE_FP32>(more[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
  }
  if (OVEC && n == 8) embed_write<OTY, true>(a, to, n, old, sum);
  else embed_write<OTY, false>(a, to, n, old, sum);
}

}  // namespace prsgd
