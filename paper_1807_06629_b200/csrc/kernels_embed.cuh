// Token embeddings: out_t = scale * table[id_t], and its gradient dtable_v = scale * sum_{t: id_t = v} dout_t.
//
// The lookup moves rows: its floor is the rows read once and written once.  The gradient sorts the tokens of a group by id (stable,
// least significant digits first) and adds the rows of each run of equal ids in the tokens' order, so that no two blocks
// add to one place and the result does not depend on their order.  The sorted tokens are dealt out in units of equal length,
// whatever the runs' lengths (the most frequent token of a text makes up several percent of it): a run inside a unit is
// finished there, one that crosses a border leaves its parts in the workspace for a last launch that adds them in order.
#pragma once
#include "rows_io.cuh"

namespace prsgd {

struct EmbedArgs {
  RowWalk walk;                                  // of a group's tokens
  const void* table; int64_t row, group;
  const int32_t* ids;
  void* out; int64_t out_row, out_group;
  int64_t tokens, vocab;
  float scale;
};

template <int TY, int OTY, bool VEC>
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
  int64_t row[kRowUnroll];
  uint32_t chunk[kRowUnroll];
  int id[kRowUnroll];
  float v[kRowUnroll][8];
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    const uint32_t i = s.chunk + u * kRowThreads + threadIdx.x, over = a.walk.by_chunks.div(i);
    row[u] = s.row + over;
    chunk[u] = i - over * a.walk.chunks;
    id[u] = row[u] < a.walk.rows ? ids[row[u]] : -1;
  }
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    const int n = (int)min((int64_t)8, a.walk.cols - (int64_t)chunk[u] * 8);
    const bool some = id[u] >= 0 && id[u] < a.vocab;
    load8<TY, VEC>(table + (some ? id[u] : 0) * a.row + (int64_t)chunk[u] * 8, some ? n : 0, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kRowUnroll; ++u) {
    if (row[u] >= a.walk.rows) break;
    const int n = (int)min((int64_t)8, a.walk.cols - (int64_t)chunk[u] * 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[u][i] *= a.scale;
    store8<OTY, VEC>(out + row[u] * a.out_row + (int64_t)chunk[u] * 8, n, v[u]);
  }
}

// ---- gradient -------------------------------------------------------------------------------------------------
constexpr int kSortBits = 9, kSortDigits = 1 << kSortBits, kSortWarps = 32, kSortPitch = kSortDigits + 1;
constexpr size_t kSortSmem = (size_t)kSortWarps * kSortPitch * 4;

struct EmbedGradArgs {
  const void* dout; int64_t row, group;
  const int32_t* ids;
  void* dtable; int64_t t_row, t_group;
  int64_t groups, tokens, vocab;
  int dim, chunks;
  float scale;
  int accumulate;
  int passes;                                    // digits of an id
  int unit, units;                               // sorted tokens of a unit; units of a group
  int lanes;                                     // threads side by side along a row; kRowThreads / lanes units share a block
  uint2* keys[2];                                // [groups][tokens] (id, token), sorted ones in keys[passes & 1]
  int* live;                                     // [groups]
  float* parts;                                  // [groups][units][2][chunks * 8]: sum of the run that began in an earlier unit; of the one that goes on
  DeviceStatus* status;
};

// Tokens of a group by id.  A warp takes an equal share of them, counts its digits, and places them behind those of smaller
// digits and of earlier warps; within a warp's 32 the order is the lanes'.
__device__ void embed_sort(const EmbedGradArgs& a, int64_t g, uint32_t* counts) {
  __shared__ uint32_t sums[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int32_t* ids = a.ids + g * a.tokens;
  uint32_t* mine = counts + warp * kSortPitch;
  int64_t n = a.tokens;
  for (int p = 0; p < a.passes; ++p) {
    const uint2* from = a.keys[p & 1] + g * a.tokens;
    uint2* to = a.keys[(p + 1) & 1] + g * a.tokens;
    const int64_t share = ((n + kSortWarps - 1) / kSortWarps + 31) / 32 * 32, begin = warp * share, end = min(n, begin + share);
    auto get = [&](int64_t i) -> uint2 {         // (digit out of range: none)
      if (i >= end) return make_uint2(0xFFFFFFFFu, 0u);
      if (p == 0) {
        const int id = ids[i];
        return id >= 0 && id < a.vocab ? make_uint2((uint32_t)id, (uint32_t)i) : make_uint2(0xFFFFFFFFu, 0u);
      }
      return from[i];
    };
    for (int d = lane; d < kSortDigits; d += 32) mine[d] = 0;
    __syncwarp();
    for (int64_t i = begin + lane; i - lane < end; i += 32) {
      const uint2 k = get(i);
      if (k.x != 0xFFFFFFFFu) atomicAdd(mine + ((k.x >> (p * kSortBits)) & (kSortDigits - 1)), 1u);
    }
    __syncthreads();
    // exclusive sums, digit by digit and within one warp by warp: a thread takes half the warps of a digit
    {
      const int d = threadIdx.x >> 1, w0 = (threadIdx.x & 1) * (kSortWarps / 2);
      uint32_t total = 0;
      for (int w = 0; w < kSortWarps / 2; ++w) total += counts[(w0 + w) * kSortPitch + d];
      uint32_t run = total;
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += up;
      }
      if (lane == 31) sums[warp] = run;
      __syncthreads();
      if (warp == 0) {
        uint32_t s = sums[lane];
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t up = __shfl_up_sync(0xffffffffu, s, o);
          if (lane >= o) s += up;
        }
        sums[lane] = s;
      }
      __syncthreads();
      run += (warp > 0 ? sums[warp - 1] : 0u) - total;
      n = sums[kSortWarps - 1];
      for (int w = 0; w < kSortWarps / 2; ++w) {
        uint32_t* c = counts + (w0 + w) * kSortPitch + d;
        const uint32_t here = *c;
        *c = run;
        run += here;
      }
    }
    __syncthreads();
    for (int64_t i = begin + lane; i - lane < end; i += 32) {
      const uint2 k = get(i);
      const bool some = k.x != 0xFFFFFFFFu;
      const uint32_t digit = some ? (k.x >> (p * kSortBits)) & (kSortDigits - 1) : kSortDigits;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      uint32_t at = 0;
      if (some) at = mine[digit] + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (some && (same >> lane) == 1u) mine[digit] = at + 1u;      // (the last of its digit)
      __syncwarp();
      if (some) to[at] = k;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) a.live[g] = (int)n;
}

// The first `groups` blocks sort; the others write zeros meanwhile, rows whose ids occur included (their sums follow).
template <int OTY, bool VEC>
__global__ void __launch_bounds__(1024) embed_sort_kernel(const EmbedGradArgs a) {
  extern __shared__ uint32_t counts[];
  op_pdl_wait();
  op_pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x < sizeof(DeviceStatus) / 4) reinterpret_cast<unsigned int*>(a.status)[threadIdx.x] = 0u;
  if (blockIdx.x < a.groups) {
    embed_sort(a, blockIdx.x, counts);
    return;
  }
  using O = typename ElemOf<OTY>::type;
  const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int64_t rows = a.groups * a.vocab, blocks = gridDim.x - a.groups;
  const int per = 1024 / a.lanes, sub = threadIdx.x / a.lanes, c0 = threadIdx.x - sub * a.lanes;
  if (sub >= per) return;
  for (int64_t r = (blockIdx.x - a.groups) * per + sub; r < rows; r += blocks * per) {
    const int64_t g = r / a.vocab;
    O* to = static_cast<O*>(a.dtable) + g * a.t_group + (r - g * a.vocab) * a.t_row;
    for (int c = c0; c < a.chunks; c += a.lanes) store8<OTY, VEC>(to + c * 8, min(8, a.dim - c * 8), zero);
  }
}

template <int OTY, bool VEC>
__device__ __forceinline__ void embed_write(const EmbedGradArgs& a, int64_t g, int64_t id, int c, const float (&sum)[8]) {
  using O = typename ElemOf<OTY>::type;
  O* to = static_cast<O*>(a.dtable) + g * a.t_group + id * a.t_row + c * 8;
  const int n = min(8, a.dim - c * 8);
  float v[8];
  if (a.accumulate) {
    load8<OTY, VEC>(to, n, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(a.scale, sum[i], v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.scale * sum[i];
  }
  store8<OTY, VEC>(to, n, v);
}

template <int TY, int OTY, bool VEC, bool OVEC>
__global__ void __launch_bounds__(kRowThreads) embed_sum_kernel(const EmbedGradArgs a) {
  using T = typename ElemOf<TY>::type;
  constexpr int kAhead = 8;
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int per = kRowThreads / a.lanes, sub = threadIdx.x / a.lanes;
  const int u = blockIdx.x * per + sub, c = blockIdx.y * a.lanes + threadIdx.x - sub * a.lanes;
  if (sub >= per || u >= a.units || c >= a.chunks) return;
  const int live = a.live[g], begin = u * a.unit, end = min(live, begin + a.unit);
  if (begin >= end) return;
  const uint2* keys = a.keys[a.passes & 1] + g * a.tokens;
  const T* dout = static_cast<const T*>(a.dout) + g * a.group + c * 8;
  float* parts = a.parts + ((g * a.units + u) * 2) * (int64_t)a.chunks * 8 + c * 8;
  const int n = min(8, a.dim - c * 8);
  bool inner = begin == 0 || keys[begin - 1].x != keys[begin].x;        // the current run began in this unit
  const bool goes_on = end < live && keys[end].x == keys[end - 1].x;    // the last run does not end in it
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  uint32_t id = keys[begin].x;
  for (int i = begin; i < end; i += kAhead) {
    uint2 k[kAhead];
    float v[kAhead][8];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) k[j] = i + j < end ? keys[i + j] : make_uint2(0u, 0u);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) load8<TY, VEC>(dout + (int64_t)k[j].y * a.row, i + j < end ? n : 0, v[j]);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i + j >= end) break;
      if (k[j].x != id) {
        if (inner) embed_write<OTY, OVEC>(a, g, id, c, sum);
        else store8<PRSGD_TYPE_FP32, true>(parts, 8, sum);
        inner = true;
        id = k[j].x;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[j][e];
    }
  }
  if (inner && !goes_on) embed_write<OTY, OVEC>(a, g, id, c, sum);
  else store8<PRSGD_TYPE_FP32, true>(inner ? parts + (int64_t)a.chunks * 8 : parts, 8, sum);
}

// The runs that cross borders: the unit in which a run begins adds the parts behind it, in order.
template <int OTY, bool OVEC>
__global__ void __launch_bounds__(kRowThreads) embed_join_kernel(const EmbedGradArgs a) {
  op_pdl_wait();
  op_pdl_trigger();
  const int64_t g = blockIdx.z;
  const int per = kRowThreads / a.lanes, sub = threadIdx.x / a.lanes;
  const int u = blockIdx.x * per + sub, c = blockIdx.y * a.lanes + threadIdx.x - sub * a.lanes;
  if (sub >= per || u >= a.units || c >= a.chunks) return;
  const int live = a.live[g], begin = u * a.unit, end = min(live, begin + a.unit);
  if (begin >= end || end >= live) return;
  const uint2* keys = a.keys[a.passes & 1] + g * a.tokens;
  const uint32_t id = keys[end - 1].x;
  if (keys[end].x != id) return;                                        // ends here
  if (begin > 0 && keys[begin].x == id && keys[begin - 1].x == id) return;      // began earlier
  const int64_t pitch = (int64_t)a.chunks * 8;
  const float* part = a.parts + ((g * a.units + u) * 2 + 1) * pitch + c * 8;
  float sum[8], more[8];
  load8<PRSGD_TYPE_FP32, true>(part, 8, sum);
  for (int w = u + 1; (int64_t)w * a.unit < live && keys[(int64_t)w * a.unit].x == id; ++w) {
    load8<PRSGD_TYPE_FP32, true>(a.parts + (g * a.units + w) * 2 * pitch + c * 8, 8, more);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += more[e];
  }
  embed_write<OTY, OVEC>(a, g, id, c, sum);
}

}  // namespace prsgd
