// C entries of the cross entropy over a vocabulary.  See include/prsgd.h for the contract.
#include <mutex>
#include "kernels_vocab_few.cuh"
#include "kernels_vocab_tc.cuh"

using namespace prsgd;

namespace {

int check_vocab(int type, int64_t groups, int64_t tokens, int64_t vocab, int dim) {
  if (!type_known(type)) return op_fail(PRSGD_ERR_ARG, "unknown element type");
  if (groups < 0 || tokens < 0 || vocab < 1 || dim < 1) return op_fail(PRSGD_ERR_ARG, "need groups >= 0, tokens >= 0, vocab >= 1, dim >= 1");
  if (groups > 4096 || tokens > (1ll << 22) || vocab > PRSGD_VOCAB_MAX || dim > 65536)
    return op_fail(PRSGD_ERR_SIZE, "more than 4096 groups, 2^22 tokens, PRSGD_VOCAB_MAX classes or 65536 columns");
  return PRSGD_OK;
}

// How a call is cut up and what its workspace holds.
struct VocabPlan {
  VocabPrep prep{};
  VocabChain chain{};
  bool grad = false, split = false, copy_w = false, longest = false;
  int64_t tasks = 0;         // at most
  size_t bytes = 0;
};

VocabPlan vocab_plan(int type, int64_t groups, int64_t T, int64_t V, int D, bool w_aligned, bool grad, unsigned char* base) {
  VocabPlan p;
  p.grad = grad; p.split = type == PRSGD_TYPE_FP32; p.copy_w = p.split || !w_aligned;
  const int planes = p.split ? 2 : 1;
  VocabPrep& a = p.prep;
  VocabChain& c = p.chain;
  a.groups = groups; a.T = T; a.V = V; a.D = D; a.grad = grad; a.h_type = type;
  const VocabCuts cuts = vocab_cuts(p.split, grad, groups, T, V, D);
  a.Tp = cuts.Tp; a.pitch = (int)round_up(D, 8);
  a.w_groups = (int)groups;
  c.groups = (int)groups; c.D = D; c.T = T; c.V = V; c.Tp = a.Tp; c.bf16 = type == PRSGD_TYPE_BF16;
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* q = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  a.status = c.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  c.live = a.live = reinterpret_cast<int*>(take(4 * (size_t)groups));
  c.scale = a.scale = reinterpret_cast<VocabScale*>(take(sizeof(VocabScale) * (size_t)groups));
  a.Vp = c.Vp = round_up(V, 256);
  a.Dp = c.Dp = (int)round_up(D, 256);
  if (p.split) {
    c.rowf = a.rowf = reinterpret_cast<float2*>(take(8 * (size_t)groups * a.Tp));
    c.colf = a.colf = reinterpret_cast<float2*>(take(8 * (size_t)groups * a.Vp));
  }
  c.rowy = a.rowy = reinterpret_cast<int*>(take(4 * (size_t)groups * a.Tp));
  c.index = a.index = reinterpret_cast<int*>(take(4 * (size_t)groups * a.Tp));
  for (int i = 0; i < planes; ++i) {
    a.Hc[i] = reinterpret_cast<uint16_t*>(take(2 * (size_t)groups * a.Tp * a.pitch));
    a.Wc[i] = reinterpret_cast<uint16_t*>(take(p.copy_w ? 2 * (size_t)groups * V * a.pitch : 0));
  }
  if (grad && type != PRSGD_TYPE_BF16) {
    for (int i = 0; i < planes; ++i) a.Hm[i] = reinterpret_cast<uint16_t*>(take(2 * (size_t)groups * a.Tp * a.pitch));
    c.rowg = a.rowg = reinterpret_cast<float2*>(take(8 * (size_t)groups * a.Tp));
  }
  if (grad && type == PRSGD_TYPE_FP16 && T > kLargestApart) a.largest = reinterpret_cast<float*>(take(4 * (size_t)groups));
  if (p.split && grad) {
    for (int i = 0; i < planes; ++i) a.Wm[i] = reinterpret_cast<uint16_t*>(take(2 * (size_t)groups * V * a.pitch));
    c.dhf = a.dhf = reinterpret_cast<float2*>(take(8 * (size_t)groups * a.Dp));
    c.dwf = a.dwf = reinterpret_cast<float2*>(take(8 * (size_t)groups * a.Dp));
    a.most = reinterpret_cast<unsigned int*>(take(4 * 2 * (size_t)groups * a.Dp));
  }
  c.tiles = cuts.tiles; c.td = cuts.td; c.kd = cuts.kd; c.by_td = FastDiv((uint32_t)cuts.td);
  p.tasks = cuts.tasks; p.longest = cuts.longest != 0;
  if (!grad) {
    c.run = cuts.run; c.runs = cuts.runs;
    c.part = reinterpret_cast<float2*>(take(8 * (size_t)groups * c.runs * a.Tp));
    c.zy = reinterpret_cast<float*>(take(4 * (size_t)groups * a.Tp));
    a.n_counters = 1;
    a.counters = c.claim = reinterpret_cast<unsigned int*>(take(4));
    p.bytes = off;
    return p;
  }
  c.rowp = a.rowp = reinterpret_cast<float4*>(take(16 * (size_t)groups * a.Tp));
  c.piece = cuts.piece; c.pieces = cuts.pieces; c.gp = cuts.gp; c.parts = cuts.parts; c.kpart = cuts.kpart; c.run_w = cuts.run_w;
  c.h_first = cuts.h_first; c.last_tiles = cuts.last_tiles; c.last_blocks = cuts.last_blocks; c.lag = cuts.lag; c.slots = cuts.slots;
  c.by_run_w = FastDiv((uint32_t)c.run_w);
  const int64_t seqs = cuts.seqs;
  for (int i = 0; i < planes; ++i) c.G[i] = reinterpret_cast<uint16_t*>(take(2 * (size_t)c.slots * a.Tp * c.gp));
  c.acc_pitch = (int)round_up(D, 8);
  c.acc = reinterpret_cast<float*>(take(c.pieces * c.parts > 1 ? 4 * (size_t)groups * c.parts * a.Tp * c.acc_pitch : 0));
  if (c.pieces * c.parts == 1) c.acc = nullptr;
  a.n_counters = (int)(1 + 2 * seqs);
  a.counters = c.claim = reinterpret_cast<unsigned int*>(take(4 * (size_t)a.n_counters));
  c.done_g = c.claim + 1; c.done_u = c.done_g + seqs;
  p.bytes = off;
  return p;
}

VocabFew vocab_few_plan(int64_t groups, int64_t T, int64_t V, int D, unsigned char* base, size_t* bytes) {
  VocabFew a{};
  a.T = (int)T; a.V = V; a.D = D; a.dp = (int)round_up(D, 8);
  // as many blocks as run at a time by their registers: three an SM for one token, else two (four, in two rounds: 24 us for 20)
  const int64_t turn = kFewWarps * kFewRows, most = std::max<int64_t>(1, 148 * (T <= 1 ? 3 : 2) / std::max<int64_t>(groups, 1));
  a.turns = (int)up(std::max<int64_t>(T, 1), kFewTurn);
  const int64_t blocks = std::max<int64_t>(1, std::min(most / a.turns, up(V, turn)));
  a.per = up(up(V, turn), blocks) * turn;
  a.blocks = (int)up(V, a.per);
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* q = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  a.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  a.part = reinterpret_cast<float2*>(take(8 * (size_t)groups * T * a.blocks));
  a.zy = reinterpret_cast<float*>(take(4 * (size_t)groups * T));
  *bytes = off;
  return a;
}

VocabFewGrad vocab_few_grad_plan(int64_t groups, int64_t T, int64_t V, int D, unsigned char* base, size_t* bytes) {
  VocabFewGrad b{};
  VocabFew& a = b.f;
  a.T = (int)T; a.V = V; a.D = D; a.dp = (int)round_up(D, 8);
  const int64_t turns = up(V, kFewTile), most = std::max<int64_t>(1, 148 * 2 / std::max<int64_t>(groups, 1));      // (two blocks an SM by their registers)
  a.per = up(turns, std::min(most, turns)) * kFewTile;
  a.blocks = (int)up(V, a.per);
  b.lanes = 1;
  while (b.lanes * 8 < D) b.lanes *= 2;
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* q = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return q; };
  a.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  b.acc = reinterpret_cast<float*>(take(4 * (size_t)groups * a.blocks * T * a.dp));
  *bytes = off;
  return b;
}

// 16-bit values, box {64, box_y, box_z}, 128-byte swizzle; zeros beyond the edges
int vt_map(CUtensorMap* m, const void* base, int64_t dx, int64_t dy, int64_t dz, int64_t sy, int64_t sz, int box_y, int box_z) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode enc = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<Encode>(f) : nullptr;
  }();
  if (!enc) return op_fail(PRSGD_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[3] = {(cuuint64_t)dx, (cuuint64_t)dy, (cuuint64_t)dz}, strides[2] = {(cuuint64_t)sy * 2, (cuuint64_t)sz * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_y, (cuuint32_t)box_z}, one[3] = {1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? PRSGD_OK : op_fail(PRSGD_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
}

// SMs of the current device; the kernels' shared memory is raised on the first call on it.
int vocab_device(int* sms) {
  static std::mutex lock;
  static int known[64];
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= 64)) return op_fail(PRSGD_ERR_ARG, "device ordinal out of range");
  std::lock_guard<std::mutex> hold(lock);
  if (e == cudaSuccess && known[dev] == 0) {
    int n = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    auto raise = [&](auto kernel, bool grad) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)vt_smem(grad)); };
    raise(vocab_chain_kernel<false, false>, false); raise(vocab_chain_kernel<false, true>, false);
    raise(vocab_chain_kernel<true, false>, true); raise(vocab_chain_kernel<true, false, true>, true); raise(vocab_chain_kernel<true, true>, true);
    auto few = [&](auto ty, auto nt) {
      for (auto kernel : {vocab_few_kernel<decltype(ty)::value, true, decltype(nt)::value>, vocab_few_kernel<decltype(ty)::value, false, decltype(nt)::value>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
    };
    for (int t : {PRSGD_TYPE_FP32, PRSGD_TYPE_BF16, PRSGD_TYPE_FP16})
      with_type(t, [&](auto ty) { few(ty, std::integral_constant<int, 1>()); few(ty, std::integral_constant<int, 2>()); few(ty, std::integral_constant<int, 4>()); });
    if (e == cudaSuccess) known[dev] = n;
  }
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("vocab_loss: ") + cudaGetErrorString(e));
  *sms = known[dev];
  return PRSGD_OK;
}

// The passes before the products, and the products.
int vocab_run(VocabPlan& p, cudaStream_t st) {
  int sms = 0;
  int rc = vocab_device(&sms);
  if (rc != PRSGD_OK) return rc;
  VocabPrep& a = p.prep;
  VocabChain& c = p.chain;
  const int planes = p.split ? 2 : 1, D = a.D;
  const int64_t G = a.groups;
  c.w_shared = a.w_groups == 1;
  VocabMaps maps{};
  for (int i = 0; i < planes && rc == PRSGD_OK; ++i) {
    rc = vt_map(&maps.hk[i], a.Hc[i], D, a.Tp, G, a.pitch, a.Tp * a.pitch, 128, 1);
    if (rc == PRSGD_OK && p.grad) rc = vt_map(&maps.hm[i], a.Hm[i] ? a.Hm[i] : a.Hc[i], D, a.T, G, a.pitch, a.Tp * a.pitch, 64, 1);
    const int64_t row = p.copy_w ? a.pitch : a.w_row, group = a.w_groups == 1 ? row : p.copy_w ? a.V * a.pitch : a.w_group;
    c.w_swap = a.w_groups > 1 && group < row;
    for (int mn = 0; mn < (p.grad ? 2 : 1) && rc == PRSGD_OK; ++mn) {
      CUtensorMap* to = mn ? &maps.wm[i] : &maps.wk[i];
      const int box = mn ? 64 : 128;
      const void* w = !p.copy_w ? a.W : mn && a.Wm[i] ? a.Wm[i] : a.Wc[i];
      rc = c.w_swap ? vt_map(to, w, D, a.w_groups, a.V, group, row, 1, box) : vt_map(to, w, D, a.V, a.w_groups, row, group, box, 1);
    }
    if (!p.grad) continue;
    if (rc == PRSGD_OK) rc = vt_map(&maps.gk[i], c.G[i], c.gp, a.Tp, c.slots, c.gp, a.Tp * c.gp, 128, 1);
    if (rc == PRSGD_OK) rc = vt_map(&maps.gm[i], c.G[i], c.gp, a.T, c.slots, c.gp, a.Tp * c.gp, 64, 1);
  }
  if (rc != PRSGD_OK) return rc;
  // eight rows a block and turn, two rounds of blocks over all groups
  const int64_t most = std::max<int64_t>(1, 148 * 8 / G);
  a.h_blocks = (int)std::min<int64_t>(up(a.T, 8), most);
  a.w_blocks = p.copy_w ? (int)std::min<int64_t>(up(a.V, 8), most) : 0;
  if (p.split && p.grad) {
    const int64_t n = 2 * G * a.Dp;
    launch_pdl(vocab_zero_kernel, dim3((unsigned)std::min<int64_t>(up(n, 256), 148 * 8)), dim3(256), 0, st, a.most, n);
    // blocks of 64 rows or more, eight an SM over all groups and strips of 128 columns
    const int64_t strips = up(D, 128), share = std::max<int64_t>(1, 148 * 8 / (G * strips));
    a.most_rows = (int)round_up(std::max<int64_t>(64, up(a.T + a.V, share)), 32);
    a.most_h = a.Hm[0] ? (int)up(a.T, a.most_rows) : 0;
    a.most_w = a.Wm[0] ? (int)up(a.V, a.most_rows) : 0;
    launch_pdl(vocab_columns_kernel, dim3((unsigned)(a.most_h + a.most_w), (unsigned)strips, (unsigned)G), dim3(256), 0, st, a);
  }
  if (a.largest) launch_pdl(vocab_largest_kernel, dim3((unsigned)G), dim3(1024), 0, st, a);
  with_type(a.h_type, [&](auto ty) { launch_pdl(vocab_prep_kernel<decltype(ty)::value>, dim3((unsigned)(a.h_blocks + a.w_blocks), (unsigned)G), dim3(256), 0, st, a); });
  const dim3 grid(2 * (unsigned)std::min<int64_t>(sms / 2, p.tasks));
  auto go = [&](auto kernel) { launch_pdl_cluster(kernel, grid, dim3(kVtThreads), vt_smem(p.grad), st, 2, maps, c); };
  if (p.grad && p.split) go(vocab_chain_kernel<true, true>);
  else if (p.longest) go(vocab_chain_kernel<true, false, true>);
  else if (p.grad) go(vocab_chain_kernel<true, false>);
  else if (p.split) go(vocab_chain_kernel<false, true>);
  else go(vocab_chain_kernel<false, false>);
  return PRSGD_OK;
}

int check_inputs(const void* H, int64_t hr, int64_t hg, const void* W, int64_t wr, int64_t wg, int type, const int32_t* labels, int64_t G, int64_t T, int64_t V, int D) {
  int rc = check_rows("H", H, type, hr, hg, G, T, D, false);
  if (rc == PRSGD_OK) rc = check_rows("W", W, type, wr, wg, G, V, D, false);
  if (rc != PRSGD_OK) return rc;
  if (labels == nullptr) return op_fail(PRSGD_ERR_ARG, "labels is NULL");
  return PRSGD_OK;
}

int check_tasks(int64_t tasks) {
  return tasks < (1ll << 31) ? PRSGD_OK : op_fail(PRSGD_ERR_SIZE, "too many tiles in one call: take fewer tokens or classes");
}

int check_work(const void* work, size_t bytes, size_t need) {
  if (!work || bytes < need) return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than its *_workspace_bytes function says");
  if (((uintptr_t)work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  return PRSGD_OK;
}

void set_inputs(VocabPrep& a, const void* H, int64_t hr, int64_t hg, const void* W, int64_t wr, int64_t wg, int type, const int32_t* labels) {
  a.H = H; a.h_row = hr; a.h_group = hg; a.vec_h = rows_16(H, type, hr, hg);
  a.W = W; a.w_row = wr; a.w_group = wg; a.vec_w = rows_16(W, type, wr, wg);
  if (wg == 0) a.w_groups = 1;
  a.labels = labels;
}

int check_floats(const void* a, const void* b, const void* c, const void* d) {
  if (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) % 4)
    return op_fail(PRSGD_ERR_ALIGN, "labels, loss, stats, dloss and dlse must be 4-byte aligned");
  return PRSGD_OK;
}

// loss [n] and stats [2 n] are apart
int check_outputs(const float* loss, const float* stats, int64_t n) {
  const uintptr_t l = (uintptr_t)loss, s = (uintptr_t)stats;
  return l < s + 8 * (uintptr_t)n && s < l + 4 * (uintptr_t)n ? op_fail(PRSGD_ERR_ARG, "loss and stats overlap") : PRSGD_OK;
}

}  // namespace

extern "C" {

int prsgd_vocab_loss_workspace_bytes(int32_t type, int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, int32_t w_aligned, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  const int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (vocab_few(type == PRSGD_TYPE_FP32, groups, tokens, vocab, dim)) vocab_few_plan(groups, tokens, vocab, dim, nullptr, bytes);
  else *bytes = vocab_plan(type, groups, tokens, vocab, dim, w_aligned != 0, false, nullptr).bytes;
  return PRSGD_OK;
}

int prsgd_vocab_loss_grad_workspace_bytes(int32_t type, int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, int32_t w_aligned, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  const int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (vocab_few_grad(tokens, dim)) vocab_few_grad_plan(groups, tokens, vocab, dim, nullptr, bytes);
  else *bytes = vocab_plan(type, groups, tokens, vocab, dim, w_aligned != 0, true, nullptr).bytes;
  return PRSGD_OK;
}

int prsgd_vocab_loss(const void* d_H, int64_t h_row_stride, int64_t h_group_stride,
                     const void* d_W, int64_t w_row_stride, int64_t w_group_stride, int32_t type, const int32_t* d_labels,
                     int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, float* d_loss, float* d_stats,
                     void* d_work, size_t work_bytes, void* cuda_stream) {
  int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (groups == 0 || tokens == 0) return op_clear_status(d_work, work_bytes, cuda_stream);
  rc = check_inputs(d_H, h_row_stride, h_group_stride, d_W, w_row_stride, w_group_stride, type, d_labels, groups, tokens, vocab, dim);
  if (rc == PRSGD_OK) rc = check_floats(d_labels, d_loss, d_stats, nullptr);
  if (rc != PRSGD_OK) return rc;
  if (!d_loss || !d_stats) return op_fail(PRSGD_ERR_ARG, "an output is NULL");
  if (vocab_few(type == PRSGD_TYPE_FP32, groups, tokens, vocab, dim)) {
    size_t need = 0;
    VocabFew f = vocab_few_plan(groups, tokens, vocab, dim, static_cast<unsigned char*>(d_work), &need);
    rc = check_work(d_work, work_bytes, need);
    if (rc == PRSGD_OK) rc = check_outputs(d_loss, d_stats, groups * tokens);
    int sms = 0;
    if (rc == PRSGD_OK) rc = vocab_device(&sms);
    if (rc != PRSGD_OK) return rc;
    f.H = d_H; f.h_row = h_row_stride; f.h_group = h_group_stride; f.W = d_W; f.w_row = w_row_stride; f.w_group = w_group_stride;
    f.labels = d_labels; f.loss = d_loss; f.stats = d_stats;
    const bool vec = rows_16(d_W, type, w_row_stride, w_group_stride);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const dim3 grid((unsigned)(f.blocks * f.turns), (unsigned)groups);
    with_type(type, [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      auto go = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        const size_t smem = (size_t)NT * f.dp * 4;
        if (vec) launch_pdl(vocab_few_kernel<TY, true, NT>, grid, dim3(32 * kFewWarps), smem, st, f);
        else launch_pdl(vocab_few_kernel<TY, false, NT>, grid, dim3(32 * kFewWarps), smem, st, f);
      };
      if (tokens == 1) go(std::integral_constant<int, 1>());
      else if (tokens == 2) go(std::integral_constant<int, 2>());
      else go(std::integral_constant<int, 4>());
    });
    launch_pdl(vocab_few_join_kernel, dim3((unsigned)groups), dim3((unsigned)(32 * tokens)), 0, st, f);
    return op_launched("vocab_loss");
  }
  VocabPlan p = vocab_plan(type, groups, tokens, vocab, dim, rows_16(d_W, type, w_row_stride, w_group_stride), false, static_cast<unsigned char*>(d_work));
  rc = check_tasks(p.tasks);
  if (rc == PRSGD_OK) rc = check_work(d_work, work_bytes, p.bytes);
  if (rc == PRSGD_OK) rc = check_outputs(d_loss, d_stats, groups * tokens);
  if (rc != PRSGD_OK) return rc;
  VocabPrep& a = p.prep;
  set_inputs(a, d_H, h_row_stride, h_group_stride, d_W, w_row_stride, w_group_stride, type, d_labels);
  a.loss = d_loss; a.out_stats = d_stats;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  rc = vocab_run(p, st);
  if (rc != PRSGD_OK) return rc;
  VocabJoin j{};
  j.part = p.chain.part; j.zy = p.chain.zy; j.index = a.index; j.live = a.live; j.Tp = a.Tp; j.T = tokens; j.runs = p.chain.runs;
  j.loss = d_loss; j.stats = d_stats;
  if (tokens <= 8) launch_pdl(vocab_join_kernel<1>, dim3((unsigned)tokens, (unsigned)groups), dim3(256), 0, st, j);
  else if (groups * tokens <= 16384) launch_pdl(vocab_join_kernel<8>, dim3((unsigned)up(tokens, 8), (unsigned)groups), dim3(256), 0, st, j);
  else launch_pdl(vocab_join_kernel<32>, dim3((unsigned)up(tokens, 32), (unsigned)groups), dim3(256), 0, st, j);
  return op_launched("vocab_loss");
}

int prsgd_vocab_loss_grad(const void* d_H, int64_t h_row_stride, int64_t h_group_stride,
                          const void* d_W, int64_t w_row_stride, int64_t w_group_stride, int32_t type, const int32_t* d_labels,
                          int64_t groups, int64_t tokens, int64_t vocab, int32_t dim,
                          const float* d_stats, const float* d_dloss, const float* d_dlse,
                          void* d_dH, int64_t dh_row_stride, int64_t dh_group_stride,
                          void* d_dW, int32_t dw_type, int64_t dw_row_stride, int64_t dw_group_stride, int32_t accumulate,
                          void* d_work, size_t work_bytes, void* cuda_stream) {
  int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (d_dW && dw_type != type && dw_type != PRSGD_TYPE_FP32) return op_fail(PRSGD_ERR_ARG, "dW must be of W's type or fp32");
  if (groups == 0 || (tokens == 0 && (accumulate || !d_dW))) return op_clear_status(d_work, work_bytes, cuda_stream);
  if (d_dW) rc = check_rows("dW", d_dW, dw_type, dw_row_stride, dw_group_stride, groups, vocab, dim, true);
  if (rc == PRSGD_OK && tokens > 0) {
    rc = check_inputs(d_H, h_row_stride, h_group_stride, d_W, w_row_stride, w_group_stride, type, d_labels, groups, tokens, vocab, dim);
    if (rc == PRSGD_OK && d_dH) rc = check_rows("dH", d_dH, type, dh_row_stride, dh_group_stride, groups, tokens, dim, true);
    if (rc == PRSGD_OK) rc = check_floats(d_labels, d_stats, d_dloss, d_dlse);
    if (rc == PRSGD_OK && !d_stats) rc = op_fail(PRSGD_ERR_ARG, "stats is NULL");
    if (rc == PRSGD_OK && ((d_dH && (d_dH == d_H || d_dH == d_W || d_dH == d_dW)) || (d_dW && (d_dW == d_W || d_dW == d_H))))
      rc = op_fail(PRSGD_ERR_ARG, "dH or dW is another array's memory");
  }
  if (rc != PRSGD_OK) return rc;
  if (tokens == 0) {                                     // no term in any sum
    const size_t size = (size_t)type_bytes(dw_type);
    cudaError_t e = cudaSuccess;
    for (int64_t g = 0; g < groups && e == cudaSuccess; ++g)
      e = cudaMemset2DAsync(static_cast<char*>(d_dW) + g * dw_group_stride * size, dw_row_stride * size, 0, dim * size, vocab, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("vocab_loss_grad: ") + cudaGetErrorString(e));
    return op_clear_status(d_work, work_bytes, cuda_stream);
  }
  if (!d_dH && !d_dW) return op_clear_status(d_work, work_bytes, cuda_stream);
  if (vocab_few_grad(tokens, dim)) {
    size_t need = 0;
    VocabFewGrad f = vocab_few_grad_plan(groups, tokens, vocab, dim, static_cast<unsigned char*>(d_work), &need);
    rc = check_work(d_work, work_bytes, need);
    if (rc != PRSGD_OK) return rc;
    f.f.H = d_H; f.f.h_row = h_row_stride; f.f.h_group = h_group_stride; f.f.W = d_W; f.f.w_row = w_row_stride; f.f.w_group = w_group_stride;
    f.f.labels = d_labels;
    f.in_stats = d_stats; f.dloss = d_dloss; f.dlse = d_dlse;
    f.dW = d_dW; f.dw_row = dw_row_stride; f.dw_group = dw_group_stride; f.accumulate = accumulate != 0;
    f.dH = d_dH; f.dh_row = dh_row_stride; f.dh_group = dh_group_stride;
    if (!d_dH) f.acc = nullptr;
    const bool vec = dim % 8 == 0 && rows_16(d_W, type, w_row_stride, w_group_stride) && (!d_dW || rows_16(d_dW, dw_type, dw_row_stride, dw_group_stride));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const dim3 grid((unsigned)f.f.blocks, (unsigned)groups);
    // H, or at the end the sums of the threads that share columns: 256 / lanes of them, 2048 columns in all at most
    const size_t smem = (size_t)tokens * f.f.dp * 4 * (32 * kFewWarps / f.lanes);
    with_type(type, [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      auto go = [&](auto oty, auto v, auto nt) { launch_pdl(vocab_few_grad_kernel<TY, decltype(oty)::value, decltype(v)::value, decltype(nt)::value>, grid, dim3(32 * kFewWarps), smem, st, f); };
      auto typed = [&](auto oty) {
        auto both = [&](auto v) {
          if (tokens == 1) go(oty, v, std::integral_constant<int, 1>());
          else go(oty, v, std::integral_constant<int, 2>());
        };
        if (vec) both(std::integral_constant<bool, true>());
        else both(std::integral_constant<bool, false>());
      };
      if (!d_dW || dw_type == type) typed(ty);
      else typed(std::integral_constant<int, PRSGD_TYPE_FP32>());
      if (d_dH) launch_pdl(vocab_few_sum_kernel<TY>, dim3((unsigned)up(dim, 32), (unsigned)tokens, (unsigned)groups), dim3(256), 0, st, f);
    });
    return op_launched("vocab_loss_grad");
  }
  VocabPlan p = vocab_plan(type, groups, tokens, vocab, dim, rows_16(d_W, type, w_row_stride, w_group_stride), true, static_cast<unsigned char*>(d_work));
  rc = check_tasks(p.tasks);
  if (rc == PRSGD_OK) rc = check_work(d_work, work_bytes, p.bytes);
  if (rc != PRSGD_OK) return rc;
  VocabPrep& a = p.prep;
  VocabChain& c = p.chain;
  set_inputs(a, d_H, h_row_stride, h_group_stride, d_W, w_row_stride, w_group_stride, type, d_labels);
  a.stats = d_stats; a.dloss = d_dloss; a.dlse = d_dlse;
  if (!d_dH) a.Wm[0] = a.Wm[1] = nullptr;
  if (!d_dW) a.Hm[0] = a.Hm[1] = nullptr;
  a.dH = d_dH; a.dh_row = dh_row_stride; a.dh_group = dh_group_stride; a.vec_dh = d_dH && rows_16(d_dH, type, dh_row_stride, dh_group_stride);
  c.dH = d_dH; c.dh_row = dh_row_stride; c.dh_group = dh_group_stride; c.dh_type = type; c.vec_dh = a.vec_dh;
  c.dW = d_dW; c.dw_row = dw_row_stride; c.dw_group = dw_group_stride; c.dw_type = dw_type; c.accumulate = accumulate != 0;
  c.vec_dw = d_dW && rows_16(d_dW, dw_type, dw_row_stride, dw_group_stride);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  rc = vocab_run(p, st);
  if (rc != PRSGD_OK) return rc;
  if (d_dH && c.acc) {
    VocabSum s{};
    s.acc = c.acc; s.index = a.index; s.live = a.live; s.Tp = a.Tp; s.groups = groups; s.parts = c.parts; s.acc_pitch = c.acc_pitch; s.D = dim;
    s.dH = d_dH; s.dh_row = dh_row_stride; s.dh_group = dh_group_stride;
    // eight rows a block, or, where they are few and their parts many, one whose parts the warps share
    const bool shared = c.parts >= 8 && groups * tokens <= 1024;
    const dim3 grid((unsigned)std::min<int64_t>(shared ? tokens : up(tokens, 8), 65536), (unsigned)up(dim, 256), (unsigned)groups);
    with_type(type, [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      auto go = [&](auto kernel) { launch_pdl(kernel, grid, dim3(256), 0, st, s); };
      if (shared) { if (a.vec_dh) go(vocab_sum_kernel<TY, true, true>); else go(vocab_sum_kernel<TY, false, true>); }
      else if (a.vec_dh) go(vocab_sum_kernel<TY, true, false>);
      else go(vocab_sum_kernel<TY, false, false>);
    });
  }
  return op_launched("vocab_loss_grad");
}

}  // extern "C"
