// C entries of the token embedding and its gradient.  See include/prsgd.h for the contract.
#include <cmath>
#include <mutex>
#include "kernels_embed.cuh"

using namespace prsgd;

namespace {

int check_tokens(const int32_t* ids, int64_t groups, int64_t tokens, int64_t vocab, int dim) {
  if (groups < 0 || tokens < 0 || vocab < 1 || dim < 0) return op_fail(PRSGD_ERR_ARG, "need groups >= 0, tokens >= 0, vocab >= 1, dim >= 0");
  if (groups > 65535 || tokens > (1ll << 24) || vocab > PRSGD_VOCAB_MAX || dim > 65536)
    return op_fail(PRSGD_ERR_SIZE, "more than 65535 groups, 2^24 tokens, PRSGD_VOCAB_MAX ids or 65536 columns");
  if (groups > 0 && tokens > 0 && dim > 0) {
    if (ids == nullptr) return op_fail(PRSGD_ERR_ARG, "ids is NULL");
    if (((uintptr_t)ids) % 4) return op_fail(PRSGD_ERR_ALIGN, "ids must be 4-byte aligned");
  }
  return PRSGD_OK;
}

// Sorted tokens of a unit, at whose borders a run's sum is cut: by the number of tokens alone, so that a group's sums have the same bits whatever
// other groups are in the call.  Few of them, so that short calls have many units (2 x 500 x 100: 8 22 us, 16 28, 32 37 with cold caches; 32 x 512 x 256 28, 30, 38);
// more, so that long ones have few parts to join (1 x 8192 x 2048 back to back: 8 40 us, 16 35, 32 33; 4 x 8192 x 2048 108, 97, 92; 16 x 16384 x 64 84, 71, 72).
int embed_unit(int64_t tokens) { return (int)std::max<int64_t>(8, std::min<int64_t>(32, tokens / 256 / 8 * 8)); }

EmbedGradArgs embed_grad_carve(int64_t groups, int64_t tokens, int64_t vocab, int dim, unsigned char* base, size_t* bytes) {
  EmbedGradArgs a{};
  a.groups = groups; a.tokens = tokens; a.vocab = vocab; a.dim = dim;
  a.chunks = (dim + 7) / 8;
  a.lanes = std::min(a.chunks, kRowThreads);
  int bits = 1;
  while ((1ll << bits) < vocab) ++bits;
  a.passes = (bits + kSortBits - 1) / kSortBits;
  a.bits = (bits + a.passes - 1) / a.passes;
  // as many blocks as have a turn each, so that up to 8192 tokens take one
  a.ctas = 1;
  while (a.ctas < kSortCtas && a.ctas * kSortTurn < tokens) a.ctas *= 2;
  a.turns = (int)std::max<int64_t>(1, (tokens + a.ctas * kSortTurn - 1) / (a.ctas * kSortTurn));
  a.unit = embed_unit(tokens);
  a.units = (int)((tokens + a.unit - 1) / a.unit);
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* p = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return p; };
  a.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  a.live = reinterpret_cast<int*>(take(4 * (size_t)groups));
  for (int i = 0; i < 2; ++i) a.keys[i] = reinterpret_cast<uint2*>(take(8 * (size_t)groups * tokens));
  a.parts = reinterpret_cast<float*>(take((size_t)groups * a.units * 2 * a.chunks * 32));
  *bytes = off;
  return a;
}

// The sorting kernels' shared memory, raised on the first call on a device.
int embed_prepare() {
  static std::mutex lock;
  static bool known[64];
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= 64)) return op_fail(PRSGD_ERR_ARG, "device ordinal out of range");
  std::lock_guard<std::mutex> hold(lock);
  if (e == cudaSuccess && !known[dev]) {
    auto raise = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSortSmem); };
    raise(embed_sort_kernel<PRSGD_TYPE_FP32, true>); raise(embed_sort_kernel<PRSGD_TYPE_BF16, true>); raise(embed_sort_kernel<PRSGD_TYPE_FP16, true>);
    raise(embed_sort_kernel<PRSGD_TYPE_FP32, false>); raise(embed_sort_kernel<PRSGD_TYPE_BF16, false>); raise(embed_sort_kernel<PRSGD_TYPE_FP16, false>);
    known[dev] = e == cudaSuccess;
  }
  return e == cudaSuccess ? PRSGD_OK : op_fail(PRSGD_ERR_CUDA, std::string("embed_grad: ") + cudaGetErrorString(e));
}

}  // namespace

extern "C" {

int prsgd_embed(const void* d_table, int32_t type, int64_t row_stride, int64_t group_stride, const int32_t* d_ids,
                int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, float scale,
                void* d_out, int32_t out_type, int64_t out_row_stride, int64_t out_group_stride, void* cuda_stream) {
  int rc = check_tokens(d_ids, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (!type_known(type) || !type_known(out_type)) return op_fail(PRSGD_ERR_ARG, "unknown element type");
  if (!std::isfinite(scale)) return op_fail(PRSGD_ERR_ARG, "scale must be finite");
  if (groups == 0 || tokens == 0 || dim == 0) return PRSGD_OK;
  rc = check_rows("table", d_table, type, row_stride, group_stride, groups, vocab, dim, false);
  if (rc == PRSGD_OK) rc = check_rows("out", d_out, out_type, out_row_stride, out_group_stride, groups, tokens, dim, true);
  if (rc != PRSGD_OK) return rc;
  if (d_out == d_table) return op_fail(PRSGD_ERR_ARG, "out and table are the same memory");
  EmbedArgs a{};
  a.walk = row_walk(tokens, dim);
  a.table = d_table; a.row = row_stride; a.group = group_stride; a.ids = d_ids;
  a.out = d_out; a.out_row = out_row_stride; a.out_group = out_group_stride;
  a.tokens = tokens; a.vocab = vocab; a.scale = scale;
  const dim3 grid((unsigned)((a.walk.items + kRowItems - 1) / kRowItems), (unsigned)groups);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool whole = dim % 8 == 0 && rows_16(d_table, type, row_stride, group_stride) && rows_16(d_out, out_type, out_row_stride, out_group_stride);
  with_type(type, [&](auto ty) {
    with_type(out_type, [&](auto oty) {
      if (whole) launch_pdl(embed_kernel<decltype(ty)::value, decltype(oty)::value>, grid, dim3(kRowThreads), 0, st, a);
      else launch_pdl(embed_any_kernel<decltype(ty)::value, decltype(oty)::value>, grid, dim3(kRowThreads), 0, st, a);
    });
  });
  return op_launched("embed");
}

int prsgd_embed_grad_workspace_bytes(int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  static const int32_t none = 0;
  const int rc = check_tokens(&none, groups, tokens, vocab, dim);
  if (rc == PRSGD_OK) embed_grad_carve(groups, tokens, vocab, dim, nullptr, bytes);
  return rc;
}

int prsgd_embed_grad(const void* d_dout, int32_t type, int64_t row_stride, int64_t group_stride, const int32_t* d_ids,
                     int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, float scale,
                     void* d_dtable, int32_t dtable_type, int64_t dtable_row_stride, int64_t dtable_group_stride, int32_t accumulate,
                     void* d_work, size_t work_bytes, void* cuda_stream) {
  int rc = check_tokens(d_ids, groups, tokens, vocab, dim);
  if (rc != PRSGD_OK) return rc;
  if (!type_known(type) || !type_known(dtable_type)) return op_fail(PRSGD_ERR_ARG, "unknown element type");
  if (!std::isfinite(scale)) return op_fail(PRSGD_ERR_ARG, "scale must be finite");
  if (groups == 0 || dim == 0 || (tokens == 0 && accumulate)) return op_clear_status(d_work, work_bytes, cuda_stream);
  if (tokens > 0) rc = check_rows("dout", d_dout, type, row_stride, group_stride, groups, tokens, dim, false);
  if (rc == PRSGD_OK) rc = check_rows("dtable", d_dtable, dtable_type, dtable_row_stride, dtable_group_stride, groups, vocab, dim, true);
  if (rc != PRSGD_OK) return rc;
  if (d_dout == d_dtable) return op_fail(PRSGD_ERR_ARG, "dtable and dout are the same memory");
  size_t need = 0;
  EmbedGradArgs a = embed_grad_carve(groups, tokens, vocab, dim, static_cast<unsigned char*>(d_work), &need);
  if (!d_work || work_bytes < need) return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than prsgd_embed_grad_workspace_bytes");
  if (((uintptr_t)d_work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  rc = embed_prepare();
  if (rc != PRSGD_OK) return rc;
  a.dout = d_dout; a.row = row_stride; a.group = group_stride; a.ids = d_ids;
  a.dtable = d_dtable; a.t_row = dtable_row_stride; a.t_group = dtable_group_stride;
  a.scale = scale; a.accumulate = accumulate != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool vec = rows_16(d_dout, type, row_stride, group_stride), ovec = rows_16(d_dtable, dtable_type, dtable_row_stride, dtable_group_stride);
  // blocks that write zeros: about 64 KB each
  const int64_t zero_rows = accumulate ? 0 : groups * vocab;
  const int64_t zeros = zero_rows == 0 ? 0 : std::max<int64_t>(1, std::min<int64_t>(zero_rows * dim / 16384, 148 * 16));
  with_type(dtable_type, [&](auto oty) {
    constexpr int OTY = decltype(oty)::value;
    auto both = [&](auto ov) {
      constexpr bool OV = decltype(ov)::value;
      const unsigned grid = (unsigned)((groups * a.ctas + zeros + a.ctas - 1) / a.ctas * a.ctas);
      launch_pdl_cluster(embed_sort_kernel<OTY, OV>, dim3(grid), dim3(1024), kSortSmem, st, (unsigned)a.ctas, a);
      if (tokens == 0) return;
      // threads of a block: whole rows of lanes, fewer of them while that gives the GPU more blocks
      int threads = kRowThreads;
      while (threads > 64 && threads / 2 >= a.lanes && groups * a.units * a.lanes / threads < 148 * 4) threads /= 2;
      const int per = threads / a.lanes;
      const dim3 sum_grid((unsigned)((a.units + per - 1) / per), (unsigned)((a.chunks + a.lanes - 1) / a.lanes), (unsigned)groups);
      with_type(type, [&](auto ty) {
        if (vec) launch_pdl(embed_sum_kernel<decltype(ty)::value, OTY, true, OV>, sum_grid, dim3(threads), 0, st, a);
        else launch_pdl(embed_sum_kernel<decltype(ty)::value, OTY, false, OV>, sum_grid, dim3(threads), 0, st, a);
      });
      if (a.units > 1) launch_pdl(embed_join_kernel<OTY, OV>, sum_grid, dim3(threads), 0, st, a);
    };
    if (ovec) both(std::integral_constant<bool, true>());
    else both(std::integral_constant<bool, false>());
  });
  return op_launched("embed_grad");
}

}  // extern "C"
