// C entries of the cross entropy over a vocabulary.  See include/prsgd.h for the contract.
#include "kernels_vocab.cuh"

using namespace prsgd;

namespace {

int check_vocab(int type, int64_t groups, int64_t tokens, int64_t vocab, int dim) {
  if (!type_known(type)) return op_fail(PRSGD_ERR_ARG, "unknown element type");
  if (groups < 0 || tokens < 0 || vocab < 1 || dim < 1) return op_fail(PRSGD_ERR_ARG, "need groups >= 0, tokens >= 0, vocab >= 1, dim >= 1");
  if (groups > 4096 || tokens > (1ll << 22) || vocab > PRSGD_VOCAB_MAX || dim > 65536)
    return op_fail(PRSGD_ERR_SIZE, "more than 4096 groups, 2^22 tokens, PRSGD_VOCAB_MAX classes or 65536 columns");
  return PRSGD_OK;
}

VocabArgs vocab_carve(int64_t groups, int64_t tokens, int64_t vocab, int dim, bool grad, unsigned char* base, size_t* bytes) {
  VocabArgs a{};
  a.T = tokens; a.V = vocab; a.D = dim;
  a.runs = (int)((vocab + kVocabRun * kVocabTile - 1) / (kVocabRun * kVocabTile));
  a.piece = std::min<int64_t>(vocab, 8192);
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* p = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return p; };
  a.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  if (grad) {
    a.G = reinterpret_cast<float*>(take(4 * (size_t)groups * tokens * a.piece));
    a.acc = reinterpret_cast<float*>(take(4 * (size_t)groups * tokens * dim));
  } else {
    a.part = reinterpret_cast<float2*>(take(8 * (size_t)groups * tokens * a.runs));
    a.zy = reinterpret_cast<float*>(take(4 * (size_t)groups * tokens));
  }
  *bytes = off;
  return a;
}

int check_inputs(const void* H, int64_t hr, int64_t hg, const void* W, int64_t wr, int64_t wg, int type, const int32_t* labels, int64_t G, int64_t T, int64_t V, int D) {
  int rc = check_rows("H", H, type, hr, hg, G, T, D, false);
  if (rc == PRSGD_OK) rc = check_rows("W", W, type, wr, wg, G, V, D, false);
  if (rc != PRSGD_OK) return rc;
  if (labels == nullptr) return op_fail(PRSGD_ERR_ARG, "labels is NULL");
  return PRSGD_OK;
}

int check_floats(const void* a, const void* b, const void* c, const void* d) {
  if (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) % 4)
    return op_fail(PRSGD_ERR_ALIGN, "labels, loss, stats, dloss and dlse must be 4-byte aligned");
  return PRSGD_OK;
}

}  // namespace

extern "C" {

int prsgd_vocab_loss_workspace_bytes(int32_t type, int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, int32_t w_aligned, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  const int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc == PRSGD_OK) vocab_carve(groups, tokens, vocab, dim, false, nullptr, bytes);
  return rc;
}

int prsgd_vocab_loss_grad_workspace_bytes(int32_t type, int64_t groups, int64_t tokens, int64_t vocab, int32_t dim, int32_t w_aligned, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  const int rc = check_vocab(type, groups, tokens, vocab, dim);
  if (rc == PRSGD_OK) vocab_carve(groups, tokens, vocab, dim, true, nullptr, bytes);
  return rc;
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
  size_t need = 0;
  VocabArgs a = vocab_carve(groups, tokens, vocab, dim, false, static_cast<unsigned char*>(d_work), &need);
  if (!d_work || work_bytes < need) return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than prsgd_vocab_loss_workspace_bytes");
  if (((uintptr_t)d_work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  a.H = d_H; a.h_row = h_row_stride; a.h_group = h_group_stride; a.W = d_W; a.w_row = w_row_stride; a.w_group = w_group_stride;
  a.labels = d_labels; a.loss = d_loss; a.stats = d_stats;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const dim3 grid((unsigned)((tokens + kVocabTile - 1) / kVocabTile), (unsigned)a.runs, (unsigned)groups);
  with_type(type, [&](auto ty) { launch_pdl(vocab_stats_kernel<decltype(ty)::value>, grid, dim3(256), 0, st, a); });
  launch_pdl(vocab_join_kernel, dim3((unsigned)((tokens + 255) / 256), (unsigned)groups), dim3(256), 0, st, a);
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
  size_t need = 0;
  VocabArgs a = vocab_carve(groups, tokens, vocab, dim, true, static_cast<unsigned char*>(d_work), &need);
  if (!d_work || work_bytes < need) return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than prsgd_vocab_loss_grad_workspace_bytes");
  if (((uintptr_t)d_work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  a.H = d_H; a.h_row = h_row_stride; a.h_group = h_group_stride; a.W = d_W; a.w_row = w_row_stride; a.w_group = w_group_stride;
  a.labels = d_labels; a.in_stats = d_stats; a.dloss = d_dloss; a.dlse = d_dlse;
  a.dH = d_dH; a.dh_row = dh_row_stride; a.dh_group = dh_group_stride;
  a.dW = d_dW; a.dw_row = dw_row_stride; a.dw_group = dw_group_stride; a.accumulate = accumulate != 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  rc = op_clear_status(d_work, work_bytes, cuda_stream);
  if (rc != PRSGD_OK) return rc;
  const unsigned tt = (unsigned)((tokens + kVocabTile - 1) / kVocabTile), dt = (unsigned)((dim + kVocabTile - 1) / kVocabTile), G = (unsigned)groups;
  with_type(type, [&](auto ty) {
    constexpr int TY = decltype(ty)::value;
    for (a.v0 = 0; a.v0 < vocab; a.v0 += a.piece) {
      a.pv = std::min(a.piece, vocab - a.v0);
      const unsigned vt = (unsigned)((a.pv + kVocabTile - 1) / kVocabTile);
      if (tt > 0) launch_pdl(vocab_g_kernel<TY>, dim3(tt, vt, G), dim3(256), 0, st, a);
      if (d_dH && tt > 0) launch_pdl(vocab_dh_kernel<TY>, dim3(tt, dt, G), dim3(256), 0, st, a);
      if (!d_dW) continue;
      if (dw_type == TY) launch_pdl(vocab_dw_kernel<TY, TY>, dim3(vt, dt, G), dim3(256), 0, st, a);
      else launch_pdl(vocab_dw_kernel<TY, PRSGD_TYPE_FP32>, dim3(vt, dt, G), dim3(256), 0, st, a);
    }
  });
  return op_launched("vocab_loss_grad");
}

}  // extern "C"
