// C entries of the top-k router (prsgd_route, prsgd_route_grad).  See include/prsgd.h for the contract.
#include <initializer_list>
#include "kernels_route.cuh"

using namespace prsgd;

namespace {

// Blocks of a group: its tokens are dealt out in turns of `per_block` to no more blocks than the GPU holds at a time (two
// an SM by the kernels' launch bounds), so that there is no second, partly filled round of them.
int route_blocks(int64_t G, int64_t T, int per_block) {
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kRouteBlocks, 148 * 2 / G));
  return (int)std::min<int64_t>((T + per_block - 1) / per_block, most);
}
int lanes_per_token(int E) { return E <= 8 ? 1 : E <= 16 ? 2 : E <= 128 ? 4 : E <= 256 ? 8 : E <= 512 ? 16 : 32; }

int check_route(const void* logits, int type, int64_t row_stride, int64_t group_stride, int64_t G, int64_t T, int E, int k) {
  if (!type_known(type)) return op_fail(PRSGD_ERR_ARG, "unknown element type of the logits");
  if (G < 0 || T < 0 || E < 1 || k < 1) return op_fail(PRSGD_ERR_ARG, "need groups >= 0, tokens >= 0, experts >= 1, top_k >= 1");
  if (E > kRouteMaxExperts) return op_fail(PRSGD_ERR_SIZE, "more than PRSGD_ROUTE_MAX_EXPERTS experts");
  if (k > E || k > kRouteMaxK) return op_fail(PRSGD_ERR_ARG, "top_k exceeds the experts or PRSGD_ROUTE_MAX_K");
  if (G > 65535) return op_fail(PRSGD_ERR_SIZE, "more than 65535 groups");
  if (T > (1ll << 31) / k - 1 || T > (1ll << 24)) return op_fail(PRSGD_ERR_SIZE, "more than 2^24 tokens in a group");
  if (G > 0 && T > 0 && logits == nullptr) return op_fail(PRSGD_ERR_ARG, "logits is NULL");
  if (row_stride < E || group_stride < 0) return op_fail(PRSGD_ERR_ARG, "need row_stride >= experts, group_stride >= 0");
  if (((uintptr_t)logits) % type_bytes(type)) return op_fail(PRSGD_ERR_ALIGN, "logits is not aligned to its element type");
  return PRSGD_OK;
}

// The arrays of 32-bit words are read and written as such.
int check_words(std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (((uintptr_t)p) % 4) return op_fail(PRSGD_ERR_ALIGN, "experts, weights, counts, mean and loss, and the gradients of weights and loss, must be 4-byte aligned");
  return PRSGD_OK;
}

template <typename F> void with_per(int E, F&& f) {
  if (E <= 32) f(std::integral_constant<int, 1>());
  else if (E <= 64) f(std::integral_constant<int, 2>());
  else if (E <= 128) f(std::integral_constant<int, 4>());
  else if (E <= 256) f(std::integral_constant<int, 8>());
  else if (E <= 512) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
}

// f(elements per lane, lanes per token): PER * L >= E
template <typename F> void with_lanes(int E, F&& f) {
  using std::integral_constant;
  if (E <= 8) f(integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (E <= 16) f(integral_constant<int, 8>(), integral_constant<int, 2>());
  else if (E <= 32) f(integral_constant<int, 8>(), integral_constant<int, 4>());
  else if (E <= 64) f(integral_constant<int, 16>(), integral_constant<int, 4>());
  else if (E <= 128) f(integral_constant<int, 32>(), integral_constant<int, 4>());
  else if (E <= 256) f(integral_constant<int, 32>(), integral_constant<int, 8>());
  else if (E <= 512) f(integral_constant<int, 32>(), integral_constant<int, 16>());
  else f(integral_constant<int, 32>(), integral_constant<int, 32>());
}

// The gradient keeps half as many elements a lane where a row is long: it needs registers for more than the row.
template <typename F> void with_grad_lanes(int E, F&& f) {
  using std::integral_constant;
  if (E <= 64) with_lanes(E, f);
  else if (E <= 128) f(integral_constant<int, 16>(), integral_constant<int, 8>());
  else if (E <= 256) f(integral_constant<int, 16>(), integral_constant<int, 16>());
  else if (E <= 512) f(integral_constant<int, 16>(), integral_constant<int, 32>());
  else f(integral_constant<int, 32>(), integral_constant<int, 32>());
}
int grad_lanes_per_token(int E) { return E <= 64 ? lanes_per_token(E) : E <= 128 ? 8 : E <= 256 ? 16 : 32; }

int rows_vectorise(const void* p, int type, int64_t row_stride, int64_t group_stride, int E) {
  const int v = 16 / type_bytes(type);
  return (uintptr_t)p % 16 == 0 && row_stride % v == 0 && group_stride % v == 0 && E % v == 0;
}

}  // namespace

extern "C" {

int prsgd_route_workspace_bytes(int64_t groups, int64_t tokens, int32_t experts, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  if (groups < 0 || tokens < 0 || experts < 1 || experts > kRouteMaxExperts)
    return op_fail(PRSGD_ERR_ARG, "need groups >= 0, tokens >= 0, experts in 1..PRSGD_ROUTE_MAX_EXPERTS");
  const size_t slots = (size_t)groups * (size_t)std::max<int64_t>(1, std::min<int64_t>(kRouteBlocks, (tokens + 7) / 8));
  *bytes = 256 + slots * ((size_t)experts * 8 + 4) + 256;
  return PRSGD_OK;
}

int prsgd_route(const void* d_logits, int32_t type, int64_t row_stride, int64_t group_stride, const uint8_t* d_live,
                int64_t groups, int64_t tokens, int32_t experts, int32_t top_k, int32_t normalize, float coef,
                int32_t* d_experts, float* d_weights, int32_t* d_counts, float* d_mean, float* d_loss,
                void* d_work, size_t work_bytes, void* cuda_stream) {
  int rc = check_route(d_logits, type, row_stride, group_stride, groups, tokens, experts, top_k);
  if (rc != PRSGD_OK) return rc;
  if (groups == 0) return op_clear_status(d_work, work_bytes, cuda_stream);
  if (!d_counts || !d_mean || !d_loss || (tokens > 0 && (!d_experts || !d_weights))) return op_fail(PRSGD_ERR_ARG, "an output is NULL");
  rc = check_words({d_experts, d_weights, d_counts, d_mean, d_loss});
  if (rc != PRSGD_OK) return rc;
  size_t need = 0;
  prsgd_route_workspace_bytes(groups, tokens, experts, &need);
  if (!d_work || work_bytes < need) return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than prsgd_route_workspace_bytes");
  if (((uintptr_t)d_work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  RouteArgs a{};
  a.logits = d_logits; a.row_stride = row_stride; a.group_stride = group_stride; a.live = d_live;
  a.G = groups; a.T = tokens; a.E = experts; a.k = top_k; a.normalize = normalize != 0; a.coef = coef;
  a.experts = d_experts; a.weights = d_weights; a.counts = d_counts; a.mean = d_mean; a.loss = d_loss;
  const bool lanes = top_k <= 8;
  a.blocks = route_blocks(groups, tokens, lanes ? 8 * 32 / lanes_per_token(experts) : 8);
  a.vec = rows_vectorise(d_logits, type, row_stride, group_stride, experts);
  // A group of few tokens is one cluster that finishes itself, without a second launch: up to two turns of tokens a block, while
  // all blocks run at a time (us: 16 x 500 x 128 11.6 -> 9.9, 140 x 128 x 64 11.0 -> 8.9, 16 x 256 x 512 28 -> 22; but with
  // 512 blocks, 64 x 1024 x 64, 12 -> 14, and with four turns, 16 x 2048 x 128, 15.8 -> 17.0).
  const int64_t turn = 8 * 32 / lanes_per_token(experts);
  const int64_t cluster = std::min<int64_t>((tokens + turn - 1) / turn, kRouteCluster);
  if (lanes && cluster > 1 && tokens <= 2 * kRouteCluster * turn && groups * cluster <= 148 * 2) {
    a.clustered = 1;
    a.blocks = (int)cluster;
  }
  a.status = static_cast<DeviceStatus*>(d_work);
  unsigned char* w = static_cast<unsigned char*>(d_work) + 256;
  a.part_p = reinterpret_cast<float*>(w);
  a.part_c = reinterpret_cast<int32_t*>(a.part_p + (size_t)groups * a.blocks * experts);
  a.part_n = a.part_c + (size_t)groups * a.blocks * experts;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (a.blocks > 0) {
    const dim3 grid((unsigned)a.blocks, (unsigned)groups);
    with_type(type, [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      if (!lanes) {
        with_per(experts, [&](auto per) { launch_pdl(route_kernel<TY, decltype(per)::value>, grid, dim3(256), 0, st, a); });
      } else {
        with_lanes(experts, [&](auto per, auto l) {
          constexpr int PER = decltype(per)::value, L = decltype(l)::value;
          auto go = [&](auto kernel) {
            if (a.clustered) launch_pdl_cluster(kernel, grid, dim3(256), 0, st, (unsigned)a.blocks, a);
            else launch_pdl(kernel, grid, dim3(256), 0, st, a);
          };
          if (top_k <= 4) go(route_lanes_kernel<TY, PER, L, 4>);
          else go(route_lanes_kernel<TY, PER, L, 8>);
        });
      }
    });
  }
  if (a.blocks != 1 && !a.clustered) {                   // (a single block finishes itself)
    const unsigned parts = (unsigned)route_finish_blocks(experts);
    launch_pdl_cluster(route_finish_kernel, dim3(parts, (unsigned)groups), dim3(256), 0, st, parts, a);
  }
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("route: ") + cudaGetErrorString(e));
  return PRSGD_OK;
}

int prsgd_route_grad(const void* d_logits, int32_t type, int64_t row_stride, int64_t group_stride, const uint8_t* d_live,
                     int64_t groups, int64_t tokens, int32_t experts, int32_t top_k, int32_t normalize, float coef,
                     const int32_t* d_experts, const int32_t* d_counts, const float* d_dweights, const float* d_dloss,
                     void* d_dlogits, int64_t d_row_stride, int64_t d_group_stride, void* cuda_stream) {
  int rc = check_route(d_logits, type, row_stride, group_stride, groups, tokens, experts, top_k);
  if (rc != PRSGD_OK) return rc;
  if (groups == 0 || tokens == 0) return PRSGD_OK;
  if (!d_counts || !d_dlogits || (d_dweights && !d_experts)) return op_fail(PRSGD_ERR_ARG, "counts, dlogits or experts is NULL");
  rc = check_words({d_experts, d_counts, d_dweights, d_dloss});
  if (rc != PRSGD_OK) return rc;
  if (d_row_stride < experts || d_group_stride < 0 || !rows_apart(groups, d_group_stride, tokens, d_row_stride, experts))
    return op_fail(PRSGD_ERR_ARG, "the rows of dlogits overlap");
  if (d_dlogits == d_logits && !same_layout(groups, group_stride, d_group_stride, tokens, row_stride, d_row_stride))
    return op_fail(PRSGD_ERR_ARG, "dlogits are the logits' memory with other strides");
  if (((uintptr_t)d_dlogits) % type_bytes(type)) return op_fail(PRSGD_ERR_ALIGN, "dlogits is not aligned to its element type");
  RouteArgs a{};
  a.logits = d_logits; a.row_stride = row_stride; a.group_stride = group_stride; a.live = d_live;
  a.G = groups; a.T = tokens; a.E = experts; a.k = top_k; a.normalize = normalize != 0; a.coef = coef;
  a.experts = const_cast<int32_t*>(d_experts); a.counts = const_cast<int32_t*>(d_counts);
  a.dweights = d_dweights; a.dloss = d_dloss; a.dlogits = d_dlogits; a.d_row_stride = d_row_stride; a.d_group_stride = d_group_stride;
  a.vec = rows_vectorise(d_logits, type, row_stride, group_stride, experts);
  a.vec_out = rows_vectorise(d_dlogits, type, d_row_stride, d_group_stride, experts);
  const int64_t per_block = 8 * 32 / grad_lanes_per_token(experts);
  const int64_t resident = 148 * (experts <= 512 ? route_grad_blocks(16) : route_grad_blocks(32));
  const int64_t blocks = std::min<int64_t>((tokens + per_block - 1) / per_block, std::max<int64_t>(1, resident / groups));
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  with_type(type, [&](auto ty) {
    with_grad_lanes(experts, [&](auto per, auto l) {
      constexpr int TY = decltype(ty)::value, PER = decltype(per)::value, L = decltype(l)::value;
      const dim3 grid((unsigned)blocks, (unsigned)groups);
      if (top_k <= 8) launch_pdl(route_grad_kernel<TY, PER, L, (8 + L - 1) / L>, grid, dim3(256), 0, st, a);
      else launch_pdl(route_grad_kernel<TY, PER, L, (kRouteMaxK + L - 1) / L>, grid, dim3(256), 0, st, a);
    });
  });
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("route_grad: ") + cudaGetErrorString(e));
  return PRSGD_OK;
}

}  // extern "C"
