// C entries of the Newton-Schulz orthogonalisation and of the Muon step.  See include/prsgd.h for the contract.
#include <cmath>
#include <mutex>
#include "kernels_ortho_small.cuh"
#include "ops_internal.h"

using namespace prsgd;

namespace prsgd {

// Into how many parts the contraction of A = X X^T is cut: while A has fewer tiles than there are pairs of CTAs (74), as
// many as there are pairs for, but no part below 12 blocks of 64 products (6 us of products against about 4 for leaving a
// part's sum and adding it up).  4 x 500 x 1900, fp32: 12 tiles in 6 parts.
static int ns_parts(const NsShape& sh, int precision) {
  const int64_t s = std::min(sh.rows, sh.cols), l = std::max(sh.rows, sh.cols), ts = (s + 255) / 256, kb = (l + 63) / 64;
  const int64_t tiles = (int64_t)sh.batch * ts * (ts + 1) / 2, blocks = kb * (precision == PRSGD_PRECISION_FP32 ? 3 : 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(74 / std::max<int64_t>(tiles, 1), blocks / 12), std::min<int64_t>(kb, 16)));
}

static NsBuffers ns_carve(const NsShape& sh, int precision, unsigned char* base, size_t* bytes) {
  NsBuffers b{};
  const int64_t s = std::min(sh.rows, sh.cols);
  const bool split = precision == PRSGD_PRECISION_FP32;
  b.xp = round_up(sh.cols, 8); b.sp = round_up(s, 8);
  const int64_t per = (int64_t)sh.rows * sh.cols;
  b.panels = (int)((s + 255) / 256);
  b.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(kNsChunks, sh.rows), (per + 8191) / 8192));
  size_t off = 0;
  auto take = [&](size_t n) { unsigned char* p = base ? base + off : nullptr; off += (n + 255) / 256 * 256; return p; };
  b.status = reinterpret_cast<DeviceStatus*>(take(sizeof(DeviceStatus)));
  b.claim = reinterpret_cast<unsigned int*>(take(4));
  b.done = reinterpret_cast<unsigned int*>(take(4 * (size_t)sh.batch * b.panels));
  b.part = reinterpret_cast<double*>(take(8 * (size_t)sh.batch * b.chunks));
  b.parts = ns_parts(sh, precision); b.gram_tiles = b.panels * (b.panels + 1) / 2;
  const size_t sums = b.parts > 1 ? (size_t)sh.batch * b.gram_tiles : 0;
  b.part_count = reinterpret_cast<unsigned int*>(take(sums * 16 * 4));
  b.part_sums = reinterpret_cast<float*>(take(sums * b.parts * 16 * 4096 * 4));
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) b.x[i][j] = reinterpret_cast<__half*>(take(2 * (size_t)sh.batch * sh.rows * b.xp));
  for (int j = 0; j < 2; ++j) {
    b.A[j] = reinterpret_cast<__half*>(j == 0 || split ? take(2 * (size_t)sh.batch * s * b.sp) : nullptr);
    b.P[j] = reinterpret_cast<__half*>(j == 0 || split ? take(2 * (size_t)sh.batch * s * b.sp) : nullptr);
  }
  *bytes = off;
  return b;
}

// fp16 [batch][d1][pitch] with d0 elements of a row in use, boxes of 64 x box_rows, 128-byte swizzle; beyond the edges zeros
static int ns_map(CUtensorMap* m, const void* base, int64_t d0, int64_t d1, int64_t batch, int64_t pitch, int box_rows) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode enc = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<Encode>(f) : nullptr;
  }();
  if (!enc) return op_fail(PRSGD_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[3] = {(cuuint64_t)d0, (cuuint64_t)d1, (cuuint64_t)batch};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)pitch * (cuuint64_t)d1 * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? PRSGD_OK : op_fail(PRSGD_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string((int)r));
}

// The current device: its SM count, and how many clusters of 1 to 8 CTAs of ns_small_kernel run at a time (a cluster lies
// within one group of SMs, so that is fewer than the SMs divided by its size).  Found out, and the kernels'
// shared-memory limits raised, on the first call.
struct NsDevice { int sms, clusters[kNsSmallCtas + 1]; };
static int ns_device(NsDevice* out) {
  static std::mutex lock;
  static NsDevice known[64];
  int dev = -1;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev < 0 || dev >= 64)) return op_fail(PRSGD_ERR_ARG, "device ordinal out of range");
  std::lock_guard<std::mutex> hold(lock);
  if (e == cudaSuccess && known[dev].sms == 0) {
    int n = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(ns_chain_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kNsSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(ns_chain_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kNsSmem);
    auto small = [&](auto vec) {
      constexpr int V = decltype(vec)::value;
      auto raise = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kNsSmallSmem); };
      raise(ns_small_kernel<PRSGD_TYPE_FP32, 0, V>); raise(ns_small_kernel<PRSGD_TYPE_BF16, 0, V>); raise(ns_small_kernel<PRSGD_TYPE_FP16, 0, V>);
      raise(ns_small_kernel<PRSGD_TYPE_FP32, 2, V>); raise(ns_small_kernel<PRSGD_TYPE_BF16, 2, V>); raise(ns_small_kernel<PRSGD_TYPE_FP16, 2, V>);
      raise(ns_small_kernel<PRSGD_TYPE_FP32, 1, V>);
    };
    small(std::integral_constant<int, 1>()); small(std::integral_constant<int, 4>());
    for (int c = 1; c <= kNsSmallCtas && e == cudaSuccess; ++c) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)c); cfg.blockDim = dim3(kNsSmallThreads); cfg.dynamicSmemBytes = kNsSmallSmem;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = (unsigned)c; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr; cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&known[dev].clusters[c], ns_small_kernel<PRSGD_TYPE_FP32, 0, 4>, &cfg);
    }
    if (e == cudaSuccess) known[dev].sms = n;
  }
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("orthogonalize: ") + cudaGetErrorString(e));
  *out = known[dev];
  return PRSGD_OK;
}

int ns_prepare() { NsDevice d; return ns_device(&d); }

size_t ns_workspace_bytes(const NsShape& sh, int precision) {
  size_t n = 0;
  ns_carve(sh, precision, nullptr, &n);
  return n;
}

// Matrices of a short side up to 128 and a long one up to 2048 (short side up to 64) or 1536: a cluster each.
static int ns_run_small(const NsPlan& p, const NsBuffers& buf, bool vec_in, int vec_out, const NsDevice& dev, cudaStream_t st, int64_t* launches) {
  NsSmallArgs a{};
  a.sh = p.shape; a.src = p.src; a.dst = p.dst; a.status = buf.status; a.own_status = buf.own_status;
  a.steps = p.steps; a.tall = p.shape.rows > p.shape.cols; a.s = std::min(p.shape.rows, p.shape.cols); a.l = std::max(p.shape.rows, p.shape.cols);
  a.a = p.a; a.b = p.b; a.c = p.c; a.eps = p.eps; a.vec_out = vec_out;
  a.sp = (a.s + 15) / 16 * 16;
  // As few CTAs as hold the matrix, or, while all clusters run at a time, more with fewer columns (down to 128).  (16 matrices
  // of 10 x 1024 in clusters of 8, of which 14 run at a time, took 1.6 times as long as in clusters of 6; 8 of 64 x 1024 with 128
  // columns a CTA 40 us, with 192 46, with 256 49.)
  a.ctas = (a.l + ns_small_cols(a.s) - 1) / ns_small_cols(a.s);
  while (a.ctas < kNsSmallCtas && (a.l + a.ctas - 1) / a.ctas > 128 && p.shape.batch <= dev.clusters[a.ctas + 1]) ++a.ctas;
  a.w = ((a.l + a.ctas - 1) / a.ctas + 63) / 64 * 64;
  a.ctas = (a.l + a.w - 1) / a.w;
  const dim3 grid((unsigned)(p.shape.batch * a.ctas));
  auto go = [&](auto kernel) { launch_pdl_cluster(kernel, grid, dim3(kNsSmallThreads), kNsSmallSmem, st, (unsigned)a.ctas, a); };
  auto modes = [&](auto vec) {
    constexpr int V = decltype(vec)::value;
    if (p.src.V == nullptr) with_type(p.g_type, [&](auto ty) { go(ns_small_kernel<decltype(ty)::value, 0, V>); });
    else if (p.src.G != nullptr) with_type(p.g_type, [&](auto ty) { go(ns_small_kernel<decltype(ty)::value, 2, V>); });
    else go(ns_small_kernel<PRSGD_TYPE_FP32, 1, V>);
  };
  if (vec_in && !a.tall) modes(std::integral_constant<int, 4>());
  else modes(std::integral_constant<int, 1>());
  if (launches) *launches += 1;
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("orthogonalize: ") + cudaGetErrorString(e));
  return PRSGD_OK;
}

int ns_run(const NsPlan& p, void* d_work, cudaStream_t st, int64_t* launches) {
  size_t bytes = 0;
  NsBuffers buf = ns_carve(p.shape, p.precision, static_cast<unsigned char*>(d_work), &bytes);
  buf.own_status = p.status == nullptr ? 1 : 0;
  if (p.status != nullptr) buf.status = p.status;
  const int s = std::min(p.shape.rows, p.shape.cols);
  const bool split = p.precision == PRSGD_PRECISION_FP32;
  auto fits4 = [](const void* q, int64_t row, int64_t batch, int esz) {
    return q == nullptr || ((uintptr_t)q % (4 * esz) == 0 && row % 4 == 0 && batch % 4 == 0);
  };
  const bool vec = p.shape.cols % 4 == 0 && fits4(p.src.G, p.src.g_row, p.src.g_batch, type_bytes(p.g_type)) &&
                   fits4(p.src.V, p.src.v_tiled ? 0 : p.src.v_row, p.src.v_batch, 4);
  const dim3 grid((unsigned)buf.chunks, (unsigned)p.shape.batch);
  NsDevice dev;
  int rc = ns_device(&dev);
  const int sms = dev.sms;
  if (rc != PRSGD_OK) return rc;
  const int esz = type_bytes(p.dst.type);
  const int vec_out = (uintptr_t)p.dst.out % 16 == 0 && (p.dst.tiled || p.dst.row * esz % 16 == 0) && p.dst.batch * esz % 16 == 0;
  const int l = std::max(p.shape.rows, p.shape.cols);
  if (s <= kNsSmallSide && l <= ns_small_cols(s) * kNsSmallCtas) return ns_run_small(p, buf, vec, vec_out, dev, st, launches);
  with_type(p.g_type, [&](auto ty) {
    constexpr int TY = decltype(ty)::value;
    auto passes = [&](auto norm, auto pack) {
      launch_pdl(norm, grid, dim3(256), 0, st, p.shape, p.src, buf);
      launch_pdl(pack, grid, dim3(256), 0, st, p.shape, p.src, buf, p.eps);
    };
    if (p.src.V == nullptr) {
      if (vec) passes(ns_norm_kernel<TY, 4, 0>, ns_pack_kernel<TY, 4, 0>);
      else passes(ns_norm_kernel<TY, 1, 0>, ns_pack_kernel<TY, 1, 0>);
    } else if (p.src.G != nullptr) {
      if (vec) passes(ns_norm_kernel<TY, 4, 2>, ns_pack_kernel<TY, 4, 2>);
      else passes(ns_norm_kernel<TY, 1, 2>, ns_pack_kernel<TY, 1, 2>);
    } else {                                             // (G's type does not matter)
      if (vec) passes(ns_norm_kernel<PRSGD_TYPE_FP32, 4, 1>, ns_pack_kernel<PRSGD_TYPE_FP32, 4, 1>);
      else passes(ns_norm_kernel<PRSGD_TYPE_FP32, 1, 1>, ns_pack_kernel<PRSGD_TYPE_FP32, 1, 1>);
    }
  });
  if (launches) *launches += 2;
  NsChainArgs a{};
  a.sh = p.shape; a.buf = buf; a.dst = p.dst; a.steps = p.steps; a.split = split ? 1 : 0;
  a.tall = p.shape.rows > p.shape.cols; a.s = s; a.l = std::max(p.shape.rows, p.shape.cols);
  a.a = p.a; a.b = p.b; a.c = p.c;
  const int ts = (s + 255) / 256;
  a.tsym = ts * (ts + 1) / 2; a.tr = (p.shape.rows + 255) / 256; a.tc = (p.shape.cols + 255) / 256;
  a.ts = ts; a.parts = buf.parts; a.per_step = a.tsym * (a.parts + 1) + a.tr * a.tc; a.per_panel = 2 * ts + (a.tall ? a.tr : a.tc);
  const int64_t total = (int64_t)p.shape.batch * p.steps * a.per_step;
  if (total > 0x3fffffffll) return op_fail(PRSGD_ERR_SIZE, "orthogonalize: too many tiles in one call");
  a.total = (int)total;
  // Groups: while the last tiles of a product of one matrix drain, at least two rounds of tiles of other matrices
  // are to be claimed before its next product's.
  a.group = std::min(p.shape.batch, (sms + a.tsym - 1) / a.tsym + 1);
  a.vec_out = vec_out;
  NsMaps maps{};
  const int64_t rows = p.shape.rows, cols = p.shape.cols, batch = p.shape.batch;
  auto map_x = [&](CUtensorMap* to, const __half* p, int box) { if (rc == PRSGD_OK) rc = ns_map(to, p, cols, rows, batch, buf.xp, box); };
  auto map_s = [&](CUtensorMap* to, const __half* p, int box) { if (rc == PRSGD_OK) rc = ns_map(to, p, s, s, batch, buf.sp, box); };
  for (int j = 0; j < (split ? 2 : 1); ++j) {            // lo is an operand with 32-bit precision only
    for (int i = 0; i < 2; ++i) {
      map_x(&maps.x[i][j], buf.x[i][j], 64);
      map_x(&maps.xk[i][j], buf.x[i][j], 128);
    }
    map_s(&maps.A[j], buf.A[j], 64); map_s(&maps.Ak[j], buf.A[j], 128);
    map_s(&maps.P[j], buf.P[j], 64); map_s(&maps.Pk[j], buf.P[j], 128);
  }
  if (rc != PRSGD_OK) return rc;
  const int pairs = (int)std::min<int64_t>(sms / 2, batch * std::max(a.tsym * a.parts, a.tr * a.tc));
  if (split) launch_pdl_cluster(ns_chain_kernel<true>, dim3(2 * pairs), dim3(kNsThreads), kNsSmem, st, 2, maps, a);
  else launch_pdl_cluster(ns_chain_kernel<false>, dim3(2 * pairs), dim3(kNsThreads), kNsSmem, st, 2, maps, a);
  if (launches) *launches += 1;
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("orthogonalize: ") + cudaGetErrorString(e));
  return PRSGD_OK;
}

}  // namespace prsgd

namespace {

constexpr float kDefaultCoefs[3] = {3.4445f, -4.7750f, 2.0315f};

// One strided batch of matrices: pointer, alignment, strides.
int check_matrices(const char* name, const void* p, int type, int64_t row, int64_t batch_stride, int batch, int rows, int cols, bool written) {
  if (p == nullptr) return op_fail(PRSGD_ERR_ARG, std::string(name) + " is NULL");
  if (!type_known(type)) return op_fail(PRSGD_ERR_ARG, std::string("unknown element type of ") + name);
  if (((uintptr_t)p) % type_bytes(type)) return op_fail(PRSGD_ERR_ALIGN, std::string(name) + " is not aligned to its element type");
  if (row < cols) return op_fail(PRSGD_ERR_ARG, std::string("row stride of ") + name + " is below its columns");
  if (batch_stride < 0 || (written && !rows_apart(batch, batch_stride, rows, row, cols)))
    return op_fail(PRSGD_ERR_ARG, std::string("the matrices of ") + name + " overlap");
  return PRSGD_OK;
}

int check_sizes(int batch, int rows, int cols, int precision) {
  if (batch < 0 || rows < 0 || cols < 0) return op_fail(PRSGD_ERR_ARG, "need batch, rows, cols >= 0");
  if (batch > 65535 || rows > PRSGD_ORTHO_MAX_SIDE || cols > PRSGD_ORTHO_MAX_SIDE)
    return op_fail(PRSGD_ERR_SIZE, "more than 65535 matrices or a side above PRSGD_ORTHO_MAX_SIDE");
  if (precision != PRSGD_PRECISION_FP32 && precision != PRSGD_PRECISION_BF16) return op_fail(PRSGD_ERR_ARG, "unknown precision");
  return PRSGD_OK;
}

int check_chain(int steps, const float* coefs, float eps, NsPlan* p) {
  if (steps < 1 || steps > PRSGD_ORTHO_MAX_STEPS) return op_fail(PRSGD_ERR_ARG, "steps must be in 1..PRSGD_ORTHO_MAX_STEPS");
  if (!(eps >= 0.f) || std::isinf(eps)) return op_fail(PRSGD_ERR_ARG, "eps must be finite and >= 0");
  const float* q = coefs ? coefs : kDefaultCoefs;
  for (int i = 0; i < 3; ++i)
    if (!(std::fabs(q[i]) <= 16.f)) return op_fail(PRSGD_ERR_ARG, "a coefficient is NaN or beyond 16 in magnitude");
  p->steps = steps; p->a = q[0]; p->b = q[1]; p->c = q[2]; p->eps = eps;
  return PRSGD_OK;
}

int check_work(const NsShape& sh, int precision, const void* work, size_t bytes) {
  if (work == nullptr || bytes < ns_workspace_bytes(sh, precision))
    return op_fail(PRSGD_ERR_SIZE, "workspace is NULL or smaller than prsgd_orthogonalize_workspace_bytes");
  if (((uintptr_t)work) % 256) return op_fail(PRSGD_ERR_ALIGN, "d_work must be 256-byte aligned");
  return PRSGD_OK;
}

}  // namespace

extern "C" {

int prsgd_orthogonalize_workspace_bytes(int32_t batch, int32_t rows, int32_t cols, int32_t precision, size_t* bytes) {
  if (!bytes) return op_fail(PRSGD_ERR_ARG, "bytes is NULL");
  int rc = check_sizes(batch, rows, cols, precision);
  if (rc != PRSGD_OK) return rc;
  *bytes = ns_workspace_bytes({batch, rows, cols}, precision);
  return PRSGD_OK;
}

int prsgd_orthogonalize(const void* d_G, int32_t g_type, int64_t g_row_stride, int64_t g_batch_stride,
                        void* d_out, int32_t out_type, int64_t out_row_stride, int64_t out_batch_stride,
                        int32_t batch, int32_t rows, int32_t cols, int32_t steps, const float* h_coefs, float scale,
                        float eps, int32_t precision, void* d_work, size_t work_bytes, void* cuda_stream) {
  NsPlan p{};
  int rc = check_sizes(batch, rows, cols, precision);
  if (rc == PRSGD_OK) rc = check_chain(steps, h_coefs, eps, &p);
  if (rc != PRSGD_OK) return rc;
  if (!std::isfinite(scale)) return op_fail(PRSGD_ERR_ARG, "scale must be finite");
  if (batch == 0 || rows == 0 || cols == 0) return op_clear_status(d_work, work_bytes, cuda_stream);
  rc = check_matrices("G", d_G, g_type, g_row_stride, g_batch_stride, batch, rows, cols, false);
  if (rc == PRSGD_OK) rc = check_matrices("out", d_out, out_type, out_row_stride, out_batch_stride, batch, rows, cols, true);
  if (rc == PRSGD_OK && d_out == d_G && (g_type != out_type || !same_layout(batch, g_batch_stride, out_batch_stride, rows, g_row_stride, out_row_stride)))
    return op_fail(PRSGD_ERR_ARG, "out is G's memory with another type or other strides");
  p.shape = {batch, rows, cols}; p.precision = precision; p.g_type = g_type;
  if (rc == PRSGD_OK) rc = check_work(p.shape, precision, d_work, work_bytes);
  if (rc != PRSGD_OK) return rc;
  p.src.G = d_G; p.src.g_row = g_row_stride; p.src.g_batch = g_batch_stride;
  p.dst.out = d_out; p.dst.type = out_type; p.dst.row = out_row_stride; p.dst.batch = out_batch_stride;
  p.dst.alpha = scale; p.dst.beta = 0.f;
  return ns_run(p, d_work, static_cast<cudaStream_t>(cuda_stream), nullptr);
}

int prsgd_muon_step(void* d_W, int32_t w_type, int64_t w_row_stride, int64_t w_batch_stride,
                    float* d_V, int64_t v_row_stride, int64_t v_batch_stride,
                    const void* d_G, int32_t g_type, int64_t g_row_stride, int64_t g_batch_stride,
                    int32_t batch, int32_t rows, int32_t cols, float lr, float mu, int32_t nesterov, float weight_decay,
                    int32_t steps, const float* h_coefs, float scale, float eps, int32_t precision,
                    void* d_work, size_t work_bytes, void* cuda_stream) {
  NsPlan p{};
  int rc = check_sizes(batch, rows, cols, precision);
  if (rc == PRSGD_OK) rc = check_chain(steps, h_coefs, eps, &p);
  if (rc != PRSGD_OK) return rc;
  if (!(mu >= 0.f && mu < 1.f)) return op_fail(PRSGD_ERR_ARG, "mu must be in [0, 1)");
  if (!std::isfinite(lr) || !std::isfinite(scale) || !std::isfinite(weight_decay)) return op_fail(PRSGD_ERR_ARG, "lr, scale and weight_decay must be finite");
  if (lr * weight_decay == 1.f) return op_fail(PRSGD_ERR_ARG, "lr * weight_decay must not be 1");
  if (batch == 0 || rows == 0 || cols == 0) return op_clear_status(d_work, work_bytes, cuda_stream);
  rc = check_matrices("W", d_W, w_type, w_row_stride, w_batch_stride, batch, rows, cols, true);
  if (rc == PRSGD_OK) rc = check_matrices("V", d_V, PRSGD_TYPE_FP32, v_row_stride, v_batch_stride, batch, rows, cols, true);
  if (rc == PRSGD_OK) rc = check_matrices("G", d_G, g_type, g_row_stride, g_batch_stride, batch, rows, cols, false);
  if (rc == PRSGD_OK && (d_W == static_cast<void*>(d_V) || d_W == d_G || d_V == d_G)) return op_fail(PRSGD_ERR_ARG, "two of W, V and G are the same memory");
  p.shape = {batch, rows, cols}; p.precision = precision; p.g_type = g_type;
  if (rc == PRSGD_OK) rc = check_work(p.shape, precision, d_work, work_bytes);
  if (rc != PRSGD_OK) return rc;
  p.src.G = d_G; p.src.g_row = g_row_stride; p.src.g_batch = g_batch_stride;
  p.src.V = d_V; p.src.v_row = v_row_stride; p.src.v_batch = v_batch_stride; p.src.mu = mu; p.src.nesterov = nesterov != 0;
  p.dst.out = d_W; p.dst.type = w_type; p.dst.row = w_row_stride; p.dst.batch = w_batch_stride;
  p.dst.alpha = -lr * scale; p.dst.beta = 1.f - lr * weight_decay;
  return ns_run(p, d_work, static_cast<cudaStream_t>(cuda_stream), nullptr);
}

int prsgd_work_status(const void* d_work, void* cuda_stream) {
  if (!d_work) return op_fail(PRSGD_ERR_ARG, "d_work is NULL");
  unsigned int st[2] = {0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaMemcpyAsync(st, d_work, sizeof st, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return op_fail(PRSGD_ERR_CUDA, std::string("work_status: ") + cudaGetErrorString(e));
  if (st[0] != 0u)
    return op_fail(PRSGD_ERR_DEVICE_TIMEOUT, "a bounded wait expired in an operator's kernel (code " + std::to_string(st[0]) + ", block " + std::to_string(st[1]) + ")");
  return PRSGD_OK;
}

}  // extern "C"
