// Linear layers (lqsgd_linear_forward / _grad_input / _grad_weight): argument checks, the choice of tile and split, tensor
// maps and launches.  The matrix product kernel and its epilogues are in lqsgd_linear_dev.cuh.
#include "lqsgd_linear_dev.cuh"

#include <algorithm>
#include <atomic>
#include <cstring>

namespace lqsgd {
namespace {

// Adds the partial sums of a split product in the order of the pieces and applies the epilogue: a warp per row and 32
// columns, lane by lane.
__global__ void __launch_bounds__(256)
linear_join_kernel(const float* __restrict__ partial, int64_t ld_partial, int splits, LinEpilogue e) {
  train_pdl_wait();
  const int lane = threadIdx.x & 31;
  const int groups = (e.cols + 31) / 32;
  const int64_t units = (int64_t)e.rows * groups, plane = (int64_t)e.rows * ld_partial;
  for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
    const int64_t row = u / groups;
    const int col = (int)(u - row * groups) * 32 + lane;
    const bool on = col < e.cols;
    float v = 0.f;
    if (on) {
      const float* src = partial + row * ld_partial + col;
#pragma unroll 4
      for (int s = 0; s < splits; ++s) v += src[s * plane];
    }
    finish_lane(e, row, col, on, v, on && e.bias ? __ldg(e.bias + col) : 0.f);
  }
}

// Copies a matrix of 16-bit values whose rows TMA cannot address (base or row distance not a multiple of 16 bytes) to
// rows of ld_dst elements, a multiple of 8; what lies past cols is never read.
__global__ void __launch_bounds__(256)
realign_kernel(const uint16_t* __restrict__ src, int64_t ld_src, int64_t rows, int cols, uint16_t* __restrict__ dst, int64_t ld_dst) {
  train_pdl_wait();
  const int pairs = (cols + 1) / 2;
  const int64_t units = rows * pairs;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < units; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / pairs;
    const int col = (int)(u - row * pairs) * 2;
    const uint16_t* s = src + row * ld_src + col;
    const uint32_t lo = s[0], hi = col + 1 < cols ? s[1] : 0;
    *reinterpret_cast<uint32_t*>(dst + row * ld_dst + col) = lo | (hi << 16);
  }
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn tensor_map_encoder() {
  static std::atomic<EncodeFn> cached{nullptr};
  EncodeFn fn = cached.load(std::memory_order_acquire);
  if (fn) return fn;
  void* raw = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &raw, cudaEnableDefault, &q) != cudaSuccess || !raw || q != cudaDriverEntryPointSuccess) return nullptr;
  fn = reinterpret_cast<EncodeFn>(raw);
  cached.store(fn, std::memory_order_release);
  return fn;
}
// Map over a matrix of 16-bit values: boxes of 64 columns x box_rows rows, 128-byte swizzle, zeros outside.
int encode_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  EncodeFn fn = tensor_map_encoder();
  if (!fn) return record_cuda_failure(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
  const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t stride[1] = {(cuuint64_t)(rows == 1 ? ceil_div64(cols, 8) * 8 : ld) * 2};   // one row has no distance to the next
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, es[2] = {1, 1};
  if (fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return record_cuda_failure(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  return LQSGD_OK;
}

// One operand as it lies in memory.
struct Stored {
  const void* base = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  bool packed = false;
  // One row needs no row distance.
  bool tma_ready() const { return train_aligned(base, 16) && (rows == 1 || ld % 8 == 0); }
};

struct Plan {
  int product;
  bool swap;                     // few rows: A and B exchanged
  int cg, bn;
  int64_t M, N, K;
  Stored a, b;
  int tiles_m, tiles_n, splits, kb_total, kb_per_split;
  int64_t ld_partial;
  size_t off_a, off_b, off_partial, bytes;
};

constexpr int64_t kFewRows = 64;       // at most this many rows: the weights are the operand that is streamed

// Microseconds one work item of `kb` k-blocks costs: the fixed part (filling the pipeline, draining the accumulator) and the blocks.
double item_us(int cg, int bn, int64_t kb) {
  const double per_kb = cg == 2 ? 0.32 : (bn >= 128 ? 0.24 : 0.13);
  return 2.0 + kb * per_kb;
}

int make_plan(int product, const lqsgd_linear& a, Plan* out) {
  Plan p = {};
  p.product = product;
  const int64_t rows = a.rows;
  const Stored x = {a.dev_x, rows, a.in, a.ld_x, false}, w = {a.dev_w, a.out, a.in, a.ld_w, false},
               dz = {a.dev_dz, rows, a.out, a.ld_dz, false};
  p.swap = product != LQSGD_LINEAR_GRAD_WEIGHT && rows <= kFewRows;
  int64_t out_rows = rows, out_cols;
  if (product == LQSGD_LINEAR_FORWARD) {
    p.a = x; p.b = w; p.M = rows; p.N = a.out; p.K = a.in; out_cols = a.out;
  } else if (product == LQSGD_LINEAR_GRAD_INPUT) {
    p.a = dz; p.b = w; p.M = rows; p.N = a.in; p.K = a.out; out_cols = a.in;
  } else {
    p.a = dz; p.b = x; p.M = a.out; p.N = a.in; p.K = rows; out_rows = a.out; out_cols = a.in;
    if (a.x8.dev_codes) p.b = {a.x8.dev_codes, rows, a.in, a.x8.ld_codes, true};
  }
  if (p.swap) { std::swap(p.a, p.b); std::swap(p.M, p.N); }
  p.kb_total = (int)ceil_div64(p.K, kLinBK);
  const int slots = 148;               // a constant, so that sums are cut the same way on every card
  double best = 1e30;
  auto consider = [&](int cg, int bn) {
    const int64_t tm = ceil_div64(p.M, (int64_t)kLinBM * cg), tn = ceil_div64(p.N, bn);
    if (tm * tn > (1 << 28)) return;
    const int units = slots / cg;
    for (int s = 1; s <= 148 && s <= p.kb_total; ++s) {
      if (tm * tn * s > 4 * units && s > 1) break;
      const int64_t kb = ceil_div64(p.kb_total, s);
      if (ceil_div64(p.kb_total, kb) != s) continue;         // the same pieces as a smaller s
      const int64_t waves = ceil_div64(tm * tn * s, units);
      double t = waves * item_us(cg, bn, kb);
      if (s > 1) t += 2.5 + 8.0 * s * out_rows * out_cols / 4.0e6;
      if (t < best) {
        best = t;
        p.cg = cg; p.bn = bn; p.tiles_m = (int)tm; p.tiles_n = (int)tn; p.splits = s; p.kb_per_split = (int)kb;
      }
    }
  };
  if (p.swap) {
    consider(1, p.N <= 16 ? 16 : (p.N <= 32 ? 32 : 64));
  } else {
    consider(1, 128);
    consider(2, 256);
  }
  if (best > 1e29) return LQSGD_ERR_BAD_SHAPE;
  p.ld_partial = ceil_div64(out_cols, 8) * 8;
  size_t off = 0;
  auto take = [&](size_t n) { const size_t at = off; off += (n + 255) / 256 * 256; return at; };
  auto copied = [&](const Stored& s) { return !s.packed && !s.tma_ready(); };
  if (copied(p.a)) p.off_a = take((size_t)p.a.rows * (ceil_div64(p.a.cols, 8) * 8) * 2);
  if (copied(p.b)) p.off_b = take((size_t)p.b.rows * (ceil_div64(p.b.cols, 8) * 8) * 2);
  if (p.splits > 1) p.off_partial = take((size_t)p.splits * out_rows * p.ld_partial * 4);
  p.bytes = off;
  *out = p;
  return LQSGD_OK;
}

int check_args(int product, const lqsgd_linear* a) {
  if (!a || a->struct_size != sizeof(lqsgd_linear)) return LQSGD_ERR_INVALID_ARG;
  if (a->dtype != LQSGD_BF16 && a->dtype != LQSGD_F16) return LQSGD_ERR_INVALID_ARG;
  if (!train_act_ok(a->act) || (a->accumulate != 0 && a->accumulate != 1)) return LQSGD_ERR_INVALID_ARG;
  if (product < LQSGD_LINEAR_FORWARD || product > LQSGD_LINEAR_GRAD_WEIGHT) return LQSGD_ERR_INVALID_ARG;
  if (a->rows < 0 || a->rows > 0x7fffffffll - 511 || a->in < 1 || a->out < 1 || a->in > (1 << 24) || a->out > (1 << 24)) return LQSGD_ERR_BAD_SHAPE;
  return LQSGD_OK;
}
int check_matrix(const void* p, int64_t ld, int32_t cols, int elem) {
  if (!p || ld < cols) return LQSGD_ERR_INVALID_ARG;
  return train_aligned(p, elem) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}

// TMA reads an operand in place, or a copy of it with aligned rows in the workspace.
int place(Stored* s, char* ws, size_t off, cudaStream_t st) {
  if (s->packed || s->tma_ready()) return LQSGD_OK;
  const int64_t ld = ceil_div64(s->cols, 8) * 8;
  uint16_t* dst = reinterpret_cast<uint16_t*>(ws + off);
  const int64_t blocks = std::min<int64_t>(ceil_div64(s->rows * ((s->cols + 1) / 2), 256), 148 * 16);
  TRAIN_CK(train_launch(realign_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 1, static_cast<const uint16_t*>(s->base), s->ld, s->rows,
                        (int)s->cols, dst, ld), "realign_kernel launch");
  s->base = dst;
  s->ld = ld;
  return LQSGD_OK;
}

template <int CG, int BN, int OA, int OB, bool SWAP>
int launch(const Plan& p, LinProblem& q, cudaStream_t st) {
  using S = LinCfg<CG, BN, OA, OB>;
  auto kernel = linear_kernel<CG, BN, OA, OB, SWAP>;
  static std::atomic<uint64_t> ready{0};                     // devices on which the kernel may use its shared memory
  int dev = 0;
  TRAIN_CK(cudaGetDevice(&dev), "cudaGetDevice");
  if (dev >= 64 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    TRAIN_CK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem), "cudaFuncSetAttribute(linear_kernel)");
    if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
  }
  int rc = encode_map(&q.ta, p.a.base, p.a.rows, p.a.cols, p.a.ld, OA == kOpK ? kLinBM : kLinBK);
  if (rc != LQSGD_OK) return rc;
  if (OB != kOpPacked && (rc = encode_map(&q.tb, p.b.base, p.b.rows, p.b.cols, p.b.ld, OB == kOpK ? S::kBNc : kLinBK)) != LQSGD_OK) return rc;
  const int sms = train_sm_count();
  if (sms < CG) return record_cuda_failure(cudaErrorInvalidDevice, "cudaDevAttrMultiProcessorCount");
  const int64_t items = (int64_t)p.tiles_m * p.tiles_n * p.splits;
  const int clusters = (int)std::min<int64_t>(items, sms / CG);
  TRAIN_CK(train_launch(kernel, dim3((unsigned)(clusters * CG)), dim3(S::kThreads), S::kSmem, st, CG, q), "linear_kernel launch");
  return LQSGD_OK;
}

int run(int product, const lqsgd_linear& a, LinEpilogue ep, cudaStream_t st) {
  Plan p;
  int rc = make_plan(product, a, &p);
  if (rc != LQSGD_OK) return rc;
  if (p.bytes) {
    if (!a.dev_workspace || a.workspace_bytes < p.bytes) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
    if (!train_aligned(a.dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
  }
  char* ws = static_cast<char*>(a.dev_workspace);
  if ((rc = place(&p.a, ws, p.off_a, st)) != LQSGD_OK || (rc = place(&p.b, ws, p.off_b, st)) != LQSGD_OK) return rc;
  const int es = ep.dtype == LQSGD_F32 ? 4 : 2;
  auto rows_aligned = [](const void* ptr, int64_t bytes, size_t to) { return train_aligned(ptr, to) && bytes % (int64_t)to == 0; };
  ep.vec_out = rows_aligned(ep.out, ep.ld_out * es, 32);
  ep.vec_res = rows_aligned(ep.residual, ep.ld_res * 2, 32);
  ep.vec_z8 = rows_aligned(ep.z8.dev_codes, ep.z8.ld_codes, 16);
  ep.vec_y8 = rows_aligned(ep.y8.dev_codes, ep.y8.ld_codes, 16);
  LinProblem q;
  std::memset(&q, 0, sizeof(q));
  q.ep = ep;
  q.partial = p.splits > 1 ? reinterpret_cast<float*>(ws + p.off_partial) : nullptr;
  q.ld_partial = p.ld_partial;
  q.x8 = a.x8;
  q.x8_vec = rows_aligned(a.x8.dev_codes, a.x8.ld_codes, 16);
  q.M = (int32_t)p.M; q.N = (int32_t)p.N; q.K = (int32_t)p.K;
  q.tiles_m = p.tiles_m; q.tiles_n = p.tiles_n; q.splits = p.splits; q.kb_total = p.kb_total; q.kb_per_split = p.kb_per_split;
  q.dtype = a.dtype;
  q.status = a.dev_status;
  if (product == LQSGD_LINEAR_FORWARD) {
    if (p.swap) rc = p.bn == 16 ? launch<1, 16, kOpK, kOpK, true>(p, q, st) : p.bn == 32 ? launch<1, 32, kOpK, kOpK, true>(p, q, st) : launch<1, 64, kOpK, kOpK, true>(p, q, st);
    else rc = p.cg == 2 ? launch<2, 256, kOpK, kOpK, false>(p, q, st) : launch<1, 128, kOpK, kOpK, false>(p, q, st);
  } else if (product == LQSGD_LINEAR_GRAD_INPUT) {
    if (p.swap) rc = p.bn == 16 ? launch<1, 16, kOpMN, kOpK, true>(p, q, st) : p.bn == 32 ? launch<1, 32, kOpMN, kOpK, true>(p, q, st) : launch<1, 64, kOpMN, kOpK, true>(p, q, st);
    else rc = p.cg == 2 ? launch<2, 256, kOpK, kOpMN, false>(p, q, st) : launch<1, 128, kOpK, kOpMN, false>(p, q, st);
  } else if (p.b.packed) {
    rc = p.cg == 2 ? launch<2, 256, kOpMN, kOpPacked, false>(p, q, st) : launch<1, 128, kOpMN, kOpPacked, false>(p, q, st);
  } else {
    rc = p.cg == 2 ? launch<2, 256, kOpMN, kOpMN, false>(p, q, st) : launch<1, 128, kOpMN, kOpMN, false>(p, q, st);
  }
  if (rc != LQSGD_OK) return rc;
  if (p.splits > 1) {
    const int64_t units = (int64_t)ep.rows * ((ep.cols + 31) / 32);
    TRAIN_CK(train_launch(linear_join_kernel, dim3((unsigned)std::min<int64_t>(ceil_div64(units, 8), 148 * 8)), dim3(256), 0, st, 1,
                          static_cast<const float*>(q.partial), p.ld_partial, p.splits, ep), "linear_join_kernel launch");
  }
  return LQSGD_OK;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

extern "C" int lqsgd_linear_workspace_bytes(int32_t product, const lqsgd_linear* host_args, size_t* host_bytes_out) {
  if (!host_bytes_out) return LQSGD_ERR_INVALID_ARG;
  int rc = check_args(product, host_args);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = 0;
  if (host_args->rows == 0) return LQSGD_OK;
  Plan p;
  if ((rc = make_plan(product, *host_args, &p)) != LQSGD_OK) return rc;
  *host_bytes_out = p.bytes;
  return LQSGD_OK;
}

extern "C" int lqsgd_linear_forward(const lqsgd_linear* a, void* cuda_stream) {
  int rc = check_args(LQSGD_LINEAR_FORWARD, a);
  if (rc != LQSGD_OK) return rc;
  if (a->rows == 0) return LQSGD_OK;
  if ((rc = check_matrix(a->dev_x, a->ld_x, a->in, 2)) != LQSGD_OK || (rc = check_matrix(a->dev_w, a->ld_w, a->in, 2)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_out, a->ld_out, a->out, 2)) != LQSGD_OK)
    return rc;
  if (a->dev_residual && (rc = check_matrix(a->dev_residual, a->ld_residual, a->out, 2)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_bias, 4) || !train_aligned(a->dev_status, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->z8.dev_codes && (rc = check_packed8(a->z8, a->out)) != LQSGD_OK) return rc;
  if (a->y8.dev_codes && (rc = check_packed8(a->y8, a->out)) != LQSGD_OK) return rc;
  LinEpilogue ep = {};
  ep.out = a->dev_out; ep.ld_out = a->ld_out; ep.bias = a->dev_bias;
  ep.residual = a->dev_residual; ep.ld_res = a->ld_residual;
  ep.z8 = a->z8; ep.y8 = a->y8;
  ep.rows = (int32_t)a->rows; ep.cols = a->out; ep.dtype = a->dtype; ep.act = a->act;
  return run(LQSGD_LINEAR_FORWARD, *a, ep, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int lqsgd_linear_grad_input(const lqsgd_linear* a, void* cuda_stream) {
  int rc = check_args(LQSGD_LINEAR_GRAD_INPUT, a);
  if (rc != LQSGD_OK) return rc;
  if (a->rows == 0) return LQSGD_OK;
  if ((rc = check_matrix(a->dev_dz, a->ld_dz, a->out, 2)) != LQSGD_OK || (rc = check_matrix(a->dev_w, a->ld_w, a->in, 2)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_out, a->ld_out, a->in, 2)) != LQSGD_OK)
    return rc;
  if (a->dev_residual && (rc = check_matrix(a->dev_residual, a->ld_residual, a->in, 2)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_status, 4)) return LQSGD_ERR_MISALIGNED;
  LinEpilogue ep = {};
  ep.out = a->dev_out; ep.ld_out = a->ld_out;
  ep.residual = a->dev_residual; ep.ld_res = a->ld_residual;
  ep.rows = (int32_t)a->rows; ep.cols = a->in; ep.dtype = a->dtype; ep.act = LQSGD_ACT_NONE;
  return run(LQSGD_LINEAR_GRAD_INPUT, *a, ep, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int lqsgd_linear_grad_weight(const lqsgd_linear* a, void* cuda_stream) {
  int rc = check_args(LQSGD_LINEAR_GRAD_WEIGHT, a);
  if (rc != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if ((rc = check_matrix(a->dev_out, a->ld_out, a->in, 4)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_status, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->rows == 0) {                                       // an empty sum
    if (!a->accumulate)
      TRAIN_CK(cudaMemset2DAsync(a->dev_out, (size_t)a->ld_out * 4, 0, (size_t)a->in * 4, a->out, st), "cudaMemset2DAsync(dw)");
    return LQSGD_OK;
  }
  if ((rc = check_matrix(a->dev_dz, a->ld_dz, a->out, 2)) != LQSGD_OK) return rc;
  if (a->x8.dev_codes) rc = check_packed8(a->x8, a->in);
  else rc = check_matrix(a->dev_x, a->ld_x, a->in, 2);
  if (rc != LQSGD_OK) return rc;
  LinEpilogue ep = {};
  ep.out = a->dev_out; ep.ld_out = a->ld_out;
  ep.rows = a->out; ep.cols = a->in; ep.dtype = LQSGD_F32; ep.act = LQSGD_ACT_NONE; ep.accumulate = a->accumulate;
  return run(LQSGD_LINEAR_GRAD_WEIGHT, *a, ep, st);
}
