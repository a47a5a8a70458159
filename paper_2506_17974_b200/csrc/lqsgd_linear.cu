// Linear layers (lqsgd_linear_forward / _grad_input / _grad_weight): argument checks, the choice of tile and split, tensor
// maps and launches.  The matrix product kernel and its epilogues are in lqsgd_linear_dev.cuh.
#include "lqsgd_linear_dev.cuh"

#include <algorithm>
#include <atomic>
#include <cstring>

namespace lqsgd {
namespace {

// Adds the pieces of tiles that several clusters summed, in the order of the clusters, and applies the epilogue.  A block takes
// `rows` rows of a tile, a warp 128 columns of a row.  With many pieces the block's 8 warps take turns at them (WAYS = 8) and
// meet in shared memory: one warp alone would wait for them one after the other.
struct LinPieces {
  const float* partial;
  uint32_t tiles_m, tiles_n, kb_total, share, cg, bn, rows;
};
template <uint32_t WAYS>
__global__ void __launch_bounds__(256)
linear_join_kernel(LinPieces q, LinEpilogue e) {
  __shared__ float4 sums[8][32];
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t high = q.cg * kLinBM, parts = high / q.rows;
  const uint32_t t = quick_div(blockIdx.x, parts), part = blockIdx.x - t * parts;
  const uint32_t first = t * q.kb_total, g0 = quick_div(first, q.share), g1 = quick_div(first + q.kb_total - 1, q.share);
  int m_tile, n_tile;
  LinWalk::place(q.tiles_m, q.tiles_n, t, m_tile, n_tile);
  const uint32_t row0 = m_tile * high + part * q.rows;
  train_pdl_wait();
  if (g0 == g1 || row0 >= (uint32_t)e.rows) return;                 // one cluster had the tile and finished it
  const size_t tile = (size_t)high * q.bn;
  const uint32_t sub = warp % WAYS, strips = q.bn / 128, units = q.rows * strips;
  for (uint32_t u0 = 0; u0 < units; u0 += 8 / WAYS) {
    const uint32_t u = u0 + warp / WAYS, r = u / strips, strip = u - r * strips;
    const int64_t row = row0 + r;
    const bool mine = u < units && row < e.rows && (int)(n_tile * q.bn + strip * 128) < e.cols;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine && (int)(n_tile * q.bn + strip * 128 + 4 * lane) < e.cols) {
      const float* src = q.partial + (size_t)(part * q.rows + r) * q.bn + strip * 128 + 4 * lane;
#pragma unroll 6
      for (uint32_t g = g0 + sub; g <= g1; g += WAYS) {
        const float4 s = *reinterpret_cast<const float4*>(src + (2 * g + (g * q.share < first ? 1 : 0)) * tile);
        v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
      }
    }
    if (WAYS > 1) {
      sums[warp][lane] = make_float4(v[0], v[1], v[2], v[3]);
      __syncthreads();
      if (sub == 0)
        for (uint32_t k = 1; k < WAYS; ++k) {
          const float4 s = sums[warp + k][lane];
          v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
        }
      __syncthreads();
    }
    if (mine && sub == 0) finish_quad(e, row, n_tile * q.bn + strip * 128 + 4 * lane, v);
  }
}

// Copies a matrix whose rows TMA cannot address (base or row distance not a multiple of 16 bytes) to rows of ld_dst elements, a
// multiple of 16 bytes, zeros past cols; what lies past cols is never read.  A warp takes 256 columns of a row at a time, a thread
// 8 of them: words where the row starts on one, else 16-bit values.
constexpr int kRealignCols = 256;
__global__ void __launch_bounds__(256)
realign_kernel(const uint16_t* __restrict__ src, int64_t ld_src, int64_t rows, int cols, uint16_t* __restrict__ dst, int64_t ld_dst) {
  train_pdl_wait();
  const int lane = threadIdx.x & 31, strips = (cols + kRealignCols - 1) / kRealignCols, warps = (int)gridDim.x * 8;
  const int first = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
  int strip = first % strips;
  for (int64_t row = first / strips; row < rows; row += warps / strips) {
    const int col = strip * kRealignCols + 8 * lane, have = cols - col;
    if (have > 0) {
      const uint16_t* s = src + row * ld_src + col;
      uint32_t w[4];
      if (have >= 8 && (reinterpret_cast<uintptr_t>(s) & 3) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t*>(s) + i);
      } else {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < have ? __ldg(s + i) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (h[2 * i + 1] << 16);
      }
      *reinterpret_cast<uint4*>(dst + row * ld_dst + col) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    strip += warps % strips;
    if (strip >= strips) { strip -= strips; ++row; }
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
// One operand as it lies in memory, 16-bit values.
struct Stored {
  const void* base = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  int64_t aligned_ld() const { return ceil_div64(cols, 8) * 8; }
  // One row needs no row distance.
  bool tma_ready() const { return train_aligned(base, 16) && (rows == 1 || ld % 8 == 0); }
  size_t copy_bytes() const { return tma_ready() ? 0 : (size_t)rows * aligned_ld() * 2; }
};
// Map over an operand: boxes of 64 columns x box_rows, 128-byte swizzle, zeros outside.
int encode_map(CUtensorMap* map, const Stored& s, int box_rows) {
  EncodeFn fn = tensor_map_encoder();
  if (!fn) return record_cuda_failure(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
  const cuuint64_t dim[2] = {(cuuint64_t)s.cols, (cuuint64_t)s.rows};
  const cuuint64_t stride[1] = {(cuuint64_t)(s.rows == 1 ? s.aligned_ld() : s.ld) * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, es[2] = {1, 1};
  if (fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(s.base), dim, stride, box, es,
         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return record_cuda_failure(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  return LQSGD_OK;
}

struct Plan {
  int64_t M, N, K;
  Stored a, b;
  bool unpacked;                 // b is x8, decoded into the workspace first
  int cg, bn, tiles_m, tiles_n, kb_total, deal, share, meet, clusters;
  size_t off_a, off_b, off_x, off_partial, bytes;
};

constexpr size_t kPieceAlign = 32;     // of the pieces of sums in the workspace: the kernels move them in 32-byte accesses
constexpr int kSms = 148;              // sums are cut for this many SMs whatever the card has: results do not depend on it

int make_plan(int product, const lqsgd_linear& a, Plan* out) {
  Plan p = {};
  const int64_t rows = a.rows;
  const Stored x = {a.dev_x, rows, a.in, a.ld_x}, w = {a.dev_w, a.out, a.in, a.ld_w}, dz = {a.dev_dz, rows, a.out, a.ld_dz};
  if (product == LQSGD_LINEAR_FORWARD) {
    p.a = x; p.b = w; p.M = rows; p.N = a.out; p.K = a.in;
  } else if (product == LQSGD_LINEAR_GRAD_INPUT) {
    p.a = dz; p.b = w; p.M = rows; p.N = a.in; p.K = a.out;
  } else {
    p.a = dz; p.b = x; p.M = a.out; p.N = a.in; p.K = rows;
    p.unpacked = a.x8.dev_codes != nullptr;
    if (p.unpacked) p.b = {nullptr, rows, a.in, ceil_div64(a.in, 8) * 8};
  }
  p.kb_total = (int)ceil_div64(p.K, kLinBK);
  // The cheapest of the ways to deal the tiles out, by what they were measured to cost (microseconds).  Pairs of SMs on tiles of
  // 256 x 256 or single ones on 128 x 128: 94 against 134 us at 4096 x 4096 x 4096, but 10.7 against 9.2 at 1024 x 1024 x 1024, where
  // 16 pairs would work.  A forward product of 256 x 3136 x 512 takes 17.6 us in whole tiles, 12.6 in shares, 9.9 with the sums
  // of a cluster's CTAs meeting; a weight gradient of 65536 rows, 64 x 128, 281 us in whole tiles and 14.4 in shares; one of
  // 8192 rows, 512 x 512, 39.9, 18.1, and 14.4 where they meet.  8 x 4096 x 16384, 128 tiles: 27.7 us whole, 30.0 in shares.
  constexpr double kTileUs = 2.2, kMeetUs = 4.0, kJoinUs = 4.0;
  double best = 1e30;
  auto consider = [&](int cg, int bn) {
    const int64_t tm = ceil_div64(p.M, (int64_t)kLinBM * cg), tn = ceil_div64(p.N, bn), tiles = tm * tn;
    if (tiles > (1 << 28)) return;
    const int units = kSms / cg;
    const double per = cg == 2 ? 0.31 : 0.22;
    auto take = [&](double t, int deal, int64_t share, int meet, int64_t clusters) {
      if (t >= best) return;
      best = t;
      p.cg = cg; p.bn = bn; p.tiles_m = (int)tm; p.tiles_n = (int)tn;
      p.deal = deal; p.share = (int)share; p.meet = meet; p.clusters = (int)clusters;
    };
    take(ceil_div64(tiles, units) * (kTileUs + p.kb_total * per), kWhole, 0, 1, std::min<int64_t>(tiles, units));
    // how many clusters of 2 .. 8 such CTAs a B200 runs at once (SMs of one cluster lie in one GPC)
    constexpr int kAtOnce[9] = {0, 0, 74, 45, 33, 26, 22, 15, 15};
    for (int meet = 2; cg == 1 && meet <= 8; ++meet) {
      const int64_t share = ceil_div64(p.kb_total, meet);
      if (tiles <= kAtOnce[meet] && ceil_div64(p.kb_total, share) == meet) take(kTileUs + share * per + kMeetUs, kMeet, share, meet, tiles * meet);
    }
    // equal shares of at least 4 k blocks each, where tiles are few
    const int64_t pairs = tiles * p.kb_total;
    if (tiles >= 2 * units || p.kb_total < 8 || pairs >= (1ll << 31)) return;
    const int64_t share = std::max<int64_t>(4, ceil_div64(pairs, units)), clusters = ceil_div64(pairs, share);
    const double bytes = 4.0 * kLinBM * cg * bn * (double)clusters;
    take(kTileUs * (share >= p.kb_total ? 2 : 1) + share * per + kJoinUs + bytes / 2.0e6, kShares, share, 1, clusters);
  };
  consider(1, 128);
  consider(2, 256);
  if (best > 1e29) return LQSGD_ERR_BAD_SHAPE;
  size_t off = 0;
  auto room = [&](size_t n) { const size_t at = off; off += (n + 255) / 256 * 256; return at; };
  if (p.unpacked) p.off_x = room((size_t)rows * p.b.ld * 2);
  p.off_a = room(p.a.copy_bytes());
  p.off_b = room(p.b.copy_bytes());
  // The pieces are written and read 32 bytes at a time, and the caller's workspace starts on 16: room to move their start.
  if (p.deal == kShares) p.off_partial = room((size_t)2 * p.clusters * kLinBM * p.cg * p.bn * 4 + kPieceAlign);
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
  if (s->tma_ready()) return LQSGD_OK;
  const int64_t ld = s->aligned_ld();
  const int64_t blocks = std::min<int64_t>(ceil_div64(s->rows * ceil_div64(s->cols, kRealignCols), 8), kSms * 8);
  TRAIN_CK(train_launch(realign_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 1, static_cast<const uint16_t*>(s->base), s->ld, s->rows,
                        (int)s->cols, reinterpret_cast<uint16_t*>(ws + off), ld), "realign_kernel launch");
  s->base = ws + off;
  s->ld = ld;
  return LQSGD_OK;
}

template <int CG, int BN, int OA, int OB, bool WF32>
int launch(const Plan& p, LinProblem& q, cudaStream_t st) {
  using S = LinCfg<CG, BN, OA, OB, WF32>;
  auto kernel = linear_kernel<CG, BN, OA, OB, WF32>;
  static std::atomic<uint64_t> ready{0};                     // devices on which the kernel may use its shared memory
  int dev = 0;
  TRAIN_CK(cudaGetDevice(&dev), "cudaGetDevice");
  if (dev >= 64 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    TRAIN_CK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem), "cudaFuncSetAttribute(linear_kernel)");
    if (S::kMoveRegs) {                                      // the epilogue's warps would wait for registers that nobody brought
      cudaFuncAttributes fa;
      TRAIN_CK(cudaFuncGetAttributes(&fa, kernel), "cudaFuncGetAttributes(linear_kernel)");
      if (fa.numRegs * S::kThreads < S::kRegsAll) return record_cuda_failure(cudaErrorInvalidConfiguration, "registers of linear_kernel");
    }
    if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
  }
  q.box_a = OA == kOpK ? (uint32_t)std::min<int64_t>(kLinBM, ceil_div64(p.M, 8) * 8) : kLinBM;
  int rc = encode_map(&q.ta, p.a, OA == kOpK ? (int)q.box_a : kLinBK);
  if (rc != LQSGD_OK || (rc = encode_map(&q.tb, p.b, OB == kOpK ? S::kBNc : kLinBK)) != LQSGD_OK) return rc;
  const int sms = train_sm_count();
  if (sms < CG) return record_cuda_failure(cudaErrorInvalidDevice, "cudaDevAttrMultiProcessorCount");
  // Whole tiles may be dealt to any number of clusters; the others were cut for p.clusters (on a smaller card they run in turn).
  const int clusters = p.deal == kWhole ? (int)std::min<int64_t>((int64_t)p.tiles_m * p.tiles_n, sms / CG) : p.clusters;
  TRAIN_CK(train_launch(kernel, dim3((unsigned)(clusters * CG)), dim3(S::kThreads), S::kSmem, st, CG * p.meet, q), "linear_kernel launch");
  return LQSGD_OK;
}

// What lqsgd_test_linear_wait asked of this host thread's next product.
struct TestWait { uint32_t limit = 0, after = 0; int32_t role = kNoRole; };
thread_local TestWait test_wait;

int run(int product, const lqsgd_linear& a, LinEpilogue ep, cudaStream_t st) {
  const TestWait test = test_wait;
  test_wait = TestWait();
  Plan p;
  int rc = make_plan(product, a, &p);
  if (rc != LQSGD_OK) return rc;
  if (p.bytes) {
    if (!a.dev_workspace || a.workspace_bytes < p.bytes) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
    if (!train_aligned(a.dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
  }
  char* ws = static_cast<char*>(a.dev_workspace);
  if (p.unpacked) {
    p.b.base = ws + p.off_x;
    if ((rc = lqsgd_unpack8(&a.x8, a.rows, a.in, ws + p.off_x, p.b.ld, a.dtype, st)) != LQSGD_OK) return rc;
  }
  if ((rc = place(&p.a, ws, p.off_a, st)) != LQSGD_OK || (rc = place(&p.b, ws, p.off_b, st)) != LQSGD_OK) return rc;
  const int es = ep.dtype == LQSGD_F32 ? 4 : 2;
  auto rows_aligned = [](const void* ptr, int64_t bytes, size_t to) { return train_aligned(ptr, to) && bytes % (int64_t)to == 0; };
  auto rows_vec = [&](const void* q, int64_t ld) { return rows_aligned(q, ld, 32) ? 2 : rows_aligned(q, ld, 16) ? 1 : 0; };
  ep.vec_out = rows_vec(ep.out, ep.ld_out * es);
  ep.vec_res = rows_vec(ep.residual, ep.ld_res * 2);
  ep.vec_z8 = rows_vec(ep.z8.dev_codes, ep.z8.ld_codes);
  ep.vec_y8 = rows_vec(ep.y8.dev_codes, ep.y8.ld_codes);
  LinProblem q;
  std::memset(&q, 0, sizeof(q));
  q.ep = ep;
  q.partial = p.deal == kShares ? reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(ws + p.off_partial) + kPieceAlign - 1) & ~(uintptr_t)(kPieceAlign - 1)) : nullptr;
  q.M = (int32_t)p.M; q.N = (int32_t)p.N; q.K = (int32_t)p.K;
  q.tiles_m = p.tiles_m; q.tiles_n = p.tiles_n; q.kb_total = p.kb_total;
  q.deal = p.deal; q.share = p.share; q.meet = p.meet;
  q.first_chunk = pair_chunk(p.kb_total);
  q.dtype = a.dtype;
  q.status = a.dev_status;
  q.test_limit = test.limit; q.test_after = test.after; q.test_role = test.role;
  if (product == LQSGD_LINEAR_FORWARD)
    rc = p.cg == 2 ? launch<2, 256, kOpK, kOpK, false>(p, q, st) : launch<1, 128, kOpK, kOpK, false>(p, q, st);
  else if (product == LQSGD_LINEAR_GRAD_INPUT)
    rc = p.cg == 2 ? launch<2, 256, kOpK, kOpMN, false>(p, q, st) : launch<1, 128, kOpK, kOpMN, false>(p, q, st);
  else
    rc = p.cg == 2 ? launch<2, 256, kOpMN, kOpMN, true>(p, q, st) : launch<1, 128, kOpMN, kOpMN, true>(p, q, st);
  if (rc != LQSGD_OK) return rc;
  if (p.deal == kShares) {
    const int most = (int)((p.kb_total - 1) / p.share + 2);           // pieces of one tile
    const uint32_t tiles = (uint32_t)p.tiles_m * p.tiles_n, high = kLinBM * p.cg;
    uint32_t rows = 32;                                               // fewer per block until the card is full
    while (rows > (most >= 8 ? 1u : 8u) && tiles * (high / rows) < kSms * 4) rows /= 2;
    const LinPieces j = {q.partial, (uint32_t)p.tiles_m, (uint32_t)p.tiles_n, (uint32_t)p.kb_total, (uint32_t)p.share, (uint32_t)p.cg, (uint32_t)p.bn, rows};
    const dim3 grid(tiles * (high / rows));
    if (most >= 8) TRAIN_CK(train_launch(linear_join_kernel<8>, grid, dim3(256), 0, st, 1, j, ep), "linear_join_kernel launch");
    else TRAIN_CK(train_launch(linear_join_kernel<1>, grid, dim3(256), 0, st, 1, j, ep), "linear_join_kernel launch");
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

extern "C" int lqsgd_test_linear_wait(int32_t role, int32_t after, uint32_t wait_limit) {
  if (role < LQSGD_LINEAR_ROLE_LOADER || role > LQSGD_LINEAR_ROLE_MMA || after < 0 || wait_limit < 16 || wait_limit > kWaitLimit) return LQSGD_ERR_INVALID_ARG;
  test_wait.limit = wait_limit;
  test_wait.after = (uint32_t)after;
  test_wait.role = role;
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
