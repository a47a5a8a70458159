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
template <uint32_t WAYS, int KIND>
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
        v[0] = add_sums<KIND>(v[0], s.x); v[1] = add_sums<KIND>(v[1], s.y); v[2] = add_sums<KIND>(v[2], s.z); v[3] = add_sums<KIND>(v[3], s.w);
      }
    }
    if (WAYS > 1) {
      sums[warp][lane] = make_float4(v[0], v[1], v[2], v[3]);
      __syncthreads();
      if (sub == 0)
        for (uint32_t k = 1; k < WAYS; ++k) {
          const float4 s = sums[warp + k][lane];
          v[0] = add_sums<KIND>(v[0], s.x); v[1] = add_sums<KIND>(v[1], s.y); v[2] = add_sums<KIND>(v[2], s.z); v[3] = add_sums<KIND>(v[3], s.w);
        }
      __syncthreads();
    }
    if (mine && sub == 0) finish_quad<KIND>(e, row, n_tile * q.bn + strip * 128 + 4 * lane, v);
  }
}

// Copies a matrix whose rows TMA cannot address (base or row distance not a multiple of 16 bytes) to rows of ld_dst elements, a
// multiple of 16 bytes, zeros past cols; what lies past cols is never read.  A warp takes 512 bytes of a row at a time, a thread
// 16 of them: words where the row starts on one, else the elements (T: of 16 or of 8 bits).
constexpr int kRealignBytes = 512;
template <typename T>
__global__ void __launch_bounds__(256)
realign_kernel(const T* __restrict__ src, int64_t ld_src, int64_t rows, int cols, T* __restrict__ dst, int64_t ld_dst) {
  train_pdl_wait();
  const int lane = threadIdx.x & 31, kEach = 16 / (int)sizeof(T), strips = (cols + 32 * kEach - 1) / (32 * kEach), warps = (int)gridDim.x * 8;
  const int first = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
  int strip = first % strips;
  for (int64_t row = first / strips; row < rows; row += warps / strips) {
    const int col = (strip * 32 + lane) * kEach, have = cols - col;
    if (have > 0) {
      const T* s = src + row * ld_src + col;
      uint32_t w[4];
      if (have >= kEach && (reinterpret_cast<uintptr_t>(s) & 3) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t*>(s) + i);
      } else {
        uint32_t h[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) h[i] = i < have ? __ldg(s + i) : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = 0;
#pragma unroll
          for (int j = 0; j < kEach / 4; ++j) w[i] |= h[kEach / 4 * i + j] << (8 * (int)sizeof(T) * j);
        }
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
// One operand as it lies in memory, values of `elem` bytes.
struct Stored {
  const void* base = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
  int elem = 2;
  int64_t aligned_ld() const { return ceil_div64(cols * elem, 16) * 16 / elem; }
  // One row needs no row distance.
  bool tma_ready() const { return train_aligned(base, 16) && (rows == 1 || ld * elem % 16 == 0); }
  size_t copy_bytes() const { return tma_ready() ? 0 : (size_t)rows * aligned_ld() * elem; }
};
// Map over an operand: boxes of 128 bytes (64 columns, 128 of 8 bits) x box_rows, 128-byte swizzle, zeros outside.
int encode_map(CUtensorMap* map, const Stored& s, int box_rows) {
  EncodeFn fn = tensor_map_encoder();
  if (!fn) return record_cuda_failure(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
  const cuuint64_t dim[2] = {(cuuint64_t)s.cols, (cuuint64_t)s.rows};
  const cuuint64_t stride[1] = {(cuuint64_t)(s.rows == 1 ? s.aligned_ld() : s.ld) * (cuuint64_t)s.elem};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / s.elem), (cuuint32_t)box_rows}, es[2] = {1, 1};
  if (fn(map, s.elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(s.base), dim, stride, box, es,
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

int deal_out(Plan p, int bk, Plan* out);
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
  return deal_out(p, kLinBK, out);
}
int make_plan(const lqsgd_linear_rows8& a, Plan* out) {
  Plan p = {};
  p.a = {a.x.dev_codes, a.rows, a.in, a.x.ld_codes, 1};
  p.b = {a.w.dev_codes, a.out, a.in, a.w.ld_codes, 1};
  p.M = a.rows; p.N = a.out; p.K = a.in;
  return deal_out(p, lin_bk<kInt8>(), out);
}
// Tiles and shares for the operands and sizes that p has; bk: k per block.
int deal_out(Plan p, int bk, Plan* out) {
  p.kb_total = (int)ceil_div64(p.K, bk);
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
  if (p.unpacked) p.off_x = room((size_t)p.b.rows * p.b.ld * 2);
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
  const int64_t blocks = std::min<int64_t>(ceil_div64(s->rows * ceil_div64(s->cols * s->elem, kRealignBytes), 8), kSms * 8);
  if (s->elem == 1)
    TRAIN_CK(train_launch(realign_kernel<uint8_t>, dim3((unsigned)blocks), dim3(256), 0, st, 1, static_cast<const uint8_t*>(s->base), s->ld, s->rows,
                          (int)s->cols, reinterpret_cast<uint8_t*>(ws + off), ld), "realign_kernel launch");
  else
    TRAIN_CK(train_launch(realign_kernel<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, st, 1, static_cast<const uint16_t*>(s->base), s->ld, s->rows,
                          (int)s->cols, reinterpret_cast<uint16_t*>(ws + off), ld), "realign_kernel launch");
  s->base = ws + off;
  s->ld = ld;
  return LQSGD_OK;
}

template <int CG, int BN, int OA, int OB, bool WF32, int KIND = kHalf>
int launch(const Plan& p, LinProblem& q, cudaStream_t st) {
  using S = LinCfg<CG, BN, OA, OB, WF32, KIND>;
  auto kernel = linear_kernel<CG, BN, OA, OB, WF32, KIND>;
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

// What both forms of a product share: checks of the workspace `ws`, aligned copies, the kernel (started by `go`) and the join of pieces.
template <int KIND, typename Go>
int run_plan(Plan p, LinEpilogue ep, int dtype, uint32_t* status, char* ws, cudaStream_t st, Go&& go) {
  const TestWait test = test_wait;
  test_wait = TestWait();
  int rc;
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
  q.dtype = dtype;
  q.status = status;
  q.test_limit = test.limit; q.test_after = test.after; q.test_role = test.role;
  if ((rc = go(p, q)) != LQSGD_OK) return rc;
  if (p.deal == kShares) {
    const int most = (int)((p.kb_total - 1) / p.share + 2);           // pieces of one tile
    const uint32_t tiles = (uint32_t)p.tiles_m * p.tiles_n, high = kLinBM * p.cg;
    uint32_t rows = 32;                                               // fewer per block until the card is full
    while (rows > (most >= 8 ? 1u : 8u) && tiles * (high / rows) < kSms * 4) rows /= 2;
    const LinPieces j = {q.partial, (uint32_t)p.tiles_m, (uint32_t)p.tiles_n, (uint32_t)p.kb_total, (uint32_t)p.share, (uint32_t)p.cg, (uint32_t)p.bn, rows};
    const dim3 grid(tiles * (high / rows));
    if (most >= 8) TRAIN_CK(train_launch(linear_join_kernel<8, KIND>, grid, dim3(256), 0, st, 1, j, ep), "linear_join_kernel launch");
    else TRAIN_CK(train_launch(linear_join_kernel<1, KIND>, grid, dim3(256), 0, st, 1, j, ep), "linear_join_kernel launch");
  }
  return LQSGD_OK;
}
int check_workspace(const Plan& p, const void* ws, size_t bytes) {
  if (!p.bytes) return LQSGD_OK;
  if (!ws || bytes < p.bytes) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
  return train_aligned(ws, 16) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}

int run(int product, const lqsgd_linear& a, const LinEpilogue& ep, cudaStream_t st) {
  Plan p;
  int rc = make_plan(product, a, &p);
  if (rc == LQSGD_OK) rc = check_workspace(p, a.dev_workspace, a.workspace_bytes);
  char* ws = static_cast<char*>(a.dev_workspace);
  if (rc == LQSGD_OK && p.unpacked) {
    p.b.base = ws + p.off_x;
    rc = lqsgd_unpack8(&a.x8, a.rows, a.in, ws + p.off_x, p.b.ld, a.dtype, st);
  }
  if (rc != LQSGD_OK) {
    test_wait = TestWait();
    return rc;
  }
  return run_plan<kHalf>(p, ep, a.dtype, a.dev_status, ws, st, [&](const Plan& plan, LinProblem& q) {
    if (product == LQSGD_LINEAR_FORWARD)
      return plan.cg == 2 ? launch<2, 256, kOpK, kOpK, false>(plan, q, st) : launch<1, 128, kOpK, kOpK, false>(plan, q, st);
    if (product == LQSGD_LINEAR_GRAD_INPUT)
      return plan.cg == 2 ? launch<2, 256, kOpK, kOpMN, false>(plan, q, st) : launch<1, 128, kOpK, kOpMN, false>(plan, q, st);
    return plan.cg == 2 ? launch<2, 256, kOpMN, kOpMN, true>(plan, q, st) : launch<1, 128, kOpMN, kOpMN, true>(plan, q, st);
  });
}
int run_few(const lqsgd_linear_rows8& a, const LinEpilogue& ep, cudaStream_t st);
bool few_rows(const lqsgd_linear_rows8& a);
int run(const lqsgd_linear_rows8& a, const LinEpilogue& ep, cudaStream_t st) {
  if (few_rows(a)) {
    test_wait = TestWait();
    return run_few(a, ep, st);
  }
  Plan p;
  int rc = make_plan(a, &p);
  if (rc == LQSGD_OK) rc = check_workspace(p, a.dev_workspace, a.workspace_bytes);
  if (rc != LQSGD_OK) {
    test_wait = TestWait();
    return rc;
  }
  return run_plan<kInt8>(p, ep, a.dtype, a.dev_status, static_cast<char*>(a.dev_workspace), st, [&](const Plan& plan, LinProblem& q) {
    return plan.cg == 2 ? launch<2, 256, kOpK, kOpK, false, kInt8>(plan, q, st) : launch<1, 128, kOpK, kOpK, false, kInt8>(plan, q, st);
  });
}

// ---- products of codes for one or two rows (a token between two layers): w is read once, and its bytes are all that the call costs.  The tensor
// cores' tile fills 128 of the SMs for 16384 channels and starts with a tensor map, tensor memory and a first copy's latency; plain wide
// loads of w, straight into integer dot products of four codes, start at once and fill the card: 1 x 4096 x 16384 in 14.2 us (4.7 TB/s)
// against 15.6 on the tensor cores, 1 x 512 x 10 in 1.7 against 5.  With four rows the dot products take longer than the loads (25 us against
// 15.8).  A warp takes four channels, so that a piece of x is loaded once for them; where there are few channels, several warps of a
// block share the terms of a sum.
constexpr int kFewRows = 2, kFewChannels = 4;
template <int R>
__global__ void __launch_bounds__(256)
rows8_few_kernel(const int8_t* __restrict__ x, int64_t ld_x, const int8_t* __restrict__ w, int64_t ld_w, int cin, int ksplit, const __grid_constant__ LinEpilogue e) {
  __shared__ int parts[8][R * kFewChannels];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = warp % ksplit, group = warp / ksplit, channel0 = ((int)blockIdx.x * ((int)(blockDim.x >> 5) / ksplit) + group) * kFewChannels;
  train_pdl_wait();
  int acc[R][kFewChannels] = {};
  const int pieces = cin / 16;
  const int8_t* wr[kFewChannels];
#pragma unroll
  for (int c = 0; c < kFewChannels; ++c) wr[c] = w + (int64_t)min(channel0 + c, e.cols - 1) * ld_w;      // channels past the last are not written
#pragma unroll 4
  for (int k = part * 32 + lane; k < pieces; k += 32 * ksplit) {
    int4 a[R], b[kFewChannels];
#pragma unroll
    for (int c = 0; c < kFewChannels; ++c) b[c] = __ldg(reinterpret_cast<const int4*>(wr[c]) + k);
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = r < e.rows ? __ldg(reinterpret_cast<const int4*>(x + r * ld_x) + k) : make_int4(0, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < kFewChannels; ++c)
        acc[r][c] = __dp4a(a[r].w, b[c].w, __dp4a(a[r].z, b[c].z, __dp4a(a[r].y, b[c].y, __dp4a(a[r].x, b[c].x, acc[r][c]))));
  }
  const int k = pieces * 16 + lane;                                       // the last piece, if it is not whole
  if (part == 0 && lane < 16 && k < cin) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < kFewChannels; ++c)
        if (r < e.rows) acc[r][c] += (int)x[r * ld_x + k] * (int)wr[c][k];
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int c = 0; c < kFewChannels; ++c) {
      acc[r][c] = __reduce_add_sync(0xffffffffu, acc[r][c]);
      if (ksplit > 1 && lane == 0) parts[warp][r * kFewChannels + c] = acc[r][c];
    }
  if (ksplit > 1) {
    __syncthreads();
    if (part != 0) return;
  }
  if (lane >= R * kFewChannels) return;
  const int r = lane / kFewChannels, c = lane % kFewChannels, channel = channel0 + c;
  if (r >= e.rows || channel >= e.cols) return;
  int sum = 0;
  if (ksplit > 1) {
    for (int p = 0; p < ksplit; ++p) sum += parts[warp + p][lane];
  } else {
#pragma unroll
    for (int i = 0; i < R * kFewChannels; ++i)
      if (i == lane) sum = acc[i / kFewChannels][i % kFewChannels];
  }
  float v[2] = {finish_sum(sum, __ldg(e.row_scale + r), __ldg(e.col_scale + channel), e.bias ? __ldg(e.bias + channel) : 0.f), 0.f};
  act_pairs(e.act, v);
  if (e.residual) v[0] = add_residual<kInt8>(v[0], unpack1(e.dtype, static_cast<const uint16_t*>(e.residual)[r * e.ld_res + channel]));
  static_cast<uint16_t*>(e.out)[r * e.ld_out + channel] = pack1(e.dtype, v[0]);
}
// Whether the call takes that way: rows on 16 bytes, and no copies in 8 bits (their groups of 32 channels span warps).
bool few_rows(const lqsgd_linear_rows8& a) {
  return a.rows <= kFewRows && !a.z8.dev_codes && !a.y8.dev_codes && train_aligned(a.x.dev_codes, 16) && train_aligned(a.w.dev_codes, 16) &&
         (a.rows == 1 || a.x.ld_codes % 16 == 0) && (a.out == 1 || a.w.ld_codes % 16 == 0);
}
int run_few(const lqsgd_linear_rows8& a, const LinEpilogue& ep, cudaStream_t st) {
  const int64_t warps = ceil_div64(a.out, kFewChannels);
  // Warps that share a sum: until the card has four a scheduler, or a lane two pieces of it (1 x 4096 x 4096: 10.7 us with one, 5.1 so; eight
  // pieces a lane 10.7, one 6.2).
  int ksplit = 1;
  while (ksplit < 8 && warps * ksplit < kSms * 16 && a.in > 32 * 16 * 2 * ksplit) ksplit *= 2;
  const int together = std::max(4, ksplit);                               // warps of a block: small ones deal out evenly
  const dim3 grid((unsigned)ceil_div64(warps, together / ksplit));
  auto go = [&](auto kernel) { return train_launch(kernel, grid, dim3(32 * together), 0, st, 1, a.x.dev_codes, a.x.ld_codes, a.w.dev_codes, a.w.ld_codes, a.in, ksplit, ep); };
  TRAIN_CK(a.rows == 1 ? go(rows8_few_kernel<1>) : go(rows8_few_kernel<2>), "rows8_few_kernel launch");
  return LQSGD_OK;
}

int check_rows8_args(const lqsgd_linear_rows8* a) {
  if (!a || a->struct_size != sizeof(lqsgd_linear_rows8)) return LQSGD_ERR_INVALID_ARG;
  if ((a->dtype != LQSGD_BF16 && a->dtype != LQSGD_F16) || !train_act_ok(a->act) || a->reserved) return LQSGD_ERR_INVALID_ARG;
  // 128^2 terms of at most 131071 stay below 2^31
  if (a->rows < 0 || a->rows > 0x7fffffffll - 511 || a->in < 1 || a->out < 1 || a->in > 131071 || a->out > (1 << 24)) return LQSGD_ERR_BAD_SHAPE;
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

extern "C" int lqsgd_linear_rows8_workspace_bytes(const lqsgd_linear_rows8* host_args, size_t* host_bytes_out) {
  if (!host_bytes_out) return LQSGD_ERR_INVALID_ARG;
  int rc = check_rows8_args(host_args);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = 0;
  if (host_args->rows == 0 || few_rows(*host_args)) return LQSGD_OK;
  Plan p;
  if ((rc = make_plan(*host_args, &p)) != LQSGD_OK) return rc;
  *host_bytes_out = p.bytes;
  return LQSGD_OK;
}

extern "C" int lqsgd_linear_rows8_forward(const lqsgd_linear_rows8* a, void* cuda_stream) {
  int rc = check_rows8_args(a);
  if (rc != LQSGD_OK) return rc;
  if (a->rows == 0) return LQSGD_OK;
  if ((rc = check_rows8(a->x, a->in)) != LQSGD_OK || (rc = check_rows8(a->w, a->in)) != LQSGD_OK || (rc = check_matrix(a->dev_out, a->ld_out, a->out, 2)) != LQSGD_OK)
    return rc;
  if (a->dev_residual && (rc = check_matrix(a->dev_residual, a->ld_residual, a->out, 2)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_bias, 4) || !train_aligned(a->dev_status, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->z8.dev_codes && (rc = check_packed8(a->z8, a->out)) != LQSGD_OK) return rc;
  if (a->y8.dev_codes && (rc = check_packed8(a->y8, a->out)) != LQSGD_OK) return rc;
  LinEpilogue ep = {};
  ep.out = a->dev_out; ep.ld_out = a->ld_out; ep.bias = a->dev_bias;
  ep.row_scale = a->x.dev_scales; ep.col_scale = a->w.dev_scales;
  ep.residual = a->dev_residual; ep.ld_res = a->ld_residual;
  ep.z8 = a->z8; ep.y8 = a->y8;
  ep.rows = (int32_t)a->rows; ep.cols = a->out; ep.dtype = a->dtype; ep.act = a->act;
  return run(*a, ep, static_cast<cudaStream_t>(cuda_stream));
}
