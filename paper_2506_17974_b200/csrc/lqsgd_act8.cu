// Activations kept in 8 bits: packing, unpacking, and the activation's backward step that reads them.
//
// All three are streams: each value is read once and written once, and what bounds them is HBM.  A thread owns 8
// consecutive columns (16 bytes of a 16-bit type, 8 bytes of codes) of a row, so four neighbouring lanes hold one group of
// 32 and agree on its exponent with two shuffles.  A warp covers `lanes` x 8 columns of 32 / lanes rows, lanes = 4 .. 32
// by the row length, so that short rows do not leave lanes idle.
#include "lqsgd_train_dev.cuh"

#include <algorithm>
#include <mutex>

namespace lqsgd {

int train_sm_count() {
  static std::mutex mu;
  static int cached[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  std::lock_guard<std::mutex> lock(mu);
  if (!cached[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    cached[dev] = n;
  }
  return cached[dev];
}

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kRun = 8;                      // columns per thread

// How a matrix is dealt out: warps of 32 / lanes rows x (8 lanes) columns; blockIdx.x = column segment, blockIdx.y = row block.
struct Deal {
  int64_t rows, rows_per_block;
  int32_t cols, lane_shift;                  // lanes = 1 << lane_shift
};
struct Spot {
  int64_t row, row_end, row_step;            // rows row, row + row_step, ... < row_end
  int col, have;                             // first column; how many of its 8 exist (<= 0: none)
};
__device__ __forceinline__ Spot spot_of(const Deal& d) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int lanes = 1 << d.lane_shift, sub = lane >> d.lane_shift, per_warp = 32 >> d.lane_shift;
  Spot s;
  s.col = ((int)blockIdx.x * lanes + (lane & (lanes - 1))) * kRun;
  s.have = min(kRun, d.cols - s.col);
  const int64_t first = (int64_t)blockIdx.y * d.rows_per_block;
  s.row = first + warp * per_warp + sub;
  s.row_end = min(d.rows, first + d.rows_per_block);
  s.row_step = kWarps * per_warp;
  return s;
}
Deal make_deal(int64_t rows, int32_t cols, int ctas_wanted, dim3* grid) {
  Deal d;
  d.rows = rows;
  d.cols = cols;
  d.lane_shift = 2;
  while (d.lane_shift < 5 && (8 << d.lane_shift) < cols) ++d.lane_shift;
  const int64_t segs = ceil_div64(cols, 8ll << d.lane_shift);
  const int64_t step = kWarps * (32 >> d.lane_shift);              // rows one pass of a block covers
  const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>({ceil_div64(rows, step), ceil_div64(ctas_wanted, segs), 65535}));
  d.rows_per_block = ceil_div64(ceil_div64(rows, blocks), step) * step;
  *grid = dim3((unsigned)segs, (unsigned)std::max<int64_t>(1, ceil_div64(rows, d.rows_per_block)));
  return d;
}

// Largest magnitude of the group of 32 columns that four neighbouring lanes hold, as its bit pattern: for numbers without
// sign the order of the patterns is the order of the values, and NaN comes out on top.
__device__ __forceinline__ float group_top(const float (&v)[kRun]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  return __uint_as_float(top);
}
__device__ __forceinline__ void store_codes(uint8_t* p, bool vec, int have, uint2 w) {
  if (vec) {
    *reinterpret_cast<uint2*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      if (j < have) p[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
  }
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* __restrict__ p, bool vec, int have) {
  if (vec) return *reinterpret_cast<const uint2*>(p);
  uint2 w = make_uint2(0u, 0u);
#pragma unroll
  for (int j = 0; j < kRun; ++j)
    if (j < have) (j < 4 ? w.x : w.y) |= (uint32_t)p[j] << (8 * (j & 3));
  return w;
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
pack8_kernel(Deal d, const void* __restrict__ x, int64_t ld_x, bool vec_x, lqsgd_packed8 out, bool vec_c) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  const Spot s = spot_of(d);
  const int sub = (threadIdx.x & 31) >> d.lane_shift;
  // a warp whose last rows lie past the end stays together for the shuffles: those lanes hold zeros and store nothing
  for (int64_t r0 = s.row; r0 - sub < s.row_end; r0 += s.row_step) {
    const bool on = r0 < s.row_end && s.have > 0;
    float v[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = 0.f;
    if (on) load_run<DT, kRun>(static_cast<const T*>(x) + r0 * ld_x + s.col, vec_x && s.have == kRun, s.have, v);
    const int eb = exp_byte(group_top(v));
    const float inv = inv_step(eb);
    if (on) {
      const uint2 w = make_uint2(code_word(v[0], v[1], v[2], v[3], inv), code_word(v[4], v[5], v[6], v[7], inv));
      store_codes(out.dev_codes + r0 * out.ld_codes + s.col, vec_c && s.have == kRun, s.have, w);
      if ((s.col & (kGroup - 1)) == 0) out.dev_exps[r0 * out.ld_exps + s.col / kGroup] = (uint8_t)eb;
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
unpack8_kernel(Deal d, lqsgd_packed8 in, bool vec_c, void* __restrict__ y, int64_t ld_y, bool vec_y) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  const Spot s = spot_of(d);
  if (s.have <= 0) return;
  for (int64_t r = s.row; r < s.row_end; r += s.row_step) {
    const uint2 w = load_codes(in.dev_codes + r * in.ld_codes + s.col, vec_c && s.have == kRun, s.have);
    const float step = step_of(in.dev_exps[r * in.ld_exps + s.col / kGroup]);
    float v[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      v[j] = decode8((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255u, step);
      // only sources wider than the target can exceed its range: the largest finite value then (a NaN stays)
      constexpr float kTop = DT == LQSGD_F16 ? 65504.f : (DT == LQSGD_BF16 ? 3.3895314e38f : 3.402823466e38f);
      if (fabsf(v[j]) > kTop) v[j] = copysignf(kTop, v[j]);
    }
    store_run<DT, kRun>(static_cast<T*>(y) + r * ld_y + s.col, vec_y && s.have == kRun, s.have, v);
  }
}

// dz = dy act'(z); the block's column sums of dz go to partial[blockIdx.y][cols].
template <int DT>
__global__ void __launch_bounds__(kThreads)
act_grad_kernel(Deal d, const void* dy, int64_t ld_dy, bool vec_dy, lqsgd_packed8 z8, bool vec_c, int act,
                void* dz, int64_t ld_dz, bool vec_dz, float* __restrict__ partial) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  __shared__ float sums[kWarps][32][kRun + 1];
  const Spot s = spot_of(d);
  float acc[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) acc[j] = 0.f;
  if (s.have > 0)
    for (int64_t r = s.row; r < s.row_end; r += s.row_step) {
      float g[kRun];
      load_run<DT, kRun>(static_cast<const T*>(dy) + r * ld_dy + s.col, vec_dy && s.have == kRun, s.have, g);
      if (act != LQSGD_ACT_NONE) {
        const uint2 w = load_codes(z8.dev_codes + r * z8.ld_codes + s.col, vec_c && s.have == kRun, s.have);
        const float step = step_of(z8.dev_exps[r * z8.ld_exps + s.col / kGroup]);
        float z[kRun];
#pragma unroll
        for (int j = 0; j < kRun; ++j) z[j] = decode8((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255u, step);
        slope_run(act, z);
#pragma unroll
        for (int j = 0; j < kRun; ++j) g[j] *= z[j];
      }
      if (dz) store_run<DT, kRun>(static_cast<T*>(dz) + r * ld_dz + s.col, vec_dz && s.have == kRun, s.have, g);
#pragma unroll
      for (int j = 0; j < kRun; ++j) acc[j] += g[j];
    }
  if (!partial) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int j = 0; j < kRun; ++j) sums[warp][lane][j] = acc[j];
  __syncthreads();
  const int lanes = 1 << d.lane_shift;
  for (int c = threadIdx.x; c < lanes * kRun; c += kThreads) {
    const int col = (int)blockIdx.x * lanes * kRun + c;
    if (col >= d.cols) continue;
    float t = 0.f;
    for (int w = 0; w < kWarps; ++w)
      for (int sub = 0; sub < (32 >> d.lane_shift); ++sub) t += sums[w][(sub << d.lane_shift) + c / kRun][c % kRun];
    partial[(size_t)blockIdx.y * d.cols + col] = t;
  }
}

// out[c] = sum over b of partial[b][c], 32 columns x 8 threads per block, fixed order.
__global__ void __launch_bounds__(kThreads)
join_columns_kernel(const float* __restrict__ partial, int blocks, int cols, float* __restrict__ out) {
  train_pdl_wait();
  __shared__ float part[kWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 32 + lane;
  float t = 0.f;
  if (col < cols)
    for (int b = warp; b < blocks; b += kWarps) t += partial[(size_t)b * cols + col];
  part[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && col < cols) {
    float u = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) u += part[w][lane];
    out[col] = u;
  }
}

// CTAs that fill the card: 148 SMs x 8 blocks of 256 threads.  A constant, so that the order of the sums (and the
// workspace) depends on the sizes alone.
constexpr int kCtas = 148 * 8;

int check_matrix(int64_t rows, int32_t cols) {
  return rows < 0 || cols < 1 || rows > (int64_t)1 << 40 ? LQSGD_ERR_BAD_SHAPE : LQSGD_OK;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

#define BY_DTYPE(dtype, kernel, ...)                                               \
  ((dtype) == LQSGD_BF16 ? train_launch(kernel<LQSGD_BF16>, __VA_ARGS__)           \
   : (dtype) == LQSGD_F16 ? train_launch(kernel<LQSGD_F16>, __VA_ARGS__)           \
                          : train_launch(kernel<LQSGD_F32>, __VA_ARGS__))

static bool vec_rows(const void* p, int64_t ld, int elem, int bytes) {
  return train_aligned(p, bytes) && (ld * elem) % bytes == 0;
}

extern "C" int lqsgd_pack8(const void* dev_x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t cols,
                           const lqsgd_packed8* host_out, void* cuda_stream) {
  if (!host_out || !train_dtype_ok(dtype)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_matrix(rows, cols);
  if (rc != LQSGD_OK) return rc;
  if (rows == 0) return LQSGD_OK;
  if (!dev_x || ld_x < cols) return LQSGD_ERR_INVALID_ARG;
  if ((rc = check_packed8(*host_out, cols)) != LQSGD_OK) return rc;
  const int es = train_elem(dtype);
  if (!train_aligned(dev_x, es)) return LQSGD_ERR_MISALIGNED;
  dim3 grid;
  const Deal d = make_deal(rows, cols, kCtas, &grid);
  const bool vx = vec_rows(dev_x, ld_x, es, 16), vc = vec_rows(host_out->dev_codes, host_out->ld_codes, 1, 8);
  TRAIN_CK(BY_DTYPE(dtype, pack8_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, dev_x, ld_x, vx, *host_out, vc), "pack8_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_unpack8(const lqsgd_packed8* host_in, int64_t rows, int32_t cols, void* dev_y, int64_t ld_y,
                             int32_t dtype, void* cuda_stream) {
  if (!host_in || !train_dtype_ok(dtype)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_matrix(rows, cols);
  if (rc != LQSGD_OK) return rc;
  if (rows == 0) return LQSGD_OK;
  if (!dev_y || ld_y < cols) return LQSGD_ERR_INVALID_ARG;
  if ((rc = check_packed8(*host_in, cols)) != LQSGD_OK) return rc;
  const int es = train_elem(dtype);
  if (!train_aligned(dev_y, es)) return LQSGD_ERR_MISALIGNED;
  dim3 grid;
  const Deal d = make_deal(rows, cols, kCtas, &grid);
  const bool vy = vec_rows(dev_y, ld_y, es, 16), vc = vec_rows(host_in->dev_codes, host_in->ld_codes, 1, 8);
  TRAIN_CK(BY_DTYPE(dtype, unpack8_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, *host_in, vc, dev_y, ld_y, vy), "unpack8_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_act_grad_workspace_bytes(int64_t rows, int32_t cols, size_t* host_bytes_out) {
  if (!host_bytes_out) return LQSGD_ERR_INVALID_ARG;
  const int rc = check_matrix(rows, cols);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = 0;
  if (rows == 0) return LQSGD_OK;
  dim3 grid;
  make_deal(rows, cols, kCtas, &grid);
  *host_bytes_out = grid.y > 1 ? (size_t)grid.y * cols * sizeof(float) : 0;
  return LQSGD_OK;
}

extern "C" int lqsgd_act_grad(const void* dev_dy, int64_t ld_dy, const lqsgd_packed8* host_z8, int32_t act, int32_t dtype,
                              int64_t rows, int32_t cols, void* dev_dz, int64_t ld_dz, float* dev_db, void* dev_workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  if (!train_dtype_ok(dtype) || !train_act_ok(act)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_matrix(rows, cols);
  if (rc != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!train_aligned(dev_db, 4)) return LQSGD_ERR_MISALIGNED;
  if (rows == 0) {
    if (dev_db) TRAIN_CK(cudaMemsetAsync(dev_db, 0, (size_t)cols * sizeof(float), st), "cudaMemsetAsync(db)");
    return LQSGD_OK;
  }
  if (!dev_dz && (!dev_db || act != LQSGD_ACT_NONE)) return LQSGD_ERR_INVALID_ARG;
  if (!dev_dy || ld_dy < cols || (dev_dz && ld_dz < cols)) return LQSGD_ERR_INVALID_ARG;
  lqsgd_packed8 z8 = {};
  if (act != LQSGD_ACT_NONE) {
    if (!host_z8) return LQSGD_ERR_INVALID_ARG;
    z8 = *host_z8;
    if ((rc = check_packed8(z8, cols)) != LQSGD_OK) return rc;
  }
  const int es = train_elem(dtype);
  if (!train_aligned(dev_dy, es) || !train_aligned(dev_dz, es)) return LQSGD_ERR_MISALIGNED;
  dim3 grid;
  const Deal d = make_deal(rows, cols, kCtas, &grid);
  float* partial = dev_db;
  if (dev_db && grid.y > 1) {
    if (!dev_workspace || workspace_bytes < (size_t)grid.y * cols * sizeof(float)) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
    if (!train_aligned(dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
    partial = static_cast<float*>(dev_workspace);
  }
  TRAIN_CK(BY_DTYPE(dtype, act_grad_kernel, grid, dim3(kThreads), 0, st, 1, d, dev_dy, ld_dy, vec_rows(dev_dy, ld_dy, es, 16), z8,
                    vec_rows(z8.dev_codes, z8.ld_codes, 1, 8), act, dev_dz, ld_dz, vec_rows(dev_dz, ld_dz, es, 16), partial),
           "act_grad_kernel launch");
  if (partial != dev_db)
    TRAIN_CK(train_launch(join_columns_kernel, dim3((cols + 31) / 32), dim3(kThreads), 0, st, 1, partial, (int)grid.y, cols, dev_db), "join_columns_kernel launch");
  return LQSGD_OK;
}
