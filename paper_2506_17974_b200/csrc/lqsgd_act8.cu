// Activations kept in 8 bits: packing, unpacking, and the activation's backward step that reads them.
//
// All three are streams: each value is read once and written once, and what bounds them is HBM.  A thread works on runs of 8
// consecutive columns of a row, so four neighbouring lanes hold one group of 32 and agree on its exponent with two
// shuffles.  A warp covers `lanes` x 8 columns of 32 / lanes rows, lanes = 4 .. 32 by the row length, so that short rows do
// not leave lanes idle.  Rows of 16-byte pieces are read and written as such (RUNS).  Rows at any other alignment are
// read and written 32 neighbouring elements at a time, a lane each (a run of 8 taken element by element touches 32
// places instead), and turned between the two forms in shared memory: 1021 x 25087 in fp32 packs in 26 us so and unpacks in 20,
// where runs taken element by element took 39 and 35.
// A thread takes several rows at a time, all their loads first: one row in flight per thread does not fill HBM's latency.
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

// How a matrix is dealt out: a warp takes 32 / lanes rows x (8 lanes) columns; a block's 8 warps stand 1 << wide_shift side by
// side (up to four: a block then reads two kilobytes of a row, which HBM serves up to 1.6 times faster than the same bytes
// from many rows) and the rest below one another; blockIdx.x = column segment, blockIdx.y = row block.
struct Deal {
  int64_t rows, rows_per_block;
  int32_t cols, lane_shift, wide_shift;      // lanes = 1 << lane_shift
};
struct Spot {
  int64_t row, row_end, row_step;            // rows row, row + row_step, ... < row_end
  int col, have;                             // first column of the run; how many of its 8 exist (<= 0: none)
  int side;                                  // the warp's first column + lane: columns side, side + 32, ... of the other form
  int sub;                                   // which of the warp's rows
  __device__ __forceinline__ explicit Spot(const Deal& d) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int lanes = 1 << d.lane_shift, per_warp = 32 >> d.lane_shift;
    sub = lane >> d.lane_shift;
    const int seg = ((((int)blockIdx.x << d.wide_shift) + (warp & ((1 << d.wide_shift) - 1))) << d.lane_shift) * kRun;
    col = seg + (lane & (lanes - 1)) * kRun;
    have = min(kRun, d.cols - col);
    side = seg + lane;
    const int64_t first = (int64_t)blockIdx.y * d.rows_per_block;
    row = first + (warp >> d.wide_shift) * per_warp + sub;
    row_end = min(d.rows, first + d.rows_per_block);
    row_step = (kWarps >> d.wide_shift) * per_warp;
  }
};
Deal make_deal(int64_t rows, int32_t cols, bool runs, int ctas_wanted, int64_t least_rows, dim3* grid) {
  Deal d;
  d.rows = rows;
  d.cols = cols;
  d.lane_shift = runs ? 2 : 5;
  while (d.lane_shift < 5 && (8 << d.lane_shift) < cols) ++d.lane_shift;
  d.wide_shift = 0;
  while (d.wide_shift < 2 && (8ll << (d.lane_shift + d.wide_shift)) < cols) ++d.wide_shift;
  const int64_t segs = ceil_div64(cols, 8ll << (d.lane_shift + d.wide_shift));
  const int64_t step = (kWarps >> d.wide_shift) * (32 >> d.lane_shift);   // rows one pass of a block covers
  const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>({ceil_div64(rows, step * least_rows), ceil_div64(ctas_wanted, segs), 65535}));
  d.rows_per_block = ceil_div64(ceil_div64(rows, blocks), step) * step;
  *grid = dim3((unsigned)segs, (unsigned)std::max<int64_t>(1, ceil_div64(rows, d.rows_per_block)));
  return d;
}
// Runs where the values have 16-byte pieces, or where the rows are too short for a warp's 256 columns.
bool use_runs(bool vec, int32_t cols) { return vec || cols <= 128; }

// Raw pieces, so that several rows' loads can be outstanding before any is converted.
template <int DT> struct Piece { uint32_t w[kRun * sizeof(typename Elem<DT>::T) / 4]; };
// row: the row's first element.  What does not exist reads as 0.
template <int DT, bool RUNS>
__device__ __forceinline__ void load_piece(const typename Elem<DT>::T* row, const Spot& s, int cols, bool vec, Piece<DT>& out) {
  using T = typename Elem<DT>::T;
  T* t = reinterpret_cast<T*>(out.w);
  if (!RUNS) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) t[j] = s.side + 32 * j < cols ? row[s.side + 32 * j] : Elem<DT>::down(0.f);
  } else if (vec) {
#pragma unroll
    for (int i = 0; i < kRun * (int)sizeof(T) / 16; ++i) *reinterpret_cast<uint4*>(out.w + 4 * i) = reinterpret_cast<const uint4*>(row + s.col)[i];
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j) t[j] = j < s.have ? row[s.col + j] : Elem<DT>::down(0.f);
  }
}
// The run as floats; `turn` is the warp's 256 elements of shared memory (unused with RUNS).
template <int DT, bool RUNS>
__device__ __forceinline__ void open_piece(const Piece<DT>& in, typename Elem<DT>::T* turn, float (&v)[kRun]) {
  using T = typename Elem<DT>::T;
  const T* t = reinterpret_cast<const T*>(in.w);
  if (RUNS) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = Elem<DT>::up(t[j]);
  } else {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < kRun; ++j) turn[32 * j + lane] = t[j];
    __syncwarp();
    load_run<DT, kRun>(turn + kRun * lane, true, kRun, v);
    __syncwarp();
  }
}
template <int DT, bool RUNS>
__device__ __forceinline__ void store_piece(typename Elem<DT>::T* row, const Spot& s, int cols, bool vec, typename Elem<DT>::T* turn, const float (&v)[kRun]) {
  if (RUNS) {
    store_run<DT, kRun>(row + s.col, vec, s.have, v);
  } else {
    const int lane = threadIdx.x & 31;
    store_run<DT, kRun>(turn + kRun * lane, true, kRun, v);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      if (s.side + 32 * j < cols) row[s.side + 32 * j] = turn[32 * j + lane];
    __syncwarp();
  }
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
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, bool vec, int have) {
  if (vec) return *reinterpret_cast<const uint2*>(p);
  uint2 w = make_uint2(0u, 0u);
#pragma unroll
  for (int j = 0; j < kRun; ++j)
    if (j < have) (j < 4 ? w.x : w.y) |= (uint32_t)p[j] << (8 * (j & 3));
  return w;
}

template <int DT, bool RUNS>
__global__ void __launch_bounds__(kThreads)
pack8_kernel(Deal d, const void* __restrict__ x, int64_t ld_x, bool vec_x, lqsgd_packed8 out, bool vec_c) {
  constexpr int kRows = DT == LQSGD_F32 ? 2 : 4;
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turn[RUNS ? 1 : kWarps][RUNS ? 8 : 256];
  train_pdl_wait();
  const Spot s(d);
  const bool vx = vec_x && s.have == kRun, vc = vec_c && s.have == kRun;
  T* mine = turn[RUNS ? 0 : threadIdx.x >> 5];
  // a warp whose last rows lie past the end stays together for the shuffles: those lanes hold zeros and store nothing
  for (int64_t r0 = s.row; r0 - s.sub < s.row_end; r0 += kRows * s.row_step) {
    Piece<DT> raw[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * s.row_step;
#pragma unroll
      for (int i = 0; i < (int)(sizeof(raw[u].w) / 4); ++i) raw[u].w[i] = 0u;
      if (r < s.row_end && (!RUNS || s.have > 0)) load_piece<DT, RUNS>(static_cast<const T*>(x) + r * ld_x, s, d.cols, vx, raw[u]);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * s.row_step;
      if (r - s.sub >= s.row_end) break;
      float v[kRun];
      open_piece<DT, RUNS>(raw[u], mine, v);
      // magnitudes as bit patterns: their order is the values', and NaN comes out on top
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int eb = exp_byte(__uint_as_float(top));
      const float inv = inv_step(eb);
      if (r < s.row_end && s.have > 0) {
        store_codes(out.dev_codes + r * out.ld_codes + s.col, vc, s.have,
                    make_uint2(code_word(v[0], v[1], v[2], v[3], inv), code_word(v[4], v[5], v[6], v[7], inv)));
        if ((s.col & (kGroup - 1)) == 0) out.dev_exps[r * out.ld_exps + s.col / kGroup] = (uint8_t)eb;
      }
    }
  }
}

template <int DT, bool RUNS>
__global__ void __launch_bounds__(kThreads)
unpack8_kernel(Deal d, lqsgd_packed8 in, bool vec_c, void* __restrict__ y, int64_t ld_y, bool vec_y) {
  constexpr int kRows = 4;
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turn[RUNS ? 1 : kWarps][RUNS ? 8 : 256];
  train_pdl_wait();
  const Spot s(d);
  if (RUNS && s.have <= 0) return;
  const bool vy = vec_y && s.have == kRun, vc = vec_c && s.have == kRun;
  for (int64_t r0 = s.row; r0 < s.row_end; r0 += kRows * s.row_step) {
    uint2 w[kRows];
    int e[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = min(r0 + u * s.row_step, s.row_end - 1);
      w[u] = make_uint2(0u, 0u);
      e[u] = kExpBias;
      if (s.have > 0) {
        w[u] = load_codes(in.dev_codes + r * in.ld_codes + s.col, vc, s.have);
        e[u] = in.dev_exps[r * in.ld_exps + s.col / kGroup];
      }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * s.row_step;
      if (r >= s.row_end) break;
      float v[kRun];
      decode_run(w[u], e[u], v);
      // only sources wider than the target can exceed its range: the largest finite value then (a NaN stays)
      constexpr float kTop = DT == LQSGD_F16 ? 65504.f : (DT == LQSGD_BF16 ? 3.3895314e38f : 3.402823466e38f);
      if (DT != LQSGD_F32 && e[u] >= (DT == LQSGD_F16 ? kExpBias + 9 : kQuickByte)) {
#pragma unroll
        for (int j = 0; j < kRun; ++j)
          if (fabsf(v[j]) > kTop) v[j] = copysignf(kTop, v[j]);
      }
      store_piece<DT, RUNS>(static_cast<T*>(y) + r * ld_y, s, d.cols, vy, turn[RUNS ? 0 : threadIdx.x >> 5], v);
    }
  }
}

// dz = dy act'(z); the block's column sums of dz go to partial[blockIdx.y][cols].
// GELU's and SiLU's slopes cost 20 to 30 instructions, more than HBM leaves time for.  But z takes few values: 128 magnitudes
// times a step, and both slopes satisfy s(z) = 1 - s(-z).  So a block that has work enough first tabulates the slopes s(-|z|) for
// the steps 2^-16 .. 2^4; groups with other steps, and blocks with little work, compute them.  Either way it is the side of the
// negative values that is computed: their slopes go to 0, and 1 minus their mirror image has lost its digits there (silu at
// -15.5: 28 % of the slope), while 1 - s(-z) for positive z is near 1 and loses nothing.
// Rows in flight per thread and blocks per SM, measured on 8192 x 16384 in bf16: without z, one row and six blocks (48 us; two
// rows 72); with z, four rows and three blocks (gelu 122 us, two rows and four blocks 148, one and six 142).
template <int DT, bool RUNS, int KIND>
struct SumShape {
  static constexpr int kRows = KIND == 0 ? 1 : (DT == LQSGD_F32 || !RUNS ? 2 : 4);
  static constexpr int kBlocks = KIND == 0 ? 6 : 3;
};
enum SlopeKind { kSlopeNone = 0, kSlopeRelu = 1, kSlopeCurve = 2 };
constexpr int kTabLow = kExpBias - 16, kTabSteps = 21;
template <int DT, bool RUNS, int KIND>
__global__ void __launch_bounds__(kThreads, SumShape<DT, RUNS, KIND>::kBlocks)
act_grad_kernel(Deal d, const void* dy, int64_t ld_dy, bool vec_dy, lqsgd_packed8 z8, bool vec_c, int act, bool table,
                void* dz, int64_t ld_dz, bool vec_dz, float* __restrict__ partial) {
  constexpr int kRows = SumShape<DT, RUNS, KIND>::kRows;
  using T = typename Elem<DT>::T;
  __shared__ float tab[KIND == kSlopeCurve ? kTabSteps * 128 : 1];
  __shared__ __align__(16) float sums[kWarps][32][kRun + 1];
  const Spot s(d);
  if (KIND == kSlopeCurve && table) {
    for (int i = threadIdx.x; i < kTabSteps * 128; i += kThreads) {
      const float z = -((float)(i & 127) * step_of(kTabLow + (i >> 7)));
      tab[i] = act == LQSGD_ACT_GELU ? act_slope<LQSGD_ACT_GELU>(z) : act_slope<LQSGD_ACT_SILU>(z);
    }
    __syncthreads();
  }
  train_pdl_wait();
  // the warp's place for turning rows is the one that its sums take at the end
  T* turn = reinterpret_cast<T*>(&sums[threadIdx.x >> 5][0][0]);
  const bool vg = vec_dy && s.have == kRun, vz = vec_dz && s.have == kRun, vc = vec_c && s.have == kRun;
  float acc[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) acc[j] = 0.f;
  if (!RUNS || s.have > 0)
    for (int64_t r0 = s.row; r0 < s.row_end; r0 += kRows * s.row_step) {
      Piece<DT> raw[kRows];
      uint2 w[kRows];
      uint32_t e[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int64_t r = min(r0 + u * s.row_step, s.row_end - 1);
        load_piece<DT, RUNS>(static_cast<const T*>(dy) + r * ld_dy, s, d.cols, vg, raw[u]);
        w[u] = make_uint2(0u, 0u);
        e[u] = kExpBias;
        if (KIND != kSlopeNone && s.have > 0) {
          w[u] = load_codes(z8.dev_codes + r * z8.ld_codes + s.col, vc, s.have);
          e[u] = z8.dev_exps[r * z8.ld_exps + s.col / kGroup];
        }
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int64_t r = r0 + u * s.row_step;
        if (r >= s.row_end) break;
        float g[kRun];
        open_piece<DT, RUNS>(raw[u], turn, g);
        if (KIND == kSlopeRelu) {
          // 1 for a positive value, 0 for the others, NaN for a group that is not finite
          const float one = e[u] == kExpNonFinite ? step_of(kExpNonFinite) : 1.f, none = one - one;
#pragma unroll
          for (int j = 0; j < kRun; ++j) {
            const uint32_t c = (j < 4 ? w[u].x : w[u].y) >> (8 * (j & 3)) & 255u;
            g[j] *= c - 1u < 127u ? one : none;
          }
        } else if (KIND == kSlopeCurve) {
          if (table && e[u] - kTabLow < (uint32_t)kTabSteps) {
            const float* row = tab + (e[u] - kTabLow) * 128;
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
              const uint32_t c = (j < 4 ? w[u].x : w[u].y) >> (8 * (j & 3));
              const float t = row[c & 127u];
              g[j] *= c & 128u ? t : 1.f - t;
            }
          } else {
            float z[kRun];
            decode_run(w[u], (int)e[u], z);
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
              const float t = act == LQSGD_ACT_GELU ? act_slope<LQSGD_ACT_GELU>(-fabsf(z[j])) : act_slope<LQSGD_ACT_SILU>(-fabsf(z[j]));
              g[j] *= signbit(z[j]) ? t : 1.f - t;
            }
          }
        }
        if (dz) store_piece<DT, RUNS>(static_cast<T*>(dz) + r * ld_dz, s, d.cols, vz, turn, g);
#pragma unroll
        for (int j = 0; j < kRun; ++j) acc[j] += g[j];
      }
    }
  if (!partial) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kRun; ++j) sums[warp][lane][j] = acc[j];
  __syncthreads();
  const int warp_cols = kRun << d.lane_shift;
  for (int c = threadIdx.x; c < warp_cols << d.wide_shift; c += kThreads) {
    const int col = (int)blockIdx.x * (warp_cols << d.wide_shift) + c;
    if (col >= d.cols) continue;
    const int beside = c / warp_cols, in = c - beside * warp_cols;
    float t = 0.f;
    for (int w = beside; w < kWarps; w += 1 << d.wide_shift)
      for (int sub = 0; sub < (32 >> d.lane_shift); ++sub) t += sums[w][(sub << d.lane_shift) + in / kRun][in % kRun];
    partial[(size_t)blockIdx.y * d.cols + col] = t;
  }
}

// out[c] = sum over b of partial[b][c]: 32 columns x 32 warps per block, fixed order.
__global__ void __launch_bounds__(1024)
join_columns_kernel(const float* __restrict__ partial, int blocks, int cols, float* __restrict__ out) {
  train_pdl_wait();
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 32 + lane;
  float t = 0.f;
  if (col < cols) {
#pragma unroll 8
    for (int b = warp; b < blocks; b += 32) t += partial[(size_t)b * cols + col];
  }
  part[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && col < cols) {
    float u = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) u += part[w][lane];
    out[col] = u;
  }
}

// CTAs that fill the card: 148 SMs x 8 blocks of 256 threads (x 6 where they leave column sums behind to be joined).  Constants,
// so that the order of the sums, and the workspace, depend on the sizes alone.
constexpr int kCtas = 148 * 8, kCtasSums = 148 * 6;
Deal deal_sums(int64_t rows, int32_t cols, bool runs, dim3* grid) { return make_deal(rows, cols, runs, kCtasSums, 8, grid); }

int check_matrix(int64_t rows, int32_t cols) {
  return rows < 0 || cols < 1 || rows > (int64_t)1 << 40 ? LQSGD_ERR_BAD_SHAPE : LQSGD_OK;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

#define BY_DTYPE(dtype, runs, kernel, ...)                                                       \
  ((dtype) == LQSGD_BF16 ? ((runs) ? train_launch(kernel<LQSGD_BF16, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_BF16, false>, __VA_ARGS__)) \
   : (dtype) == LQSGD_F16 ? ((runs) ? train_launch(kernel<LQSGD_F16, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_F16, false>, __VA_ARGS__))  \
                          : ((runs) ? train_launch(kernel<LQSGD_F32, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_F32, false>, __VA_ARGS__)))

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
  const bool vx = vec_rows(dev_x, ld_x, es, 16), vc = vec_rows(host_out->dev_codes, host_out->ld_codes, 1, 8);
  const bool runs = use_runs(vx, cols);
  dim3 grid;
  const Deal d = make_deal(rows, cols, runs, kCtas, 1, &grid);
  TRAIN_CK(BY_DTYPE(dtype, runs, pack8_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, dev_x, ld_x, vx, *host_out, vc), "pack8_kernel launch");
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
  const bool vy = vec_rows(dev_y, ld_y, es, 16), vc = vec_rows(host_in->dev_codes, host_in->ld_codes, 1, 8);
  const bool runs = use_runs(vy, cols);
  dim3 grid;
  const Deal d = make_deal(rows, cols, runs, kCtas, 1, &grid);
  TRAIN_CK(BY_DTYPE(dtype, runs, unpack8_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, *host_in, vc, dev_y, ld_y, vy), "unpack8_kernel launch");
  return LQSGD_OK;
}

// Row blocks of act_grad's column sums; the workspace has room for either layout.
static size_t sums_bytes(const dim3& grid, int32_t cols) { return grid.y > 1 ? (size_t)grid.y * cols * sizeof(float) : 0; }

extern "C" int lqsgd_act_grad_workspace_bytes(int64_t rows, int32_t cols, size_t* host_bytes_out) {
  if (!host_bytes_out) return LQSGD_ERR_INVALID_ARG;
  const int rc = check_matrix(rows, cols);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = 0;
  if (rows == 0) return LQSGD_OK;
  dim3 a, b;
  deal_sums(rows, cols, true, &a);
  deal_sums(rows, cols, cols <= 128, &b);
  *host_bytes_out = std::max(sums_bytes(a, cols), sums_bytes(b, cols));
  return LQSGD_OK;
}

template <int DT, bool RUNS>
static cudaError_t launch_act_grad(int act, dim3 grid, cudaStream_t st, const Deal& d, const void* dy, int64_t ld_dy, bool vg, const lqsgd_packed8& z8,
                                   bool vc, void* dz, int64_t ld_dz, bool vz, float* partial) {
  if (act == LQSGD_ACT_NONE)
    return train_launch(act_grad_kernel<DT, RUNS, kSlopeNone>, grid, dim3(kThreads), 0, st, 1, d, dy, ld_dy, vg, z8, vc, act, false, dz, ld_dz, vz, partial);
  if (act == LQSGD_ACT_RELU)
    return train_launch(act_grad_kernel<DT, RUNS, kSlopeRelu>, grid, dim3(kThreads), 0, st, 1, d, dy, ld_dy, vg, z8, vc, act, false, dz, ld_dz, vz, partial);
  // a block's table takes about ten slopes per thread: worth it from four times as many values on
  const bool table = d.rows_per_block * (kRun << (d.lane_shift + d.wide_shift)) >= 40 * kThreads;
  return train_launch(act_grad_kernel<DT, RUNS, kSlopeCurve>, grid, dim3(kThreads), 0, st, 1, d, dy, ld_dy, vg, z8, vc, act, table, dz, ld_dz, vz, partial);
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
  const bool vg = vec_rows(dev_dy, ld_dy, es, 16), vz = !dev_dz || vec_rows(dev_dz, ld_dz, es, 16),
             vc = act == LQSGD_ACT_NONE || vec_rows(z8.dev_codes, z8.ld_codes, 1, 8);
  const bool runs = use_runs(vg && vz, cols);
  dim3 grid;
  const Deal d = deal_sums(rows, cols, runs, &grid);
  float* partial = dev_db;
  if (dev_db && grid.y > 1) {
    if (!dev_workspace || workspace_bytes < sums_bytes(grid, cols)) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
    if (!train_aligned(dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
    partial = static_cast<float*>(dev_workspace);
  }
  cudaError_t e;
  if (dtype == LQSGD_BF16)
    e = runs ? launch_act_grad<LQSGD_BF16, true>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial)
             : launch_act_grad<LQSGD_BF16, false>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial);
  else if (dtype == LQSGD_F16)
    e = runs ? launch_act_grad<LQSGD_F16, true>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial)
             : launch_act_grad<LQSGD_F16, false>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial);
  else
    e = runs ? launch_act_grad<LQSGD_F32, true>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial)
             : launch_act_grad<LQSGD_F32, false>(act, grid, st, d, dev_dy, ld_dy, vg, z8, vc, dev_dz, ld_dz, vz, partial);
  TRAIN_CK(e, "act_grad_kernel launch");
  if (partial != dev_db)
    TRAIN_CK(train_launch(join_columns_kernel, dim3((unsigned)ceil_div64(cols, 32)), dim3(1024), 0, st, 1, partial, (int)grid.y, cols, dev_db), "join_columns_kernel launch");
  return LQSGD_OK;
}
