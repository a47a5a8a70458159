// Streams over the rows of a matrix: how it is dealt out to threads in runs of 8 columns, and how such runs are read and
// written at any alignment (lqsgd_act8.cu has the measurements behind it).
#pragma once
#include "lqsgd_train_dev.cuh"

#include <algorithm>

namespace lqsgd {
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
struct Place {
  int col, have;                             // first column of the run; how many of its 8 exist (<= 0: none)
  int side;                                  // the warp's first column + lane: columns side, side + 32, ... of the other form
};
struct Spot : Place {
  int64_t row, row_end, row_step;            // rows row, row + row_step, ... < row_end
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
__device__ __forceinline__ void load_piece(const typename Elem<DT>::T* row, const Place& s, int cols, bool vec, Piece<DT>& out) {
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
__device__ __forceinline__ void store_piece(typename Elem<DT>::T* row, const Place& s, int cols, bool vec, typename Elem<DT>::T* turn, const float (&v)[kRun]) {
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

// CTAs that fill the card: 148 SMs x 8 blocks of 256 threads.  A constant, so that results depend on the sizes alone.
constexpr int kCtas = 148 * 8;
static inline bool vec_rows(const void* p, int64_t ld, int elem, int bytes) { return train_aligned(p, bytes) && (ld * elem) % bytes == 0; }

}  // namespace
}  // namespace lqsgd

// kernel<type, runs>(...) launched for a type known at run time
#define BY_DTYPE(dtype, runs, kernel, ...)                                                       \
  ((dtype) == LQSGD_BF16 ? ((runs) ? train_launch(kernel<LQSGD_BF16, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_BF16, false>, __VA_ARGS__)) \
   : (dtype) == LQSGD_F16 ? ((runs) ? train_launch(kernel<LQSGD_F16, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_F16, false>, __VA_ARGS__))  \
                          : ((runs) ? train_launch(kernel<LQSGD_F32, true>, __VA_ARGS__) : train_launch(kernel<LQSGD_F32, false>, __VA_ARGS__)))
