// Root-mean-square norm of rows with dropout and the residual's addition in front of it (lqsgd_rms_norm_*).
//
// Both directions are streams that need one sum per row before they can write: a row is read once, stays in registers while
// its threads agree on the sum, and is written from there.  What bounds them is HBM.  Rows of up to 1024 columns are held by 4 to 32
// lanes of a warp, longer ones by a block; rows beyond what a block holds are read twice.
#include "lqsgd_rows_dev.cuh"

namespace lqsgd {
namespace {

struct RmsArgs {
  const void *x, *residual, *dy, *skip;
  void *h, *y, *dx, *dresidual;
  int64_t ld_x, ld_residual, ld_dy, ld_skip, ld_h, ld_y, ld_dx, ld_dresidual;
  const float* gamma;
  float *rstd, *partial;
  lqsgd_packed8 h8, y8;
  lqsgd_rows8 r8;
  Drop drop;
  int64_t rows;
  int32_t cols, lane_shift;
  float eps;
  bool vec_x, vec_residual, vec_dy, vec_skip, vec_h, vec_y, vec_dx, vec_dresidual, vec_gamma, vec_h8, vec_y8, vec_r8;
};

// h = residual + dropout(x) of one run, as stored.
template <int DT, bool RUNS>
__device__ __forceinline__ void open_h(const RmsArgs& a, const Piece<DT>& x, const Piece<DT>& res, uint64_t block, typename Elem<DT>::T* turn, float (&v)[kRun]) {
  open_piece<DT, RUNS>(x, turn, v);
  float r[kRun] = {};
  if (a.residual) open_piece<DT, RUNS>(res, turn, r);
  if (a.drop.threshold) drop_run(a.drop, block, v, r);
  else if (a.residual) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] += r[j];
  }
#pragma unroll
  for (int j = 0; j < kRun; ++j) v[j] = as_stored<DT>(v[j]);
}
// Squares into `sum`, the largest |h gamma| into `top`.
__device__ __forceinline__ void add_squares(const RmsArgs& a, const Place& s, const float (&v)[kRun], float& sum, uint32_t& top) {
#pragma unroll
  for (int j = 0; j < kRun; ++j) sum = fmaf(v[j], v[j], sum);
  if (a.r8.dev_codes) {
    float g[kRun];
    load_vector(a.gamma, s, a.vec_gamma, g);
#pragma unroll
    for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j] * g[j]) & 0x7fffffffu);
  }
}
// y of one run and its copies in 8 bits.
template <int DT, bool RUNS>
__device__ __forceinline__ void put_y(const RmsArgs& a, int64_t row, const Place& s, bool on, float rstd, float inv, typename Elem<DT>::T* turn, float (&v)[kRun]) {
  using T = typename Elem<DT>::T;
  if (a.h8.dev_codes) put_packed_run(a.h8, a.vec_h8, row, s, on && s.have > 0, v);
  float g[kRun];
  load_vector(a.gamma, s, a.vec_gamma, g);
#pragma unroll
  for (int j = 0; j < kRun; ++j) v[j] = v[j] * rstd * g[j];
  if (a.r8.dev_codes && on && s.have > 0)
    store_codes(reinterpret_cast<uint8_t*>(a.r8.dev_codes) + row * a.r8.ld_codes + s.col, a.vec_r8 && s.have == kRun, s.have,
                make_uint2(signed_word(v, inv), signed_word(v + 4, inv)));
  if (a.y && on && (!RUNS || s.have > 0)) store_piece<DT, RUNS>(static_cast<T*>(a.y) + row * a.ld_y, s, a.cols, a.vec_y && s.have == kRun, turn, v);
  if (a.y8.dev_codes) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = as_stored<DT>(v[j]);
    put_packed_run(a.y8, a.vec_y8, row, s, on && s.have > 0, v);
  }
}
__device__ __forceinline__ float inverse_rms(float sum, int cols, float eps) { return 1.f / sqrtf(sum / (float)cols + eps); }

template <int DT, int N, bool NARROW, bool RUNS>
__global__ void __launch_bounds__(NARROW ? 256 : 512)
rms_forward_kernel(RmsArgs a) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : NARROW ? 8 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[32];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<NARROW> team(a.lane_shift);
  const int64_t row = team.row;
  const bool on = !NARROW || row < a.rows;
  train_pdl_wait();
  open_drop(a.drop);
  Piece<DT> x[N], res[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Place s = team.place(i, a.cols);
#pragma unroll
    for (int k = 0; k < (int)(sizeof(x[i].w) / 4); ++k) x[i].w[k] = res[i].w[k] = 0u;
    if (on && (!RUNS || s.have > 0)) {
      load_piece<DT, RUNS>(static_cast<const T*>(a.x) + row * a.ld_x, s, a.cols, a.vec_x && s.have == kRun, x[i]);
      if (a.residual) load_piece<DT, RUNS>(static_cast<const T*>(a.residual) + row * a.ld_residual, s, a.cols, a.vec_residual && s.have == kRun, res[i]);
    }
  }
  float v[N][kRun], sum = 0.f;
  uint32_t top = 0;
  const uint64_t block0 = (uint64_t)row * ((a.cols + kRun - 1) / kRun);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Place s = team.place(i, a.cols);
    open_h<DT, RUNS>(a, x[i], res[i], block0 + s.col / kRun, turn, v[i]);
    if (a.h && on && (!RUNS || s.have > 0)) store_piece<DT, RUNS>(static_cast<T*>(a.h) + row * a.ld_h, s, a.cols, a.vec_h && s.have == kRun, turn, v[i]);
    add_squares(a, s, v[i], sum, top);
  }
  team.join(sum, top, slots);
  const float rstd = inverse_rms(sum, a.cols, a.eps);
  float scale = 0.f, inv = 0.f;
  if (a.r8.dev_codes) row_scale(__uint_as_float(top) * rstd, scale, inv);
  if (on && team.t == 0) {
    a.rstd[row] = rstd;
    if (a.r8.dev_codes) a.r8.dev_scales[row] = scale;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) put_y<DT, RUNS>(a, row, team.place(i, a.cols), on, rstd, inv, turn, v[i]);
}

// Rows longer than a block holds: h is computed (and stored) in a first pass and computed again in a second.
template <int DT, bool RUNS>
__global__ void __launch_bounds__(512)
rms_forward_long_kernel(RmsArgs a) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[32];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<false> team(0);
  const int64_t row = team.row;
  train_pdl_wait();
  open_drop(a.drop);
  const uint64_t block0 = (uint64_t)row * ((a.cols + kRun - 1) / kRun);
  const int steps = team.steps(a.cols);
  auto fetch = [&](const Place& s, float (&v)[kRun]) {
    Piece<DT> x = {}, res = {};
    if (!RUNS || s.have > 0) {
      load_piece<DT, RUNS>(static_cast<const T*>(a.x) + row * a.ld_x, s, a.cols, a.vec_x && s.have == kRun, x);
      if (a.residual) load_piece<DT, RUNS>(static_cast<const T*>(a.residual) + row * a.ld_residual, s, a.cols, a.vec_residual && s.have == kRun, res);
    }
    open_h<DT, RUNS>(a, x, res, block0 + s.col / kRun, turn, v);
  };
  float sum = 0.f;
  uint32_t top = 0;
  for (int i = 0; i < steps; ++i) {
    const Place s = team.place(i, a.cols);
    float v[kRun];
    fetch(s, v);
    if (a.h && (!RUNS || s.have > 0)) store_piece<DT, RUNS>(static_cast<T*>(a.h) + row * a.ld_h, s, a.cols, a.vec_h && s.have == kRun, turn, v);
    add_squares(a, s, v, sum, top);
  }
  team.join(sum, top, slots);
  const float rstd = inverse_rms(sum, a.cols, a.eps);
  float scale = 0.f, inv = 0.f;
  if (a.r8.dev_codes) row_scale(__uint_as_float(top) * rstd, scale, inv);
  if (team.t == 0) {
    a.rstd[row] = rstd;
    if (a.r8.dev_codes) a.r8.dev_scales[row] = scale;
  }
  for (int i = 0; i < steps; ++i) {
    const Place s = team.place(i, a.cols);
    float v[kRun];
    fetch(s, v);
    put_y<DT, RUNS>(a, row, s, true, rstd, inv, turn, v);
  }
}

// ---- backward
// dy and h of one run, whichever form h has.
template <int DT, bool RUNS>
struct GradPieces {
  Piece<DT> dy, h, skip;
  uint2 codes;
  uint32_t exp;
  __device__ __forceinline__ void load(const RmsArgs& a, int64_t row, const Place& s, bool on, bool with_skip) {
    using T = typename Elem<DT>::T;
#pragma unroll
    for (int k = 0; k < (int)(sizeof(dy.w) / 4); ++k) dy.w[k] = h.w[k] = skip.w[k] = 0u;
    codes = make_uint2(0u, 0u);
    exp = kExpBias;
    if (!on || (RUNS && s.have <= 0)) return;
    load_piece<DT, RUNS>(static_cast<const T*>(a.dy) + row * a.ld_dy, s, a.cols, a.vec_dy && s.have == kRun, dy);
    if (!a.h8.dev_codes) {
      load_piece<DT, RUNS>(static_cast<const T*>(a.h) + row * a.ld_h, s, a.cols, a.vec_h && s.have == kRun, h);
    } else if (s.have > 0) {
      codes = load_codes(a.h8.dev_codes + row * a.h8.ld_codes + s.col, a.vec_h8 && s.have == kRun, s.have);
      exp = a.h8.dev_exps[row * a.h8.ld_exps + s.col / kGroup];
    }
    if (with_skip && a.skip) load_piece<DT, RUNS>(static_cast<const T*>(a.skip) + row * a.ld_skip, s, a.cols, a.vec_skip && s.have == kRun, skip);
  }
  __device__ __forceinline__ void open_h(const RmsArgs& a, typename Elem<DT>::T* turn, float (&v)[kRun]) const {
    if (a.h8.dev_codes) decode_run(codes, (int)exp, v);
    else open_piece<DT, RUNS>(h, turn, v);
  }
};
// d of one run into dx and dresidual.
template <int DT, bool RUNS>
__device__ __forceinline__ void put_d(const RmsArgs& a, int64_t row, const Place& s, bool on, uint64_t block, const Piece<DT>& skip, typename Elem<DT>::T* turn, float (&d)[kRun]) {
  using T = typename Elem<DT>::T;
  if (a.skip) {
    float k[kRun];
    open_piece<DT, RUNS>(skip, turn, k);
#pragma unroll
    for (int j = 0; j < kRun; ++j) d[j] += k[j];
  }
  if (!on || (RUNS && s.have <= 0)) return;
  if (a.dresidual) store_piece<DT, RUNS>(static_cast<T*>(a.dresidual) + row * a.ld_dresidual, s, a.cols, a.vec_dresidual && s.have == kRun, turn, d);
  if (a.dx) {
    const float none[kRun] = {};
    if (a.drop.threshold) drop_run(a.drop, block, d, none);
    store_piece<DT, RUNS>(static_cast<T*>(a.dx) + row * a.ld_dx, s, a.cols, a.vec_dx && s.have == kRun, turn, d);
  }
}

template <int DT, int N, bool NARROW, bool RUNS>
__global__ void __launch_bounds__(NARROW ? 256 : 512)
rms_backward_kernel(RmsArgs a) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : NARROW ? 8 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[2][32];
  __shared__ float sums[NARROW ? 256 * (kRun + 1) : 1];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<NARROW> team(a.lane_shift);
  train_pdl_wait();
  open_drop(a.drop);
  const float mean = 1.f / (float)a.cols;
  float acc[N][kRun];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < kRun; ++j) acc[i][j] = 0.f;
  const int step = team.rows_per_grid();
  int turn_of = 0;
  // NARROW: a warp stays together while one of its rows exists
  const int64_t first = NARROW ? team.row - ((threadIdx.x & 31) >> a.lane_shift) : team.row;
  for (int64_t r0 = first; r0 < a.rows; r0 += step) {
    const int64_t row = team.row + (r0 - first);
    const bool on = row < a.rows;
    GradPieces<DT, RUNS> p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) p[i].load(a, row, team.place(i, a.cols), on, true);
    const float rstd = on ? a.rstd[row] : 0.f;
    float xh[N][kRun], u[N][kRun], sum = 0.f;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const Place s = team.place(i, a.cols);
      float g[kRun];
      p[i].open_h(a, turn, xh[i]);
      open_piece<DT, RUNS>(p[i].dy, turn, u[i]);
      load_vector(a.gamma, s, a.vec_gamma, g);
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        xh[i][j] *= rstd;
        acc[i][j] = fmaf(u[i][j], xh[i][j], acc[i][j]);
        u[i][j] *= g[j];
        sum = fmaf(u[i][j], xh[i][j], sum);
      }
    }
    team.join(sum, top, slots[turn_of]);
    turn_of ^= 1;
    sum *= mean;
    const uint64_t block0 = (uint64_t)row * ((a.cols + kRun - 1) / kRun);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const Place s = team.place(i, a.cols);
#pragma unroll
      for (int j = 0; j < kRun; ++j) u[i][j] = rstd * (u[i][j] - xh[i][j] * sum);
      put_d<DT, RUNS>(a, row, s, on, block0 + s.col / kRun, p[i].skip, turn, u[i]);
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (size_t)blockIdx.x * a.cols;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Place s = team.place(i, a.cols);
    if (NARROW) {                                          // the block's rows meet in shared memory
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kRun; ++j) sums[threadIdx.x * (kRun + 1) + j] = acc[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < team.size * kRun; c += 256) {
        const int col = i * team.size * kRun + c;
        if (col >= a.cols) continue;
        float t = 0.f;
        for (int k = 0; k < 256 >> a.lane_shift; ++k) t += sums[((k << a.lane_shift) + c / kRun) * (kRun + 1) + c % kRun];
        out[col] = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (j < s.have) out[s.col + j] = acc[i][j];
    }
  }
}

// Rows longer than a block holds: <u xh> of each in a first kernel, the rest as a stream over columns.
template <int DT, bool RUNS>
__global__ void __launch_bounds__(512)
rms_dot_kernel(RmsArgs a, float* dots) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[32];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<false> team(0);
  const int64_t row = team.row;
  train_pdl_wait();
  const float rstd = a.rstd[row];
  float sum = 0.f;
  uint32_t top = 0;
  const int steps = team.steps(a.cols);
  for (int i = 0; i < steps; ++i) {
    const Place s = team.place(i, a.cols);
    GradPieces<DT, RUNS> p;
    p.load(a, row, s, true, false);
    float h[kRun], u[kRun], g[kRun];
    p.open_h(a, turn, h);
    open_piece<DT, RUNS>(p.dy, turn, u);
    load_vector(a.gamma, s, a.vec_gamma, g);
#pragma unroll
    for (int j = 0; j < kRun; ++j) sum = fmaf(u[j] * g[j], h[j] * rstd, sum);
  }
  team.join(sum, top, slots);
  if (team.t == 0) dots[row] = sum / (float)a.cols;
}
template <int DT, bool RUNS>
__global__ void __launch_bounds__(kThreads)
rms_columns_kernel(RmsArgs a, Deal d, const float* dots) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) float sums[kWarps][32][kRun + 1];
  T* turn = reinterpret_cast<T*>(&sums[threadIdx.x >> 5][0][0]);
  train_pdl_wait();
  open_drop(a.drop);
  const Spot s(d);
  float acc[kRun] = {}, g[kRun];
  load_vector(a.gamma, s, a.vec_gamma, g);
  for (int64_t row = s.row; row < s.row_end; row += s.row_step) {
    GradPieces<DT, RUNS> p;
    p.load(a, row, s, true, true);
    const float rstd = a.rstd[row], dot = dots[row];
    float h[kRun], u[kRun];
    p.open_h(a, turn, h);
    open_piece<DT, RUNS>(p.dy, turn, u);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      h[j] *= rstd;
      acc[j] = fmaf(u[j], h[j], acc[j]);
      u[j] = rstd * (u[j] * g[j] - h[j] * dot);
    }
    put_d<DT, RUNS>(a, row, s, true, (uint64_t)row * ((a.cols + kRun - 1) / kRun) + s.col / kRun, p.skip, turn, u);
  }
  if (!a.partial) return;
  // the rows that the block's warps have of one column: warps side by side hold other columns
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warp_cols = kRun * 32;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kRun; ++j) sums[warp][lane][j] = acc[j];
  __syncthreads();
  for (int c = threadIdx.x; c < warp_cols << d.wide_shift; c += kThreads) {
    const int col = (int)blockIdx.x * (warp_cols << d.wide_shift) + c;
    if (col >= a.cols) continue;
    const int beside = c / warp_cols, in = c - beside * warp_cols;
    float t = 0.f;
    for (int w = beside; w < kWarps; w += 1 << d.wide_shift) t += sums[w][in / kRun][in % kRun];
    a.partial[(size_t)blockIdx.y * a.cols + col] = t;
  }
}

// ---- choice of kernel: how a row is dealt out
constexpr int kNarrow = 1024, kMostForward = 512 * kRun * 8, kMostBackward = 512 * kRun * 4;
struct Shape {
  bool narrow;
  int lane_shift, threads, n;                // n: runs per thread
  int64_t teams;                             // rows per block
};
// Rows of up to 1024 columns in a warp or less, then in blocks of up to 512 threads; the fewest runs per thread that hold the row.
Shape shape_of(int32_t cols) {
  Shape s = {};
  const int runs = (int)ceil_div64(cols, kRun);
  s.narrow = cols <= kNarrow;
  if (s.narrow) {
    s.lane_shift = 2;
    while (s.lane_shift < 5 && (1 << s.lane_shift) < runs) ++s.lane_shift;
    s.n = 1;
    while ((s.n << s.lane_shift) < runs) s.n *= 2;
    s.threads = 256;
    s.teams = 256 >> s.lane_shift;
  } else {
    s.n = 1;
    while (s.n * 512 < runs) s.n *= 2;
    s.threads = (int)ceil_div64(ceil_div64(runs, s.n), 32) * 32;
    s.teams = 1;
  }
  return s;
}
bool whole_warps(int32_t cols) { return cols > 128; }                    // rows of fewer columns leave lanes of a warp to other rows

constexpr int kSms = 148;
int64_t backward_blocks(const Shape& s, int64_t rows) {
  const int64_t per_sm = s.narrow ? 4 : std::max(1, 1024 / s.threads);
  return std::min<int64_t>(ceil_div64(rows, s.teams), kSms * per_sm);
}
constexpr int kCtasColumns = kSms * 6;

struct GradPlan {
  bool wide;                                 // the two kernels for long rows
  Shape shape;
  Deal deal;
  dim3 grid;
  int blocks;                                // of the sums over rows
  size_t off_partial, bytes;
};
GradPlan plan_backward(const lqsgd_rms_norm& a, bool runs) {
  GradPlan p = {};
  p.wide = a.cols > kMostBackward;
  if (p.wide) {
    p.deal = make_deal(a.rows, a.cols, runs, kCtasColumns, 8, &p.grid);
    p.blocks = (int)p.grid.y;
    p.off_partial = (size_t)ceil_div64(a.rows * 4, 256) * 256;
  } else {
    p.shape = shape_of(a.cols);
    p.blocks = (int)backward_blocks(p.shape, a.rows);
  }
  p.bytes = p.off_partial + (a.dev_dgamma && p.blocks > 1 ? (size_t)p.blocks * a.cols * 4 : 0);
  return p;
}

template <int DT, bool RUNS>
cudaError_t launch_forward(const Shape& s, bool wide, const RmsArgs& a, cudaStream_t st) {
  if (wide) return train_launch(rms_forward_long_kernel<DT, RUNS>, dim3((unsigned)a.rows), dim3(512), 0, st, 1, a);
  const dim3 grid((unsigned)ceil_div64(a.rows, s.teams)), block(s.threads);
#define GO(N, NARROW) train_launch(rms_forward_kernel<DT, N, NARROW, RUNS>, grid, block, 0, st, 1, a)
  if (s.narrow) return s.n == 1 ? GO(1, true) : s.n == 2 ? GO(2, true) : GO(4, true);
  return s.n == 1 ? GO(1, false) : s.n == 2 ? GO(2, false) : s.n == 4 ? GO(4, false) : GO(8, false);
#undef GO
}
template <int DT, bool RUNS>
cudaError_t launch_backward(const GradPlan& p, const RmsArgs& a, float* dots, cudaStream_t st) {
  if (p.wide) {
    const cudaError_t e = train_launch(rms_dot_kernel<DT, RUNS>, dim3((unsigned)a.rows), dim3(512), 0, st, 1, a, dots);
    return e != cudaSuccess ? e : train_launch(rms_columns_kernel<DT, RUNS>, p.grid, dim3(kThreads), 0, st, 1, a, p.deal, dots);
  }
  const dim3 grid((unsigned)p.blocks), block(p.shape.threads);
#define GO(N, NARROW) train_launch(rms_backward_kernel<DT, N, NARROW, RUNS>, grid, block, 0, st, 1, a)
  if (p.shape.narrow) return p.shape.n == 1 ? GO(1, true) : p.shape.n == 2 ? GO(2, true) : GO(4, true);
  return p.shape.n == 1 ? GO(1, false) : p.shape.n == 2 ? GO(2, false) : GO(4, false);
#undef GO
}
#define BY_TYPE(dtype, runs, f, ...)                                                                       \
  ((dtype) == LQSGD_BF16 ? ((runs) ? f<LQSGD_BF16, true>(__VA_ARGS__) : f<LQSGD_BF16, false>(__VA_ARGS__)) \
   : (dtype) == LQSGD_F16 ? ((runs) ? f<LQSGD_F16, true>(__VA_ARGS__) : f<LQSGD_F16, false>(__VA_ARGS__))  \
                          : ((runs) ? f<LQSGD_F32, true>(__VA_ARGS__) : f<LQSGD_F32, false>(__VA_ARGS__)))

int check_args(const lqsgd_rms_norm* a) {
  if (!a || a->struct_size != sizeof(lqsgd_rms_norm) || !train_dtype_ok(a->dtype)) return LQSGD_ERR_INVALID_ARG;
  if (a->rows < 0 || a->rows > 0x7fffffffll || a->cols < 1 || a->cols > (1 << 24)) return LQSGD_ERR_BAD_SHAPE;
  return check_drop(a->drop);
}
// A matrix argument: *vec tells whether its rows start on 16 bytes (an absent one does not stand in the way).
int check_matrix(const void* p, int64_t ld, const lqsgd_rms_norm& a, bool* vec) {
  const int es = train_elem(a.dtype);
  *vec = !p || vec_rows(p, ld, es, 16) || (a.rows == 1 && train_aligned(p, 16));
  if (!p) return LQSGD_OK;
  if (ld < a.cols) return LQSGD_ERR_INVALID_ARG;
  return train_aligned(p, es) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

extern "C" int lqsgd_rms_norm_workspace_bytes(int32_t backward, const lqsgd_rms_norm* a, size_t* host_bytes_out) {
  if (!host_bytes_out || (backward != 0 && backward != 1)) return LQSGD_ERR_INVALID_ARG;
  const int rc = check_args(a);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = backward && a->rows > 0 ? plan_backward(*a, true).bytes : 0;
  return LQSGD_OK;
}

extern "C" int lqsgd_rms_norm_forward(const lqsgd_rms_norm* a, void* cuda_stream) {
  int rc = check_args(a);
  if (rc != LQSGD_OK) return rc;
  if (!(a->eps >= 0.f) || a->eps > 3.402823466e38f) return LQSGD_ERR_INVALID_ARG;
  if (a->rows == 0) return LQSGD_OK;
  if (!a->dev_x || !a->dev_gamma || !a->dev_rstd) return LQSGD_ERR_INVALID_ARG;
  if (!a->dev_h && (a->dev_residual || a->drop.p > 0.f)) return LQSGD_ERR_INVALID_ARG;
  RmsArgs k = {};
  if ((rc = check_matrix(a->dev_x, a->ld_x, *a, &k.vec_x)) != LQSGD_OK || (rc = check_matrix(a->dev_residual, a->ld_residual, *a, &k.vec_residual)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_h, a->ld_h, *a, &k.vec_h)) != LQSGD_OK || (rc = check_matrix(a->dev_y, a->ld_y, *a, &k.vec_y)) != LQSGD_OK)
    return rc;
  if (a->h8.dev_codes && (rc = check_packed8(a->h8, a->cols)) != LQSGD_OK) return rc;
  if (a->y8.dev_codes && (rc = check_packed8(a->y8, a->cols)) != LQSGD_OK) return rc;
  if (a->rows8.dev_codes && (rc = check_rows8(a->rows8, a->cols)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  k.x = a->dev_x; k.ld_x = a->ld_x; k.residual = a->dev_residual; k.ld_residual = a->ld_residual;
  k.h = a->dev_h; k.ld_h = a->ld_h; k.y = a->dev_y; k.ld_y = a->ld_y;
  k.gamma = a->dev_gamma; k.rstd = a->dev_rstd;
  k.h8 = a->h8; k.y8 = a->y8; k.r8 = a->rows8;
  k.drop = make_drop(a->drop);
  k.rows = a->rows; k.cols = a->cols; k.eps = a->eps;
  k.vec_gamma = train_aligned(a->dev_gamma, 16);
  k.vec_h8 = vec_rows(a->h8.dev_codes, a->h8.ld_codes, 1, 8);
  k.vec_y8 = vec_rows(a->y8.dev_codes, a->y8.ld_codes, 1, 8);
  k.vec_r8 = vec_rows(a->rows8.dev_codes, a->rows8.ld_codes, 1, 8);
  const bool wide = a->cols > kMostForward, runs = (k.vec_x && k.vec_residual && k.vec_h && k.vec_y) || !whole_warps(a->cols);
  const Shape s = wide ? Shape{} : shape_of(a->cols);
  k.lane_shift = s.lane_shift;
  TRAIN_CK(BY_TYPE(a->dtype, runs, launch_forward, s, wide, k, static_cast<cudaStream_t>(cuda_stream)), "rms_forward_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_rms_norm_backward(const lqsgd_rms_norm* a, void* cuda_stream) {
  int rc = check_args(a);
  if (rc != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!a->dev_dx && !a->dev_dresidual && !a->dev_dgamma) return LQSGD_ERR_INVALID_ARG;
  if (!train_aligned(a->dev_dgamma, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->rows == 0) {
    if (a->dev_dgamma) TRAIN_CK(cudaMemsetAsync(a->dev_dgamma, 0, (size_t)a->cols * sizeof(float), st), "cudaMemsetAsync(dgamma)");
    return LQSGD_OK;
  }
  const bool kept = a->h8.dev_codes != nullptr;
  if (!a->dev_dy || !a->dev_gamma || !a->dev_rstd || (!kept && !a->dev_h)) return LQSGD_ERR_INVALID_ARG;
  RmsArgs k = {};
  if ((rc = check_matrix(a->dev_dy, a->ld_dy, *a, &k.vec_dy)) != LQSGD_OK || (rc = check_matrix(a->dev_skip, a->ld_skip, *a, &k.vec_skip)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_dx, a->ld_dx, *a, &k.vec_dx)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_dresidual, a->ld_dresidual, *a, &k.vec_dresidual)) != LQSGD_OK ||
      (rc = check_matrix(kept ? nullptr : a->dev_h, a->ld_h, *a, &k.vec_h)) != LQSGD_OK)
    return rc;
  if (kept && (rc = check_packed8(a->h8, a->cols)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  const bool runs = (k.vec_dy && k.vec_skip && k.vec_dx && k.vec_dresidual && k.vec_h) || !whole_warps(a->cols);
  const GradPlan p = plan_backward(*a, runs);
  if (p.bytes) {
    if (!a->dev_workspace || a->workspace_bytes < p.bytes) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
    if (!train_aligned(a->dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
  }
  char* ws = static_cast<char*>(a->dev_workspace);
  k.dy = a->dev_dy; k.ld_dy = a->ld_dy; k.skip = a->dev_skip; k.ld_skip = a->ld_skip;
  k.dx = a->dev_dx; k.ld_dx = a->ld_dx; k.dresidual = a->dev_dresidual; k.ld_dresidual = a->ld_dresidual;
  k.h = kept ? nullptr : a->dev_h; k.ld_h = a->ld_h; k.h8 = a->h8;
  k.gamma = a->dev_gamma; k.rstd = a->dev_rstd;
  k.partial = !a->dev_dgamma ? nullptr : p.blocks > 1 ? reinterpret_cast<float*>(ws + p.off_partial) : a->dev_dgamma;
  k.drop = make_drop(a->drop);
  k.rows = a->rows; k.cols = a->cols; k.lane_shift = p.shape.lane_shift;
  k.vec_gamma = train_aligned(a->dev_gamma, 16);
  k.vec_h8 = vec_rows(a->h8.dev_codes, a->h8.ld_codes, 1, 8);
  TRAIN_CK(BY_TYPE(a->dtype, runs, launch_backward, p, k, reinterpret_cast<float*>(ws), st), "rms_backward_kernel launch");
  return a->dev_dgamma && p.blocks > 1 ? join_columns(k.partial, p.blocks, a->cols, a->dev_dgamma, st) : LQSGD_OK;
}
