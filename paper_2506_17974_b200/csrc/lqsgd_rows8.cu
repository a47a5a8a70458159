// Rows of signed 8-bit codes with one scale each, to and from them, and dropout by itself.  All are streams bounded by HBM; packing
// needs the row's largest magnitude first, so a row stays in the registers of its threads in between.
#include "lqsgd_rows_dev.cuh"

namespace lqsgd {
namespace {

struct PackArgs {
  const void* x;
  int64_t ld_x, rows;
  lqsgd_rows8 out;
  int32_t cols, lane_shift;
  bool vec_x, vec_c;
};
__device__ __forceinline__ uint32_t largest(const float (&v)[kRun], uint32_t top) {
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ void put_row_codes(const PackArgs& a, int64_t row, const Place& s, float inv, const float (&v)[kRun]) {
  store_codes(reinterpret_cast<uint8_t*>(a.out.dev_codes) + row * a.out.ld_codes + s.col, a.vec_c && s.have == kRun, s.have,
              make_uint2(signed_word(v, inv), signed_word(v + 4, inv)));
}

template <int DT, int N, bool NARROW, bool RUNS>
__global__ void __launch_bounds__(NARROW ? 256 : 512)
pack_rows8_kernel(PackArgs a) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : NARROW ? 8 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[32];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<NARROW> team(a.lane_shift);
  const int64_t row = team.row;
  const bool on = !NARROW || row < a.rows;
  train_pdl_wait();
  Piece<DT> x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Place s = team.place(i, a.cols);
#pragma unroll
    for (int k = 0; k < (int)(sizeof(x[i].w) / 4); ++k) x[i].w[k] = 0u;
    if (on && (!RUNS || s.have > 0)) load_piece<DT, RUNS>(static_cast<const T*>(a.x) + row * a.ld_x, s, a.cols, a.vec_x && s.have == kRun, x[i]);
  }
  float v[N][kRun], none = 0.f;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    open_piece<DT, RUNS>(x[i], turn, v[i]);
    top = largest(v[i], top);
  }
  team.join(none, top, slots);
  float scale, inv;
  row_scale(__uint_as_float(top), scale, inv);
  if (!on) return;
  if (team.t == 0) a.out.dev_scales[row] = scale;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Place s = team.place(i, a.cols);
    if (s.have > 0) put_row_codes(a, row, s, inv, v[i]);
  }
}

// Rows longer than a block holds: read twice.
template <int DT, bool RUNS>
__global__ void __launch_bounds__(512)
pack_rows8_long_kernel(PackArgs a) {
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : 16][RUNS ? 8 : 256];
  __shared__ float2 slots[32];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  const Team<false> team(0);
  const int64_t row = team.row;
  train_pdl_wait();
  const int steps = team.steps(a.cols);
  auto fetch = [&](const Place& s, float (&v)[kRun]) {
    Piece<DT> x = {};
    if (!RUNS || s.have > 0) load_piece<DT, RUNS>(static_cast<const T*>(a.x) + row * a.ld_x, s, a.cols, a.vec_x && s.have == kRun, x);
    open_piece<DT, RUNS>(x, turn, v);
  };
  float none = 0.f;
  uint32_t top = 0;
  for (int i = 0; i < steps; ++i) {
    float v[kRun];
    fetch(team.place(i, a.cols), v);
    top = largest(v, top);
  }
  team.join(none, top, slots);
  float scale, inv;
  row_scale(__uint_as_float(top), scale, inv);
  if (team.t == 0) a.out.dev_scales[row] = scale;
  for (int i = 0; i < steps; ++i) {
    const Place s = team.place(i, a.cols);
    float v[kRun];
    fetch(s, v);
    if (s.have > 0) put_row_codes(a, row, s, inv, v);
  }
}

template <int DT, bool RUNS>
__global__ void __launch_bounds__(kThreads)
unpack_rows8_kernel(Deal d, lqsgd_rows8 in, bool vec_c, void* __restrict__ y, int64_t ld_y, bool vec_y) {
  constexpr int kRows = 4;
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turn[RUNS ? 1 : kWarps][RUNS ? 8 : 256];
  train_pdl_wait();
  const Spot s(d);
  if (RUNS && s.have <= 0) return;
  const bool vy = vec_y && s.have == kRun, vc = vec_c && s.have == kRun;
  for (int64_t r0 = s.row; r0 < s.row_end; r0 += kRows * s.row_step) {
    uint2 w[kRows];
    float scale[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = min(r0 + u * s.row_step, s.row_end - 1);
      w[u] = make_uint2(0u, 0u);
      if (s.have > 0) w[u] = load_codes(reinterpret_cast<const uint8_t*>(in.dev_codes) + r * in.ld_codes + s.col, vc, s.have);
      scale[u] = in.dev_scales[r];
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * s.row_step;
      if (r >= s.row_end) break;
      float v[kRun];
#pragma unroll
      for (int j = 0; j < kRun; ++j) v[j] = (float)(int8_t)((j < 4 ? w[u].x : w[u].y) >> (8 * (j & 3))) * scale[u];
      // past the type's range (for the source's own type: only by the scale's rounding): the largest finite value; a NaN stays
      constexpr float kTop = DT == LQSGD_F16 ? 65504.f : (DT == LQSGD_BF16 ? 3.3895314e38f : 3.402823466e38f);
      if (scale[u] > kTop / 128.5f) {
#pragma unroll
        for (int j = 0; j < kRun; ++j)
          if (fabsf(v[j]) > kTop) v[j] = copysignf(kTop, v[j]);
      }
      store_piece<DT, RUNS>(static_cast<T*>(y) + r * ld_y, s, d.cols, vy, turn[RUNS ? 0 : threadIdx.x >> 5], v);
    }
  }
}

template <int DT, bool RUNS>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(Deal d, const void* x, int64_t ld_x, bool vec_x, const void* residual, int64_t ld_r, bool vec_r, Drop drop,
               void* out, int64_t ld_o, bool vec_o) {
  constexpr int kRows = DT == LQSGD_F32 ? 1 : 2;
  using T = typename Elem<DT>::T;
  __shared__ __align__(16) T turns[RUNS ? 1 : kWarps][RUNS ? 8 : 256];
  T* turn = turns[RUNS ? 0 : threadIdx.x >> 5];
  train_pdl_wait();
  open_drop(drop);
  const Spot s(d);
  if (RUNS && s.have <= 0) return;
  const bool vx = vec_x && s.have == kRun, vr = vec_r && s.have == kRun, vo = vec_o && s.have == kRun;
  const uint64_t blocks = (uint64_t)((d.cols + kRun - 1) / kRun);
  for (int64_t r0 = s.row; r0 < s.row_end; r0 += kRows * s.row_step) {
    Piece<DT> px[kRows], pr[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = min(r0 + u * s.row_step, s.row_end - 1);
      load_piece<DT, RUNS>(static_cast<const T*>(x) + r * ld_x, s, d.cols, vx, px[u]);
      if (residual) load_piece<DT, RUNS>(static_cast<const T*>(residual) + r * ld_r, s, d.cols, vr, pr[u]);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int64_t r = r0 + u * s.row_step;
      if (r >= s.row_end) break;
      float v[kRun], add[kRun] = {};
      open_piece<DT, RUNS>(px[u], turn, v);
      if (residual) open_piece<DT, RUNS>(pr[u], turn, add);
      drop_run(drop, (uint64_t)r * blocks + s.col / kRun, v, add);
      store_piece<DT, RUNS>(static_cast<T*>(out) + r * ld_o, s, d.cols, vo, turn, v);
    }
  }
}

constexpr int kNarrow = 1024, kMostHeld = 512 * kRun * 8;
template <int DT, bool RUNS>
cudaError_t launch_pack(const PackArgs& a0, cudaStream_t st) {
  PackArgs a = a0;
  const int runs = (int)ceil_div64(a.cols, kRun);
  if (a.cols > kMostHeld) return train_launch(pack_rows8_long_kernel<DT, RUNS>, dim3((unsigned)a.rows), dim3(512), 0, st, 1, a);
#define GO(N, NARROW) train_launch(pack_rows8_kernel<DT, N, NARROW, RUNS>, grid, block, 0, st, 1, a)
  int n = 1;
  if (a.cols <= kNarrow) {
    a.lane_shift = 2;
    while (a.lane_shift < 5 && (1 << a.lane_shift) < runs) ++a.lane_shift;
    while ((n << a.lane_shift) < runs) n *= 2;
    const dim3 grid((unsigned)ceil_div64(a.rows, 256 >> a.lane_shift)), block(256);
    return n == 1 ? GO(1, true) : n == 2 ? GO(2, true) : GO(4, true);
  }
  while (n * 512 < runs) n *= 2;
  const dim3 grid((unsigned)a.rows), block((unsigned)(ceil_div64(ceil_div64(runs, n), 32) * 32));
  return n == 1 ? GO(1, false) : n == 2 ? GO(2, false) : n == 4 ? GO(4, false) : GO(8, false);
#undef GO
}

int check_shape(int64_t rows, int32_t cols) {
  return rows < 0 || rows > 0x7fffffffll || cols < 1 || cols > (1 << 24) ? LQSGD_ERR_BAD_SHAPE : LQSGD_OK;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

extern "C" int lqsgd_pack_rows8(const void* dev_x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t cols,
                                const lqsgd_rows8* host_out, void* cuda_stream) {
  if (!host_out || !train_dtype_ok(dtype)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_shape(rows, cols);
  if (rc != LQSGD_OK) return rc;
  if (rows == 0) return LQSGD_OK;
  if (!dev_x || ld_x < cols) return LQSGD_ERR_INVALID_ARG;
  if ((rc = check_rows8(*host_out, cols)) != LQSGD_OK) return rc;
  const int es = train_elem(dtype);
  if (!train_aligned(dev_x, es)) return LQSGD_ERR_MISALIGNED;
  const bool vx = vec_rows(dev_x, ld_x, es, 16), vc = vec_rows(host_out->dev_codes, host_out->ld_codes, 1, 8);
  const PackArgs a = {dev_x, ld_x, rows, *host_out, cols, 0, vx, vc};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool runs = use_runs(vx, cols);
  TRAIN_CK(dtype == LQSGD_BF16 ? (runs ? launch_pack<LQSGD_BF16, true>(a, st) : launch_pack<LQSGD_BF16, false>(a, st))
           : dtype == LQSGD_F16 ? (runs ? launch_pack<LQSGD_F16, true>(a, st) : launch_pack<LQSGD_F16, false>(a, st))
                                : (runs ? launch_pack<LQSGD_F32, true>(a, st) : launch_pack<LQSGD_F32, false>(a, st)), "pack_rows8_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_unpack_rows8(const lqsgd_rows8* host_in, int64_t rows, int32_t cols, void* dev_y, int64_t ld_y,
                                  int32_t dtype, void* cuda_stream) {
  if (!host_in || !train_dtype_ok(dtype)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_shape(rows, cols);
  if (rc != LQSGD_OK) return rc;
  if (rows == 0) return LQSGD_OK;
  if (!dev_y || ld_y < cols) return LQSGD_ERR_INVALID_ARG;
  if ((rc = check_rows8(*host_in, cols)) != LQSGD_OK) return rc;
  const int es = train_elem(dtype);
  if (!train_aligned(dev_y, es)) return LQSGD_ERR_MISALIGNED;
  const bool vy = vec_rows(dev_y, ld_y, es, 16), vc = vec_rows(host_in->dev_codes, host_in->ld_codes, 1, 8);
  const bool runs = use_runs(vy, cols);
  dim3 grid;
  const Deal d = make_deal(rows, cols, runs, kCtas, 1, &grid);
  TRAIN_CK(BY_DTYPE(dtype, runs, unpack_rows8_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, *host_in, vc, dev_y, ld_y, vy), "unpack_rows8_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_dropout(const void* dev_x, int64_t ld_x, const void* dev_residual, int64_t ld_residual, int32_t dtype, int64_t rows,
                             int32_t cols, const lqsgd_drop* host_drop, void* dev_out, int64_t ld_out, void* cuda_stream) {
  if (!host_drop || !train_dtype_ok(dtype)) return LQSGD_ERR_INVALID_ARG;
  int rc = check_shape(rows, cols);
  if (rc != LQSGD_OK || (rc = check_drop(*host_drop)) != LQSGD_OK) return rc;
  if (rows == 0) return LQSGD_OK;
  if (!dev_x || ld_x < cols || !dev_out || ld_out < cols || (dev_residual && ld_residual < cols)) return LQSGD_ERR_INVALID_ARG;
  const int es = train_elem(dtype);
  if (!train_aligned(dev_x, es) || !train_aligned(dev_residual, es) || !train_aligned(dev_out, es)) return LQSGD_ERR_MISALIGNED;
  const bool vx = vec_rows(dev_x, ld_x, es, 16), vr = !dev_residual || vec_rows(dev_residual, ld_residual, es, 16), vo = vec_rows(dev_out, ld_out, es, 16);
  const bool runs = use_runs(vx && vr && vo, cols);
  dim3 grid;
  const Deal d = make_deal(rows, cols, runs, kCtas, 1, &grid);
  TRAIN_CK(BY_DTYPE(dtype, runs, dropout_kernel, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(cuda_stream), 1, d, dev_x, ld_x, vx, dev_residual,
                    ld_residual, vr, make_drop(*host_drop), dev_out, ld_out, vo), "dropout_kernel launch");
  return LQSGD_OK;
}
