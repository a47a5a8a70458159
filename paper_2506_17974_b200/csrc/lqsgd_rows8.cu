// Rows of signed 8-bit codes with one scale each, to and from them, and dropout by itself.  All are streams bounded by HBM; packing
// needs the row's largest magnitude first, so a row stays in the registers of its threads in between, a long one in their shared memory.
// A thread has 64 bytes of a row (four runs of a 16-bit type) on their way at once.
// Measured: 16384 x 4096 packed from bf16 30 us (6.7 TB/s), from fp32 48 (7.0), unpacked to bf16 31 (6.4); dropout of 8192 x 16384 bf16 89 (6.0 TB/s;
// the generator is a third of its 125 instructions per run), 8192 x 8192 with a residual 58 (7.0).
#include "lqsgd_rows_dev.cuh"

namespace lqsgd {
namespace {

struct PackArgs {
  const void* x;
  int64_t ld_x, rows;
  lqsgd_rows8 out;
  int32_t cols, lane_shift;
  bool vec_c;
};
__device__ __forceinline__ uint8_t* codes_of(const lqsgd_rows8& r, int64_t row, int col) { return reinterpret_cast<uint8_t*>(r.dev_codes) + row * r.ld_codes + col; }

constexpr int kPackThreads = 512;
template <int DT, int N, bool NARROW, int HOW>
__global__ void __launch_bounds__(NARROW ? 256 : kPackThreads, NARROW || HOW == kShift ? 1 : 3)
pack_rows8_kernel(const __grid_constant__ PackArgs a) {
  __shared__ float2 slots[16];
  const Team<NARROW, N> team(a.lane_shift);
  const int64_t row = team.row;
  const Lanes l = team.lanes(a.cols, !NARROW || row < a.rows);
  const Cursor<DT, HOW> x(a.x, row * a.ld_x, l);
  train_pdl_wait();
  Raw<DT, HOW> raw[N];
#pragma unroll
  for (int i = 0; i < N; ++i) fetch(x, l, i, raw[i]);
  Piece<DT> p[N];
  float none = 0.f, top = 0.f;
  settle(raw, x, l, p);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[kRun];
    open_words<DT>(p[i], v);
    top = largest(top, v);
  }
  team.template join<true>(none, top, slots);
  float scale, inv;
  row_scale(top, scale, inv);
  if (team.first() && l.on) a.out.dev_scales[row] = scale;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[kRun];
    open_words<DT>(p[i], v);
    put_codes<HOW>(codes_of(a.out, row, l.col), a.vec_c, l, i, signed_codes(v, inv));
  }
}

// Rows longer than a block's registers hold: in shared memory between two passes (1021 x 25087 bf16 21 us, read twice 25; fp32 32 and 39), where two
// blocks of an SM have room for them.
template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kPackThreads, 2)
pack_rows8_long_kernel(const __grid_constant__ PackArgs a, bool keep) {
  extern __shared__ uint4 kept[];
  __shared__ float2 slots[16];
  const Team<false, N> team(0);
  const int64_t row = team.row;
  train_pdl_wait();
  if (threadIdx.x == 0) ahead(static_cast<const typename Elem<DT>::T*>(a.x) + row * a.ld_x, (int64_t)a.cols * (int)sizeof(typename Elem<DT>::T));
  const int each = blockDim.x * N * kRun, steps = (a.cols + each - 1) / each;
  float none = 0.f, top = 0.f, scale, inv = 0.f;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int k = 0; k < steps; ++k) {
      const Lanes l = team.lanes(a.cols, true, k);
      Piece<DT> p[N];
      if (pass == 1 && keep) {
        kept_runs<DT>(kept, k, p);
      } else {
        const Cursor<DT, HOW> x(a.x, row * a.ld_x, l);
        Raw<DT, HOW> raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) fetch(x, l, i, raw[i]);
        settle(raw, x, l, p);
        if (keep) keep_runs<DT>(kept, k, p);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float v[kRun];
        open_words<DT>(p[i], v);
        if (pass == 0) top = largest(top, v);
        else put_codes<HOW>(codes_of(a.out, row, l.col), a.vec_c, l, i, signed_codes(v, inv));
      }
    }
    if (pass == 0) {
      team.template join<true>(none, top, slots);
      row_scale(top, scale, inv);
      if (team.first()) a.out.dev_scales[row] = scale;
    }
  }
}

// ---- streams: a warp takes a strip of N runs per lane of one row, or, of rows of up to 128 columns, one run per lane of several rows
struct Strips {
  int64_t rows;
  int32_t cols, lane_shift;
  uint32_t per_row;                          // strips
};
template <int N>
struct Strip {
  Lanes l;
  int64_t row;
  __device__ __forceinline__ explicit Strip(const Strips& s) {
    const uint32_t warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), me = threadIdx.x & 31;
    l.lanes = 1 << s.lane_shift;
    l.lane = me & (l.lanes - 1);
    uint32_t in = 0;
    if (s.lane_shift < 5) {
      row = (int64_t)warp * (32 >> s.lane_shift) + (me >> s.lane_shift);
    } else {
      row = warp / s.per_row;
      in = warp - (uint32_t)row * s.per_row;
    }
    l.col = (int)in * N * kWarpCols + l.lane * kRun;
    l.left = s.cols - l.col;
    l.on = row < s.rows;
  }
};

template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kThreads)
unpack_rows8_kernel(const __grid_constant__ Strips s, lqsgd_rows8 in, bool vec_c, void* y, int64_t ld_y) {
  const Strip<N> w(s);
  const Lanes& l = w.l;
  train_pdl_wait();
  uint2 c[N];
  float scale = 0.f;
  if (l.on) scale = in.dev_scales[w.row];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    c[i] = make_uint2(0u, 0u);
    if (l.on && l.have(i) > 0) c[i] = load_codes(codes_of(in, w.row, l.col) + i * kWarpCols, HOW == kWhole || (vec_c && l.have(i) >= kRun), min(l.have(i), kRun));
  }
  const Cursor<DT, HOW> out(y, w.row * ld_y, l);
  Piece<DT> p[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = (float)(int8_t)((j < 4 ? c[i].x : c[i].y) >> (8 * (j & 3))) * scale;
    // past the type's range (for the source's own type: only by the scale's rounding): the largest finite value; a NaN stays
    constexpr float kTop = DT == LQSGD_F16 ? 65504.f : (DT == LQSGD_BF16 ? 3.3895314e38f : 3.402823466e38f);
    if (scale > kTop / 128.5f) {
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (fabsf(v[j]) > kTop) v[j] = copysignf(kTop, v[j]);
    }
    close_words<DT>(v, p[i]);
  }
  put(out, l, p);
}

template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kThreads, 3)
dropout_kernel(const __grid_constant__ Strips s, const void* x, int64_t ld_x, const void* residual, int64_t ld_r, const __grid_constant__ Drop drop, void* out, int64_t ld_o) {
  __shared__ uint32_t room[kDropRoom];
  const Strip<N> w(s);
  const Lanes& l = w.l;
  const Cursor<DT, HOW> cx(x, w.row * ld_x, l), cr(residual, w.row * ld_r, l), co(out, w.row * ld_o, l);
  train_pdl_wait();
  open_drop(drop, room);
  Raw<DT, HOW> rx[N], rr[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    fetch(cx, l, i, rx[i]);
    if (residual) fetch(cr, l, i, rr[i]);
  }
  const uint64_t block = (uint64_t)w.row * (uint32_t)((s.cols + kRun - 1) / kRun) + l.col / kRun;
  Piece<DT> p[N], pr[N];
  settle(rx, cx, l, p);
  if (residual) settle(rr, cr, l, pr);
  uint4 bits[N];
  drop_bits(drop, room, block, bits);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[kRun], sum[kRun];
    clear_run(sum);
    if (residual) open_words<DT>(pr[i], sum);
    open_words<DT>(p[i], v);
    drop_run(drop, bits[i], v, sum);
    close_words<DT>(sum, p[i]);
  }
  put(co, l, p);
}

template <int DT, int HOW>
cudaError_t launch_pack(PackArgs a, cudaStream_t st) {
  constexpr int kRuns = DT == LQSGD_F32 ? 2 : 4;              // 64 bytes per thread
  const RowShape s = shape_of(a.cols, kRuns, 1024, kPackThreads);
  if (!s.held) {
    static std::atomic<uint64_t> ready{0};
    auto kernel = pack_rows8_long_kernel<DT, kRuns, HOW>;
    const int threads = long_threads(a.cols, kRuns, kPackThreads);
    const size_t keep = long_keep(a.cols, kRuns, (int)sizeof(typename Elem<DT>::T), threads);
    const cudaError_t e = allow_keep(reinterpret_cast<const void*>(kernel), ready);
    return e != cudaSuccess ? e : train_launch(kernel, dim3((unsigned)a.rows), dim3(threads), keep, st, 1, a, keep > 0);
  }
  a.lane_shift = s.lane_shift;
  const dim3 grid((unsigned)ceil_div64(a.rows, s.teams)), block(s.threads);
#define GO(N, NARROW) train_launch(pack_rows8_kernel<DT, N, NARROW, HOW>, grid, block, 0, st, 1, a)
  if (s.narrow) return s.n == 1 ? GO(1, true) : s.n == 2 ? GO(2, true) : GO(4, true);
  return GO(kRuns, false);
#undef GO
}
// Strips of up to `most` runs per lane.
Strips strips_of(int64_t rows, int32_t cols, int most, int* n, dim3* grid) {
  Strips s = {rows, cols, 2, 1};
  while (s.lane_shift < 5 && (kRun << s.lane_shift) < cols) ++s.lane_shift;
  *n = 1;
  while (*n < most && *n * kWarpCols < cols) *n *= 2;
  s.per_row = (uint32_t)ceil_div64(cols, (int64_t)*n * kWarpCols);
  const int64_t warps = s.lane_shift < 5 ? ceil_div64(rows, 32 >> s.lane_shift) : rows * s.per_row;
  *grid = dim3((unsigned)ceil_div64(warps, kWarps));
  return s;
}
template <int DT, int HOW>
cudaError_t launch_unpack(int64_t rows, int32_t cols, cudaStream_t st, const lqsgd_rows8& in, bool vec_c, void* y, int64_t ld_y) {
  int n;
  dim3 grid;
  const Strips s = strips_of(rows, cols, 4, &n, &grid);
#define GO(N) train_launch(unpack_rows8_kernel<DT, N, HOW>, grid, dim3(kThreads), 0, st, 1, s, in, vec_c, y, ld_y)
  return n == 1 ? GO(1) : n == 2 ? GO(2) : GO(4);
#undef GO
}
template <int DT, int HOW>
cudaError_t launch_dropout(int64_t rows, int32_t cols, cudaStream_t st, const void* x, int64_t ld_x, const void* r, int64_t ld_r, const Drop& drop, void* out, int64_t ld_o) {
  int n;
  dim3 grid;
  const Strips s = strips_of(rows, cols, DT == LQSGD_F32 ? 2 : 4, &n, &grid);
#define GO(N) train_launch(dropout_kernel<DT, N, HOW>, grid, dim3(kThreads), 0, st, 1, s, x, ld_x, r, ld_r, drop, out, ld_o)
  if constexpr (DT == LQSGD_F32) return n == 1 ? GO(1) : GO(2);
  else return n == 1 ? GO(1) : n == 2 ? GO(2) : GO(4);
#undef GO
}

int check_shape(int64_t rows, int32_t cols) {
  return rows < 0 || rows > (1 << 28) || cols < 1 || cols > (1 << 24) || rows * cols > (1ll << 40) ? LQSGD_ERR_BAD_SHAPE : LQSGD_OK;
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
  const PackArgs a = {dev_x, ld_x, rows, *host_out, cols, 0, vc};
  TRAIN_CK(BY_TYPE(dtype, access_of(vx, vc, cols), launch_pack, a, static_cast<cudaStream_t>(cuda_stream)), "pack_rows8_kernel launch");
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
  TRAIN_CK(BY_TYPE(dtype, access_of(vy, vc, cols), launch_unpack, rows, cols, static_cast<cudaStream_t>(cuda_stream), *host_in, vc, dev_y, ld_y), "unpack_rows8_kernel launch");
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
  TRAIN_CK(BY_TYPE(dtype, access_of(vx && vr && vo, true, cols), launch_dropout, rows, cols, static_cast<cudaStream_t>(cuda_stream), dev_x, ld_x, dev_residual,
                   ld_residual, make_drop(*host_drop), dev_out, ld_out), "dropout_kernel launch");
  return LQSGD_OK;
}
