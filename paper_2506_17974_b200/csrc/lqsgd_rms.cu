// Root-mean-square norm of rows with dropout and the residual's addition in front of it (lqsgd_rms_norm_*).
//
// Both directions are streams that need one sum per row before they can write, and what bounds them is HBM, closely followed by the
// instructions: random bits, two 8-bit forms and the sum cost 350 a run of 8 columns, where HBM leaves time for 330.  So a row's values are
// read once and stay in registers, as they are stored, while its threads agree on the sum; the steps of a thread's runs interleave
// without branches between them; and arithmetic goes two values to an instruction.
// Rows of up to 1024 columns (512 backward) are held by 4 to 32 lanes of a warp, longer ones by a block: forward up to 13312 columns (10240 at any
// alignment; fp32 6656), backward up to 8192.  Rows beyond are read twice: forward by one block, the second time from L2; backward by two kernels, each
// over the whole matrix, so that what does not fit L2 comes from HBM twice (1021 x 25088 bf16 72 us, of which 28 are its bytes read once).
// Measured, 8192 x 4096 bf16: norm alone 27 us (5.0 TB/s), with a residual 43 (6.2 TB/s), with dropout, residual and both kept copies 57 (6.0 TB/s);
// its gradient with skip 59 (4.5 TB/s), with dropout from 8-bit h 81 (3.7 TB/s).  Gradients of fp32, two runs
// a thread as of 16 bits, spill registers: 64 bytes a thread in the aligned block (8192 x 4096 127 us), 540 at any alignment; 244 and 656 where rows
// are narrow, 228 and 412 in strips.
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
  float eps, per_col;                        // 1 / cols
  bool vec_gamma, vec_h8, vec_y8, vec_r8;    // on 16 bytes; rows of 8-bit copies on 8
};
// Forward: 64 bytes of each matrix per thread (4 runs of a 16-bit type), and blocks of as many threads as leave registers for a second block on
// an SM, which loads while the first one waits for its sum (16384 columns of bf16 in one block of 512: 82 us at 4000 rows, read twice 60; 12000 with
// everything in two blocks of 384: 50 at 2000 rows, read twice 71).
constexpr int kNarrow = 1024, kForwardThreads = 416;
template <int DT> constexpr int kForwardRuns = DT == LQSGD_F32 ? 2 : 4;
template <int DT> constexpr int kLongRuns = DT == LQSGD_F32 ? 1 : 2;     // rows in steps: twice the threads in their place (four runs, balanced: 75 us to 58)
constexpr int forward_threads(int dtype, int how) { return how == kWhole || dtype == LQSGD_F32 ? kForwardThreads : 320; }
constexpr int kLongThreads = 448, kGradThreads = 512, kGradRuns = 2;

// What a thread touches of one row of the forward call.
template <int DT, int HOW>
struct ForwardRow {
  const RmsArgs& a;
  const uint32_t (&room)[kDropRoom];
  Lanes l;
  int64_t row;
  Cursor<DT, HOW> x, residual, h, y;
  const float* gamma;
  uint64_t block;                            // dropout's of the thread's first run
  __device__ __forceinline__ ForwardRow(const RmsArgs& a_, const uint32_t (&room_)[kDropRoom], int64_t row_, const Lanes& l_)
      : a(a_), room(room_), l(l_), row(row_), x(a.x, row * a.ld_x, l), residual(a.residual, row * a.ld_residual, l), h(a.h, row * a.ld_h, l),
        y(a.y, row * a.ld_y, l), gamma(a.gamma + l.col), block((uint64_t)row * (uint32_t)((a.cols + kRun - 1) / kRun) + l.col / kRun) {}
  __device__ __forceinline__ void ask(int i, Raw<DT, HOW>& rx, Raw<DT, HOW>& rr) const {
    fetch(x, l, i, rx);
    if (a.residual) fetch(residual, l, i, rr);
  }
  // h = residual + dropout(x) of all runs, as it is stored
  template <int N>
  __device__ __forceinline__ void make_h(const Raw<DT, HOW> (&rx)[N], const Raw<DT, HOW> (&rr)[N], Piece<DT> (&ph)[N]) const {
    settle(rx, x, l, ph);
    if (!a.h) return;
    Piece<DT> pr[N];
    if (a.residual) settle(rr, residual, l, pr);
    float v[kRun], r[kRun];
    if (a.drop.threshold) {
      uint4 bits[N];
      drop_bits(a.drop, room, block, bits);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        clear_run(r);
        if (a.residual) open_words<DT>(pr[i], r);
        open_words<DT>(ph[i], v);
        drop_run(a.drop, bits[i], v, r);
        close_words<DT>(r, ph[i]);
      }
    } else if (a.residual) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        open_words<DT>(pr[i], r);
        open_words<DT>(ph[i], v);
        add_run(r, r, v);
        close_words<DT>(r, ph[i]);
      }
    }
  }
  // squares into `sum`, the largest |h gamma| into `top`
  __device__ __forceinline__ void add_squares(int i, const Piece<DT>& ph, float (&sum)[2], float& top) const {
    float v[kRun];
    open_words<DT>(ph, v);
    dot_run(sum, v, v);
    if (a.r8.dev_codes) {
      float g[kRun];
      fetch_vector<HOW>(gamma, a.vec_gamma, l, i, g);
      mul_run(g, g, v);
      top = largest(top, g);
    }
  }
  // The row's figures, written by one of its threads.  A product h gamma is off by up to 2^-150 at the range's lower end, which a large rstd (no
  // eps, small rows) carries up: with twice the smallest number on top of the largest one no code passes 127.
  __device__ __forceinline__ void figures(bool mine, float sum, float top, float& rstd, float& inv) const {
    rstd = rsqrtf(fmaf(sum, a.per_col, a.eps));
    float scale = 0.f;
    if (a.r8.dev_codes) row_scale((top + 2.80259693e-45f) * rstd, scale, inv);
    if (mine && l.on) {
      a.rstd[row] = rstd;
      if (a.r8.dev_codes) a.r8.dev_scales[row] = scale;
    }
  }
  // y of all runs and the copies in 8 bits
  template <int N>
  __device__ __forceinline__ void put_y(float rstd, float inv, const Piece<DT> (&ph)[N]) const {
    Piece<DT> py[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v[kRun], g[kRun];
      open_words<DT>(ph[i], v);
      fetch_vector<HOW>(gamma, a.vec_gamma, l, i, g);
      if (a.h8.dev_codes) put_packed_run<HOW>(a.h8.dev_codes + row * a.h8.ld_codes + l.col, a.h8.dev_exps + row * a.h8.ld_exps + l.col / kGroup, a.vec_h8, l, i, v);
      mul_run(v, v, rstd);
      mul_run(v, v, g);
      if (a.r8.dev_codes) put_codes<HOW>(reinterpret_cast<uint8_t*>(a.r8.dev_codes) + row * a.r8.ld_codes + l.col, a.vec_r8, l, i, signed_codes(v, inv));
      if (!a.y && !a.y8.dev_codes) continue;
      close_words<DT>(v, py[i]);
      if (a.y8.dev_codes) {
        open_words<DT>(py[i], v);
        put_packed_run<HOW>(a.y8.dev_codes + row * a.y8.ld_codes + l.col, a.y8.dev_exps + row * a.y8.ld_exps + l.col / kGroup, a.vec_y8, l, i, v);
      }
    }
    if (a.y) put(y, l, py);
  }
};

template <int DT, int N, bool NARROW, int HOW>
__global__ void __launch_bounds__(NARROW ? 256 : kForwardThreads)
rms_forward_kernel(const __grid_constant__ RmsArgs a) {
  __shared__ float2 slots[16];
  __shared__ uint32_t room[kDropRoom];
  const Team<NARROW, N> team(a.lane_shift);
  const ForwardRow<DT, HOW> io(a, room, team.row, team.lanes(a.cols, !NARROW || team.row < a.rows));
  train_pdl_wait();
  open_drop(a.drop, room);
  Raw<DT, HOW> x[N], res[N];
#pragma unroll
  for (int i = 0; i < N; ++i) io.ask(i, x[i], res[i]);
  Piece<DT> h[N];
  float sum[2] = {0.f, 0.f}, top = 0.f, rstd, inv = 0.f;
  io.make_h(x, res, h);
  if (a.h) put(io.h, io.l, h);
#pragma unroll
  for (int i = 0; i < N; ++i) io.add_squares(i, h[i], sum, top);
  sum[0] += sum[1];
  if (a.r8.dev_codes) team.template join<true>(sum[0], top, slots);
  else team.template join<false>(sum[0], top, slots);
  io.figures(team.first(), sum[0], top, rstd, inv);
  io.put_y(rstd, inv, h);
}

// Rows longer than a block holds: h is computed (and stored) in a first pass and read again, from L2, in a second.
template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kLongThreads, 2)
rms_forward_long_kernel(const __grid_constant__ RmsArgs a) {
  __shared__ float2 slots[16];
  __shared__ uint32_t room[kDropRoom];
  constexpr int kSize = (int)sizeof(typename Elem<DT>::T);
  const Team<false, N> team(0);
  train_pdl_wait();
  if (threadIdx.x == 0) {                                  // the whole row on its way: the first pass waits for its first step only
    ahead(static_cast<const char*>(a.x) + team.row * a.ld_x * kSize, (int64_t)a.cols * kSize);
    if (a.residual) ahead(static_cast<const char*>(a.residual) + team.row * a.ld_residual * kSize, (int64_t)a.cols * kSize);
  }
  open_drop(a.drop, room);
  const int each = blockDim.x * N * kRun, steps = (a.cols + each - 1) / each;
  float sum[2] = {0.f, 0.f}, top = 0.f, rstd = 0.f, inv = 0.f;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int k = 0; k < steps; ++k) {
      const ForwardRow<DT, HOW> io(a, room, team.row, team.lanes(a.cols, true, k));
      Piece<DT> h[N];
      if (pass == 0) {
        Raw<DT, HOW> x[N], res[N];
#pragma unroll
        for (int i = 0; i < N; ++i) io.ask(i, x[i], res[i]);
        io.make_h(x, res, h);
        if (a.h) put(io.h, io.l, h);
#pragma unroll
        for (int i = 0; i < N; ++i) io.add_squares(i, h[i], sum, top);
      } else {                                               // what other threads of the block wrote of it lies behind the sum's barrier
        const Cursor<DT, HOW>& from = a.h ? io.h : io.x;
        Raw<DT, HOW> raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) fetch(from, io.l, i, raw[i]);
        settle(raw, from, io.l, h);
        io.put_y(rstd, inv, h);
      }
    }
    if (pass == 0) {
      sum[0] += sum[1];
      team.template join<true>(sum[0], top, slots);
      ForwardRow<DT, HOW>(a, room, team.row, team.lanes(a.cols, true)).figures(team.first(), sum[0], top, rstd, inv);
    }
  }
}

// ---- backward
// A row needs <u xh>, xh = h rstd, and then d = (gamma rstd) dy - (rstd <u xh>) xh + skip.  (With h itself in the place of xh a run takes 8
// multiplications less, but products of very large or small rows leave fp32's range on the way.)
// A team walks rows: loads of all runs, the sum, stores; its columns' sums for dgamma stay in registers.  That leaves at most 16 warps an SM (a block
// of 9 to 16 alone from 4097 columns on: 4000 x 4097 bf16 81 us, 4000 x 7168 58, at floors of 18 and 26), too few to hide HBM's latency, so one thread asks L2 for the next row meanwhile (8192 x 4096 without dropout, at that step, 75 -> 61 us, fp32 136 -> 122).  h from its
// 8-bit form is decoded once, to bf16, in which it is exact.
// Eight codes as bf16: |128 + m| with the magnitude m below is a bf16 number (0x4300 | m), and (128 + m) 2^e - 128 2^e is m 2^e exactly; the
// signs are put on top.  For exponents from kQuickByte on 128 2^e leaves the range.
__device__ __forceinline__ void decode_bf16(uint2 c, uint32_t eb, uint32_t (&w)[4]) {
  if (eb <= kQuickByte) {
    const uint32_t step = ((eb + 1) << 7) * 0x00010001u, off = (((eb + 8) << 7) | 0x8000u) * 0x00010001u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t of = j < 2 ? c.x : c.y, m = of & 0x7f7f7f7fu;
      const uint32_t big = __byte_perm(m, 0x43u, j & 1 ? 0x4342 : 0x4140), sign = __byte_perm(of, 0u, j & 1 ? 0x3424 : 0x1404);
      uint32_t r;
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(big), "r"(step), "r"(off));
      w[j] = r | (sign & 0x80008000u);
    }
  } else {
    float v[kRun];
    decode_run(c, (int)eb, v);
    constexpr float kTop = 3.3895314e38f;                  // of bf16; a NaN stays
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = fabsf(v[j]) > kTop ? copysignf(kTop, v[j]) : v[j];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_pair<LQSGD_BF16>(v[2 * j], v[2 * j + 1]);
  }
}
__device__ __forceinline__ void open_bf16(const uint32_t (&w)[4], float (&v)[kRun]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = open_pair<LQSGD_BF16>(w[j]);
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
}
// What a thread reads of one row of the backward call.
template <int DT, int HOW>
struct BackwardRow {
  Lanes l;
  int64_t row;
  Cursor<DT, HOW> dy, h, skip;
  __device__ __forceinline__ BackwardRow(const RmsArgs& a, int64_t row_, const Lanes& l_)
      : l(l_), row(row_), dy(a.dy, row * a.ld_dy, l), h(a.h, row * a.ld_h, l), skip(a.skip, row * a.ld_skip, l) {}
  // codes and exponent of run i of h's 8-bit form
  __device__ __forceinline__ uint2 codes(const RmsArgs& a, int i) const {
    const uint8_t* c = a.h8.dev_codes + row * a.h8.ld_codes + l.col + i * kWarpCols;
    if (!l.has(i)) return make_uint2(0u, 0u);
    return load_codes(c, HOW == kWhole || (a.vec_h8 && l.have(i) >= kRun), min(l.have(i), kRun));
  }
  __device__ __forceinline__ uint32_t exponent(const RmsArgs& a, int i) const {
    return l.has(i) ? a.h8.dev_exps[row * a.h8.ld_exps + l.col / kGroup + i * (kWarpCols / kGroup)] : kExpBias;
  }
};
template <int DT>
__device__ __forceinline__ void open_h(const RmsArgs& a, const Piece<DT>& h, float (&v)[kRun]) {
  if (DT != LQSGD_BF16 && a.h8.dev_codes) {
    const uint32_t w[4] = {h.w[0], h.w[1], h.w[2], h.w[3]};
    open_bf16(w, v);
  } else {
    open_words<DT>(h, v);
  }
}
// d of a thread's N runs into dx and dresidual.
template <int DT, int HOW, int N>
__device__ __forceinline__ void put_d(const RmsArgs& a, const uint32_t (&room)[kDropRoom], const BackwardRow<DT, HOW>& r, float (&d)[N][kRun]) {
  Piece<DT> out[N];
  auto write = [&](void* matrix, int64_t ld) {
    put(Cursor<DT, HOW>(matrix, r.row * ld, r.l), r.l, out);
  };
  if (a.dresidual || !a.drop.threshold) {
#pragma unroll
    for (int i = 0; i < N; ++i) close_words<DT>(d[i], out[i]);
  }
  if (a.dresidual) write(a.dresidual, a.ld_dresidual);
  if (!a.dx) return;
  if (a.drop.threshold) {
    uint4 bits[N];
    drop_bits(a.drop, room, (uint64_t)r.row * (uint32_t)((a.cols + kRun - 1) / kRun) + r.l.col / kRun, bits);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t[kRun];
      clear_run(t);
      drop_run(a.drop, bits[i], d[i], t);
      close_words<DT>(t, out[i]);
    }
  }
  write(a.dx, a.ld_dx);
}

// The rows that a team comes to next.
template <int DT>
__device__ __forceinline__ void rows_ahead(const RmsArgs& a, int64_t row, bool with_skip) {
  constexpr int kSize = (int)sizeof(typename Elem<DT>::T);
  if (row >= a.rows) return;
  ahead(static_cast<const char*>(a.dy) + row * a.ld_dy * kSize, (int64_t)a.cols * kSize);
  if (with_skip && a.skip) ahead(static_cast<const char*>(a.skip) + row * a.ld_skip * kSize, (int64_t)a.cols * kSize);
  if (a.h8.dev_codes) ahead(a.h8.dev_codes + row * a.h8.ld_codes, a.cols);
  else ahead(static_cast<const char*>(a.h) + row * a.ld_h * kSize, (int64_t)a.cols * kSize);
}

template <int DT, int N, bool NARROW, int HOW>
__global__ void __launch_bounds__(NARROW ? 256 : kGradThreads, NARROW ? 2 : 1)
rms_backward_kernel(const __grid_constant__ RmsArgs a) {
  __shared__ float2 slots[2][16];
  __shared__ float sums[NARROW ? 256 * (kRun + 1) : 1];
  __shared__ uint32_t room[kDropRoom];
  const Team<NARROW, N> team(a.lane_shift);
  train_pdl_wait();
  open_drop(a.drop, room);
  float acc[N][kRun];
#pragma unroll
  for (int i = 0; i < N; ++i) clear_run(acc[i]);
  int turn = 0;
  // NARROW: a warp stays together while one of its rows exists
  const int64_t first = NARROW ? team.row - ((threadIdx.x & 31) >> team.shift) : team.row;
#pragma unroll 1
  for (int64_t r0 = first; r0 < a.rows; r0 += team.rows_per_grid) {
    const int64_t row = team.row + (r0 - first);
    if (!NARROW && threadIdx.x == 0) rows_ahead<DT>(a, row + team.rows_per_grid, true);
    const BackwardRow<DT, HOW> r(a, row, team.lanes(a.cols, row < a.rows));
    const float* gamma = a.gamma + r.l.col;
    // Skip is needed behind the sum only: fetched in front of the barrier it takes no registers before (8192 x 4096 fp32 140 -> 126 us).  Runs at any
    // alignment and narrow rows, which have no barrier, lose 3 to 6 % that way.
    constexpr bool kLate = !NARROW && HOW == kWhole;
    Raw<DT, HOW> raw_skip[N];
    auto ask_skip = [&] {
      if (!a.skip) return;
#pragma unroll
      for (int i = 0; i < N; ++i) fetch(r.skip, r.l, i, raw_skip[i]);
    };
    Piece<DT> dy[N], h[N], skip[N];
    {
      Raw<DT, HOW> raw_dy[N], raw_h[N];
      uint2 codes[N];
      uint32_t exps[N];
#pragma unroll
      for (int i = 0; i < N; ++i) fetch(r.dy, r.l, i, raw_dy[i]);
      if (a.h8.dev_codes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          codes[i] = r.codes(a, i);
          exps[i] = r.exponent(a, i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) fetch(r.h, r.l, i, raw_h[i]);
      }
      if (!kLate) ask_skip();
      if (a.h8.dev_codes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          uint32_t w[4];
          decode_bf16(codes[i], exps[i], w);
#pragma unroll
          for (int k = 0; k < 4; ++k) h[i].w[k] = w[k];
        }
      } else {
        settle(raw_h, r.h, r.l, h);
      }
      settle(raw_dy, r.dy, r.l, dy);
      if (!kLate && a.skip) settle(raw_skip, r.skip, r.l, skip);
    }
    const float rstd = r.l.on ? a.rstd[row] : 0.f;
    float sum[2] = {0.f, 0.f}, none = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float u[kRun], v[kRun], g[kRun];
      open_words<DT>(dy[i], u);
      open_h<DT>(a, h[i], v);
      fetch_vector<HOW>(gamma, a.vec_gamma, r.l, i, g);
      mul_run(v, v, rstd);
      fma_run(acc[i], u, v, acc[i]);
      mul_run(u, u, g);
      dot_run(sum, u, v);
    }
    if (kLate) ask_skip();
    sum[0] += sum[1];
    team.template join<false>(sum[0], none, slots[turn]);
    turn ^= 1;
    if (kLate && a.skip) settle(raw_skip, r.skip, r.l, skip);
    const float k = rstd * (sum[0] * a.per_col);
    float d[N][kRun];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v[kRun], g[kRun];
      clear_run(d[i]);
      if (a.skip) open_words<DT>(skip[i], d[i]);
      open_h<DT>(a, h[i], v);
      mul_run(v, v, rstd);
      fma_run(d[i], v, -k, d[i]);
      open_words<DT>(dy[i], v);
      fetch_vector<HOW>(gamma, a.vec_gamma, r.l, i, g);
      mul_run(g, g, rstd);
      fma_run(d[i], g, v, d[i]);
    }
    put_d<DT, HOW, N>(a, room, r, d);
  }
  if (!a.partial) return;
  float* out = a.partial + (size_t)blockIdx.x * a.cols;
  const Lanes l = team.lanes(a.cols, true);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (NARROW) {                                          // the block's rows meet in shared memory
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kRun; ++j) sums[threadIdx.x * (kRun + 1) + j] = acc[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < l.lanes * kRun; c += 256) {
        const int col = i * kWarpCols + c;
        if (col >= a.cols) continue;
        float t = 0.f;
        for (int k = 0; k < 256 >> team.shift; ++k) t += sums[((k << team.shift) + c / kRun) * (kRun + 1) + c % kRun];
        out[col] = t;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (j < l.have(i)) out[l.col + i * kWarpCols + j] = acc[i][j];
    }
  }
}

// Rows longer than a block holds: <u xh> of each in a first kernel, the rest as a stream over columns.
// A thread's N runs of a row as they are fetched.
template <int DT, int N, int HOW>
struct GradRuns {
  BackwardRow<DT, HOW> r;
  Raw<DT, HOW> dy[N], h[N], skip[N];
  uint2 codes[N];
  uint32_t exps[N];
  __device__ __forceinline__ GradRuns(const RmsArgs& a, int64_t row, const Lanes& l, bool with_skip) : r(a, row, l) {
#pragma unroll
    for (int i = 0; i < N; ++i) fetch(r.dy, l, i, dy[i]);
    if (a.h8.dev_codes) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        codes[i] = r.codes(a, i);
        exps[i] = r.exponent(a, i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) fetch(r.h, l, i, h[i]);
    }
    if (with_skip && a.skip) {
#pragma unroll
      for (int i = 0; i < N; ++i) fetch(r.skip, l, i, skip[i]);
    }
  }
  // dy and h as words (h from its 8-bit form as bf16: open_h)
  __device__ __forceinline__ void settle_dy_h(const RmsArgs& a, Piece<DT> (&pd)[N], Piece<DT> (&ph)[N]) const {
    settle(dy, r.dy, r.l, pd);
    if (a.h8.dev_codes) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint32_t w[4];
        decode_bf16(codes[i], exps[i], w);
#pragma unroll
        for (int k = 0; k < 4; ++k) ph[i].w[k] = w[k];
      }
    } else {
      settle(h, r.h, r.l, ph);
    }
  }
};
template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kLongThreads, 2)
rms_dot_kernel(const __grid_constant__ RmsArgs a, float* dots) {
  __shared__ float2 slots[16];
  const Team<false, N> team(0);
  train_pdl_wait();
  if (threadIdx.x == 0) rows_ahead<DT>(a, team.row, false);
  const float rstd = a.rstd[team.row];
  float sum[2] = {0.f, 0.f}, top = 0.f;
  const int each = blockDim.x * N * kRun, steps = (a.cols + each - 1) / each;
#pragma unroll 1
  for (int k = 0; k < steps; ++k) {
    const GradRuns<DT, N, HOW> p(a, team.row, team.lanes(a.cols, true, k), false);
    Piece<DT> dy[N], h[N];
    p.settle_dy_h(a, dy, h);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float u[kRun], v[kRun], g[kRun];
      open_words<DT>(dy[i], u);
      open_h<DT>(a, h[i], v);
      fetch_vector<HOW>(a.gamma + p.r.l.col, a.vec_gamma, p.r.l, i, g);
      mul_run(v, v, rstd);
      mul_run(u, u, g);
      dot_run(sum, u, v);
    }
  }
  sum[0] += sum[1];
  team.template join<false>(sum[0], top, slots);
  if (team.first()) dots[team.row] = sum[0] * a.per_col;
}
// A warp walks down N runs per lane; a block's warps stand side by side, so that a row's piece is several kilobytes (each of eight rows of their
// own: 1021 x 40000 118 us, so 103; 25088, whose last strip is ragged, 69 and 72).  blockIdx.x = strip, blockIdx.y = block of rows.
template <int DT, int N, int HOW>
__global__ void __launch_bounds__(kThreads, 2)
rms_columns_kernel(const __grid_constant__ RmsArgs a, int64_t rows_per_block, const float* dots) {
  __shared__ uint32_t room[kDropRoom];
  constexpr int kSize = (int)sizeof(typename Elem<DT>::T);
  train_pdl_wait();
  open_drop(a.drop, room);
  const int lane = threadIdx.x & 31, strip = (int)(blockIdx.x * kWarps + (threadIdx.x >> 5)) * N * kWarpCols, wide = min(N * kWarpCols, a.cols - strip);
  if (wide <= 0) return;
  const Lanes l = {strip + lane * kRun, a.cols - strip - lane * kRun, lane, 32, true};
  float acc[N][kRun];
#pragma unroll
  for (int i = 0; i < N; ++i) clear_run(acc[i]);
  const int64_t end = min(a.rows, (int64_t)(blockIdx.y + 1) * rows_per_block);
#pragma unroll 1
  for (int64_t row = blockIdx.y * rows_per_block; row < end; ++row) {
    if (lane == 0 && row + 1 < end) {
      const int64_t next = row + 1;
      ahead(static_cast<const char*>(a.dy) + (next * a.ld_dy + strip) * kSize, wide * kSize);
      if (a.skip) ahead(static_cast<const char*>(a.skip) + (next * a.ld_skip + strip) * kSize, wide * kSize);
      if (a.h8.dev_codes) ahead(a.h8.dev_codes + next * a.h8.ld_codes + strip, wide);
      else ahead(static_cast<const char*>(a.h) + (next * a.ld_h + strip) * kSize, wide * kSize);
    }
    const GradRuns<DT, N, HOW> p(a, row, l, true);
    const float rstd = a.rstd[row], k = rstd * dots[row];
    Piece<DT> dy[N], h[N], skip[N];
    p.settle_dy_h(a, dy, h);
    if (a.skip) settle(p.skip, p.r.skip, l, skip);
    float d[N][kRun];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float u[kRun], v[kRun], g[kRun];
      open_words<DT>(dy[i], u);
      open_h<DT>(a, h[i], v);
      clear_run(d[i]);
      if (a.skip) open_words<DT>(skip[i], d[i]);
      mul_run(v, v, rstd);
      fma_run(d[i], v, -k, d[i]);
      fma_run(acc[i], u, v, acc[i]);
      fetch_vector<HOW>(a.gamma + l.col, a.vec_gamma, l, i, g);
      mul_run(g, g, rstd);
      fma_run(d[i], u, g, d[i]);
    }
    put_d<DT, HOW, N>(a, room, p.r, d);
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      if (j < l.have(i)) a.partial[(size_t)blockIdx.y * a.cols + l.col + i * kWarpCols + j] = acc[i][j];
}

// ---- choice of kernel
constexpr int kSms = 148;
struct GradPlan {
  RowShape shape;
  dim3 grid;
  int64_t rows_per_block;                    // of the kernel for long rows' columns
  int blocks;                                // of the sums over rows
  size_t off_partial, bytes;
};
GradPlan plan_backward(const lqsgd_rms_norm& a) {
  GradPlan p = {};
  p.shape = shape_of(a.cols, kGradRuns, 512, kGradThreads);
  if (!p.shape.held) {
    // blocks that fill the card, as many of them below one another as the strips of a row leave, of two rows at least
    const int64_t strips = ceil_div64(a.cols, kWarps * kGradRuns * kWarpCols);
    const int64_t below = std::max<int64_t>(1, std::min<int64_t>(kSms * 2 / strips, ceil_div64(a.rows, 2)));
    p.rows_per_block = ceil_div64(a.rows, below);
    p.grid = dim3((unsigned)strips, (unsigned)ceil_div64(a.rows, p.rows_per_block));
    p.blocks = (int)p.grid.y;
    p.off_partial = (size_t)ceil_div64(a.rows * 4, 256) * 256;
  } else {
    p.blocks = (int)std::min<int64_t>(ceil_div64(a.rows, p.shape.teams), kSms * (512 / p.shape.threads));    // what registers hold
    p.grid = dim3((unsigned)p.blocks);
  }
  p.bytes = p.off_partial + (a.dev_dgamma && p.blocks > 1 ? (size_t)p.blocks * a.cols * 4 : 0);
  return p;
}

// Blocks of equal steps (1021 x 25087 fp16 into codes: 58 us, in four steps of 256 threads of which the last is nearly empty 70), two of them on an SM; one step more
// if smaller blocks then fill the SM better (4000 x 16384: four steps of 256 threads, three blocks, 55 us; three steps of 352, two blocks, 64).
int walk_threads(int32_t cols, int n) {
  const int64_t runs = ceil_div64(cols, kRun), steps = ceil_div64(runs, (int64_t)n * kLongThreads);
  const int few = long_threads(runs, n, steps), more = long_threads(runs, n, steps + 1);
  return 2 * kLongThreads / few * few >= 2 * kLongThreads / more * more ? few : more;
}
template <int DT, int HOW>
cudaError_t launch_forward(RmsArgs a, cudaStream_t st) {
  const RowShape s = shape_of(a.cols, kForwardRuns<DT>, kNarrow, forward_threads(DT, HOW));
  a.lane_shift = s.lane_shift;
  if (!s.held) {
    const int threads = walk_threads(a.cols, kLongRuns<DT>);
    return train_launch(rms_forward_long_kernel<DT, kLongRuns<DT>, HOW>, dim3((unsigned)a.rows), dim3(threads), 0, st, 1, a);
  }
  const dim3 grid((unsigned)ceil_div64(a.rows, s.teams)), block(s.threads);
#define GO(N, NARROW) train_launch(rms_forward_kernel<DT, N, NARROW, HOW>, grid, block, 0, st, 1, a)
  if (s.narrow) return s.n == 1 ? GO(1, true) : s.n == 2 ? GO(2, true) : GO(4, true);
  return GO(kForwardRuns<DT>, false);
#undef GO
}
template <int DT, int HOW>
cudaError_t launch_backward(const GradPlan& p, const RmsArgs& a, float* dots, cudaStream_t st) {
  if (!p.shape.held) {
    const int threads = walk_threads(a.cols, kLongRuns<DT>);
    const cudaError_t e = train_launch(rms_dot_kernel<DT, kLongRuns<DT>, HOW>, dim3((unsigned)a.rows), dim3(threads), 0, st, 1, a, dots);
    return e != cudaSuccess ? e : train_launch(rms_columns_kernel<DT, kGradRuns, HOW>, p.grid, dim3(kThreads), 0, st, 1, a, p.rows_per_block, dots);
  }
  const RowShape& s = p.shape;
#define GO(N, NARROW) train_launch(rms_backward_kernel<DT, N, NARROW, HOW>, p.grid, dim3(s.threads), 0, st, 1, a)
  if (s.narrow) return s.n == 1 ? GO(1, true) : GO(2, true);
  return GO(kGradRuns, false);
#undef GO
}

int check_args(const lqsgd_rms_norm* a) {
  if (!a || a->struct_size != sizeof(lqsgd_rms_norm) || !train_dtype_ok(a->dtype)) return LQSGD_ERR_INVALID_ARG;
  if (a->rows < 0 || a->rows > (1 << 28) || a->cols < 1 || a->cols > (1 << 24) || a->rows * a->cols > (1ll << 40)) return LQSGD_ERR_BAD_SHAPE;
  return check_drop(a->drop);
}
// A matrix argument, or none.
int check_matrix(const void* p, int64_t ld, const lqsgd_rms_norm& a) {
  if (!p) return LQSGD_OK;
  if (ld < a.cols) return LQSGD_ERR_INVALID_ARG;
  return train_aligned(p, train_elem(a.dtype)) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}
// Whether its rows start on 16 bytes (an absent one does not stand in the way).
bool on16(const void* p, int64_t ld, const lqsgd_rms_norm& a) {
  return !p || (train_aligned(p, 16) && (a.rows == 1 || ld * train_elem(a.dtype) % 16 == 0));
}
bool on8(const void* p, int64_t ld, int64_t rows) { return !p || (train_aligned(p, 8) && (rows == 1 || ld % 8 == 0)); }
int backward_access(const lqsgd_rms_norm& a) {
  const bool rows = on16(a.dev_dy, a.ld_dy, a) && on16(a.dev_skip, a.ld_skip, a) && on16(a.dev_dx, a.ld_dx, a) && on16(a.dev_dresidual, a.ld_dresidual, a) &&
                    (a.h8.dev_codes || on16(a.dev_h, a.ld_h, a));
  return access_of(rows, train_aligned(a.dev_gamma, 16) && on8(a.h8.dev_codes, a.h8.ld_codes, a.rows), a.cols);
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

extern "C" int lqsgd_rms_norm_workspace_bytes(int32_t backward, const lqsgd_rms_norm* a, size_t* host_bytes_out) {
  if (!host_bytes_out || (backward != 0 && backward != 1)) return LQSGD_ERR_INVALID_ARG;
  const int rc = check_args(a);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = backward && a->rows > 0 ? plan_backward(*a).bytes : 0;
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
  if ((rc = check_matrix(a->dev_x, a->ld_x, *a)) != LQSGD_OK || (rc = check_matrix(a->dev_residual, a->ld_residual, *a)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_h, a->ld_h, *a)) != LQSGD_OK || (rc = check_matrix(a->dev_y, a->ld_y, *a)) != LQSGD_OK)
    return rc;
  const bool rows16 = on16(a->dev_x, a->ld_x, *a) && on16(a->dev_residual, a->ld_residual, *a) && on16(a->dev_h, a->ld_h, *a) && on16(a->dev_y, a->ld_y, *a);
  if (a->h8.dev_codes && (rc = check_packed8(a->h8, a->cols)) != LQSGD_OK) return rc;
  if (a->y8.dev_codes && (rc = check_packed8(a->y8, a->cols)) != LQSGD_OK) return rc;
  if (a->rows8.dev_codes && (rc = check_rows8(a->rows8, a->cols)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  k.x = a->dev_x; k.ld_x = a->ld_x; k.residual = a->dev_residual; k.ld_residual = a->ld_residual;
  k.h = a->dev_h; k.ld_h = a->ld_h; k.y = a->dev_y; k.ld_y = a->ld_y;
  k.gamma = a->dev_gamma; k.rstd = a->dev_rstd;
  k.h8 = a->h8; k.y8 = a->y8; k.r8 = a->rows8;
  k.drop = make_drop(a->drop);
  k.rows = a->rows; k.cols = a->cols; k.per_col = (float)(1.0 / a->cols); k.eps = a->eps;
  k.vec_gamma = train_aligned(a->dev_gamma, 16);
  k.vec_h8 = on8(a->h8.dev_codes, a->h8.ld_codes, a->rows);
  k.vec_y8 = on8(a->y8.dev_codes, a->y8.ld_codes, a->rows);
  k.vec_r8 = on8(a->rows8.dev_codes, a->rows8.ld_codes, a->rows);
  const int how = access_of(rows16, k.vec_gamma && k.vec_h8 && k.vec_y8 && k.vec_r8, a->cols);
  TRAIN_CK(BY_TYPE(a->dtype, how, launch_forward, k, static_cast<cudaStream_t>(cuda_stream)), "rms_forward_kernel launch");
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
  if ((rc = check_matrix(a->dev_dy, a->ld_dy, *a)) != LQSGD_OK || (rc = check_matrix(a->dev_skip, a->ld_skip, *a)) != LQSGD_OK ||
      (rc = check_matrix(a->dev_dx, a->ld_dx, *a)) != LQSGD_OK || (rc = check_matrix(a->dev_dresidual, a->ld_dresidual, *a)) != LQSGD_OK ||
      (rc = check_matrix(kept ? nullptr : a->dev_h, a->ld_h, *a)) != LQSGD_OK)
    return rc;
  if (kept && (rc = check_packed8(a->h8, a->cols)) != LQSGD_OK) return rc;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  k.vec_gamma = train_aligned(a->dev_gamma, 16);
  k.vec_h8 = on8(a->h8.dev_codes, a->h8.ld_codes, a->rows);
  const int how = backward_access(*a);
  const GradPlan p = plan_backward(*a);
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
  k.rows = a->rows; k.cols = a->cols; k.per_col = (float)(1.0 / a->cols); k.lane_shift = p.shape.lane_shift;
  TRAIN_CK(BY_TYPE(a->dtype, how, launch_backward, p, k, reinterpret_cast<float*>(ws), st), "rms_backward_kernel launch");
  return a->dev_dgamma && p.blocks > 1 ? join_columns(k.partial, p.blocks, a->cols, a->dev_dgamma, st) : LQSGD_OK;
}
