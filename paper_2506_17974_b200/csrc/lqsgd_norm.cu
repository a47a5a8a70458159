// Group norm with an activation on channels-last tensors, forward and backward.
//
// A thread owns 8 consecutive channels and walks over pixels, so that a warp reads whole 16-byte pieces of neighbouring
// pixels, and what it sums stays in its registers per channel: groups of any width, and rows of any alignment, need no
// special case.  Per-channel sums of a chunk of pixels meet in a small kernel, which forms the groups' figures; the
// last kernel reads the tensor a second time and applies them.
//
// Forward sums are kept as (mean, sum of squared distances from it) about a value of the channel itself and merged
// pairwise: a mean far from zero cancels nothing.
#include "lqsgd_train_dev.cuh"

#include <algorithm>

namespace lqsgd {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kRun = 8;

struct NormDev {
  int32_t n, hw, c, groups, cpg, act;
  int32_t lane_shift, segs, chunks, chunk_rows;
  float eps;
  const void* x;  int64_t ld_x, sample_x;
  const void* dy; int64_t ld_dy, sample_dy;
  void* out;      int64_t ld_out, sample_out;
  const float* gamma;
  const float* beta;
  float* mean;
  float* rstd;
  float* dgamma;
  float* dbeta;
  lqsgd_packed8 x8, y8;
  int32_t vec_x, vec_dy, vec_out, vec_x8, vec_y8;
  float* part0;                       // [n][chunks][c]: means (forward), sums of dh (backward)
  float* part1;                       // [n][chunks][c]: squared distances (forward), sums of dh xh (backward)
  float* group0;                      // [n][groups]: <u> (backward)
  float* group1;                      // [n][groups]: <u xh> (backward)
};

struct Spot {
  int sample, chunk;
  int pix, pix_end, pix_step;         // pixels pix, pix + pix_step, ... < pix_end of the sample
  int col, have;
  int sub;                            // which of the warp's pixels this lane has
};
__device__ __forceinline__ Spot spot_of(const NormDev& d) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int lanes = 1 << d.lane_shift, per_warp = 32 >> d.lane_shift;
  const int seg = (int)(blockIdx.x % (unsigned)d.segs);
  const unsigned rest = blockIdx.x / (unsigned)d.segs;
  Spot s;
  s.chunk = (int)(rest % (unsigned)d.chunks);
  s.sample = (int)(rest / (unsigned)d.chunks);
  s.sub = lane >> d.lane_shift;
  s.col = (seg * lanes + (lane & (lanes - 1))) * kRun;
  s.have = min(kRun, d.c - s.col);
  const int first = s.chunk * d.chunk_rows;
  s.pix = first + warp * per_warp + s.sub;
  s.pix_end = min(d.hw, first + d.chunk_rows);
  s.pix_step = kWarps * per_warp;
  return s;
}

template <int DT>
__device__ __forceinline__ void load_x(const NormDev& d, const Spot& s, int pix, float (&v)[kRun]) {
  using T = typename Elem<DT>::T;
  if (d.x8.dev_codes) {                                     // only the backward kernels set it as an input
    const int64_t row = (int64_t)s.sample * d.hw + pix;
    const uint8_t* p = d.x8.dev_codes + row * d.x8.ld_codes + s.col;
    const float step = step_of(d.x8.dev_exps[row * d.x8.ld_exps + s.col / kGroup]);
    uint2 w = make_uint2(0u, 0u);
    if (d.vec_x8 && s.have == kRun) {
      w = *reinterpret_cast<const uint2*>(p);
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (j < s.have) (j < 4 ? w.x : w.y) |= (uint32_t)p[j] << (8 * (j & 3));
    }
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = decode8((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255u, step);
    return;
  }
  load_run<DT, kRun>(static_cast<const T*>(d.x) + s.sample * d.sample_x + pix * d.ld_x + s.col, d.vec_x && s.have == kRun, s.have, v);
}

// (count, mean, squared distances) of the union of two sets
__device__ __forceinline__ void merge(float& n, float& m, float& q, float n2, float m2, float q2) {
  if (n2 == 0.f) return;
  if (n == 0.f) { n = n2; m = m2; q = q2; return; }
  const float t = n + n2, dist = m2 - m, f = n2 / t;
  m += dist * f;
  q += q2 + dist * dist * n * f;
  n = t;
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
norm_stats_kernel(NormDev d) {
  train_pdl_wait();
  __shared__ float smean[kWarps * 32][kRun + 1], sq[kWarps * 32][kRun + 1], scount[kWarps * 32];
  const Spot s = spot_of(d);
  d.x8.dev_codes = nullptr;
  float ref[kRun], sum[kRun], sum2[kRun];
  int count = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) ref[j] = sum[j] = sum2[j] = 0.f;
  if (s.have > 0)
    for (int p = s.pix; p < s.pix_end; p += s.pix_step, ++count) {
      float v[kRun];
      load_x<DT>(d, s, p, v);
      if (count == 0) {
#pragma unroll
        for (int j = 0; j < kRun; ++j) ref[j] = v[j];
      } else {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
          const float t = v[j] - ref[j];
          sum[j] += t;
          sum2[j] = fmaf(t, t, sum2[j]);
        }
      }
    }
  const float inv = count ? 1.f / count : 0.f;
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    smean[threadIdx.x][j] = fmaf(sum[j], inv, ref[j]);
    sq[threadIdx.x][j] = fmaxf(fmaf(-sum[j] * inv, sum[j], sum2[j]), 0.f) + 0.f * sum2[j];   // the last term keeps NaN
  }
  scount[threadIdx.x] = (float)count;
  __syncthreads();
  const int lanes = 1 << d.lane_shift;
  for (int ch = threadIdx.x; ch < lanes * kRun; ch += kThreads) {
    const int col = (int)(blockIdx.x % (unsigned)d.segs) * lanes * kRun + ch;
    if (col >= d.c) continue;
    float n = 0.f, m = 0.f, q = 0.f;
    for (int t = ch / kRun; t < kThreads; t += lanes) merge(n, m, q, scount[t], smean[t][ch % kRun], sq[t][ch % kRun]);
    const size_t at = ((size_t)s.sample * d.chunks + s.chunk) * d.c + col;
    d.part0[at] = m;
    d.part1[at] = q;
  }
}

// A warp per (sample, group): merges the group's channels and chunks.
__global__ void __launch_bounds__(kThreads)
norm_group_kernel(NormDev d) {
  train_pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t u = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (u >= (int64_t)d.n * d.groups) return;
  const int sample = (int)(u / d.groups), g = (int)(u - (int64_t)sample * d.groups);
  float n = 0.f, m = 0.f, q = 0.f;
  for (int i = lane; i < d.chunks * d.cpg; i += 32) {
    const int chunk = i / d.cpg, ch = g * d.cpg + i % d.cpg;
    const size_t at = ((size_t)sample * d.chunks + chunk) * d.c + ch;
    merge(n, m, q, (float)(min(d.hw, (chunk + 1) * d.chunk_rows) - chunk * d.chunk_rows), d.part0[at], d.part1[at]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float n2 = __shfl_down_sync(0xffffffffu, n, o), m2 = __shfl_down_sync(0xffffffffu, m, o), q2 = __shfl_down_sync(0xffffffffu, q, o);
    merge(n, m, q, n2, m2, q2);
  }
  if (lane == 0) {
    d.mean[u] = m;
    d.rstd[u] = 1.f / sqrtf(q / n + d.eps);
  }
}

__device__ __forceinline__ void channel_figures(const NormDev& d, const Spot& s, float (&mean)[kRun], float (&rstd)[kRun], float (&gamma)[kRun], float (&beta)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    const int ch = s.col + (j < s.have ? j : 0);
    const size_t at = (size_t)s.sample * d.groups + ch / d.cpg;
    mean[j] = d.mean[at];
    rstd[j] = d.rstd[at];
    gamma[j] = d.gamma[ch];
    beta[j] = d.beta[ch];
  }
}

// Packs 8 of a row's columns per thread, four neighbouring lanes to a group of 32; the whole warp calls it.
__device__ __forceinline__ void pack_run(const lqsgd_packed8& out, bool vec, int64_t row, int col, int have, bool on, const float (&v)[kRun]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, on && j < have ? __float_as_uint(v[j]) & 0x7fffffffu : 0u);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int eb = exp_byte(__uint_as_float(top));
  if (!on) return;
  const float inv = inv_step(eb);
  const uint32_t lo = code_word(v[0], v[1], v[2], v[3], inv), hi = code_word(v[4], v[5], v[6], v[7], inv);
  uint8_t* p = out.dev_codes + row * out.ld_codes + col;
  if (vec && have == kRun) {
    *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      if (j < have) p[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
  }
  if ((col & (kGroup - 1)) == 0) out.dev_exps[row * out.ld_exps + col / kGroup] = (uint8_t)eb;
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
norm_apply_kernel(NormDev d) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  const Spot s = spot_of(d);
  const lqsgd_packed8 x8 = d.x8;
  d.x8.dev_codes = nullptr;
  float mean[kRun], scale[kRun], gamma[kRun], beta[kRun];
  const bool mine = s.have > 0;
  if (mine) channel_figures(d, s, mean, scale, gamma, beta);
#pragma unroll
  for (int j = 0; j < kRun; ++j) scale[j] *= gamma[j];
  for (int p = s.pix; p - s.sub < s.pix_end; p += s.pix_step) {
    const bool on = mine && p < s.pix_end;
    const int64_t row = (int64_t)s.sample * d.hw + p;
    float v[kRun];
    if (on) load_x<DT>(d, s, p, v);
    if (x8.dev_codes) pack_run(x8, d.vec_x8, row, s.col, s.have, on, v);
    if (on) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) v[j] = fmaf(v[j] - mean[j], scale[j], beta[j]);
      act_run(d.act, v);
      store_run<DT, kRun>(static_cast<T*>(d.out) + s.sample * d.sample_out + p * d.ld_out + s.col, d.vec_out && s.have == kRun, s.have, v);
    }
    if (d.y8.dev_codes) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) v[j] = as_stored<DT>(v[j]);
      pack_run(d.y8, d.vec_y8, row, s.col, s.have, on, v);
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
norm_grad_sums_kernel(NormDev d) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  __shared__ float s0[kThreads][kRun + 1], s1[kThreads][kRun + 1];
  const Spot s = spot_of(d);
  float a[kRun], b[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) a[j] = b[j] = 0.f;
  if (s.have > 0) {
    float mean[kRun], rstd[kRun], gamma[kRun], beta[kRun];
    channel_figures(d, s, mean, rstd, gamma, beta);
    for (int p = s.pix; p < s.pix_end; p += s.pix_step) {
      float v[kRun], g[kRun];
      load_x<DT>(d, s, p, v);
      load_run<DT, kRun>(static_cast<const T*>(d.dy) + s.sample * d.sample_dy + p * d.ld_dy + s.col, d.vec_dy && s.have == kRun, s.have, g);
      float h[kRun];
#pragma unroll
      for (int j = 0; j < kRun; ++j) { v[j] = (v[j] - mean[j]) * rstd[j]; h[j] = fmaf(v[j], gamma[j], beta[j]); }
      slope_run(d.act, h);
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const float dh = g[j] * h[j];
        a[j] += dh;
        b[j] = fmaf(dh, v[j], b[j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kRun; ++j) { s0[threadIdx.x][j] = a[j]; s1[threadIdx.x][j] = b[j]; }
  __syncthreads();
  const int lanes = 1 << d.lane_shift;
  for (int ch = threadIdx.x; ch < lanes * kRun; ch += kThreads) {
    const int col = (int)(blockIdx.x % (unsigned)d.segs) * lanes * kRun + ch;
    if (col >= d.c) continue;
    float u = 0.f, w = 0.f;
    for (int t = ch / kRun; t < kThreads; t += lanes) { u += s0[t][ch % kRun]; w += s1[t][ch % kRun]; }
    const size_t at = ((size_t)s.sample * d.chunks + s.chunk) * d.c + col;
    d.part0[at] = u;
    d.part1[at] = w;
  }
}

// Blocks [0, group_blocks): a warp per (sample, group) forms <u> and <u xh>.  The others: 32 channels each, dgamma and dbeta.
__global__ void __launch_bounds__(kThreads)
norm_grad_join_kernel(NormDev d, int group_blocks) {
  train_pdl_wait();
  __shared__ float s0[kWarps][33], s1[kWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < group_blocks) {
    const int64_t u = (int64_t)blockIdx.x * kWarps + warp;
    if (u >= (int64_t)d.n * d.groups) return;
    const int sample = (int)(u / d.groups), g = (int)(u - (int64_t)sample * d.groups);
    float a = 0.f, b = 0.f;
    for (int i = lane; i < d.chunks * d.cpg; i += 32) {
      const int chunk = i / d.cpg, ch = g * d.cpg + i % d.cpg;
      const size_t at = ((size_t)sample * d.chunks + chunk) * d.c + ch;
      a = fmaf(d.gamma[ch], d.part0[at], a);
      b = fmaf(d.gamma[ch], d.part1[at], b);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      a += __shfl_down_sync(0xffffffffu, a, o);
      b += __shfl_down_sync(0xffffffffu, b, o);
    }
    if (lane == 0) {
      const float inv = 1.f / ((float)d.hw * (float)d.cpg);
      d.group0[u] = a * inv;
      d.group1[u] = b * inv;
    }
    return;
  }
  const int col = ((int)blockIdx.x - group_blocks) * 32 + lane;
  float a = 0.f, b = 0.f;
  if (col < d.c)
    for (int64_t r = warp; r < (int64_t)d.n * d.chunks; r += kWarps) {
      a += d.part0[(size_t)r * d.c + col];
      b += d.part1[(size_t)r * d.c + col];
    }
  s0[warp][lane] = a;
  s1[warp][lane] = b;
  __syncthreads();
  if (warp == 0 && col < d.c) {
    float u = 0.f, w = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) { u += s0[k][lane]; w += s1[k][lane]; }
    d.dbeta[col] = u;
    d.dgamma[col] = w;
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
norm_grad_apply_kernel(NormDev d) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  const Spot s = spot_of(d);
  if (s.have <= 0) return;
  float mean[kRun], rstd[kRun], gamma[kRun], beta[kRun], c0[kRun], c1[kRun];
  channel_figures(d, s, mean, rstd, gamma, beta);
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    const size_t at = (size_t)s.sample * d.groups + (s.col + (j < s.have ? j : 0)) / d.cpg;
    c0[j] = d.group0[at];
    c1[j] = d.group1[at];
  }
  for (int p = s.pix; p < s.pix_end; p += s.pix_step) {
    float v[kRun], g[kRun];
    load_x<DT>(d, s, p, v);
    load_run<DT, kRun>(static_cast<const T*>(d.dy) + s.sample * d.sample_dy + p * d.ld_dy + s.col, d.vec_dy && s.have == kRun, s.have, g);
    float h[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) { v[j] = (v[j] - mean[j]) * rstd[j]; h[j] = fmaf(v[j], gamma[j], beta[j]); }
    slope_run(d.act, h);
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = rstd[j] * (gamma[j] * g[j] * h[j] - c0[j] - v[j] * c1[j]);
    store_run<DT, kRun>(static_cast<T*>(d.out) + s.sample * d.sample_out + p * d.ld_out + s.col, d.vec_out && s.have == kRun, s.have, v);
  }
}

void make_geometry(NormDev* d) {
  d->cpg = d->c / d->groups;
  d->lane_shift = 2;
  while (d->lane_shift < 5 && (8 << d->lane_shift) < d->c) ++d->lane_shift;
  d->segs = (int)ceil_div64(d->c, 8ll << d->lane_shift);
  const int step = kWarps * (32 >> d->lane_shift);          // pixels one pass of a block covers
  // enough blocks for 148 SMs x 8, at least two passes each where there are that many; by the sizes alone
  const int64_t wanted = ceil_div64(148 * 8, std::max<int64_t>(1, (int64_t)d->n * d->segs));
  const int64_t most = std::max<int64_t>(1, d->hw / (2 * step));
  const int64_t chunks = std::max<int64_t>(1, std::min(wanted, most));
  d->chunk_rows = (int)(ceil_div64(ceil_div64(d->hw, chunks), step) * step);
  d->chunks = (int)ceil_div64(d->hw, d->chunk_rows);
}
size_t part_floats(const NormDev& d) { return ((size_t)d.n * d.chunks * d.c + 63) / 64 * 64; }
size_t workspace_of(const NormDev& d, bool backward) {
  const size_t groups = ((size_t)d.n * d.groups + 63) / 64 * 64;
  return 4 * (2 * part_floats(d) + (backward ? 2 * groups : 0));
}

int check_common(const lqsgd_group_norm* a) {
  if (!a || a->struct_size != sizeof(lqsgd_group_norm)) return LQSGD_ERR_INVALID_ARG;
  if (!train_dtype_ok(a->dtype) || !train_act_ok(a->act)) return LQSGD_ERR_INVALID_ARG;
  if (a->n < 0 || a->hw < 1 || a->c < 1 || a->c > 65536 || a->groups < 1 || a->c % a->groups) return LQSGD_ERR_BAD_SHAPE;
  const int64_t segs = ceil_div64(a->c, 32);
  // one block per sample, chunk and segment: the grid's limit; chunks beyond 1 only come with few samples
  if ((int64_t)a->n * segs > (1ll << 30)) return LQSGD_ERR_BAD_SHAPE;
  return LQSGD_OK;
}
int check_tensor(const void* p, int64_t ld, int64_t sample, const lqsgd_group_norm* a) {
  if (!p || ld < a->c || (a->n > 1 && sample < (int64_t)(a->hw - 1) * ld + a->c)) return LQSGD_ERR_INVALID_ARG;
  return train_aligned(p, train_elem(a->dtype)) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}
NormDev to_dev(const lqsgd_group_norm& a) {
  NormDev d = {};
  d.n = a.n; d.hw = a.hw; d.c = a.c; d.groups = a.groups; d.act = a.act; d.eps = a.eps;
  d.x = a.dev_x; d.ld_x = a.ld_x; d.sample_x = a.sample_x;
  d.dy = a.dev_dy; d.ld_dy = a.ld_dy; d.sample_dy = a.sample_dy;
  d.out = a.dev_out; d.ld_out = a.ld_out; d.sample_out = a.sample_out;
  d.gamma = a.dev_gamma; d.beta = a.dev_beta; d.mean = a.dev_mean; d.rstd = a.dev_rstd;
  d.dgamma = a.dev_dgamma; d.dbeta = a.dev_dbeta; d.x8 = a.x8; d.y8 = a.y8;
  const int es = train_elem(a.dtype);
  auto vec = [&](const void* p, int64_t ld, int64_t sample) { return train_aligned(p, 16) && (ld * es) % 16 == 0 && (a.n == 1 || (sample * es) % 16 == 0); };
  d.vec_x = vec(d.x, d.ld_x, d.sample_x);
  d.vec_dy = vec(d.dy, d.ld_dy, d.sample_dy);
  d.vec_out = vec(d.out, d.ld_out, d.sample_out);
  d.vec_x8 = train_aligned(d.x8.dev_codes, 8) && d.x8.ld_codes % 8 == 0;
  d.vec_y8 = train_aligned(d.y8.dev_codes, 8) && d.y8.ld_codes % 8 == 0;
  make_geometry(&d);
  return d;
}
int place_workspace(NormDev* d, const lqsgd_group_norm& a, bool backward) {
  if (!a.dev_workspace || a.workspace_bytes < workspace_of(*d, backward)) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
  if (!train_aligned(a.dev_workspace, 16)) return LQSGD_ERR_MISALIGNED;
  d->part0 = static_cast<float*>(a.dev_workspace);
  d->part1 = d->part0 + part_floats(*d);
  d->group0 = d->part1 + part_floats(*d);
  d->group1 = d->group0 + ((size_t)d->n * d->groups + 63) / 64 * 64;
  return LQSGD_OK;
}

}  // namespace
}  // namespace lqsgd

using namespace lqsgd;

#define NORM_BY_DTYPE(dtype, kernel, ...)                                          \
  ((dtype) == LQSGD_BF16 ? train_launch(kernel<LQSGD_BF16>, __VA_ARGS__)           \
   : (dtype) == LQSGD_F16 ? train_launch(kernel<LQSGD_F16>, __VA_ARGS__)           \
                          : train_launch(kernel<LQSGD_F32>, __VA_ARGS__))

extern "C" int lqsgd_group_norm_workspace_bytes(int32_t backward, const lqsgd_group_norm* host_args, size_t* host_bytes_out) {
  if (!host_bytes_out || (backward != 0 && backward != 1)) return LQSGD_ERR_INVALID_ARG;
  const int rc = check_common(host_args);
  if (rc != LQSGD_OK) return rc;
  *host_bytes_out = host_args->n ? workspace_of(to_dev(*host_args), backward != 0) : 0;
  return LQSGD_OK;
}

extern "C" int lqsgd_group_norm_forward(const lqsgd_group_norm* a, void* cuda_stream) {
  int rc = check_common(a);
  if (rc != LQSGD_OK) return rc;
  if (!(a->eps > 0.f) || !(a->eps < INFINITY)) return LQSGD_ERR_INVALID_ARG;
  if (a->n == 0) return LQSGD_OK;
  if ((rc = check_tensor(a->dev_x, a->ld_x, a->sample_x, a)) != LQSGD_OK || (rc = check_tensor(a->dev_out, a->ld_out, a->sample_out, a)) != LQSGD_OK) return rc;
  if (!a->dev_gamma || !a->dev_beta || !a->dev_mean || !a->dev_rstd) return LQSGD_ERR_INVALID_ARG;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_beta, 4) || !train_aligned(a->dev_mean, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->x8.dev_codes && (rc = check_packed8(a->x8, a->c)) != LQSGD_OK) return rc;
  if (a->y8.dev_codes && (rc = check_packed8(a->y8, a->c)) != LQSGD_OK) return rc;
  NormDev d = to_dev(*a);
  if ((rc = place_workspace(&d, *a, false)) != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const dim3 grid((unsigned)((int64_t)d.n * d.chunks * d.segs));
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_stats_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_stats_kernel launch");
  TRAIN_CK(train_launch(norm_group_kernel, dim3((unsigned)ceil_div64((int64_t)d.n * d.groups, kWarps)), dim3(kThreads), 0, st, 1, d), "norm_group_kernel launch");
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_apply_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_apply_kernel launch");
  return LQSGD_OK;
}

extern "C" int lqsgd_group_norm_backward(const lqsgd_group_norm* a, void* cuda_stream) {
  int rc = check_common(a);
  if (rc != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!a->dev_dgamma || !a->dev_dbeta) return LQSGD_ERR_INVALID_ARG;
  if (!train_aligned(a->dev_dgamma, 4) || !train_aligned(a->dev_dbeta, 4)) return LQSGD_ERR_MISALIGNED;
  if (a->n == 0) {
    TRAIN_CK(cudaMemsetAsync(a->dev_dgamma, 0, (size_t)a->c * 4, st), "cudaMemsetAsync(dgamma)");
    TRAIN_CK(cudaMemsetAsync(a->dev_dbeta, 0, (size_t)a->c * 4, st), "cudaMemsetAsync(dbeta)");
    return LQSGD_OK;
  }
  if ((rc = check_tensor(a->dev_dy, a->ld_dy, a->sample_dy, a)) != LQSGD_OK || (rc = check_tensor(a->dev_out, a->ld_out, a->sample_out, a)) != LQSGD_OK) return rc;
  if (a->x8.dev_codes) rc = check_packed8(a->x8, a->c);
  else rc = check_tensor(a->dev_x, a->ld_x, a->sample_x, a);
  if (rc != LQSGD_OK) return rc;
  if (!a->dev_gamma || !a->dev_beta || !a->dev_mean || !a->dev_rstd) return LQSGD_ERR_INVALID_ARG;
  if (!train_aligned(a->dev_gamma, 4) || !train_aligned(a->dev_beta, 4) || !train_aligned(a->dev_mean, 4) || !train_aligned(a->dev_rstd, 4)) return LQSGD_ERR_MISALIGNED;
  NormDev d = to_dev(*a);
  if ((rc = place_workspace(&d, *a, true)) != LQSGD_OK) return rc;
  const dim3 grid((unsigned)((int64_t)d.n * d.chunks * d.segs));
  const int group_blocks = (int)ceil_div64((int64_t)d.n * d.groups, kWarps);
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_grad_sums_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_grad_sums_kernel launch");
  TRAIN_CK(train_launch(norm_grad_join_kernel, dim3((unsigned)(group_blocks + (d.c + 31) / 32)), dim3(kThreads), 0, st, 1, d, group_blocks), "norm_grad_join_kernel launch");
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_grad_apply_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_grad_apply_kernel launch");
  return LQSGD_OK;
}
