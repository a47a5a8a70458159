// Group norm with an activation on channels-last tensors, forward and backward.
//
// A thread owns 8 consecutive channels (16 bytes of a 16-bit type) and walks over pixels; what it sums stays in its registers
// per channel, so groups of any width need no special case.  What bounds it is HBM: every tensor should be read once.
//
// Resident kernels (channels a multiple of 8, slices that fit): a cluster of 1 .. 8 CTAs takes one sample's block of whole groups
// (at least 64 bytes of a pixel), each CTA a range of its pixels, and brings it into shared memory with asynchronous
// copies of 16 bytes (no registers are held meanwhile, so the whole slice is in flight at once; rows without 16-byte pieces
// are read element by element).  Sums meet through distributed shared memory; the passes after the first read shared memory.
// A thread reads only what it copied itself.
//
// Streaming kernels (everything else): per-channel sums of a chunk of pixels meet in a small kernel, which forms the groups'
// figures, and a last kernel reads the tensor a second time (from L2 up to about 100 MB) and applies them.  A pixel is dealt to as many
// lanes as it has 8-channel pieces, so that few channels leave none idle: 431 x 9957 x 5 takes 62 us forward and 195 backward
// (80 and 202 with four pixels at once per thread: fewer threads fit then).  Their forward sums are
// (mean, squared distances from it) about a value of the channel itself, merged pairwise; the resident kernel takes the
// mean first and the distances from it in a second pass.  Either way a mean far from zero cancels nothing.
//
// 256 x 1024 x 64 in bf16, 8 groups, silu: 20 us forward resident and 36 streaming, 41 and 61 with both 8-bit copies, backward from
// the 8-bit x 45 and 83; 79 x 15713 x 8: 19 and 28, 30 and 39, 45 and 54.
#include "lqsgd_train_dev.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

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
  s.pix_end = first + min(d.chunk_rows, d.hw - first);      // first + chunk_rows can pass 2^31
  s.pix_step = kWarps * per_warp;
  return s;
}

template <int DT>
__device__ __forceinline__ void load_x(const NormDev& d, const Spot& s, int pix, float (&v)[kRun]) {
  using T = typename Elem<DT>::T;
  if (d.x8.dev_codes) {                                     // only the backward kernels set it as an input
    const int64_t row = (int64_t)s.sample * d.hw + pix;
    const uint8_t* p = d.x8.dev_codes + row * d.x8.ld_codes + s.col;
    const int eb = d.x8.dev_exps[row * d.x8.ld_exps + s.col / kGroup];
    uint2 w = make_uint2(0u, 0u);
    if (d.vec_x8 && s.have == kRun) {
      w = *reinterpret_cast<const uint2*>(p);
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j)
        if (j < s.have) (j < 4 ? w.x : w.y) |= (uint32_t)p[j] << (8 * (j & 3));
    }
    decode_run(w, eb, v);
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
  __shared__ float smean[kThreads][kRun + 1], sq[kThreads][kRun + 1], scount[kThreads];
  const Spot s = spot_of(d);
  d.x8.dev_codes = nullptr;
  float mean[kRun], sum[kRun], sum2[kRun];                  // mean: first of all a value of the channel
  int count = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) mean[j] = sum[j] = sum2[j] = 0.f;
  if (s.have > 0) {
    if (s.pix < s.pix_end) load_x<DT>(d, s, s.pix, mean), count = 1;
    for (int p = s.pix + s.pix_step; p < s.pix_end; p += s.pix_step, ++count) {
      float v[kRun];
      load_x<DT>(d, s, p, v);
#pragma unroll
      for (int j = 0; j < kRun; ++j) {
        const float t = v[j] - mean[j];
        sum[j] += t;
        sum2[j] = fmaf(t, t, sum2[j]);
      }
    }
  }
  const float inv = count ? 1.f / count : 0.f;
  float n = (float)count, q[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    mean[j] = fmaf(sum[j], inv, mean[j]);
    q[j] = fmaxf(fmaf(-sum[j] * inv, sum[j], sum2[j]), 0.f) + 0.f * sum2[j];   // the last term keeps NaN
  }
  // the warp's lanes with the same channels, then its warps
  const int lanes = 1 << d.lane_shift, lane = threadIdx.x & 31;
  for (int o = 16; o >= lanes; o >>= 1) {
    const float n2 = __shfl_down_sync(0xffffffffu, n, o), t = n + n2, f = n2 > 0.f ? n2 / t : 0.f;
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      const float m2 = __shfl_down_sync(0xffffffffu, mean[j], o), q2 = __shfl_down_sync(0xffffffffu, q[j], o);
      const float dist = m2 - mean[j];
      if (n2 > 0.f) {
        q[j] += q2 + dist * dist * n * f;
        mean[j] = n > 0.f ? fmaf(dist, f, mean[j]) : m2;
      }
    }
    n = t;
  }
  if (lane < lanes) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) { smean[threadIdx.x][j] = mean[j]; sq[threadIdx.x][j] = q[j]; }
    scount[threadIdx.x] = n;
  }
  __syncthreads();
  for (int ch = threadIdx.x; ch < lanes * kRun; ch += kThreads) {
    const int col = (int)(blockIdx.x % (unsigned)d.segs) * lanes * kRun + ch;
    if (col >= d.c) continue;
    float n1 = 0.f, m1 = 0.f, q1 = 0.f;
    for (int w = 0; w < kWarps; ++w) merge(n1, m1, q1, scount[32 * w + ch / kRun], smean[32 * w + ch / kRun][ch % kRun], sq[32 * w + ch / kRun][ch % kRun]);
    const size_t at = ((size_t)s.sample * d.chunks + s.chunk) * d.c + col;
    d.part0[at] = m1;
    d.part1[at] = q1;
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
    merge(n, m, q, (float)min(d.chunk_rows, d.hw - chunk * d.chunk_rows), d.part0[at], d.part1[at]);
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

// Packs 8 of a row's columns per thread, four neighbouring lanes to a group of 32 (a row of one or two lanes is one group);
// the whole warp calls it.
__device__ __forceinline__ void pack_run(const lqsgd_packed8& out, bool vec, int lane_shift, int64_t row, int col, int have, bool on, const float (&v)[kRun]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, on && j < have ? __float_as_uint(v[j]) & 0x7fffffffu : 0u);
  if (lane_shift > 0) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  if (lane_shift > 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
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
    if (x8.dev_codes) pack_run(x8, d.vec_x8, d.lane_shift, row, s.col, s.have, on, v);
    if (on) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) v[j] = fmaf(v[j] - mean[j], scale[j], beta[j]);
      act_run(d.act, v);
      store_run<DT, kRun>(static_cast<T*>(d.out) + s.sample * d.sample_out + p * d.ld_out + s.col, d.vec_out && s.have == kRun, s.have, v);
    }
    if (d.y8.dev_codes) {
#pragma unroll
      for (int j = 0; j < kRun; ++j) v[j] = as_stored<DT>(v[j]);
      pack_run(d.y8, d.vec_y8, d.lane_shift, row, s.col, s.have, on, v);
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kThreads)
norm_grad_sums_kernel(NormDev d) {
  train_pdl_wait();
  using T = typename Elem<DT>::T;
  __shared__ float s0[kWarps][32 * kRun], s1[kWarps][32 * kRun];
  const Spot s = spot_of(d);
  float a[kRun], b[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) a[j] = b[j] = 0.f;
  if (s.have > 0) {
    float mean[kRun], rstd[kRun], gamma[kRun], beta[kRun];
    channel_figures(d, s, mean, rstd, gamma, beta);
    for (int p = s.pix; p < s.pix_end; p += s.pix_step) {
      float v[kRun], g[kRun], h[kRun];
      load_x<DT>(d, s, p, v);
      load_run<DT, kRun>(static_cast<const T*>(d.dy) + s.sample * d.sample_dy + p * d.ld_dy + s.col, d.vec_dy && s.have == kRun, s.have, g);
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
  const int lanes = 1 << d.lane_shift, lane = threadIdx.x & 31;
  for (int o = 16; o >= lanes; o >>= 1)
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      a[j] += __shfl_down_sync(0xffffffffu, a[j], o);
      b[j] += __shfl_down_sync(0xffffffffu, b[j], o);
    }
  if (lane < lanes) {
#pragma unroll
    for (int j = 0; j < kRun; ++j) { s0[threadIdx.x >> 5][lane * kRun + j] = a[j]; s1[threadIdx.x >> 5][lane * kRun + j] = b[j]; }
  }
  __syncthreads();
  for (int ch = threadIdx.x; ch < lanes * kRun; ch += kThreads) {
    const int col = (int)(blockIdx.x % (unsigned)d.segs) * lanes * kRun + ch;
    if (col >= d.c) continue;
    float u = 0.f, w = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) { u += s0[k][ch]; w += s1[k][ch]; }
    const size_t at = ((size_t)s.sample * d.chunks + s.chunk) * d.c + col;
    d.part0[at] = u;
    d.part1[at] = w;
  }
}

constexpr int kJoinWarps = 32;
// Blocks [0, group_blocks): a warp per (sample, group) forms <u> and <u xh>.  The others: 32 channels each, dgamma and dbeta.
__global__ void __launch_bounds__(32 * kJoinWarps)
norm_grad_join_kernel(NormDev d, int group_blocks) {
  train_pdl_wait();
  __shared__ float s0[kJoinWarps][33], s1[kJoinWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < group_blocks) {
    const int64_t u = (int64_t)blockIdx.x * kJoinWarps + warp;
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
  const int rows = d.n * d.chunks;
  if (col < d.c) {
#pragma unroll 8
    for (int r = warp; r < rows; r += kJoinWarps) {
      a += d.part0[(size_t)r * d.c + col];
      b += d.part1[(size_t)r * d.c + col];
    }
  }
  s0[warp][lane] = a;
  s1[warp][lane] = b;
  __syncthreads();
  if (warp == 0 && col < d.c) {
    float u = 0.f, w = 0.f;
#pragma unroll
    for (int k = 0; k < kJoinWarps; ++k) { u += s0[k][lane]; w += s1[k][lane]; }
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
    float v[kRun], g[kRun], h[kRun];
    load_x<DT>(d, s, p, v);
    load_run<DT, kRun>(static_cast<const T*>(d.dy) + s.sample * d.sample_dy + p * d.ld_dy + s.col, d.vec_dy && s.have == kRun, s.have, g);
#pragma unroll
    for (int j = 0; j < kRun; ++j) { v[j] = (v[j] - mean[j]) * rstd[j]; h[j] = fmaf(v[j], gamma[j], beta[j]); }
    slope_run(d.act, h);
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = rstd[j] * (gamma[j] * g[j] * h[j] - c0[j] - v[j] * c1[j]);
    store_run<DT, kRun>(static_cast<T*>(d.out) + s.sample * d.sample_out + p * d.ld_out + s.col, d.vec_out && s.have == kRun, s.have, v);
  }
}

// ------------------------------------------------------------------------------------------------------- resident kernels
struct Resident {
  NormDev d;
  int32_t cb;                         // channels of a block: whole groups, a multiple of 8 (of 32 where something is packed)
  int32_t blocks;                     // blocks per sample
  int32_t lane_shift;                 // a pixel's 8-channel pieces are dealt to 1 << lane_shift threads
  int32_t parts;                      // CTAs (of one cluster) that share the pixels
  int32_t part_rows, steps;           // pixels per CTA; pieces per thread
};
constexpr int kResThreads = 256, kResWarps = kResThreads / 32;

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(dst)), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_at(dst)), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void norm_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float read_peer(const float* p, uint32_t rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_at(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

struct Place {
  int sample, c0, channels;           // the block's first channel and how many it has (the last block may have fewer)
  int part, first, rows;              // this CTA's pixels
  int col, row, row_step;             // the thread's first channel (of the tensor) and its pixels row, row + row_step, ... < rows
  bool on;
};
__device__ __forceinline__ Place place_of(const Resident& r) {
  Place q;
  q.part = r.parts > 1 ? (int)(blockIdx.x % (unsigned)r.parts) : 0;
  const unsigned unit = r.parts > 1 ? blockIdx.x / (unsigned)r.parts : blockIdx.x;
  q.sample = (int)(unit / (unsigned)r.blocks);
  q.c0 = (int)(unit - (unsigned)q.sample * r.blocks) * r.cb;
  q.channels = min(r.cb, r.d.c - q.c0);
  q.first = q.part * r.part_rows;
  q.rows = min(r.part_rows, r.d.hw - q.first);
  const int piece = threadIdx.x & ((1 << r.lane_shift) - 1);
  q.col = q.c0 + piece * kRun;
  q.row = threadIdx.x >> r.lane_shift;
  q.row_step = kResThreads >> r.lane_shift;
  q.on = piece * kRun < q.channels;
  return q;
}

// Sums over the block's threads of NV values each; threads whose piece (8 channels) is the same are added up.  On return
// scratch holds the sums of every warp that has the piece (see piece_sum).
template <int NV>
__device__ __forceinline__ void fold_rows(const Resident& r, float (&v)[NV], float* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, shift = min(r.lane_shift, 5);
  for (int o = 16; o >= (1 << r.lane_shift); o >>= 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] += __shfl_down_sync(0xffffffffu, v[j], o);
  }
  __syncthreads();                                        // scratch is free
  if (lane < (1 << shift)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) scratch[(((j * kResWarps) + warp) << shift) + lane] = v[j];
  }
  __syncthreads();
}
__device__ __forceinline__ float piece_sum(const Resident& r, const float* scratch, int v, int piece) {
  const int shift = min(r.lane_shift, 5), wide = max(1, (1 << r.lane_shift) >> 5);    // warps that a pixel spans
  float t = 0.f;
#pragma unroll 4
  for (int w = piece >> 5; w < kResWarps; w += wide) t += scratch[((v * kResWarps + w) << shift) + (piece & 31)];
  return t;
}
// NT totals of each of the block's groups over the block and the cluster: total[t * cap + g], the same bits in every CTA.
// value(t, g, i) is the i-th part of the t-th sum, `count` of them.
template <int NT, typename F>
__device__ __forceinline__ void group_totals(const Resident& r, int groups, int cap, int count, float* mine, float* total, F&& value) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int width = 32;                                         // lanes per group
  while (width > 1 && width / 2 >= count) width >>= 1;
  const int per_warp = 32 / width, sub = lane / width, in = lane & (width - 1);
  for (int g0 = warp * per_warp; g0 < groups; g0 += kResWarps * per_warp) {
    const int g = g0 + sub;
    float t[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) t[k] = 0.f;
    if (g < groups)
      for (int i = in; i < count; i += width) {
#pragma unroll
        for (int k = 0; k < NT; ++k) t[k] += value(k, g, i);
      }
    for (int o = width >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int k = 0; k < NT; ++k) t[k] += __shfl_down_sync(0xffffffffu, t[k], o);
    }
    if (in == 0 && g < groups) {
#pragma unroll
      for (int k = 0; k < NT; ++k) (r.parts > 1 ? mine : total)[k * cap + g] = t[k];
    }
  }
  if (r.parts > 1) {
    norm_cluster_sync();
    for (int i = threadIdx.x; i < NT * cap; i += kResThreads) {
      float t = 0.f;
      for (int k = 0; k < r.parts; ++k) t += read_peer(mine + i, k);
      total[i] = t;
    }
  }
  __syncthreads();
}

template <int DT>
__device__ __forceinline__ void unpack_run(const uint8_t* p, float (&v)[kRun]) {
  if constexpr (DT == LQSGD_F32) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    const float2 a = open_pair<DT>(w.x), b = open_pair<DT>(w.y), c = open_pair<DT>(w.z), e = open_pair<DT>(w.w);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = e.x; v[7] = e.y;
  }
}
// Index in 0 .. NG - 1 of channel j of a piece: ONE group per piece (8 divides the group's width), or any.
template <bool ONE>
struct Groups {
  static constexpr int kN = ONE ? 1 : kRun;
  int first, at[kN];                                                    // groups of the block
  __device__ __forceinline__ Groups(int channel, int cpg) {
    first = channel / cpg;
    at[0] = first;
    if (!ONE) {
      int left = cpg - (channel - first * cpg), g = first;
#pragma unroll
      for (int j = 1; j < kN; ++j) {
        if (--left == 0) { ++g; left = cpg; }
        at[j] = g;
      }
    }
  }
  static __device__ __forceinline__ constexpr int of(int j) { return ONE ? 0 : j; }
};

// Brings a thread's `count` pieces (8 elements, `hop` elements apart) to shared memory, `step` bytes apart; the copies are on
// their way when it returns, except those of rows without 16-byte pieces, which go through registers.
template <typename T>
__device__ __forceinline__ void fetch_pieces(uint8_t* to, int step, const T* src, int64_t hop, int count, bool vec) {
  if (vec) {
#pragma unroll 4
    for (int k = 0; k < count; ++k, src += hop, to += step) {
#pragma unroll
      for (int i = 0; i < kRun * (int)sizeof(T) / 16; ++i) copy_async<16>(to + 16 * i, reinterpret_cast<const uint8_t*>(src) + 16 * i);
    }
  } else {
#pragma unroll 2
    for (int k = 0; k < count; ++k, src += hop, to += step) {
      __align__(16) T t[kRun];
#pragma unroll
      for (int j = 0; j < kRun; ++j) t[j] = src[j];
#pragma unroll
      for (int i = 0; i < kRun * (int)sizeof(T) / 16; ++i) reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(t)[i];
    }
  }
}
// Stores a run and leaves in v what a reader of it sees.
template <int DT>
__device__ __forceinline__ void store_rounded(typename Elem<DT>::T* p, bool vec, float (&v)[kRun]) {
  if constexpr (DT == LQSGD_F32) {
    store_run<DT, kRun>(p, vec, kRun, v);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_pair<DT>(v[2 * i], v[2 * i + 1]);
    if (vec) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
      for (int j = 0; j < kRun; ++j) h[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = open_pair<DT>(w[i]); v[2 * i] = t.x; v[2 * i + 1] = t.y; }
  }
}
// pack_run for whole runs.
__device__ __forceinline__ void pack_whole(const lqsgd_packed8& out, bool vec, int lane_shift, int64_t row, int col, bool on, const float (&v)[kRun]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  if (!on) top = 0;
  if (lane_shift > 0) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  if (lane_shift > 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  if (!on) return;
  const int eb = exp_byte(__uint_as_float(top));
  const float inv = inv_step(eb);
  const uint2 w = make_uint2(code_word(v[0], v[1], v[2], v[3], inv), code_word(v[4], v[5], v[6], v[7], inv));
  uint8_t* p = out.dev_codes + row * out.ld_codes + col;
  if (vec) {
    *reinterpret_cast<uint2*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j) p[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
  }
  if ((col & (kGroup - 1)) == 0) out.dev_exps[row * out.ld_exps + col / kGroup] = (uint8_t)eb;
}

template <int DT, bool ONE>
__global__ void __launch_bounds__(kResThreads, ONE ? 4 : 3)
norm_resident_kernel(Resident r) {
  using T = typename Elem<DT>::T;
  using G = Groups<ONE>;
  constexpr int kBytes = kRun * (int)sizeof(T), kStep = kResThreads * kBytes;
  extern __shared__ __align__(16) uint8_t res_smem[];
  const NormDev& d = r.d;
  const Place q = place_of(r);
  uint8_t* data = res_smem;                                             // [steps][threads] pieces
  float* scratch = reinterpret_cast<float*>(data + (size_t)r.steps * kStep);
  const int groups_cap = r.cb / d.cpg, groups = q.channels / d.cpg;
  float* mine = scratch + (G::kN * kResWarps << min(r.lane_shift, 5));  // [2][groups of a block]
  float* mean = mine + 2 * groups_cap;                                  // [groups]
  float* rstd = mean + groups_cap;
  const int count = q.on && q.row < q.rows ? (q.rows - q.row + q.row_step - 1) / q.row_step : 0;
  uint8_t* own = data + threadIdx.x * kBytes;
  train_pdl_wait();
  {
    const T* src = static_cast<const T*>(d.x) + q.sample * d.sample_x + (int64_t)(q.first + q.row) * d.ld_x + q.col;
    fetch_pieces<T>(own, kStep, src, q.row_step * d.ld_x, count, d.vec_x);
  }
  const G at(q.col - q.c0, d.cpg);
  float gamma[kRun], beta[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    gamma[j] = q.on ? __ldg(d.gamma + q.col + j) : 0.f;
    beta[j] = q.on ? __ldg(d.beta + q.col + j) : 0.f;
  }
  copy_async_wait();
  const float inv = 1.f / ((float)d.hw * (float)d.cpg);
  const int per_group = ONE ? d.cpg / kRun : d.cpg;
  auto part = [&](int, int g, int i) {
    const int ch = ONE ? (g * per_group + i) * kRun : g * d.cpg + i;
    return piece_sum(r, scratch, ONE ? 0 : ch % kRun, ch / kRun);
  };
  float s[G::kN], v[kRun];
#pragma unroll
  for (int j = 0; j < G::kN; ++j) s[j] = 0.f;
#pragma unroll 4
  for (int k = 0; k < count; ++k) {
    unpack_run<DT>(own + k * kStep, v);
    if (ONE) s[0] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) s[G::of(j)] += v[j];
    }
  }
  fold_rows(r, s, scratch);
  group_totals<1>(r, groups, groups_cap, per_group, mine, mean, part);
  float m[G::kN];
#pragma unroll
  for (int j = 0; j < G::kN; ++j) {
    s[j] = 0.f;
    m[j] = q.on ? mean[at.at[j]] * inv : 0.f;
  }
#pragma unroll 4
  for (int k = 0; k < count; ++k) {
    unpack_run<DT>(own + k * kStep, v);
    float u[kRun];
#pragma unroll
    for (int j = 0; j < kRun; ++j) u[j] = v[j] - m[G::of(j)];
    if (ONE) {
      float t0 = u[0] * u[0], t1 = u[4] * u[4];
#pragma unroll
      for (int j = 1; j < 4; ++j) { t0 = fmaf(u[j], u[j], t0); t1 = fmaf(u[4 + j], u[4 + j], t1); }
      s[0] += t0 + t1;
    } else {
#pragma unroll
      for (int j = 0; j < kRun; ++j) s[G::of(j)] = fmaf(u[j], u[j], s[G::of(j)]);
    }
  }
  fold_rows(r, s, scratch);
  group_totals<1>(r, groups, groups_cap, per_group, mine + groups_cap, rstd, part);
  if (q.part == 0)
    for (int g = threadIdx.x; g < groups; g += kResThreads) {
      const size_t to = (size_t)q.sample * d.groups + q.c0 / d.cpg + g;
      d.mean[to] = mean[g] * inv;
      d.rstd[to] = 1.f / sqrtf(rstd[g] * inv + d.eps);
    }
  float scale[G::kN];
#pragma unroll
  for (int j = 0; j < G::kN; ++j) scale[j] = q.on ? 1.f / sqrtf(rstd[at.at[j]] * inv + d.eps) : 0.f;
#pragma unroll
  for (int j = 0; j < kRun; ++j) gamma[j] *= scale[G::of(j)];
  T* dst = static_cast<T*>(d.out) + q.sample * d.sample_out + (int64_t)(q.first + q.row) * d.ld_out + q.col;
  const int64_t hop = q.row_step * d.ld_out;
  if (!d.x8.dev_codes && !d.y8.dev_codes) {
    with_act(d.act, [&](auto tag) {
#pragma unroll 2
      for (int k = 0; k < count; ++k, dst += hop) {
        unpack_run<DT>(own + k * kStep, v);
#pragma unroll
        for (int j = 0; j < kRun; ++j) v[j] = act_value<decltype(tag)::value>(fmaf(v[j] - m[G::of(j)], gamma[j], beta[j]));
        store_run<DT, kRun>(dst, d.vec_out, kRun, v);
      }
    });
  } else {
    // groups of 32 channels need a warp's lanes together
    const int lead = (int)((threadIdx.x & 31) >> min(r.lane_shift, 5));
    with_act(d.act, [&](auto tag) {
      for (int p = q.row, k = 0; p - lead < q.rows; p += q.row_step, ++k, dst += hop) {
        const bool on = k < count;
        const int64_t row = (int64_t)q.sample * d.hw + q.first + p;
        if (on) unpack_run<DT>(own + k * kStep, v);
        if (d.x8.dev_codes) pack_whole(d.x8, d.vec_x8, r.lane_shift, row, q.col, on, v);
        if (on) {
#pragma unroll
          for (int j = 0; j < kRun; ++j) v[j] = act_value<decltype(tag)::value>(fmaf(v[j] - m[G::of(j)], gamma[j], beta[j]));
          store_rounded<DT>(dst, d.vec_out, v);
        }
        if (d.y8.dev_codes) pack_whole(d.y8, d.vec_y8, r.lane_shift, row, q.col, on, v);
      }
    });
  }
  if (r.parts > 1) norm_cluster_sync();                                 // nobody leaves while its sums may be read
}

// KEPT: x comes from its 8-bit form.
template <int DT, bool KEPT, bool ONE>
__global__ void __launch_bounds__(kResThreads, ONE ? 4 : 2)
norm_grad_resident_kernel(Resident r) {
  using T = typename Elem<DT>::T;
  using G = Groups<ONE>;
  constexpr int kDy = kRun * (int)sizeof(T), kX = KEPT ? kRun : kDy, kBytes = kDy + kX + (KEPT ? 1 : 0);
  extern __shared__ __align__(16) uint8_t res_smem[];
  const NormDev& d = r.d;
  const Place q = place_of(r);
  uint8_t* dys = res_smem;                                              // [steps][threads] pieces of dy, then of x
  uint8_t* xs = dys + (size_t)r.steps * kResThreads * kDy;
  uint8_t* es = xs + (size_t)r.steps * kResThreads * kX + threadIdx.x;   // exponent byte of every piece
  float* scratch = reinterpret_cast<float*>(res_smem + (size_t)r.steps * kResThreads * kBytes);
  const int groups_cap = r.cb / d.cpg, groups = q.channels / d.cpg;
  float* chan = scratch + (2 * kRun * kResWarps << min(r.lane_shift, 5));   // [2][channels of a block]
  float* mine = chan + 2 * r.cb;                                        // [2][groups of a block]
  float* total = mine + 2 * groups_cap;
  const int count = q.on && q.row < q.rows ? (q.rows - q.row + q.row_step - 1) / q.row_step : 0;
  uint8_t* gown = dys + threadIdx.x * kDy;
  uint8_t* xown = xs + threadIdx.x * kX;
  train_pdl_wait();
  const int64_t row0 = (int64_t)q.sample * d.hw + q.first + q.row;
  {
    fetch_pieces<T>(gown, kResThreads * kDy, static_cast<const T*>(d.dy) + q.sample * d.sample_dy + (int64_t)(q.first + q.row) * d.ld_dy + q.col,
                    q.row_step * d.ld_dy, count, d.vec_dy);
    if constexpr (KEPT) {
      const uint8_t* src = d.x8.dev_codes + row0 * d.x8.ld_codes + q.col;
      const int64_t hop = q.row_step * d.x8.ld_codes;
      if (d.vec_x8) {
#pragma unroll 4
        for (int k = 0; k < count; ++k) copy_async<8>(xown + k * (kResThreads * kX), src + k * hop);
      } else {
        for (int k = 0; k < count; ++k) {
          uint2 w = make_uint2(0u, 0u);
#pragma unroll
          for (int j = 0; j < kRun; ++j) (j < 4 ? w.x : w.y) |= (uint32_t)src[k * hop + j] << (8 * (j & 3));
          *reinterpret_cast<uint2*>(xown + k * (kResThreads * kX)) = w;
        }
      }
    } else {
      fetch_pieces<T>(xown, kResThreads * kX, static_cast<const T*>(d.x) + q.sample * d.sample_x + (int64_t)(q.first + q.row) * d.ld_x + q.col,
                      q.row_step * d.ld_x, count, d.vec_x);
    }
    if constexpr (KEPT) {
      const uint8_t* esrc = d.x8.dev_exps + row0 * d.x8.ld_exps + q.col / kGroup;
      const int64_t ehop = q.row_step * d.x8.ld_exps;
#pragma unroll 8
      for (int k = 0; k < count; ++k) es[k * kResThreads] = esrc[k * ehop];
    }
  }
  const G at(q.col - q.c0, d.cpg);
  float mean[G::kN], rstd[G::kN], gamma[kRun], beta[kRun];
#pragma unroll
  for (int j = 0; j < G::kN; ++j) {
    const size_t from = (size_t)q.sample * d.groups + (q.on ? q.c0 / d.cpg + at.at[j] : 0);
    mean[j] = d.mean[from];
    rstd[j] = d.rstd[from];
  }
#pragma unroll
  for (int j = 0; j < kRun; ++j) {
    gamma[j] = q.on ? __ldg(d.gamma + q.col + j) : 0.f;
    beta[j] = q.on ? __ldg(d.beta + q.col + j) : 0.f;
  }
  copy_async_wait();
  // With e = x - mean and f = gamma rstd:  h = f e + beta,  dh = dy act'(h),  dgamma = rstd sum of dh e,
  // dx = f dh - rstd <u> - rstd^2 <u xh> e
  float f[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) f[j] = gamma[j] * rstd[G::of(j)];
  auto piece = [&](auto tag, int k, float (&e)[kRun], float (&dh)[kRun]) {
    if constexpr (KEPT) decode_run(*reinterpret_cast<const uint2*>(xown + k * (kResThreads * kX)), es[k * kResThreads], e);
    else unpack_run<DT>(xown + k * (kResThreads * kX), e);
    unpack_run<DT>(gown + k * (kResThreads * kDy), dh);
#pragma unroll
    for (int j = 0; j < kRun; ++j) {
      e[j] -= mean[G::of(j)];
      dh[j] *= act_slope<decltype(tag)::value>(fmaf(e[j], f[j], beta[j]));
    }
  };
  float ab[2 * kRun];                                                   // sums of dh, of dh e
#pragma unroll
  for (int j = 0; j < 2 * kRun; ++j) ab[j] = 0.f;
  with_act(d.act, [&](auto tag) {
#pragma unroll 1
    for (int k = 0; k < count; ++k) {
      float e[kRun], dh[kRun];
      piece(tag, k, e, dh);
#pragma unroll
      for (int j = 0; j < kRun; ++j) { ab[j] += dh[j]; ab[kRun + j] = fmaf(dh[j], e[j], ab[kRun + j]); }
    }
  });
#pragma unroll
  for (int j = 0; j < kRun; ++j) ab[kRun + j] *= rstd[G::of(j)];
  fold_rows(r, ab, scratch);
  const size_t out_row = ((size_t)q.sample * r.parts + q.part) * d.c + q.c0;
  for (int i = threadIdx.x; i < 2 * q.channels; i += kResThreads) {
    const bool second = i >= q.channels;
    const int ch = second ? i - q.channels : i;
    const float t = piece_sum(r, scratch, (second ? kRun : 0) + ch % kRun, ch / kRun);
    (second ? d.part1 : d.part0)[out_row + ch] = t;
    chan[second * r.cb + ch] = t * __ldg(d.gamma + q.c0 + ch);
  }
  __syncthreads();
  group_totals<2>(r, groups, groups_cap, d.cpg, mine, total, [&](int t, int g, int i) { return chan[t * r.cb + g * d.cpg + i]; });
  const float inv = 1.f / ((float)d.hw * (float)d.cpg);
  float c0[G::kN], c1[G::kN];
#pragma unroll
  for (int j = 0; j < G::kN; ++j) {
    c0[j] = q.on ? -rstd[j] * total[at.at[j]] * inv : 0.f;
    c1[j] = q.on ? -rstd[j] * rstd[j] * total[groups_cap + at.at[j]] * inv : 0.f;
  }
  T* dst = static_cast<T*>(d.out) + q.sample * d.sample_out + (int64_t)(q.first + q.row) * d.ld_out + q.col;
  const int64_t hop = q.row_step * d.ld_out;
  with_act(d.act, [&](auto tag) {
    T* to = dst;
#pragma unroll 1
    for (int k = 0; k < count; ++k, to += hop) {
      float e[kRun], dh[kRun];
      piece(tag, k, e, dh);
#pragma unroll
      for (int j = 0; j < kRun; ++j) e[j] = fmaf(dh[j], f[j], fmaf(e[j], c1[G::of(j)], c0[G::of(j)]));
      store_run<DT, kRun>(to, d.vec_out, kRun, e);
    }
  });
  if (r.parts > 1) norm_cluster_sync();
}

// dgamma and dbeta: sums over the rows of part1 and part0, 32 channels per block.
__global__ void __launch_bounds__(1024)
norm_dparam_kernel(NormDev d, int rows) {
  train_pdl_wait();
  __shared__ float s0[32][33], s1[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (int)blockIdx.x * 32 + lane;
  float a = 0.f, b = 0.f;
  if (col < d.c) {
#pragma unroll 8
    for (int r = warp; r < rows; r += 32) {
      a += d.part0[(size_t)r * d.c + col];
      b += d.part1[(size_t)r * d.c + col];
    }
  }
  s0[warp][lane] = a;
  s1[warp][lane] = b;
  __syncthreads();
  if (warp < 2 && col < d.c) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) t += (warp ? s1 : s0)[k][lane];
    (warp ? d.dgamma : d.dbeta)[col] = t;
  }
}

constexpr size_t kResSmemMax = 220 * 1024;

size_t resident_smem(const Resident& r, int piece_bytes) {
  // pieces; the scratch of 16 sums per warp and piece; channel sums (two); group sums (four)
  return (size_t)r.steps * kResThreads * piece_bytes + 4 * ((size_t)(2 * kRun * kResWarps << std::min(r.lane_shift, 5)) + 2 * r.cb + 4 * (r.cb / r.d.cpg));
}
// Whether the resident kernels take a problem, and how.  piece_bytes: shared memory per 8 channels of a pixel.
bool plan_resident(const NormDev& d, bool packs, bool backward, int piece_bytes, Resident* out) {
  auto gcd = [](int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; };
  if (d.c % kRun) return false;
  const int unit = packs ? kGroup : kRun;
  const int64_t base = (int64_t)d.cpg / gcd(d.cpg, unit) * unit;
  Resident best = {};
  double best_score = 1e30;
  bool best_alone = false;                                  // more CTAs than SMs, one at a time on each
  for (int64_t cb = base;; cb += base) {
    const int64_t block = std::min<int64_t>(cb, d.c);
    if (block > kResThreads * kRun) break;
    // 64 bytes of a pixel at least, where it has them
    const bool last = block == d.c;
    if (block * (piece_bytes < 32 ? 2 : 4) < 64 && !last) continue;
    Resident r = {};
    r.d = d;
    r.cb = (int)block;
    r.blocks = (int)ceil_div64(d.c, block);
    while ((kRun << r.lane_shift) < block) ++r.lane_shift;
    const int row_step = kResThreads >> r.lane_shift;
    for (int parts = 1; parts <= 8; parts *= 2) {
      r.parts = parts;
      r.part_rows = (int)ceil_div64(d.hw, parts);
      if (parts > 1 && (int64_t)(parts - 1) * r.part_rows >= d.hw) break;
      r.steps = (int)ceil_div64(r.part_rows, row_step);
      const size_t smem = resident_smem(r, piece_bytes);
      if (smem > kResSmemMax) continue;
      const int64_t ctas = (int64_t)d.n * r.blocks * parts;
      if (ctas > 0x7fffffff) return false;
      const int per_sm = (int)std::min<size_t>(4, 226 * 1024 / (smem + 1024));
      // Fitted to the times of five shapes, forward and backward, over all these choices: 6 ns per CTA whatever it holds (9
      // where CTAs meet), 0.9 ns per 1000 values while four CTAs overlap on an SM, up to 1.9 times that with one, and a part of
      // what the last round of CTAs leaves idle.  (512 threads per CTA, or CTAs that walk over units with the next
      // one's copies under way, were built and were never the fastest.)
      const double values = (double)d.n * d.hw * d.c, wave = 148.0 * per_sm, full = std::ceil(ctas / wave) * wave / ctas;
      const double idle = (double)((1 << r.lane_shift) * kRun * r.blocks) / d.c;
      const double slow = per_sm == 1 ? 1.9 : per_sm == 2 ? 1.45 : per_sm == 3 ? 1.05 : 1.0;
      const double score = ctas * (parts > 1 ? 9e-3 : 6e-3) + values * 0.9e-6 * slow * (1 + 0.3 * std::min(full - 1, 2.0)) * idle;
      if (score < best_score) { best_score = score; best = r; best_alone = per_sm == 1 && ctas > 148; }
    }
    if (last) break;
  }
  if (best_score > 1e29) return false;
  // A forward pass that packs works long between its reads and its writes; with nothing else on the SM meanwhile the streaming
  // kernels are faster (33 x 3560 x 192, 8 groups: 98 us against 144; 38 x 6153 x 80: 85 against 136), without packing they
  // are not (67 against 44, 52 against 47), and a backward pass has more to read twice (166 against 82).
  if (packs && !backward && best_alone) return false;
  *out = best;
  return true;
}
// The last plans of this host thread, by the sizes they are made from: a training step asks for the same ones over and over.
bool make_resident(const NormDev& d, bool packs, bool backward, int piece_bytes, Resident* out) {
  struct Memo { int32_t n = -1, hw, c, groups, packs, backward, piece_bytes; bool ok; Resident r; };
  static thread_local Memo memo[16];
  static thread_local unsigned next = 0;
  for (const Memo& m : memo)
    if (m.n == d.n && m.hw == d.hw && m.c == d.c && m.groups == d.groups && m.packs == (int)packs && m.backward == (int)backward && m.piece_bytes == piece_bytes) {
      if (m.ok) { *out = m.r; out->d = d; }
      return m.ok;
    }
  Memo& m = memo[next++ % 16];
  m.ok = plan_resident(d, packs, backward, piece_bytes, &m.r);
  m.n = d.n; m.hw = d.hw; m.c = d.c; m.groups = d.groups; m.packs = packs; m.backward = backward; m.piece_bytes = piece_bytes;
  if (m.ok) *out = m.r;
  return m.ok;
}
template <void (*kernel)(Resident)>
int launch_resident(const Resident& r, int piece_bytes, cudaStream_t st, const char* what) {
  static std::atomic<uint64_t> ready{0};                    // devices on which the kernel may use its shared memory
  int dev = 0;
  TRAIN_CK(cudaGetDevice(&dev), "cudaGetDevice");
  if (dev >= 64 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    TRAIN_CK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kResSmemMax), "cudaFuncSetAttribute(norm)");
    if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
  }
  TRAIN_CK(train_launch(kernel, dim3((unsigned)((int64_t)r.d.n * r.blocks * r.parts)), dim3(kResThreads), resident_smem(r, piece_bytes), st, r.parts, r), what);
  return LQSGD_OK;
}
template <int DT>
int launch_forward(const Resident& r, cudaStream_t st) {
  const int piece = kRun * (int)sizeof(typename Elem<DT>::T);
  return r.d.cpg % kRun == 0 ? launch_resident<norm_resident_kernel<DT, true>>(r, piece, st, "norm_resident_kernel launch")
                             : launch_resident<norm_resident_kernel<DT, false>>(r, piece, st, "norm_resident_kernel launch");
}
template <int DT, bool KEPT>
int launch_backward(const Resident& r, cudaStream_t st) {
  const int dy = kRun * (int)sizeof(typename Elem<DT>::T), piece = dy + (KEPT ? kRun + 1 : dy);
  return r.d.cpg % kRun == 0 ? launch_resident<norm_grad_resident_kernel<DT, KEPT, true>>(r, piece, st, "norm_grad_resident_kernel launch")
                             : launch_resident<norm_grad_resident_kernel<DT, KEPT, false>>(r, piece, st, "norm_grad_resident_kernel launch");
}
bool forward_resident(const NormDev& d, int dtype, Resident* r) {
  return make_resident(d, d.x8.dev_codes || d.y8.dev_codes, false, kRun * train_elem(dtype), r);
}
bool backward_resident(const NormDev& d, int dtype, Resident* r) {
  const bool kept = d.x8.dev_codes != nullptr;
  return make_resident(d, kept, true, kRun * train_elem(dtype) + (kept ? kRun + 1 : kRun * train_elem(dtype)), r);
}

void make_geometry(NormDev* d) {
  d->cpg = d->c / d->groups;
  d->lane_shift = 0;
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
size_t rounded(size_t n) { return (n + 63) / 64 * 64; }
size_t workspace_of(const NormDev& d, int dtype, bool backward) {
  Resident r;
  if (backward ? backward_resident(d, dtype, &r) : forward_resident(d, dtype, &r))
    return backward ? 8 * rounded((size_t)d.n * r.parts * d.c) : 0;
  return 4 * (2 * rounded((size_t)d.n * d.chunks * d.c) + (backward ? 2 * rounded((size_t)d.n * d.groups) : 0));
}

int check_common(const lqsgd_group_norm* a) {
  if (!a || a->struct_size != sizeof(lqsgd_group_norm)) return LQSGD_ERR_INVALID_ARG;
  if (!train_dtype_ok(a->dtype) || !train_act_ok(a->act)) return LQSGD_ERR_INVALID_ARG;
  if (a->n < 0 || a->hw < 1 || a->hw > 0x7fffffff - 4095 || a->c < 1 || a->c > 65536 || a->groups < 1 || a->c % a->groups) return LQSGD_ERR_BAD_SHAPE;
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
int check_workspace(const NormDev& d, const lqsgd_group_norm& a, bool backward) {
  const size_t need = workspace_of(d, a.dtype, backward);
  if (need && (!a.dev_workspace || a.workspace_bytes < need)) return LQSGD_ERR_WORKSPACE_TOO_SMALL;
  return train_aligned(a.dev_workspace, 16) ? LQSGD_OK : LQSGD_ERR_MISALIGNED;
}
void place_workspace(NormDev* d, const lqsgd_group_norm& a, size_t part) {
  d->part0 = static_cast<float*>(a.dev_workspace);
  d->part1 = d->part0 + rounded(part);
  d->group0 = d->part1 + rounded(part);
  d->group1 = d->group0 + rounded((size_t)d->n * d->groups);
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
  *host_bytes_out = host_args->n ? workspace_of(to_dev(*host_args), host_args->dtype, backward != 0) : 0;
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
  if ((rc = check_workspace(d, *a, false)) != LQSGD_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  Resident r;
  if (forward_resident(d, a->dtype, &r)) {
    return a->dtype == LQSGD_BF16 ? launch_forward<LQSGD_BF16>(r, st) : a->dtype == LQSGD_F16 ? launch_forward<LQSGD_F16>(r, st) : launch_forward<LQSGD_F32>(r, st);
  }
  place_workspace(&d, *a, (size_t)d.n * d.chunks * d.c);
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
  if ((rc = check_workspace(d, *a, true)) != LQSGD_OK) return rc;
  Resident r;
  if (backward_resident(d, a->dtype, &r)) {
    const bool kept = d.x8.dev_codes != nullptr;
    place_workspace(&r.d, *a, (size_t)d.n * r.parts * d.c);
    if (a->dtype == LQSGD_BF16) rc = kept ? launch_backward<LQSGD_BF16, true>(r, st) : launch_backward<LQSGD_BF16, false>(r, st);
    else if (a->dtype == LQSGD_F16) rc = kept ? launch_backward<LQSGD_F16, true>(r, st) : launch_backward<LQSGD_F16, false>(r, st);
    else rc = kept ? launch_backward<LQSGD_F32, true>(r, st) : launch_backward<LQSGD_F32, false>(r, st);
    if (rc != LQSGD_OK) return rc;
    TRAIN_CK(train_launch(norm_dparam_kernel, dim3((unsigned)((d.c + 31) / 32)), dim3(1024), 0, st, 1, r.d, (int)(d.n * r.parts)), "norm_dparam_kernel launch");
    return LQSGD_OK;
  }
  place_workspace(&d, *a, (size_t)d.n * d.chunks * d.c);
  const dim3 grid((unsigned)((int64_t)d.n * d.chunks * d.segs));
  const int group_blocks = (int)ceil_div64((int64_t)d.n * d.groups, kJoinWarps);
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_grad_sums_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_grad_sums_kernel launch");
  TRAIN_CK(train_launch(norm_grad_join_kernel, dim3((unsigned)(group_blocks + (d.c + 31) / 32)), dim3(32 * kJoinWarps), 0, st, 1, d, group_blocks), "norm_grad_join_kernel launch");
  TRAIN_CK(NORM_BY_DTYPE(a->dtype, norm_grad_apply_kernel, grid, dim3(kThreads), 0, st, 1, d), "norm_grad_apply_kernel launch");
  return LQSGD_OK;
}
