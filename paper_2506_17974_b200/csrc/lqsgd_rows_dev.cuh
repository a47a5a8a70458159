// Device pieces shared by the operators that work on whole rows: the random bits of dropout, signed 8-bit codes, and how a row is
// dealt out to the threads that hold it.
#pragma once
#include "lqsgd_runs_dev.cuh"

namespace lqsgd {

// Dropout as the kernels take it: threshold T in the upper half of a word, 65536 / (65536 - T).
struct Drop {
  uint64_t seed, offset;
  const uint64_t* dev_seed;
  uint32_t threshold;                        // 0: nothing is dropped
  float scale;
};
inline Drop make_drop(const lqsgd_drop& d) {
  const int t = std::min((int)rint(65536.0 * (double)d.p), 65535);
  return {d.seed, d.offset, d.dev_seed, (uint32_t)t << 16, (float)(65536.0 / (65536 - t))};
}

namespace {

// Philox4x32, 10 rounds: a product of each even word by a constant, its high half mixed with a neighbour and the key, which grows by
// a constant every round.
__device__ __forceinline__ uint4 philox(uint64_t block, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
// Seed and offset of this launch: read on the device where the caller keeps them there.
__device__ __forceinline__ void open_drop(Drop& d) {
  if (d.threshold && d.dev_seed) {
    d.seed = d.dev_seed[0];
    d.offset += d.dev_seed[1];
  }
}
// v = r + dropout(v) for a run of 8 columns; block = row * ceil(cols / 8) + column / 8.  A half word's bits are compared in the upper half of
// a word, where what lies below them does not count.  One rounding, the same in every kernel that drops.
__device__ __forceinline__ void drop_run(const Drop& d, uint64_t block, float (&v)[kRun], const float (&r)[kRun]) {
  const uint4 bits = philox(block, d.offset, d.seed);
  const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = (w[j] << 16) >= d.threshold ? __fmaf_rn(v[2 * j], d.scale, r[2 * j]) : r[2 * j];
    v[2 * j + 1] = w[j] >= d.threshold ? __fmaf_rn(v[2 * j + 1], d.scale, r[2 * j + 1]) : r[2 * j + 1];
  }
}

// ---- rows of signed 8-bit codes
constexpr float kRowStepLow = 7.52316385e-37f, kRowInvHigh = 1.32922800e36f;      // 2^-120, 2^120
// Scale of a row, and what its values are multiplied by (0: the row is not finite, its codes are 0).
__device__ __forceinline__ void row_scale(float top, float& scale, float& inv) {
  const bool finite = __float_as_uint(top) < 0x7f800000u;
  scale = finite ? fmaxf(__fdiv_rn(top, 127.f), kRowStepLow) : __uint_as_float(0x7fc00000u);
  inv = finite ? fminf(__fdiv_rn(127.f, top), kRowInvHigh) : 0.f;
}
// Four codes rint(v inv) in a word: adding 1.5 * 2^23 to the rounded product leaves an integer in two's complement below.  v inv is rounded by
// itself, as the definition has it (no fused multiply-add).
__device__ __forceinline__ uint32_t signed_word(const float* v, float inv) {
  uint32_t b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(__fadd_rn(__fmul_rn(v[j], inv), 12582912.f));
  const uint32_t w = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  return inv == 0.f ? 0u : w;
}
// The 8-bit form of a run: four neighbouring lanes hold a group of 32.  The whole warp calls it; `store`: this lane's run is written.
__device__ __forceinline__ void put_packed_run(const lqsgd_packed8& p, bool vec, int64_t row, const Place& s, bool store, const float (&v)[kRun]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kRun; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int eb = exp_byte(__uint_as_float(top));
  const float inv = inv_step(eb);
  if (!store) return;
  store_codes(p.dev_codes + row * p.ld_codes + s.col, vec && s.have == kRun, s.have,
              make_uint2(code_word(v[0], v[1], v[2], v[3], inv), code_word(v[4], v[5], v[6], v[7], inv)));
  if ((s.col & (kGroup - 1)) == 0) p.dev_exps[row * p.ld_exps + s.col / kGroup] = (uint8_t)eb;
}

// ---- a row and its threads
// NARROW: 4, 8, 16 or 32 lanes of a warp hold a row, a block of 256 threads several rows.  Otherwise a block holds one row.
// A thread's i-th run of 8 columns is the (i * size + t)-th of the row.
template <bool NARROW>
struct Team {
  int t, size, warps;
  int64_t row;
  __device__ __forceinline__ explicit Team(int lane_shift) {
    if (NARROW) {
      size = 1 << lane_shift;
      t = threadIdx.x & (size - 1);
      warps = 1;
      row = (int64_t)blockIdx.x * (blockDim.x >> lane_shift) + (threadIdx.x >> lane_shift);
    } else {
      size = blockDim.x;
      t = threadIdx.x;
      warps = blockDim.x >> 5;
      row = blockIdx.x;
    }
  }
  __device__ __forceinline__ int rows_per_grid() const { return NARROW ? (int)gridDim.x * ((int)blockDim.x / size) : (int)gridDim.x; }
  // runs per thread of a row
  __device__ __forceinline__ int steps(int cols) const { return (cols + size * kRun - 1) / (size * kRun); }
  __device__ __forceinline__ Place place(int i, int cols) const {
    Place s;
    s.col = (i * size + t) * kRun;
    s.have = min(kRun, cols - s.col);
    s.side = (i * size + (t & ~31)) * kRun + (threadIdx.x & 31);
    return s;
  }
  // Sum and largest of the team's values, in every thread of it.  `slots`: two warps' worth of shared memory (unused by NARROW);
  // of two calls in a row the second takes other slots, or a barrier lies between them.
  __device__ __forceinline__ void join(float& sum, uint32_t& top, float2* slots) const {
    const int lanes = NARROW ? size : 32;
    for (int o = 1; o < lanes; o <<= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if (!NARROW) {
      const int lane = threadIdx.x & 31;
      if (lane == 0) slots[threadIdx.x >> 5] = make_float2(sum, __uint_as_float(top));
      __syncthreads();
      const float2 s = lane < warps ? slots[lane] : make_float2(0.f, 0.f);
      sum = s.x;
      top = __float_as_uint(s.y);
      for (int o = 1; o < 32; o <<= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
    }
  }
};
__device__ __forceinline__ void load_vector(const float* p, const Place& s, bool vec, float (&v)[kRun]) {
  if (vec && s.have == kRun) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p + s.col)), b = __ldg(reinterpret_cast<const float4*>(p + s.col) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = j < s.have ? __ldg(p + s.col + j) : 0.f;
  }
}

}  // namespace
}  // namespace lqsgd
