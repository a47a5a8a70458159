// Device side of the linear layers: the matrix product D[m, n] = sum_k A[m, k] B[n, k] on the tensor cores (tcgen05,
// fp32 accumulators in tensor memory) for the three products of a layer, with their epilogues.
//
//   product        A (rows m)          B (rows n)             contracted over      lies along memory rows
//   forward        x    [rows]         w   [out]              in                   A: k    B: k
//   grad_input     dz   [rows]         w^T [in]               out                  A: k    B: n
//   grad_weight    dz^T [out]          x^T [in]               rows                 A: m    B: n
//
// An operand whose rows hold k ("K-major") is staged as 64 k x R rows; one whose rows hold m or n ("MN-major") as blocks of
// 64 columns x 64 k: both arrive from TMA with the 128-byte swizzle that the tensor core reads, so nothing is transposed.
// x kept in 8 bits is the one operand TMA cannot bring: converter warps read its codes, decode them to 16 bits (exactly,
// see lqsgd_pack8) and write the same swizzled layout.
//
// A cluster of CG CTAs (1 or 2) works on a tile of 128 CG x BN: with CG = 2 each SM holds 128 rows of A and half of B's, and
// one tcgen05.mma.cta_group::2 drives both tensor cores, so that an SM fetches (128 + BN / 2) rows per k instead of
// 128 + BN.  Per CTA: warp 0 issues the TMA loads, warp 1 (of the cluster's first CTA) the MMAs, warps 4-11 (4-7 for a weight gradient) drain the
// accumulator (two of them, so that the next tile's sum runs under the epilogue); with x8 warp 3 loads its codes and the last
// eight warps decode them.  Clusters walk
// the work items (tile, piece of the sum) with a fixed stride.
//
// Every wait is bounded (lqsgd_stream_common.cuh): on expiry the CTA's abort flag goes up, all roles leave their loops,
// copies in flight are waited for, tensor memory is released and the caller's status word gets LQSGD_STATUS_TIMEOUT.
#pragma once
#include <cuda.h>

#include "lqsgd_stream_common.cuh"
#include "lqsgd_train_dev.cuh"

namespace lqsgd {

constexpr int kLinBM = 128;            // rows of A per CTA
constexpr int kLinBK = 64;             // k per stage: 128 bytes of a 16-bit type, one swizzle span
enum LinOperand { kOpK = 0, kOpMN = 1, kOpPacked = 2 };

// What happens to a sum: y = act(sum + bias) + residual, and the 8-bit forms.  rows x cols is the result as the caller sees it.
struct LinEpilogue {
  void* out;
  int64_t ld_out;
  const float* bias;
  const void* residual;
  int64_t ld_res;
  lqsgd_packed8 z8, y8;
  int32_t rows, cols;
  int32_t dtype;                       // of out and residual; LQSGD_F32: out is fp32 and residual is not used
  int32_t act;
  int32_t accumulate;                  // fp32 out only: add to what is there
  int32_t vec_out, vec_res, vec_z8, vec_y8;   // rows are aligned to 32 bytes (out, residual) / 16 bytes (codes)
};

struct alignas(64) LinProblem {
  CUtensorMap ta, tb;                  // operands; tb of a packed B: its codes
  CUtensorMap te;                      // exponents of a packed B
  LinEpilogue ep;
  float* partial;                      // pieces of sums: two per cluster, each a tile (see LinWalk)
  int32_t M, N, K;
  int32_t tiles_m, tiles_n, kb_total;
  int32_t share;                       // 0: clusters take whole tiles; otherwise every cluster takes this many k-blocks in a row
  int32_t dtype;                       // of the operands
  uint32_t box_a;                      // rows of A that TMA brings per stage and CTA: 128, fewer (a multiple of 8) where A has fewer and
                                       // they lie along k; what the stage holds beyond them only meets rows that do not exist
  uint32_t* status;
};

namespace {

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// shared::cluster address of the same variable in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t map_to(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// Arrival on a barrier of either CTA of the cluster.  What it announces was written through, or read by, the tensor core's side
// (after fence.proxy.async or tcgen05.fence): nothing passes through ordinary memory accesses, so it needs no release at
// cluster scope, which would wait for every load the thread has in flight (it made the weight gradient 4 times slower).
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Bounded wait: a plain try first, which costs a few cycles when the phase is complete, then the timed ones (testing in a
// loop first took 12 % off a large product's rate: the waiting warps' instructions displace the others').
__device__ __forceinline__ bool lin_wait(uint64_t* b, uint32_t parity, volatile int* abort_flag) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
  return ok ? true : mbar_wait(b, parity, abort_flag);
}
__device__ __forceinline__ bool lin_wait_warp(uint64_t* b, uint32_t parity, volatile int* abort_flag, int lane) {
  int ok = 1;
  if (lane == 0) ok = lin_wait(b, parity, abort_flag) ? 1 : 0;
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}

// For the loader and MMA warps, whose instructions take uniform operands: the whole warp waits and walks, one elected lane
// issues.  Inside `if (lane == 0)` every operand would first be moved from the lane's registers (a k block cost its lone
// thread about 690 cycles that way, more than the 512 of its MMAs).
__device__ __forceinline__ bool lin_wait_all(uint32_t bar, uint64_t* b, uint32_t parity, volatile int* abort_flag) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  if (__all_sync(0xffffffffu, ok)) return true;
  return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag));
}
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(ok));
  return ok != 0;
}

template <int CG>
__device__ __forceinline__ void lin_tma(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void lin_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 2)
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives, once every MMA issued so far has completed, on the barrier at this offset in every CTA of the cluster.
template <int CG>
__device__ __forceinline__ void lin_commit(uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void lin_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void lin_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Operand descriptor, 128-byte swizzle.  K-major: rows of 128 bytes, 8-row groups 1024 bytes apart (the stride field).
// MN-major: 128-byte rows of 64 m or n, one per k; 8 k are 1024 bytes apart (the stride field), the next 64 m or n
// 64 k x 128 bytes further (the leading field).
template <bool MN>
__device__ __forceinline__ uint64_t lin_desc(uint32_t addr) {
  uint64_t d = (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(MN ? (kLinBK * 128) >> 4 : 1) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;              // descriptor version of this architecture
  d |= (uint64_t)2 << 61;              // 128-byte swizzle
  return d;
}
// Byte step of a descriptor from one K = 16 slice to the next.
template <bool MN> __device__ __forceinline__ constexpr uint32_t lin_kstep() { return MN ? 16 * 128 : 32; }

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&f)[32]) {
  uint32_t v[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr) : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
}
// ---- 16-bit words of either operand type
__device__ __forceinline__ uint32_t pack2(int dtype, float lo, float hi) {
  if (dtype == LQSGD_BF16) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
  }
  const __half2 t = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ float2 unpack2(int dtype, uint32_t w) {
  if (dtype == LQSGD_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ uint16_t pack1(int dtype, float v) { return (uint16_t)pack2(dtype, v, 0.f); }
__device__ __forceinline__ float unpack1(int dtype, uint16_t w) { return unpack2(dtype, w).x; }

// 32 bytes in one access; the address is 32-byte aligned
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void ld_global_32(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}

// Eight-bit form of 32 values of one row in one thread (those from `have` on must be 0): the exponent byte and 8 code words.
__device__ __forceinline__ int encode32(const float (&v)[32], uint32_t (&w)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  const int eb = exp_byte(__uint_as_float(top));
  const float inv = inv_step(eb);
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = code_word(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inv);
  return eb;
}
__device__ __forceinline__ void put_packed(const lqsgd_packed8& p, bool vec, int64_t row, int col, int have, const float (&v)[32]) {
  uint32_t w[8];
  const int eb = encode32(v, w);
  uint8_t* c = p.dev_codes + row * p.ld_codes + col;
  if (vec && have == 32) {
    *reinterpret_cast<uint4*>(c) = make_uint4(w[0], w[1], w[2], w[3]);
    *(reinterpret_cast<uint4*>(c) + 1) = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < have) c[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
  p.dev_exps[row * p.ld_exps + col / kGroup] = (uint8_t)eb;
}

// Epilogues of a 32 x 32 piece held by a warp, a row per thread (on: the row exists; row0: lane 0's row): a weight gradient, ...
// Rows that are not 32-byte aligned go through the warp's scratch in shared memory, so that a warp's access is one row's
// 32 columns instead of one column of 32 rows (which costs a sector per element).
constexpr int kScratchPitch = 33;                      // words; odd, so neither rows nor columns meet on one bank
constexpr uint32_t kScratchBytes = 32 * kScratchPitch * 4, kScratchBytes16 = 32 * 34 * 2;
__device__ __forceinline__ void finish_rows_f32(const LinEpilogue& e, int64_t row0, int col, bool on, float (&v)[32], float* scratch) {
  const int lane = threadIdx.x & 31;
  const int have = min(32, e.cols - col);
  if (e.vec_out && have == 32) {
    if (!on) return;
    float* o = static_cast<float*>(e.out) + (row0 + lane) * e.ld_out + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[8];
      if (e.accumulate) {
        ld_global_32(o + 8 * i, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * i + j] += __uint_as_float(w[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * i + j]);
      st_global_32(o + 8 * i, w);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) scratch[lane * kScratchPitch + i] = v[i];
  __syncwarp();
  const int rows = (int)min((int64_t)32, e.rows - row0);
  float* o = static_cast<float*>(e.out) + row0 * e.ld_out + col + lane;
  if (lane < have) {
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
      const float t = scratch[r * kScratchPitch + lane];
      o[r * e.ld_out] = e.accumulate ? o[r * e.ld_out] + t : t;
    }
  }
  __syncwarp();
}
// ... or a layer's output.
__device__ __forceinline__ void finish_rows(const LinEpilogue& e, int64_t row0, int col, bool on, float (&v)[32], float* scratch) {
  const int lane = threadIdx.x & 31;
  const int have = min(32, e.cols - col);
  const int64_t row = row0 + lane;
  const int rows = (int)min((int64_t)32, e.rows - row0);
  uint16_t* half = reinterpret_cast<uint16_t*>(scratch);                // 16-bit values: rows of 2 x 17 halves
  constexpr int kHalfPitch = 34;
  if (e.bias) {
    if (have == 32) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] += __ldg(e.bias + col + i);
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < have) v[i] += __ldg(e.bias + col + i);
    }
  }
  if (have < 32) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i >= have) v[i] = 0.f;
  }
  if (e.z8.dev_codes && on) put_packed(e.z8, e.vec_z8, row, col, have, v);
  act_run(e.act, v);
  if (e.residual) {
    const uint16_t* r = static_cast<const uint16_t*>(e.residual) + row0 * e.ld_res + col;
    if (e.vec_res && have == 32) {
      if (on) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t w[8];
          ld_global_32(r + lane * e.ld_res + 16 * i, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 f = unpack2(e.dtype, w[j]);
            v[16 * i + 2 * j] += f.x;
            v[16 * i + 2 * j + 1] += f.y;
          }
        }
      }
    } else {
      if (lane < have) {
#pragma unroll 8
        for (int k = 0; k < rows; ++k) half[k * kHalfPitch + lane] = r[k * e.ld_res + lane];
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 f = unpack2(e.dtype, *reinterpret_cast<const uint32_t*>(half + lane * kHalfPitch + 2 * j));
        if (2 * j < have) v[2 * j] += f.x;
        if (2 * j + 1 < have) v[2 * j + 1] += f.y;
      }
      __syncwarp();
    }
  }
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = pack2(e.dtype, v[2 * i], v[2 * i + 1]);
  uint16_t* o = static_cast<uint16_t*>(e.out) + row0 * e.ld_out + col;
  if (e.vec_out && have == 32) {
    if (on) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = w[8 * i + j];
        st_global_32(o + lane * e.ld_out + 16 * i, h);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) *reinterpret_cast<uint32_t*>(half + lane * kHalfPitch + 2 * j) = w[j];
    __syncwarp();
    if (lane < have) {
#pragma unroll 8
      for (int k = 0; k < rows; ++k) o[k * e.ld_out + lane] = half[k * kHalfPitch + lane];
    }
    __syncwarp();
  }
  if (e.y8.dev_codes && on) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 f = unpack2(e.dtype, w[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
    put_packed(e.y8, e.vec_y8, row, col, have, v);
  }
}

// One value's 8-bit form where a warp holds 32 neighbouring columns of a row, lane by lane (0 in lanes past the end).
__device__ __forceinline__ void put_packed_lane(const lqsgd_packed8& p, int64_t row, int col, bool on, float v) {
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7fffffffu);
  const int eb = exp_byte(__uint_as_float(top));
  if (on) p.dev_codes[row * p.ld_codes + col] = (uint8_t)((mag_bits(v, inv_step(eb)) & 127u) | ((__float_as_uint(v) >> 24) & 128u));
  if ((threadIdx.x & 31) == 0) p.dev_exps[row * p.ld_exps + col / kGroup] = (uint8_t)eb;
}
// Epilogue of one row's 32 neighbouring columns, one per lane; col = the lane's column, on = it exists.  The whole warp calls it.
__device__ __forceinline__ void finish_lane(const LinEpilogue& e, int64_t row, int col, bool on, float v, float bias) {
  if (e.dtype == LQSGD_F32) {
    if (on) {
      float* o = static_cast<float*>(e.out) + row * e.ld_out + col;
      *o = e.accumulate ? *o + v : v;
    }
    return;
  }
  v = on ? v + bias : 0.f;
  if (e.z8.dev_codes) put_packed_lane(e.z8, row, col, on, v);
  float one[1] = {v};
  act_run(e.act, one);
  v = one[0];
  if (e.residual && on) v += unpack1(e.dtype, static_cast<const uint16_t*>(e.residual)[row * e.ld_res + col]);
  const uint16_t w = pack1(e.dtype, v);
  if (on) static_cast<uint16_t*>(e.out)[row * e.ld_out + col] = w;
  if (e.y8.dev_codes) put_packed_lane(e.y8, row, col, on, on ? unpack1(e.dtype, w) : 0.f);
}

// ---- decoding 8-bit codes into operand words: four codes (one word) -> two words of two 16-bit numbers
// bf16: 0x4300 | m is 128 + m, so (128 + m) 2^e - 128 2^e is m 2^e, exactly, in one fused operation; then the sign is put on top.
// fp16: 0x6400 | m is 1024 + m; 1024 2^e may be out of range, so the 1024 goes first.
// Codes 0 and 2 make the first word, 1 and 3 the second, which takes no byte shuffles: within every four columns the operand
// holds columns 0, 2, 1, 3, and the epilogue puts them back.
__device__ __forceinline__ void decode4_bf16(uint32_t w, uint32_t step2, uint32_t off2, uint32_t& even, uint32_t& odd) {
  const uint32_t te = (w & 0x007f007fu) | 0x43004300u, to = ((w >> 8) & 0x007f007fu) | 0x43004300u;
  const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&step2), o = *reinterpret_cast<const __nv_bfloat162*>(&off2);
  const __nv_bfloat162 e = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&te), s, o), d = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&to), s, o);
  even = *reinterpret_cast<const uint32_t*>(&e) | ((w << 8) & 0x80008000u);
  odd = *reinterpret_cast<const uint32_t*>(&d) | (w & 0x80008000u);
}
__device__ __forceinline__ void decode4_fp16(uint32_t w, uint32_t step2, uint32_t& even, uint32_t& odd) {
  const uint32_t te = (w & 0x007f007fu) | 0x64006400u, to = ((w >> 8) & 0x007f007fu) | 0x64006400u;
  const __half2 s = *reinterpret_cast<const __half2*>(&step2), k = __half2(__ushort_as_half(0x6400), __ushort_as_half(0x6400));
  const __half2 e = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&te), k), s), d = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&to), k), s);
  even = *reinterpret_cast<const uint32_t*>(&e) | ((w << 8) & 0x80008000u);
  odd = *reinterpret_cast<const uint32_t*>(&d) | (w & 0x80008000u);
}
// Any step: through fp32, saturated to the type's largest finite number (NaN stays).
__device__ __forceinline__ float decode1_any(float top, uint32_t code, int eb) {
  const float a = decode8(code & 255u, step_of(eb));
  return fabsf(a) > top ? copysignf(top, a) : a;
}
__device__ __forceinline__ void decode4_any(int dtype, uint32_t w, int eb, uint32_t& even, uint32_t& odd) {
  const float top = dtype == LQSGD_BF16 ? 3.3895314e38f : 65504.f;
  even = pack2(dtype, decode1_any(top, w, eb), decode1_any(top, w >> 16, eb));
  odd = pack2(dtype, decode1_any(top, w >> 8, eb), decode1_any(top, w >> 24, eb));
}

// ---- the walk over (tile, k block) pairs that every role of a CTA makes
// Two ways to deal them out.  Whole tiles: cluster g takes tiles g, g + G, ...  Equal shares (few tiles, long sums): all
// (tile, k block) pairs stand in one row, tile after tile, and cluster g takes pairs [g share, (g + 1) share).  A tile
// that a share begins or ends inside of is summed by several clusters: each writes what it has to a piece of the
// workspace (at most two per cluster: piece 2 g where its share begins, 2 g + 1 for a tile that its share ends
// inside of), and linear_join_kernel adds a tile's pieces in the order of the clusters.
struct LinWalk {
  uint32_t pos, end, begin;            // equal shares: pairs (fewer than 2^31); whole tiles: tiles
  uint32_t stride;
  int cluster;
  int kb, kb_end;                      // the k blocks of the current tile that are this cluster's
  int m_tile, n_tile;
  // Tiles are taken in bands of 8 rows of tiles, column by column: the clusters at work then share 8 row tiles and
  // about as many column tiles, which keeps their operands in L2.
  static __device__ __forceinline__ void place(uint32_t tiles_m, uint32_t tiles_n, uint32_t t, int& m_tile, int& n_tile) {
    constexpr uint32_t kBand = 8;
    const uint32_t band = t / (kBand * tiles_n), first = band * kBand, high = min(kBand, tiles_m - first);
    const uint32_t in = t - band * kBand * tiles_n;
    n_tile = (int)(in / high);
    m_tile = (int)(first + in - n_tile * high);
  }
  __device__ __forceinline__ void locate(const LinProblem& p) {
    uint32_t t = pos;
    kb = 0;
    kb_end = p.kb_total;
    if (p.share) {
      t = pos / (uint32_t)p.kb_total;
      kb = (int)(pos - t * p.kb_total);
      kb_end = min(p.kb_total, kb + (int)(end - pos));
    }
    place(p.tiles_m, p.tiles_n, t, m_tile, n_tile);
  }
  __device__ __forceinline__ LinWalk(const LinProblem& p, int g, int clusters) : cluster(g) {
    const uint32_t tiles = p.tiles_m * p.tiles_n;
    pos = p.share ? (uint32_t)g * p.share : (uint32_t)g;
    end = p.share ? min(tiles * p.kb_total, pos + p.share) : tiles;
    stride = clusters;
    begin = pos;
    if (pos < end) locate(p);
  }
  __device__ __forceinline__ bool done() const { return pos >= end; }
  // The piece the current tile's sum goes to, or -1: the cluster has the whole tile.
  __device__ __forceinline__ int piece(const LinProblem& p) const {
    return kb_end - kb == p.kb_total ? -1 : (pos == begin ? 2 * cluster : 2 * cluster + 1);
  }
  // To the next tile; only from the state locate() left (next() below moves kb).
  __device__ __forceinline__ void next_tile(const LinProblem& p) {
    pos += p.share ? (uint32_t)(kb_end - kb) : stride;
    if (pos < end) locate(p);
  }
  // To the next k block, of this tile or the next.
  __device__ __forceinline__ void next(const LinProblem& p) {
    if (p.share) ++pos;
    if (++kb == kb_end) {
      if (!p.share) pos += stride;
      if (pos < end) locate(p);
    }
  }
};

// WF32: the result is fp32 (a weight gradient).
template <int CG, int BN, int OA, int OB, bool WF32>
struct LinCfg {
  static constexpr int kBNc = BN / CG;                                    // rows of B per CTA
  static constexpr uint32_t kABytes = kLinBM * 128, kBBytes = kBNc * 128;
  static constexpr uint32_t kStage = kABytes + ((kBBytes + 1023) / 1024 * 1024);
  // a packed B passes through a second, small ring: 64 rows of kBNc codes and of the 16 exponents that hold the tile's
  static constexpr int kRaw = OB == kOpPacked ? 4 : 0;
  static constexpr uint32_t kRawCodes = kLinBK * kBNc, kRawBytes = kRawCodes + kLinBK * 16;
  static constexpr uint32_t kScratch = WF32 ? 4 * kScratchBytes : 8 * kScratchBytes16;   // one per epilogue warp
  static constexpr uint32_t kRoom = 225u * 1024 - kRaw * kRawBytes - kScratch;
  static constexpr int kStages = (int)(kRoom / kStage) > 12 ? 12 : (int)(kRoom / kStage);
  static constexpr uint32_t kTxB = OB == kOpPacked ? 0 : kBBytes;         // what TMA brings of B per stage and CTA
  // Two warps per quarter of tensor memory where the epilogue computes per value (GELU and the 8-bit form take as
  // long as the product of a 4096-wide layer with one).
  static constexpr int kEpiWarps = WF32 ? 4 : 8;
  // A thread decodes 32 codes of one row of x; two teams of warps take the stages in turn, because one team's
  // chain of waits, loads, decoding and hand-over (about 700 cycles) is longer than a stage's MMAs (512).
  static constexpr int kTeams = 2;
  static constexpr int kConvWarps = OB == kOpPacked ? kBNc / 16 : 0;      // of one team
  static constexpr int kConvWarp0 = 4 + kEpiWarps;
  static constexpr int kThreads = (kConvWarp0 + kTeams * kConvWarps) * 32;
  static constexpr int kTmemCols = 2 * BN < 32 ? 32 : 2 * BN;
  static constexpr int kBars = 3 * kStages + 2 * kRaw + 2 + 2 + 1;
  static constexpr uint32_t kRawBase = kStages * kStage;
  static constexpr uint32_t kScratchOff = kRawBase + kRaw * kRawBytes;
  static constexpr uint32_t kBarOff = (kScratchOff + kScratch + 7) / 8 * 8;
  static constexpr uint32_t kSmem = kBarOff + kBars * 8 + 32 + 1024;
  static_assert(kSmem <= 227 * 1024 && kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0, "one CTA per SM");
  static_assert(OB == kOpK || kBNc % 64 == 0, "MN-major operands come in blocks of 64");
  static_assert(OB != kOpPacked || kBNc == 128, "a row of codes is one 128-byte swizzle span");
};

template <int CG, int BN, int OA, int OB, bool WF32>
__global__ void __launch_bounds__(LinCfg<CG, BN, OA, OB, WF32>::kThreads, 1)
linear_kernel(const __grid_constant__ LinProblem p) {
  using S = LinCfg<CG, BN, OA, OB, WF32>;
  extern __shared__ uint8_t lin_smem[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(lin_smem) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + S::kBarOff);   // [stages] TMA bytes landed, in both CTAs (first CTA's barrier)
  uint64_t* conv = full + S::kStages;                                // [stages] decoded rows of B written, in both CTAs (first CTA's)
  uint64_t* empty = conv + S::kStages;                               // [stages] the MMAs that read the stage are done
  uint64_t* raw_full = empty + S::kStages;                           // [raw] codes and exponents of B landed in this CTA
  uint64_t* raw_empty = raw_full + S::kRaw;                          // [raw] every converter warp has them in registers
  uint64_t* d_full = raw_empty + S::kRaw;                            // [2] accumulator complete
  uint64_t* d_empty = d_full + 2;                                    // [2] accumulator drained by both CTAs (first CTA's)
  uint64_t* fin = d_empty + 2;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(fin + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(fin + 1) + 2;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
  const int cluster = (int)blockIdx.x / CG, clusters = (int)gridDim.x / CG;

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(conv + s, CG * (S::kConvWarps ? S::kConvWarps : 1));
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < S::kRaw; ++s) { mbar_init(raw_full + s, 1); mbar_init(raw_empty + s, S::kConvWarps); }
    for (int s = 0; s < 2; ++s) { mbar_init(d_full + s, 1); mbar_init(d_empty + s, S::kEpiWarps * CG); }
    mbar_init(fin, 1);
    wait_ctl_init(abort_flag, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.ta) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.tb) : "memory");
    if constexpr (OB == kOpPacked) asm volatile("prefetch.tensormap [%0];" ::"l"(&p.te) : "memory");
  }
  if (warp == 2) {
    if constexpr (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)S::kTmemCols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  lin_fence_before();
  __syncthreads();
  if constexpr (CG == 2) cluster_sync_all();
  lin_fence_after();
  const uint32_t tmem = *tmem_slot;
  train_pdl_trigger();
  // Every role first finds its place in the work, then waits for the kernel in front.
  const uint32_t base_s = smem_u32(base), full_s = smem_u32(full), conv_s = smem_u32(conv), empty_s = smem_u32(empty);

  if (warp == 0) {
    // ---- loader
    LinWalk w(p, cluster, clusters);
    train_pdl_wait();
    const uint32_t full0 = CG == 2 ? map_to(full, 0) : full_s;          // the first CTA's barriers count both CTAs' bytes
    const uint32_t tx = CG * (p.box_a * 128 + S::kTxB);
    uint32_t s = 0, turn = 0, it = 0;
    bool ok = true;
    for (; !w.done(); w.next(p), ++it) {
      if (!lin_wait_all(empty_s + 8 * s, empty + s, turn ^ 1, abort_flag)) { ok = false; break; }
      const uint32_t a = base_s + s * S::kStage, b = a + S::kABytes, bar = full0 + 8 * s;
      const int k0 = w.kb * kLinBK, m0 = (w.m_tile * CG + (int)rank) * kLinBM, n0 = w.n_tile * BN + (int)rank * S::kBNc;
      if (elect_one()) {
        if (rank == 0) mbar_arrive_expect_tx(full + s, tx);
        if constexpr (OA == kOpK) {
          lin_tma<CG>(a, &p.ta, k0, m0, bar);
        } else {
#pragma unroll
          for (int i = 0; i < kLinBM / 64; ++i) lin_tma<CG>(a + i * kLinBK * 128, &p.ta, m0 + 64 * i, k0, bar);
        }
        if constexpr (OB == kOpK) {
          lin_tma<CG>(b, &p.tb, k0, n0, bar);
        } else if constexpr (OB == kOpMN) {
#pragma unroll
          for (int i = 0; i < S::kBNc / 64; ++i) lin_tma<CG>(b + i * kLinBK * 128, &p.tb, n0 + 64 * i, k0, bar);
        }
      }
      __syncwarp();
      if (++s == S::kStages) { s = 0; turn ^= 1; }
    }
    if (!ok && rank == 0 && lane == 0) {            // copies in flight land before the CTA's memory goes away
      const uint32_t limit = wait_limit_of(abort_flag);
      for (uint32_t j = it > (uint32_t)S::kStages ? it - S::kStages : 0; j < it; ++j)
        for (uint32_t i = 0; i < limit && !mbar_try(full + j % S::kStages, (j / S::kStages) & 1); ++i) {}
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- MMA issue: the cluster's first CTA
    if (rank == 0) {
      const uint32_t fmt = p.dtype == LQSGD_BF16 ? 1u : 0u;
      // fp32 accumulator, operand type, which operands are MN-major, N / 8, M / 16
      const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((OA == kOpK ? 0u : 1u) << 15) | ((OB == kOpK ? 0u : 1u) << 16) |
                             ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((kLinBM * CG) >> 4) << 24);
      const uint64_t ad0 = lin_desc<OA != kOpK>(base_s), bd0 = lin_desc<OB != kOpK>(base_s + S::kABytes);
      const uint32_t d_full_s = smem_u32(d_full), d_empty_s = smem_u32(d_empty);
      uint32_t s = 0, turn = 0, db = 0, dturn = 0;
      bool ok = true;
      LinWalk w(p, cluster, clusters);
      for (; !w.done() && ok; w.next_tile(p)) {
        if (!lin_wait_all(d_empty_s + 8 * db, d_empty + db, dturn ^ 1, abort_flag)) { ok = false; break; }
        lin_fence_after();
        const uint32_t d = tmem + db * BN;
        uint32_t more = 0;                          // the tile's first product starts the sum
        for (int kb = w.kb; kb < w.kb_end; ++kb) {
          if (!lin_wait_all(full_s + 8 * s, full + s, turn, abort_flag)) { ok = false; break; }
          if constexpr (OB == kOpPacked) {
            if (!lin_wait_all(conv_s + 8 * s, conv + s, turn, abort_flag)) { ok = false; break; }
          }
          lin_fence_after();
          const uint64_t ad = ad0 + (uint64_t)(s * (S::kStage >> 4)), bd = bd0 + (uint64_t)(s * (S::kStage >> 4));
          if (elect_one()) {
#pragma unroll
            for (int ks = 0; ks < kLinBK / 16; ++ks)
              lin_mma<CG>(d, ad + ((ks * lin_kstep<OA != kOpK>()) >> 4), bd + ((ks * lin_kstep<OB != kOpK>()) >> 4), idesc, ks > 0 ? 1u : more);
            lin_commit<CG>(empty_s + 8 * s);
          }
          __syncwarp();
          more = 1;
          if (++s == S::kStages) { s = 0; turn ^= 1; }
        }
        if (ok && elect_one()) lin_commit<CG>(d_full_s + 8 * db);
        __syncwarp();
        db ^= 1;
        if (db == 0) dturn ^= 1;
      }
      if (elect_one()) lin_commit<CG>(smem_u32(fin));   // every MMA has completed before tensor memory is released
      __syncwarp();
      if (lane == 0) {
        const uint32_t limit = wait_limit_of(abort_flag);
        for (uint32_t i = 0; i < limit && !mbar_try(fin, 0); ++i) {}
      }
    }
    __syncwarp();
  } else if (OB == kOpPacked && warp == 3) {
    // ---- loader of the codes: one thread; each CTA brings its own part, for its own converters
    if constexpr (OB == kOpPacked) if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      LinWalk w(p, cluster, clusters);
      train_pdl_wait();
      for (; !w.done(); w.next(p), ++it) {
        const int r = it % S::kRaw;
        if (!lin_wait(raw_empty + r, ((it / S::kRaw) & 1) ^ 1, abort_flag)) { ok = false; break; }
        uint8_t* raw = base + S::kRawBase + r * S::kRawBytes;
        const int k0 = w.kb * kLinBK, n0 = w.n_tile * BN + (int)rank * S::kBNc;
        mbar_arrive_expect_tx(raw_full + r, S::kRawBytes);
        lin_tma<1>(smem_u32(raw), &p.tb, n0, k0, smem_u32(raw_full + r));
        lin_tma<1>(smem_u32(raw) + S::kRawCodes, &p.te, n0 / kGroup / 16 * 16, k0, smem_u32(raw_full + r));
      }
      if (!ok) {
        const uint32_t limit = wait_limit_of(abort_flag);
        for (uint32_t j = it > (uint32_t)S::kRaw ? it - S::kRaw : 0; j < it; ++j)
          for (uint32_t i = 0; i < limit && !mbar_try(raw_full + j % S::kRaw, (j / S::kRaw) & 1); ++i) {}
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 4 + S::kEpiWarps) {
    // ---- epilogue: a warp reads its quarter of the accumulator's rows (warp % 4), and with eight warps half of its columns
    uint32_t seq = 0;
    const int q = warp & 3;
    LinWalk w(p, cluster, clusters);
    train_pdl_wait();
    for (; !w.done(); w.next_tile(p), ++seq) {
      const uint32_t db = seq & 1;
      if (!lin_wait_warp(d_full + db, (seq >> 1) & 1, abort_flag, lane)) break;
      lin_fence_after();
      const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + db * BN;
      const int m = (w.m_tile * CG + (int)rank) * kLinBM + 32 * q + lane;
      const int n0 = w.n_tile * BN;
      const int piece = w.piece(p);
      float* part = piece >= 0 ? p.partial + (int64_t)piece * (CG * kLinBM * BN) : nullptr;
      constexpr int kStep = 32, kMine = BN / (S::kEpiWarps / 4);
      const int c0 = ((warp - 4) >> 2) * kMine;
      float* scratch = reinterpret_cast<float*>(base + S::kScratchOff + (warp - 4) * (WF32 ? kScratchBytes : kScratchBytes16));
#pragma unroll 1
      for (int c = c0; c < c0 + kMine; c += kStep) {
        float v[32];
        tmem_ld32(taddr + c, v);
        if (c + kStep >= c0 + kMine) {            // the accumulator is in registers: hand it back
          lin_fence_before();
          __syncwarp();
          if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(d_empty + db, 0)); else mbar_arrive(d_empty + db); }
        }
        if (n0 + c >= p.N || m - lane >= p.M) continue;
        if constexpr (OB == kOpPacked) {          // back from the order of the decoder
#pragma unroll
          for (int j = 0; j < 32; j += 4) { const float t = v[j + 1]; v[j + 1] = v[j + 2]; v[j + 2] = t; }
        }
        if (part) {                               // [row of the tile][BN]
          float* o = part + (int64_t)((int)rank * kLinBM + 32 * q + lane) * BN + c;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[8 * i + j]);
            st_global_32(o + 8 * i, u);
          }
        } else if constexpr (WF32) {
          finish_rows_f32(p.ep, m - lane, n0 + c, m < p.M, v, scratch);
        } else {
          finish_rows(p.ep, m - lane, n0 + c, m < p.M, v, scratch);
        }
      }
    }
  } else if (OB == kOpPacked && warp >= S::kConvWarp0) {
    // ---- converters: codes and exponents of 64 rows of x8 (k) -> the MN-major operand (n).  A warp takes 32 rows of one group
    // of 32 columns, a lane one row: its 16-byte accesses, to the codes (swizzled by TMA) and to the operand (swizzled for the
    // tensor core), then fall on different banks.  The codes come through shared memory and not straight into registers
    // because the fence before the hand-over waits for a thread's own loads, however far ahead they were issued.
    if constexpr (OB == kOpPacked) {
      const int ct = tid - S::kConvWarp0 * 32;
      const int team = ct / (S::kConvWarps * 32), krow = ct & 63, group = (ct >> 6) & 3;
      const bool bf = p.dtype == LQSGD_BF16;
      int r = 0, s = 0, turn = 0;
      uint32_t rpar = 0, spar = 1;                                       // phase parities of the raw ring and of `empty`
      for (LinWalk w(p, cluster, clusters); !w.done(); w.next(p)) {
        if (turn == team) {
          if (!lin_wait_warp(raw_full + r, rpar, abort_flag, lane)) break;
          const uint8_t* raw = base + S::kRawBase + r * S::kRawBytes;
          const uint4 lo = *reinterpret_cast<const uint4*>(raw + krow * 128 + (((2 * group) ^ (krow & 7)) << 4));
          const uint4 hi = *reinterpret_cast<const uint4*>(raw + krow * 128 + (((2 * group + 1) ^ (krow & 7)) << 4));
          const int eb = raw[S::kRawCodes + krow * 16 + (((w.n_tile * BN + (int)rank * S::kBNc) / kGroup + group) & 15)];
          __syncwarp();
          if (lane == 0) mbar_arrive(raw_empty + r);
          const uint32_t cw[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
          const int e = eb - kExpBias;
          // the step, 128 steps (bf16) and every product are normal numbers in range; anything else goes through fp32
          const bool plain = bf ? eb <= 246 : (e >= -14 && e <= 8);
          uint32_t o[16];
          if (!plain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) decode4_any(p.dtype, cw[i], eb, o[2 * i], o[2 * i + 1]);
          } else if (bf) {
            const uint32_t one = (uint32_t)(e + 127) << 7, off = 0x8000u | ((uint32_t)(e + 127 + 7) << 7);    // 2^e, -128 2^e
#pragma unroll
            for (int i = 0; i < 8; ++i) decode4_bf16(cw[i], one | (one << 16), off | (off << 16), o[2 * i], o[2 * i + 1]);
          } else {
            const uint32_t one = (uint32_t)(e + 15) << 10;
#pragma unroll
            for (int i = 0; i < 8; ++i) decode4_fp16(cw[i], one | (one << 16), o[2 * i], o[2 * i + 1]);
          }
          if (!lin_wait_warp(empty + s, spar, abort_flag, lane)) break;
          uint8_t* b = base + s * S::kStage + S::kABytes + (group >> 1) * (kLinBK * 128) + krow * 128;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(b + ((((group & 1) * 4 + i) ^ (krow & 7)) << 4)) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          fence_async_smem();
          __syncwarp();
          if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(conv + s, 0)); else mbar_arrive(conv + s); }
        }
        if (++turn == S::kTeams) turn = 0;
        if (++r == S::kRaw) { r = 0; rpar ^= 1; }
        if (++s == S::kStages) { s = 0; spar ^= 1; }
      }
    }
  }
  lin_fence_before();
  __syncthreads();
  if (tid == 0 && *abort_flag && p.status) atomicOr(p.status, kStatusTimeout);
  if constexpr (CG == 2) cluster_sync_all();        // no CTA leaves while the other may still signal its barriers
  if (warp == 2) {
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::kTmemCols) : "memory");
  }
}

}  // namespace
}  // namespace lqsgd
