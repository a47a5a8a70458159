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
// x kept in 8 bits is decoded to 16 bits into the workspace ahead of the product (exactly in bf16; in fp16 values past 65504
// saturate and those below its normal range round): 5 bytes of traffic per value, once.  Decoding inside the product (warps that turn codes into the operand's layout in shared memory)
// was built and measured: every row tile decodes x again, and the decoders' shared memory traffic and hand-over take the
// MMAs' time: 1.37 against 0.86 ms for 8192 rows, 16384 x 4096, and 22.7 against 18.4 us for 65536 rows, 64 x 128.
//
// A cluster of CG CTAs (1 or 2) works on a tile of 128 CG x BN: with CG = 2 each SM holds 128 rows of A and half of B's, and
// one tcgen05.mma.cta_group::2 drives both tensor cores, so that an SM fetches (128 + BN / 2) rows per k instead of
// 128 + BN.  Per CTA: warp 0 issues the TMA loads, warp 1 (of the cluster's first CTA) the MMAs, warps 4-11 drain the
// accumulator (two of them, so that the next tile's sum runs under the epilogue).  Clusters walk
// the work items (tile, piece of the sum) with a fixed stride.
//
// Every wait is bounded (lqsgd_stream_common.cuh) and begins after the kernel in front has ended.  On expiry the CTA's abort
// flag goes up and all roles leave their loops; then the copies that either CTA of a pair still has in flight are waited for,
// tensor memory is released and the caller's status word gets LQSGD_STATUS_TIMEOUT.
#pragma once
#include <cuda.h>

#include "lqsgd_stream_common.cuh"
#include "lqsgd_train_dev.cuh"

namespace lqsgd {

constexpr int kLinBM = 128;            // rows of A per CTA
constexpr int kLinBK = 64;             // k per stage: 128 bytes of a 16-bit type, one swizzle span
enum LinOperand { kOpK = 0, kOpMN = 1 };
enum LinDeal { kWhole = 0, kShares = 1, kMeet = 2 };

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
  int32_t vec_out, vec_res, vec_z8, vec_y8;   // rows are aligned to 32 bytes (2), to 16 bytes (1), to neither (0)
};

struct alignas(64) LinProblem {
  CUtensorMap ta, tb;                  // operands
  LinEpilogue ep;
  float* partial;                      // pieces of sums: two per cluster, each a tile (see LinWalk)
  int32_t M, N, K;
  int32_t tiles_m, tiles_n, kb_total;
  int32_t deal;                        // how the work is dealt out (LinDeal), see LinWalk
  int32_t share;                       // k blocks per cluster (kShares) or per CTA of a cluster (kMeet)
  int32_t meet;                        // CTAs that sum one tile (kMeet)
  int32_t first_chunk;                 // k blocks that a tile's first two accumulators take, for pairs with results in 16 bits (pair_chunk)
  int32_t dtype;                       // of the operands
  uint32_t box_a;                      // rows of A that TMA brings per stage and CTA: 128, fewer (a multiple of 8) where A has fewer and
                                       // they lie along k; what the stage holds beyond them only meets rows that do not exist
  uint32_t* status;
  // Test support (lqsgd_test_linear_wait; zeros in normal operation): the limit of the bounded waits, and which role of the
  // first cluster stops after how many k blocks (LinRole).
  uint32_t test_limit, test_after;
  int32_t test_role;
};
enum LinRole { kNoRole = 0, kLoader0 = 1, kLoader1 = 2, kMma = 3 };

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

// Completes `bytes` of a barrier's phase in place of a copy that was announced and never issued.
__device__ __forceinline__ void complete_tx(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
// Waits (each time with a limit) for the last copies into a CTA's stages, `issued` k blocks of them so far.
__device__ __forceinline__ void lin_drain(uint64_t* full, uint32_t stages, uint32_t issued, uint32_t limit) {
  for (uint32_t j = issued > stages ? issued - stages : 0; j < issued; ++j)
    for (uint32_t i = 0; i < limit && !mbar_try(full + j % stages, (j / stages) & 1); ++i) {}
}
// The same for a pair, whose copies all count on the first CTA's barriers: `mine` and `other` k blocks were issued by the first and
// the second CTA, `bytes` each per k block.  Where one of them went on longer (by no more than the stages: neither refills
// a stage before both have filled it and it was read), its phases are made whole first.
__device__ __forceinline__ void lin_drain_pair(uint64_t* full, uint32_t stages, uint32_t mine, uint32_t other, uint32_t bytes, uint32_t limit) {
  for (uint32_t j = other; j < mine; ++j) complete_tx(full + j % stages, bytes);             // announced for both, issued by one
  for (uint32_t j = mine; j < other; ++j) mbar_arrive_expect_tx(full + j % stages, bytes);   // issued by the second, never announced
  lin_drain(full, stages, max(mine, other), limit);
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
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&f)[16]) {
  uint32_t v[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
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

// 32 bytes of a row that is aligned to 32 (vec = 2) or 16 bytes (vec = 1)
__device__ __forceinline__ void ld_row32(const void* p, int vec, uint32_t (&w)[8]) {
  if (vec == 2) {
    ld_global_32(p, w);
  } else {
    const uint4 a = *static_cast<const uint4*>(p), b = *(static_cast<const uint4*>(p) + 1);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}
__device__ __forceinline__ void st_row32(void* p, int vec, const uint32_t (&w)[8]) {
  if (vec == 2) {
    st_global_32(p, w);
  } else {
    *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    *(static_cast<uint4*>(p) + 1) = make_uint4(w[4], w[5], w[6], w[7]);
  }
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
__device__ __forceinline__ void put_packed(const lqsgd_packed8& p, int vec, int64_t row, int col, int have, const float (&v)[32]) {
  uint32_t w[8];
  const int eb = encode32(v, w);
  uint8_t* c = p.dev_codes + row * p.ld_codes + col;
  if (vec && have == 32) {
    st_row32(c, vec, w);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < have) c[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
  p.dev_exps[row * p.ld_exps + col / kGroup] = (uint8_t)eb;
}

// Epilogue of 8 columns of a weight gradient held by a warp, a row per thread (row0: lane 0's row), where rows are not 32-byte
// aligned or the tile passes the matrix: through the warp's scratch in shared memory (rows of 9 words), so that an access is
// four rows' 8 columns instead of one column of 32 rows (which costs a sector per element).
__device__ __forceinline__ void finish_ragged_f32(const LinEpilogue& e, int64_t row0, int col, const float* v, float* scratch) {
  const int lane = threadIdx.x & 31, c = lane & 7;
#pragma unroll
  for (int i = 0; i < 8; ++i) scratch[lane * 9 + i] = v[i];
  __syncwarp();
  const int rows = (int)min((int64_t)32, e.rows - row0);
  float* o = static_cast<float*>(e.out) + row0 * e.ld_out + col + c;
  if (col + c < e.cols) {
#pragma unroll 2
    for (int r = lane >> 3; r < rows; r += 4) {
      const float t = scratch[r * 9 + c];
      o[r * e.ld_out] = e.accumulate ? o[r * e.ld_out] + t : t;
    }
  }
  __syncwarp();
}
// Epilogue of a 32 x 32 piece of a layer's output.
// bias: these columns' values in shared memory (zeros past the matrix).
__device__ __forceinline__ void finish_rows(const LinEpilogue& e, int64_t row0, int col, bool on, float (&v)[32], const float* bias, float* scratch) {
  const int lane = threadIdx.x & 31;
  const int have = min(32, e.cols - col);
  const int64_t row = row0 + lane;
  const int rows = (int)min((int64_t)32, e.rows - row0);
  uint16_t* half = reinterpret_cast<uint16_t*>(scratch);                // 16-bit values: rows of 2 x 17 halves
  constexpr int kHalfPitch = 34;
  // The residual: this row's 32 columns where rows are aligned, else a column of all 32 rows, turned in shared memory.
  const bool res_rows = e.residual && e.vec_res && have == 32, res_cols = e.residual && !res_rows;
  const uint16_t* r = static_cast<const uint16_t*>(e.residual) + row0 * e.ld_res + col;
  const int word_row = lane >> 4, word_col = 2 * (lane & 15);             // rows that start on words: two at a time
  if (res_cols) {
    if (have == 32 && ((reinterpret_cast<uintptr_t>(r) | (2 * e.ld_res)) & 3) == 0) {
      uint32_t t[16];
#pragma unroll
      for (int k = 0; k < 16; ++k)
        t[k] = 2 * k + word_row < rows ? *reinterpret_cast<const uint32_t*>(r + (2 * k + word_row) * e.ld_res + word_col) : 0u;
#pragma unroll
      for (int k = 0; k < 16; ++k) *reinterpret_cast<uint32_t*>(half + (2 * k + word_row) * kHalfPitch + word_col) = t[k];
    } else {
      uint16_t t[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) t[k] = lane < have && k < rows ? r[k * e.ld_res + lane] : (uint16_t)0;
#pragma unroll
      for (int k = 0; k < 32; ++k) half[k * kHalfPitch + lane] = t[k];
    }
    __syncwarp();
  }
  if (e.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float4 b = *(reinterpret_cast<const float4*>(bias) + i);
      v[4 * i] += b.x; v[4 * i + 1] += b.y; v[4 * i + 2] += b.z; v[4 * i + 3] += b.w;
    }
  }
  if (have < 32) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i >= have) v[i] = 0.f;
  }
  if (e.z8.dev_codes && on) put_packed(e.z8, e.vec_z8, row, col, have, v);
  act_run(e.act, v);
  if (res_rows && on) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[8];
      ld_row32(r + lane * e.ld_res + 16 * i, e.vec_res, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 f = unpack2(e.dtype, w[j]);
        v[16 * i + 2 * j] += f.x;
        v[16 * i + 2 * j + 1] += f.y;
      }
    }
  }
  if (res_cols) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float2 f = unpack2(e.dtype, *reinterpret_cast<const uint32_t*>(half + lane * kHalfPitch + 2 * j));
      if (2 * j < have) v[2 * j] += f.x;
      if (2 * j + 1 < have) v[2 * j + 1] += f.y;
    }
    __syncwarp();
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
        st_row32(o + lane * e.ld_out + 16 * i, e.vec_out, h);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) *reinterpret_cast<uint32_t*>(half + lane * kHalfPitch + 2 * j) = w[j];
    __syncwarp();
    if (have == 32 && ((reinterpret_cast<uintptr_t>(o) | (2 * e.ld_out)) & 3) == 0) {
#pragma unroll 8
      for (int k = word_row; k < rows; k += 2)
        *reinterpret_cast<uint32_t*>(o + k * e.ld_out + word_col) = *reinterpret_cast<const uint32_t*>(half + k * kHalfPitch + word_col);
    } else if (lane < have) {
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

// ---- epilogue of a row whose columns a warp holds side by side, four neighbouring ones per lane (128 in all)
// 8-bit form: eight neighbouring lanes hold a group of 32.  The values of columns that do not exist are 0.
__device__ __forceinline__ void put_packed_quad(const lqsgd_packed8& p, int64_t row, int col, int have, const float (&v)[4]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int eb = exp_byte(__uint_as_float(top));
  if (have <= 0) return;
  const uint32_t w = code_word(v[0], v[1], v[2], v[3], inv_step(eb));
  uint8_t* c = p.dev_codes + row * p.ld_codes + col;
  if (have == 4 && (reinterpret_cast<uintptr_t>(c) & 3) == 0) {
    *reinterpret_cast<uint32_t*>(c) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < have) c[i] = (uint8_t)(w >> (8 * i));
  }
  if ((col & (kGroup - 1)) == 0) p.dev_exps[row * p.ld_exps + col / kGroup] = (uint8_t)eb;
}
// The whole warp calls it; col is the lane's first column.
__device__ __forceinline__ void finish_quad(const LinEpilogue& e, int64_t row, int col, float (&v)[4]) {
  const int have = min(4, e.cols - col);
  if (e.dtype == LQSGD_F32) {
    float* o = static_cast<float*>(e.out) + row * e.ld_out + col;
    if (have == 4 && e.vec_out) {
      float4 t = make_float4(v[0], v[1], v[2], v[3]);
      if (e.accumulate) {
        const float4 u = *reinterpret_cast<const float4*>(o);
        t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
      }
      *reinterpret_cast<float4*>(o) = t;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < have) o[i] = e.accumulate ? o[i] + v[i] : v[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i >= have) v[i] = 0.f;
    else if (e.bias) v[i] += __ldg(e.bias + col + i);
  }
  if (e.z8.dev_codes) put_packed_quad(e.z8, row, col, have, v);
  act_run(e.act, v);
  if (e.residual && have > 0) {
    const uint16_t* r = static_cast<const uint16_t*>(e.residual) + row * e.ld_res + col;
    if (have == 4 && e.vec_res) {
      const uint2 w = *reinterpret_cast<const uint2*>(r);
      const float2 f = unpack2(e.dtype, w.x), g = unpack2(e.dtype, w.y);
      v[0] += f.x; v[1] += f.y; v[2] += g.x; v[3] += g.y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < have) v[i] += unpack1(e.dtype, r[i]);
    }
  }
  const uint2 w = make_uint2(pack2(e.dtype, v[0], v[1]), pack2(e.dtype, v[2], v[3]));
  uint16_t* o = static_cast<uint16_t*>(e.out) + row * e.ld_out + col;
  if (have == 4 && e.vec_out) {
    *reinterpret_cast<uint2*>(o) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < have) o[i] = (uint16_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)));
  }
  if (e.y8.dev_codes) {
    const float2 f = unpack2(e.dtype, w.x), g = unpack2(e.dtype, w.y);
    const float u[4] = {f.x, f.y, g.x, g.y};
    put_packed_quad(e.y8, row, col, have, u);
  }
}

// Sums of a row's neighbouring columns: into a piece in the workspace (32-byte aligned), into the shared memory of a CTA of the cluster.
template <int N>
__device__ __forceinline__ void store_sums(float* o, const float (&v)[N]) {
#pragma unroll
  for (int c = 0; c < N; c += 8) {
    uint32_t u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[c + j]);
    st_global_32(o + c, u);
  }
}
template <int N>
__device__ __forceinline__ void to_meeting(uint32_t o, const float (&v)[N]) {
#pragma unroll
  for (int c = 0; c < N; c += 4)
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                 ::"r"(o + 4 * c), "f"(v[c]), "f"(v[c + 1]), "f"(v[c + 2]), "f"(v[c + 3]) : "memory");
}

// a / b for a < 2^31, b >= 1: in floating point and put right, where 32-bit integer division is a long chain.
__device__ __forceinline__ uint32_t quick_div(uint32_t a, uint32_t b) {
  if (a >= (1u << 22)) return a / b;
  uint32_t q = (uint32_t)(__fdividef((float)a, (float)b));
  if (q * b > a) --q;
  if ((q + 1) * b <= a) ++q;
  return q;
}

// ---- the walk over (tile, k block) pairs that every role of a CTA makes
// Three ways to deal them out.
// kWhole: cluster g (of CG CTAs) takes tiles g, g + G, ...
// kMeet (few tiles): a cluster of up to 8 CTAs sums one tile, CTA r the k blocks [r share, (r + 1) share); the sums meet in the
//   CTAs' shared memory: each sends every other its slice of the rows, adds up what it got, in their order, and finishes it.
// kShares (few tiles, long sums): all (tile, k block) pairs stand in one row, tile after tile, and cluster g takes pairs
//   [g share, (g + 1) share).  A tile that a share begins or ends inside of is summed by several clusters: each writes what
//   it has to a piece of the workspace (at most two per cluster: piece 2 g where its share begins, 2 g + 1 for a tile that its
//   share ends inside of), and linear_join_kernel adds a tile's pieces in the order of the clusters.
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
    const uint32_t band = quick_div(t, kBand * tiles_n), first = band * kBand, high = min(kBand, tiles_m - first);
    const uint32_t in = t - band * kBand * tiles_n;
    n_tile = (int)quick_div(in, high);
    m_tile = (int)(first + in - n_tile * high);
  }
  __device__ __forceinline__ void locate(const LinProblem& p) {
    uint32_t t = pos;
    kb = 0;
    kb_end = p.kb_total;
    if (p.deal == kShares) {
      t = quick_div(pos, p.kb_total);
      kb = (int)(pos - t * p.kb_total);
      kb_end = min(p.kb_total, kb + (int)(end - pos));
    }
    place(p.tiles_m, p.tiles_n, t, m_tile, n_tile);
  }
  // g of `clusters` clusters; with kMeet the CTA `part` of the cluster that has tile g.
  __device__ __forceinline__ LinWalk(const LinProblem& p, int g, int clusters, int part) : cluster(g) {
    const uint32_t tiles = p.tiles_m * p.tiles_n;
    pos = p.deal == kShares ? (uint32_t)g * p.share : (uint32_t)g;
    end = p.deal == kShares ? min(tiles * p.kb_total, pos + p.share) : tiles;
    stride = p.deal == kMeet ? tiles : (uint32_t)clusters;
    begin = pos;
    if (pos < end) locate(p);
    if (p.deal == kMeet) {
      kb = part * p.share;
      kb_end = min(p.kb_total, kb + p.share);
    }
  }
  __device__ __forceinline__ bool done() const { return pos >= end; }
  // The piece the current tile's sum goes to, or -1: the cluster has the whole tile.
  __device__ __forceinline__ int piece(const LinProblem& p) const {
    return p.deal != kShares || kb_end - kb == p.kb_total ? -1 : (pos == begin ? 2 * cluster : 2 * cluster + 1);
  }
  // To the next tile; only from the state locate() left (next() below moves kb).
  __device__ __forceinline__ void next_tile(const LinProblem& p) {
    pos += p.deal == kShares ? (uint32_t)(kb_end - kb) : stride;
    if (pos < end) locate(p);
  }
  // To the next k block, of this tile or the next.
  __device__ __forceinline__ void next(const LinProblem& p) {
    if (p.deal == kShares) ++pos;
    if (++kb == kb_end) {
      if (p.deal != kShares) pos += stride;
      if (pos < end) locate(p);
    }
  }
};

// Rows that each of the CTAs that sum a tile together finishes: an equal part of those that exist.
__device__ __forceinline__ int meet_slice(const LinProblem& p, const LinWalk& w, int meet) {
  return (int)quick_div(min(kLinBM, p.M - w.m_tile * kLinBM) + meet - 1, meet);
}

// The tensor core's accumulator is cut toward zero at every step (K = 16) that it adds, so that its error grows with their number:
// in relative 2-norm 3.4e-7 at 256 terms, 1.25e-6 at 1024, 2.4e-6 at 2048, 1.4e-5 at 16384 and 5.7e-5 at 65536 (fp32 products on
// the CUDA cores, of normally distributed values: 2.8e-7, 5.6e-7, 8e-7, 2.3e-6, 4.6e-6).  So an accumulator takes a few k blocks of
// 64 terms, and the epilogue warps add these sums up in registers, rounding to nearest, while the next one grows: the error stays
// about that of one accumulator, however long the sum.
// Weight gradients and tiles of single SMs: 1024 terms.  8192 rows, 16384 x 4096: 695 us so, as without (512 rows: 737 us; 2048: 715);
// 7 x 16384 x 4096 takes 27.5 us (27.4 without).
// Pairs, results in 16 bits: while an epilogue runs (about 15 us with GELU and an 8-bit copy beside the MMAs) they can fill two
// accumulators and then wait, so a tile's first two take more, 1280 terms, and the later ones, which are drained at once, 512:
// error 1.4e-6 at 4096 terms, 1.0e-6 at 16384, 0.8e-6 at 65536.  8192 x 4096 x 16384 took 917 us (893 in one accumulator, 900 with
// 1344 first and an error of 1.45e-6, 1010 with 1024), its gradient of the input, with a residual, 831 us (828), 4096 x 4096 x 4096
// 107.7 (105.5).  512 terms throughout: 36 % more than one accumulator, error 0.65e-6.
// Sums of up to 2048 terms stay whole: the epilogue reads them from tensor memory piece by piece, which is what bounds them
// (4096 x 2048 x 4096 with GELU and both 8-bit copies in two accumulators: 12 % more; error 2.4e-6 and 1.3e-6).
constexpr int kChunk = 16, kLaterChunk = 8;
inline int pair_chunk(int kb_total) { return kb_total <= 32 ? 32 : 20; }

// WF32: the result is fp32 (a weight gradient).
template <int CG, int BN, int OA, int OB, bool WF32>
struct LinCfg {
  static constexpr int kBNc = BN / CG;                                    // rows of B per CTA
  static constexpr uint32_t kABytes = kLinBM * 128, kBBytes = kBNc * 128;
  static constexpr uint32_t kStage = kABytes + ((kBBytes + 1023) / 1024 * 1024);
  // Two warps per quarter of tensor memory: GELU and the 8-bit form take as long as the product of a 4096-wide layer with one;
  // with three the sums of a pair's tile no longer fit their registers.
  static constexpr int kEpiWarps = 8;
  static constexpr int kMine = BN / (kEpiWarps / 4);                      // columns per epilogue warp
  static constexpr int kThreads = (4 + kEpiWarps) * 32;
  // With 128 sums of a long chain in registers the epilogue of a layer needs more of them than the 168 that every thread starts with
  // (75 of them spilled, 8192 x 4096 x 16384 took 990 us instead of 840): the first four warps hand some over.
  static constexpr bool kMoveRegs = CG == 2 && !WF32;
  static constexpr int kRegsFront = 56, kRegsEpi = 224, kRegsAll = 128 * kRegsFront + 32 * kEpiWarps * kRegsEpi;   // the launch has to bring these
  static constexpr uint32_t kScratchWarp = WF32 ? 32 * 9 * 4 : 32 * 34 * 2 + kMine * 4, kScratch = kEpiWarps * kScratchWarp;
  static constexpr uint32_t kRoom = 225u * 1024 - kScratch;
  static constexpr int kStages = (int)(kRoom / kStage) > 12 ? 12 : (int)(kRoom / kStage);
  static constexpr int kTmemCols = 2 * BN;
  static constexpr int kBars = 2 * kStages + 2 + 2 + 1;
  static constexpr uint32_t kScratchOff = kStages * kStage;
  static constexpr uint32_t kBarOff = (kScratchOff + kScratch + 7) / 8 * 8;
  static constexpr uint32_t kSmem = kBarOff + kBars * 8 + 32 + 1024;
  // A tile summed by a cluster meets in shared memory, in the place of the operand stages: rows of BN + 4 words (a lane's
  // 16-byte accesses, a row each, then cover all banks).
  static constexpr int kMeetPitch = BN + 4;
  static_assert(kSmem <= 227 * 1024 && kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0, "one CTA per SM");
  static_assert(OB == kOpK || kBNc % 64 == 0, "MN-major operands come in blocks of 64");
  static_assert(!kMoveRegs || kRegsAll <= kThreads * 168, "the launch brings 168 per thread");
  static_assert(CG == 2 || BN == 128, "a warp finishes a row of a tile");
  static_assert(CG == 2 || (kLinBM + 7) * kMeetPitch * 4 <= kStages * kStage, "a tile, in up to 8 slices, fits in the operand stages");
};

template <int CG, int BN, int OA, int OB, bool WF32>
__global__ void __launch_bounds__(LinCfg<CG, BN, OA, OB, WF32>::kThreads, 1)
linear_kernel(const __grid_constant__ LinProblem p) {
  using S = LinCfg<CG, BN, OA, OB, WF32>;
  extern __shared__ uint8_t lin_smem[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(lin_smem) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + S::kBarOff);   // [stages] TMA bytes landed, in both CTAs (first CTA's barrier)
  uint64_t* empty = full + S::kStages;                               // [stages] the MMAs that read the stage are done
  uint64_t* d_full = empty + S::kStages;                             // [2] accumulator complete
  uint64_t* d_empty = d_full + 2;                                    // [2] accumulator drained by both CTAs (first CTA's)
  uint64_t* fin = d_empty + 2;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(fin + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(fin + 1) + 2;
  volatile uint32_t* ends = tmem_slot + 2;                           // [2] of each CTA of a pair: k blocks its loader issued * 2 + gave up

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
  const int meet = CG == 1 && p.deal == kMeet ? p.meet : 1, part_of = meet > 1 ? (int)cluster_rank() : 0;
  const int cluster = (int)blockIdx.x / (CG * meet), clusters = (int)gridDim.x / (CG * meet);

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < 2; ++s) { mbar_init(d_full + s, 1); mbar_init(d_empty + s, S::kEpiWarps * CG); }
    mbar_init(fin, 1);
    wait_ctl_init(abort_flag, p.test_limit);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.ta) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.tb) : "memory");
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
  // k blocks of a tile's n-th accumulator
  auto chunk = [&](int n) { return CG == 1 || WF32 ? kChunk : n < 2 ? p.first_chunk : kLaterChunk; };
  // Every role first finds its place in the work, then waits for the kernel in front.
  bool met = false;                    // kMeet: this warp has passed the cluster's first barrier
  const uint32_t base_s = smem_u32(base), full_s = smem_u32(full), empty_s = smem_u32(empty);
  const int test_role = cluster == 0 ? p.test_role : (int)kNoRole;
  uint32_t issued = 0;                 // k blocks whose copies this CTA's loader asked for

  if (warp < 4) {
    if constexpr (S::kMoveRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kRegsFront));
    if (warp == 0) {
    // ---- loader
    LinWalk w(p, cluster, clusters, part_of);
    train_pdl_wait();
    const uint32_t full0 = CG == 2 ? map_to(full, 0) : full_s;          // the first CTA's barriers count both CTAs' bytes
    const uint32_t tx = CG * (p.box_a * 128 + S::kBBytes);
    uint32_t s = 0, turn = 0;
    const uint32_t stop = test_role == (rank == 0 ? (int)kLoader0 : (int)kLoader1) ? p.test_after : 0xffffffffu;
    for (; !w.done(); w.next(p), ++issued) {
      if (issued == stop || !lin_wait_all(empty_s + 8 * s, empty + s, turn ^ 1, abort_flag)) break;
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
        } else {
#pragma unroll
          for (int i = 0; i < S::kBNc / 64; ++i) lin_tma<CG>(b + i * kLinBK * 128, &p.tb, n0 + 64 * i, k0, bar);
        }
      }
      __syncwarp();
      if (++s == S::kStages) { s = 0; turn ^= 1; }
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
      uint32_t s = 0, turn = 0, db = 0, dturn = 0, until = test_role == kMma ? p.test_after : 0xffffffffu;
      bool ok = true;
      LinWalk w(p, cluster, clusters, part_of);
      train_pdl_wait();
      for (; !w.done() && ok; w.next_tile(p)) {
        int nth = 0;
        uint32_t left = 0, d = 0, more = 0;         // k blocks until the accumulator changes; its first product starts the sum
        const uint32_t run = min((uint32_t)(w.kb_end - w.kb), until);
        const int stop = w.kb + (int)run;
        until -= run;
        for (int kb = w.kb; kb < stop; ++kb) {
          if (left == 0) {
            if (!lin_wait_all(d_empty_s + 8 * db, d_empty + db, dturn ^ 1, abort_flag)) { ok = false; break; }
            lin_fence_after();
            d = tmem + db * BN;
            left = min(chunk(nth++), w.kb_end - kb);
            more = 0;
          }
          if (!lin_wait_all(full_s + 8 * s, full + s, turn, abort_flag)) { ok = false; break; }
          lin_fence_after();
          const uint64_t ad = ad0 + (uint64_t)(s * (S::kStage >> 4)), bd = bd0 + (uint64_t)(s * (S::kStage >> 4));
          --left;
          if (elect_one()) {
#pragma unroll
            for (int ks = 0; ks < kLinBK / 16; ++ks)
              lin_mma<CG>(d, ad + ((ks * lin_kstep<OA != kOpK>()) >> 4), bd + ((ks * lin_kstep<OB != kOpK>()) >> 4), idesc, ks > 0 ? 1u : more);
            lin_commit<CG>(empty_s + 8 * s);
            if (left == 0) lin_commit<CG>(d_full_s + 8 * db);
          }
          __syncwarp();
          more = 1;
          if (++s == S::kStages) { s = 0; turn ^= 1; }
          if (left == 0) {
            db ^= 1;
            if (db == 0) dturn ^= 1;
          }
        }
        ok = ok && stop == w.kb_end;
      }
      if (elect_one()) lin_commit<CG>(smem_u32(fin));   // every MMA has completed before tensor memory is released
      __syncwarp();
      if (lane == 0) {
        const uint32_t limit = wait_limit_of(abort_flag);
        for (uint32_t i = 0; i < limit && !mbar_try(fin, 0); ++i) {}
      }
    }
    __syncwarp();
    }
  } else {
    if constexpr (S::kMoveRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kRegsEpi));
    // ---- epilogue: a warp reads its quarter of the accumulator's rows (warp % 4), and with eight warps half of its columns
    uint32_t seq = 0;                                                     // accumulators taken so far
    bool ok = true;
    const int q = warp & 3, c0 = ((warp - 4) >> 2) * S::kMine;
    float* scratch = reinterpret_cast<float*>(base + S::kScratchOff + (warp - 4) * S::kScratchWarp);
    LinWalk w(p, cluster, clusters, part_of);
    // What the epilogue of a layer reads besides the sum is asked for a tile ahead: the bias of this warp's columns in
    // registers, the residual into L2.
    float* bias = scratch + 32 * 34 / 2;
    float bias_next[S::kMine / 32] = {};
    auto fetch_ahead = [&](const LinWalk& t) {
      if (WF32 || meet > 1 || t.done() || t.piece(p) >= 0) return;
      const int m = (t.m_tile * CG + (int)rank) * kLinBM + 32 * q + lane, n = t.n_tile * BN + c0, have = min(S::kMine, p.N - n);
      if (p.ep.bias) {
#pragma unroll
        for (int i = 0; i < S::kMine / 32; ++i) bias_next[i] = 32 * i + lane < have ? __ldg(p.ep.bias + n + 32 * i + lane) : 0.f;
      }
      if (p.ep.residual && m < p.M && have > 0) {
        const char* r = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.ep.residual) + (int64_t)m * p.ep.ld_res + n);
#pragma unroll
        for (int b = 0; b < S::kMine * 2; b += 128)
          if (b < 2 * have) asm volatile("prefetch.global.L2 [%0];" ::"l"(r + b));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(r + 2 * have - 2));
      }
    };
    train_pdl_wait();
    fetch_ahead(w);
    for (; !w.done(); w.next_tile(p)) {
      if (!WF32 && (p.ep.residual || p.ep.bias)) {
#pragma unroll
        for (int i = 0; i < S::kMine / 32; ++i) bias[32 * i + lane] = bias_next[i];
        __syncwarp();
        LinWalk t = w;
        t.next_tile(p);
        fetch_ahead(t);
      }
      const int m = (w.m_tile * CG + (int)rank) * kLinBM + 32 * q + lane, n0 = w.n_tile * BN;
      const int piece = w.piece(p);
      float* part = piece >= 0 ? p.partial + (int64_t)piece * (CG * kLinBM * BN) : nullptr;
      // waits for the next accumulator; its columns c0.. for this warp's rows
      auto open = [&]() -> uint32_t {
        const uint32_t db = seq & 1;
        if (!lin_wait_warp(d_full + db, (seq >> 1) & 1, abort_flag, lane)) ok = false;
        lin_fence_after();
        return tmem + ((uint32_t)(32 * q) << 16) + db * BN + c0;
      };
      auto hand_back = [&]() {                        // the accumulator is in registers
        const uint32_t db = seq & 1;
        lin_fence_before();
        __syncwarp();
        if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(d_empty + db, 0)); else mbar_arrive(d_empty + db); }
        ++seq;
      };
      float* to_slice = nullptr;                      // the sums meet: this row's place in shared memory, and whose it is
      int to = 0;
      if (CG == 1 && meet > 1) {
        const int r = 32 * q + lane, slice = meet_slice(p, w, meet);
        to = min((int)quick_div(r, slice), meet - 1);
        to_slice = reinterpret_cast<float*>(base) + (part_of * slice + r - to * slice) * S::kMeetPitch;
      }
      auto meet_first = [&]() {                       // every CTA's MMAs are done with the stages that the sums go to
        if (CG == 1 && meet > 1) {
          cluster_sync_all();
          met = true;
        }
      };
      if (!WF32 && w.kb_end - w.kb <= chunk(0) && !part) {          // one accumulator has the whole sum: piece by piece from tensor memory
        const uint32_t taddr = open();
        if (!ok) break;
        meet_first();
#pragma unroll 1
        for (int c = 0; c < S::kMine; c += 32) {
          float v[32];
          tmem_ld32(taddr + c, v);
          if (c + 32 >= S::kMine) hand_back();
          if (CG == 1 && meet > 1) {
            if (m < p.M) to_meeting(map_to(to_slice + c0 + c, to), v);
          } else if (n0 + c0 + c < p.N && m - lane < p.M) {
            finish_rows(p.ep, m - lane, n0 + c0 + c, m < p.M, v, bias + c, scratch);
          }
          __syncwarp();
        }
        continue;
      }
      float acc[S::kMine];
#pragma unroll
      for (int c = 0; c < S::kMine; ++c) acc[c] = 0.f;
#pragma unroll 1
      for (int left = w.kb_end - w.kb, n = 0; left > 0; left -= chunk(n++)) {
        const uint32_t taddr = open();
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < S::kMine; c += 16) {
          float v[16];
          tmem_ld16(taddr + c, v);
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[c + j] += v[j];
        }
        hand_back();
      }
      if (!ok) break;
      meet_first();
      if (CG == 1 && meet > 1) {
        if (m < p.M) to_meeting(map_to(to_slice + c0, to), acc);
      } else if (part) {
        if (m < p.M && n0 + c0 < p.N) store_sums(part + ((int)rank * kLinBM + 32 * q + lane) * BN + c0, acc);
      } else if constexpr (WF32) {
        if (p.ep.vec_out && n0 + c0 + S::kMine <= p.N) {
          float* o = static_cast<float*>(p.ep.out) + (int64_t)m * p.ep.ld_out + n0 + c0;
          if (m < p.M) {
#pragma unroll
            for (int c = 0; c < S::kMine; c += 8) {
              uint32_t u[8];
              if (p.ep.accumulate) {
                ld_row32(o + c, p.ep.vec_out, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[c + j] += __uint_as_float(u[j]);
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(acc[c + j]);
              st_row32(o + c, p.ep.vec_out, u);
            }
          }
        } else if (m - lane < p.M) {
#pragma unroll
          for (int c = 0; c < S::kMine; c += 8)
            if (n0 + c0 + c < p.N) finish_ragged_f32(p.ep, m - lane, n0 + c0 + c, acc + c, scratch);
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < S::kMine; c += 32) {
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = acc[j];
#pragma unroll
          for (int j = 32; j < S::kMine; ++j) acc[j - 32] = acc[j];      // the next piece's: one copy of the epilogue's code, registers by number
          if (n0 + c0 + c < p.N && m - lane < p.M) finish_rows(p.ep, m - lane, n0 + c0 + c, m < p.M, v, bias + c, scratch);
          __syncwarp();
        }
      }
      __syncwarp();
    }
  }
  __syncwarp();
  if (CG == 1 && meet > 1 && !met) cluster_sync_all();
  lin_fence_before();
  __syncthreads();
  // No CTA leaves while copies into its memory are in flight, or while another may still signal its barriers: of a pair, `fin` is the
  // last thing that the MMAs signal in both CTAs (it has come when the roles have met above, unless they gave up).
  if (tid == 0) {
    const uint32_t limit = wait_limit_of(abort_flag), gave_up = *abort_flag ? 1u : 0u;
    if (gave_up && p.status) atomicOr(p.status, kStatusTimeout);
    if constexpr (CG == 2) {
      for (uint32_t i = 0; i < limit && !mbar_try(fin, 0); ++i) {}
      for (uint32_t r = 0; r < 2; ++r)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to((const void*)(ends + rank), r)), "r"(2 * issued + gave_up) : "memory");
    } else if (gave_up) {
      lin_drain(full, S::kStages, issued, limit);
    }
  }
  __syncwarp();
  if (CG == 2 || meet > 1) cluster_sync_all();      // the sums have arrived
  if constexpr (CG == 2) {
    const uint32_t first = ends[0], second = ends[1];
    if ((first | second) & 1) {
      if (tid == 0 && rank == 0)
        lin_drain_pair(full, S::kStages, first >> 1, second >> 1, p.box_a * 128 + S::kBBytes, wait_limit_of(abort_flag));
      __syncwarp();
      cluster_sync_all();
    }
  }
  if (CG == 1 && meet > 1) {
    // ---- the CTAs' sums of one tile have met: a warp takes a row of this CTA's slice, a lane four of its columns
    train_pdl_wait();                               // (the warps that had no need to yet)
    const LinWalk w(p, cluster, clusters, part_of);
    const int slice = meet_slice(p, w, meet), rows = min(slice, min(kLinBM, p.M - w.m_tile * kLinBM) - part_of * slice);
    for (int r = warp; r < rows; r += S::kThreads / 32) {
      const int row = w.m_tile * kLinBM + part_of * slice + r;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      const float* mine = reinterpret_cast<const float*>(base) + r * S::kMeetPitch + 4 * lane;
#pragma unroll 4
      for (int k = 0; k < meet; ++k) {
        const float4 t = *reinterpret_cast<const float4*>(mine + k * slice * S::kMeetPitch);
        v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
      }
      finish_quad(p.ep, row, w.n_tile * BN + 4 * lane, v);
    }
  }
  if (warp == 2) {
    if constexpr (CG == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::kTmemCols) : "memory");
  }
}

}  // namespace
}  // namespace lqsgd
