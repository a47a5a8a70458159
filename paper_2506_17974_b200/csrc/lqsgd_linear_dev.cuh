// Device side of the linear layers: the matrix product D[m, n] = sum_k A[m, k] B[n, k] on the tensor cores (tcgen05,
// fp32 accumulators in tensor memory) for the three products of a layer, with their epilogues.
//
//   product        A (rows m)          B (rows n)             contracted over      lies along memory rows
//   forward        x    [rows]         w   [out]              in                   A: k    B: k
//   grad_input     dz   [rows]         w^T [in]               out                  A: k    B: n
//   grad_weight    dz^T [out]          x^T [in]               rows                 A: m    B: n
//   few rows       w or w^T            x or dz                in / out             the first two with A and B exchanged
//
// An operand whose rows hold k ("K-major") is staged as 64 k x R rows; one whose rows hold m or n ("MN-major") as blocks of
// 64 columns x 64 k: both arrive from TMA with the 128-byte swizzle that the tensor core reads, so nothing is transposed.
// x kept in 8 bits is the one operand TMA cannot bring: converter warps read its codes, decode them to 16 bits (exactly,
// see lqsgd_pack8) and write the same swizzled layout.
//
// A cluster of CG CTAs (1 or 2) works on a tile of 128 CG x BN: with CG = 2 each SM holds 128 rows of A and half of B's, and
// one tcgen05.mma.cta_group::2 drives both tensor cores, so that an SM fetches (128 + BN / 2) rows per k instead of
// 128 + BN.  Per CTA: warp 0 issues the TMA loads, warp 1 (of the cluster's first CTA) the MMAs, warps 4-7 drain the
// accumulator (two of them, so that the next tile's sum runs under the epilogue), warps 8.. decode x8.  Clusters walk
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
  CUtensorMap ta, tb;
  LinEpilogue ep;
  float* partial;                      // [splits][rows][ld_partial] when splits > 1
  int64_t ld_partial;
  lqsgd_packed8 x8;                    // operand B when it is packed
  int32_t x8_vec;                      // its rows are 16-byte aligned
  int32_t M, N, K;
  int32_t tiles_m, tiles_n, splits, kb_total, kb_per_split;
  int32_t dtype;                       // of the operands
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
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Bounded wait that also acquires what other CTAs of the cluster released.
__device__ __forceinline__ bool lin_wait(uint64_t* b, uint32_t parity, volatile int* abort_flag) {
  const uint32_t limit = wait_limit_of(abort_flag);
  for (uint32_t i = 0; i < limit; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(smem_u32(b)), "r"(parity), "r"(1000u) : "memory");
    if (ok) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool lin_wait_warp(uint64_t* b, uint32_t parity, volatile int* abort_flag, int lane) {
  int ok = 1;
  if (lane == 0) ok = lin_wait(b, parity, abort_flag) ? 1 : 0;
  ok = __shfl_sync(0xffffffffu, ok, 0);
  return ok != 0;
}

template <int CG>
__device__ __forceinline__ void lin_tma(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
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
__device__ __forceinline__ void lin_commit(uint64_t* bar) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
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

// Epilogue of 32 consecutive columns of one row held by one thread.
__device__ __forceinline__ void finish_row32(const LinEpilogue& e, int64_t row, int col, float (&v)[32]) {
  const int have = min(32, e.cols - col);
  if (e.dtype == LQSGD_F32) {
    float* o = static_cast<float*>(e.out) + row * e.ld_out + col;
    if (e.vec_out && have == 32) {
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
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < have) o[i] = e.accumulate ? o[i] + v[i] : v[i];
    }
    return;
  }
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
  if (e.z8.dev_codes) put_packed(e.z8, e.vec_z8, row, col, have, v);
  if (e.act == LQSGD_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_value(LQSGD_ACT_RELU, v[i]);
  } else if (e.act == LQSGD_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_value(LQSGD_ACT_GELU, v[i]);
  } else if (e.act == LQSGD_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_value(LQSGD_ACT_SILU, v[i]);
  }
  if (e.residual) {
    const uint16_t* r = static_cast<const uint16_t*>(e.residual) + row * e.ld_res + col;
    if (e.vec_res && have == 32) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[8];
        ld_global_32(r + 16 * i, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 f = unpack2(e.dtype, w[j]);
          v[16 * i + 2 * j] += f.x;
          v[16 * i + 2 * j + 1] += f.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < have) v[i] += unpack1(e.dtype, r[i]);
    }
  }
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = pack2(e.dtype, v[2 * i], v[2 * i + 1]);
  uint16_t* o = static_cast<uint16_t*>(e.out) + row * e.ld_out + col;
  if (e.vec_out && have == 32) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = w[8 * i + j];
      st_global_32(o + 16 * i, h);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < have) o[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
  }
  if (e.y8.dev_codes) {
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
  v = act_value(e.act, v);
  if (e.residual && on) v += unpack1(e.dtype, static_cast<const uint16_t*>(e.residual)[row * e.ld_res + col]);
  const uint16_t w = pack1(e.dtype, v);
  if (on) static_cast<uint16_t*>(e.out)[row * e.ld_out + col] = w;
  if (e.y8.dev_codes) put_packed_lane(e.y8, row, col, on, on ? unpack1(e.dtype, w) : 0.f);
}

// ---- decoding 8-bit codes into operand words: two codes (bytes `sel`, sel + 1 of w) -> two 16-bit numbers
// bf16: 0x4300 | m is 128 + m, so subtracting 128 gives m exactly, and m 2^e has 8 significant bits.
// fp16: 0x6400 | m is 1024 + m, likewise.
__device__ __forceinline__ uint32_t decode2_bf16(uint32_t w, int hi, uint32_t step2) {
  const uint32_t p = __byte_perm(w, 0u, hi ? 0x4342 : 0x4140);             // [c0, 0, c1, 0]
  const uint32_t s = __byte_perm(w, 0u, hi ? 0x3424 : 0x1404) & 0x80008000u;  // [0, c0, 0, c1]
  uint32_t t = (p & 0x007f007fu) | 0x43004300u;
  __nv_bfloat162 m = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&t), __nv_bfloat162(__ushort_as_bfloat16(0x4300), __ushort_as_bfloat16(0x4300)));
  m = __hmul2(m, *reinterpret_cast<const __nv_bfloat162*>(&step2));
  return *reinterpret_cast<uint32_t*>(&m) | s;
}
__device__ __forceinline__ uint32_t decode2_fp16(uint32_t w, int hi, uint32_t step2) {
  const uint32_t p = __byte_perm(w, 0u, hi ? 0x4342 : 0x4140);
  const uint32_t s = __byte_perm(w, 0u, hi ? 0x3424 : 0x1404) & 0x80008000u;
  uint32_t t = (p & 0x007f007fu) | 0x64006400u;
  __half2 m = __hsub2(*reinterpret_cast<__half2*>(&t), __half2(__ushort_as_half(0x6400), __ushort_as_half(0x6400)));
  m = __hmul2(m, *reinterpret_cast<const __half2*>(&step2));
  return *reinterpret_cast<uint32_t*>(&m) | s;
}
// Any step: through fp32, saturated to the type's largest finite number (NaN stays).
__device__ __forceinline__ uint32_t decode2_any(int dtype, uint32_t w, int hi, int eb) {
  const float top = dtype == LQSGD_BF16 ? 3.3895314e38f : 65504.f;
  float a = decode8(w >> (hi ? 16 : 0) & 255u, step_of(eb)), b = decode8(w >> (hi ? 24 : 8) & 255u, step_of(eb));
  if (fabsf(a) > top) a = copysignf(top, a);
  if (fabsf(b) > top) b = copysignf(top, b);
  return pack2(dtype, a, b);
}

// ---- the walk over (work item, k block) pairs that every role of a CTA makes
struct LinWalk {
  int item, stride, items;
  int kb, kb_end;
  int m_tile, n_tile, split;
  // Tiles are taken in bands of 8 rows of tiles, column by column: 74 clusters at work then share 8 row tiles and
  // about as many column tiles, which keeps their operands in L2.
  __device__ __forceinline__ void locate(const LinProblem& p) {
    const int tiles = p.tiles_m * p.tiles_n;
    split = item / tiles;
    const int t = item - split * tiles;
    constexpr int kBand = 8;
    const int band = t / (kBand * p.tiles_n), first = band * kBand, high = min(kBand, p.tiles_m - first);
    const int in = t - band * kBand * p.tiles_n;
    m_tile = first + in % high;
    n_tile = in / high;
    kb = split * p.kb_per_split;
    kb_end = min(p.kb_total, kb + p.kb_per_split);
  }
  __device__ __forceinline__ LinWalk(const LinProblem& p, int first, int step) : item(first), stride(step) {
    items = p.tiles_m * p.tiles_n * p.splits;
    if (item < items) locate(p);
  }
  __device__ __forceinline__ bool done() const { return item >= items; }
  __device__ __forceinline__ void next_item(const LinProblem& p) {
    item += stride;
    if (item < items) locate(p);
  }
  __device__ __forceinline__ void next(const LinProblem& p) {
    if (++kb == kb_end) next_item(p);
  }
};

template <int CG, int BN, int OA, int OB>
struct LinCfg {
  static constexpr int kBNc = BN / CG;                                    // rows of B per CTA
  static constexpr uint32_t kABytes = kLinBM * 128, kBBytes = kBNc * 128;
  static constexpr uint32_t kStage = kABytes + ((kBBytes + 1023) / 1024 * 1024);
  static constexpr int kStages = (int)((216u * 1024) / kStage) > 12 ? 12 : (int)((216u * 1024) / kStage);
  static constexpr uint32_t kTxBytes = CG * (kABytes + (OB == kOpPacked ? 0 : kBBytes));
  static constexpr int kConvWarps = OB == kOpPacked ? kBNc / 16 : 0;      // a thread decodes 32 codes of one row of x
  static constexpr int kThreads = 256 + kConvWarps * 32;
  static constexpr int kTmemCols = 2 * BN < 32 ? 32 : 2 * BN;
  static constexpr int kBars = 3 * kStages + 2 + 2 + 1;
  static constexpr uint32_t kBarOff = kStages * kStage;
  static constexpr uint32_t kSmem = kBarOff + kBars * 8 + 32 + 1024;
  static_assert(kSmem <= 227 * 1024 && kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0, "one CTA per SM");
  static_assert(OB == kOpK || kBNc % 64 == 0, "MN-major operands come in blocks of 64");
};

// SWAP: A's rows are the result's columns (few rows); otherwise A's rows are its rows.
template <int CG, int BN, int OA, int OB, bool SWAP>
__global__ void __launch_bounds__(LinCfg<CG, BN, OA, OB>::kThreads, 1)
linear_kernel(const __grid_constant__ LinProblem p) {
  using S = LinCfg<CG, BN, OA, OB>;
  extern __shared__ uint8_t lin_smem[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(lin_smem) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(base + S::kBarOff);   // [stages] TMA bytes landed, in both CTAs (first CTA's barrier)
  uint64_t* conv = full + S::kStages;                                // [stages] decoded rows of B written, in both CTAs (first CTA's)
  uint64_t* empty = conv + S::kStages;                               // [stages] the MMAs that read the stage are done
  uint64_t* d_full = empty + S::kStages;                             // [2] accumulator complete
  uint64_t* d_empty = d_full + 2;                                    // [2] accumulator drained by both CTAs (first CTA's)
  uint64_t* fin = d_empty + 2;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(fin + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(fin + 1) + 2;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
  const int first_item = (int)blockIdx.x / CG, item_step = (int)gridDim.x / CG;

  if (tid == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(conv + s, CG * (S::kConvWarps ? S::kConvWarps : 1));
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < 2; ++s) { mbar_init(d_full + s, 1); mbar_init(d_empty + s, 4 * CG); }
    mbar_init(fin, 1);
    wait_ctl_init(abort_flag, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == 0 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.ta) : "memory");
    if constexpr (OB != kOpPacked) asm volatile("prefetch.tensormap [%0];" ::"l"(&p.tb) : "memory");
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
  train_pdl_wait();
  train_pdl_trigger();

  if (warp == 0) {
    // ---- loader: one thread
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (LinWalk w(p, first_item, item_step); !w.done(); w.next(p), ++it) {
        const int s = it % S::kStages;
        if (!lin_wait(empty + s, ((it / S::kStages) & 1) ^ 1, abort_flag)) { ok = false; break; }
        uint8_t* a = base + s * S::kStage;
        uint8_t* b = a + S::kABytes;
        if (rank == 0) mbar_arrive_expect_tx(full + s, S::kTxBytes);
        const uint32_t bar = CG == 2 ? map_to(full + s, 0) : smem_u32(full + s);
        const int k0 = w.kb * kLinBK, m0 = (w.m_tile * CG + (int)rank) * kLinBM;
        if constexpr (OA == kOpK) {
          lin_tma<CG>(a, &p.ta, k0, m0, bar);
        } else {
#pragma unroll
          for (int i = 0; i < kLinBM / 64; ++i) lin_tma<CG>(a + i * kLinBK * 128, &p.ta, m0 + 64 * i, k0, bar);
        }
        const int n0 = w.n_tile * BN + (int)rank * S::kBNc;
        if constexpr (OB == kOpK) {
          lin_tma<CG>(b, &p.tb, k0, n0, bar);
        } else if constexpr (OB == kOpMN) {
#pragma unroll
          for (int i = 0; i < S::kBNc / 64; ++i) lin_tma<CG>(b + i * kLinBK * 128, &p.tb, n0 + 64 * i, k0, bar);
        }
      }
      if (!ok && rank == 0) {                       // copies in flight land before the CTA's memory goes away
        const uint32_t limit = wait_limit_of(abort_flag);
        for (uint32_t j = it > (uint32_t)S::kStages ? it - S::kStages : 0; j < it; ++j)
          for (uint32_t i = 0; i < limit && !mbar_try(full + j % S::kStages, (j / S::kStages) & 1); ++i) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- MMA issue: one thread of the cluster's first CTA
    if (rank == 0 && lane == 0) {
      const uint32_t fmt = p.dtype == LQSGD_BF16 ? 1u : 0u;
      // fp32 accumulator, operand type, which operands are MN-major, N / 8, M / 16
      const uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((OA == kOpK ? 0u : 1u) << 15) | ((OB == kOpK ? 0u : 1u) << 16) |
                             ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((kLinBM * CG) >> 4) << 24);
      uint32_t it = 0, seq = 0;
      bool ok = true;
      for (LinWalk w(p, first_item, item_step); !w.done() && ok; w.next_item(p), ++seq) {
        const uint32_t db = seq & 1;
        if (!lin_wait(d_empty + db, ((seq >> 1) & 1) ^ 1, abort_flag)) { ok = false; break; }
        lin_fence_after();
        const uint32_t d = tmem + db * BN;
        for (int kb = w.kb; kb < w.kb_end; ++kb, ++it) {
          const int s = it % S::kStages;
          if (!lin_wait(full + s, (it / S::kStages) & 1, abort_flag)) { ok = false; break; }
          if constexpr (OB == kOpPacked) {
            if (!lin_wait(conv + s, (it / S::kStages) & 1, abort_flag)) { ok = false; break; }
          }
          lin_fence_after();
          const uint64_t ad = lin_desc<OA != kOpK>(smem_u32(base + s * S::kStage));
          const uint64_t bd = lin_desc<OB != kOpK>(smem_u32(base + s * S::kStage + S::kABytes));
#pragma unroll
          for (int ks = 0; ks < kLinBK / 16; ++ks)
            lin_mma<CG>(d, ad + ((ks * lin_kstep<OA != kOpK>()) >> 4), bd + ((ks * lin_kstep<OB != kOpK>()) >> 4), idesc,
                        (kb > w.kb || ks > 0) ? 1u : 0u);
          lin_commit<CG>(empty + s);
        }
        if (ok) lin_commit<CG>(d_full + db);
      }
      lin_commit<CG>(fin);                          // every MMA has completed before tensor memory is released
      const uint32_t limit = wait_limit_of(abort_flag);
      for (uint32_t i = 0; i < limit && !mbar_try(fin, 0); ++i) {}
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 8) {
    // ---- epilogue
    uint32_t seq = 0;
    const int q = warp & 3;
    for (LinWalk w(p, first_item, item_step); !w.done(); w.next_item(p), ++seq) {
      const uint32_t db = seq & 1;
      if (!lin_wait_warp(d_full + db, (seq >> 1) & 1, abort_flag, lane)) break;
      lin_fence_after();
      const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + db * BN;
      const int m = (w.m_tile * CG + (int)rank) * kLinBM + 32 * q + lane;
      const int n0 = w.n_tile * BN;
      float* part = p.splits > 1 ? p.partial + (int64_t)w.split * p.ep.rows * p.ld_partial : nullptr;
      if constexpr (!SWAP) {
        constexpr int kStep = 32;
#pragma unroll 1
        for (int c = 0; c < BN; c += kStep) {
          float v[32];
          tmem_ld32(taddr + c, v);
          if (c + kStep >= BN) {                    // the accumulator is in registers: hand it back
            lin_fence_before();
            __syncwarp();
            if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(d_empty + db, 0)); else mbar_arrive(d_empty + db); }
          }
          if (m < p.M && n0 + c < p.N) {
            if (part) {
              float* o = part + (int64_t)m * p.ld_partial + n0 + c;          // rows of 32-byte aligned runs
              const int have = min(32, p.N - n0 - c);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (8 * i < have) {
                  uint32_t u[8];
#pragma unroll
                  for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[8 * i + j]);
                  st_global_32(o + 8 * i, u);       // the row's pad takes what lies past N
                }
            } else {
              finish_row32(p.ep, m, n0 + c, v);
            }
          }
        }
      } else {
        const bool on = m < p.M;
        const float bias = (!part && p.ep.bias && on) ? __ldg(p.ep.bias + m) : 0.f;
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
          float v[16];
          tmem_ld16(taddr + c, v);
          if (c + 16 >= BN) {
            lin_fence_before();
            __syncwarp();
            if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(d_empty + db, 0)); else mbar_arrive(d_empty + db); }
          }
          if (m - lane >= p.M) continue;            // none of the warp's columns exists
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int row = n0 + c + j;
            if (row < p.N) {
              if (part) { if (on) part[(int64_t)row * p.ld_partial + m] = v[j]; }
              else finish_lane(p.ep, row, m, on, v[j], bias);
            }
          }
        }
      }
    }
  } else if (OB == kOpPacked && warp >= 8) {
    // ---- converters: rows of x8 (k) x the CTA's 32-column groups (n) -> the MN-major operand.  A warp takes 32 rows of one
    // group: its lanes' 16-byte chunks then fall on different banks (the swizzle runs over rows), and a lane's 32 codes are
    // one sector.  Loads run two stages ahead of the decoding.
    const int ct = tid - 256;
    const int krow = ct & 63, group = ct >> 6;
    struct Frag { uint32_t w[8]; int eb; };
    auto fetch = [&](const LinWalk& w, Frag& f) {
      const int k = w.kb * kLinBK + krow;
      const int col = w.n_tile * BN + (int)rank * S::kBNc + group * kGroup;
      const int have = k < p.K ? min(kGroup, p.N - col) : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) f.w[i] = 0u;
      f.eb = kExpBias;
      if (have <= 0) return;
      const uint8_t* c = p.x8.dev_codes + (int64_t)k * p.x8.ld_codes + col;
      f.eb = p.x8.dev_exps[(int64_t)k * p.x8.ld_exps + col / kGroup];
      if (have == kGroup && p.x8_vec) {
        const uint4 lo = *reinterpret_cast<const uint4*>(c), hi = *(reinterpret_cast<const uint4*>(c) + 1);
        f.w[0] = lo.x; f.w[1] = lo.y; f.w[2] = lo.z; f.w[3] = lo.w;
        f.w[4] = hi.x; f.w[5] = hi.y; f.w[6] = hi.z; f.w[7] = hi.w;
      } else if (have == kGroup) {
        // any alignment: the 4-byte words that hold the 32 codes, shifted into place (each word read holds one of them)
        const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(c) & 3);
        const uint32_t* q = reinterpret_cast<const uint32_t*>(c - off);
        uint32_t t[9];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = q[i];
        t[8] = off ? q[8] : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) f.w[i] = __funnelshift_r(t[i], t[i + 1], 8 * off);
      } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
          if (i < have) f.w[i >> 2] |= (uint32_t)c[i] << (8 * (i & 3));
      }
    };
    LinWalk ahead(p, first_item, item_step);
    Frag f0, f1, f2;
    bool v0 = !ahead.done(), v1 = false, v2 = false;
    if (v0) { fetch(ahead, f0); ahead.next(p); }
    v1 = !ahead.done();
    if (v1) { fetch(ahead, f1); ahead.next(p); }
    for (uint32_t it = 0; v0; ++it) {
      v2 = !ahead.done();
      if (v2) { fetch(ahead, f2); ahead.next(p); }
      const int s = it % S::kStages;
      if (!lin_wait_warp(empty + s, ((it / S::kStages) & 1) ^ 1, abort_flag, lane)) break;
      uint8_t* b = base + s * S::kStage + S::kABytes + (group >> 1) * (kLinBK * 128) + krow * 128;
      const bool bf = p.dtype == LQSGD_BF16;
      const int e = f0.eb - kExpBias;
      const bool plain = bf ? f0.eb <= 246 : (e >= -14 && e <= 8);          // the step and every product are normal numbers in range
      const uint32_t one = bf ? (uint32_t)(e + 127) << 7 : (uint32_t)((e + 15) & 31) << 10;
      const uint32_t step2 = one | (one << 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 o;
        uint32_t* ow = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const uint32_t cw = f0.w[2 * i + (h >> 1)];
          if (!plain) ow[h] = decode2_any(p.dtype, cw, h & 1, f0.eb);
          else ow[h] = bf ? decode2_bf16(cw, h & 1, step2) : decode2_fp16(cw, h & 1, step2);
        }
        *reinterpret_cast<uint4*>(b + ((((group & 1) * 4 + i) ^ (krow & 7)) << 4)) = o;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) { if constexpr (CG == 2) arrive_at(map_to(conv + s, 0)); else mbar_arrive(conv + s); }
      f0 = f1; f1 = f2;
      v0 = v1; v1 = v2;
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
