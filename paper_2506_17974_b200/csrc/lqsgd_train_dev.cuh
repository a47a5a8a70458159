// Device helpers of the training operators: the 8-bit form of activations, the activations and their slopes,
// and loads / stores of short runs of elements at any alignment.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdint.h>

#include "lqsgd_train.h"

namespace lqsgd {
namespace {

constexpr int kGroup = LQSGD_PACK8_GROUP;
constexpr int kExpBias = 126;            // stored exponent byte = e + 126
constexpr int kExpNonFinite = 255;       // group with an infinity or a NaN

__device__ __forceinline__ void train_pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void train_pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- element types
template <int DT> struct Elem;
template <> struct Elem<LQSGD_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float up(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T down(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<LQSGD_F16> {
  using T = __half;
  static __device__ __forceinline__ float up(T v) { return __half2float(v); }
  static __device__ __forceinline__ T down(float v) { return __float2half_rn(v); }
};
template <> struct Elem<LQSGD_F32> {
  using T = float;
  static __device__ __forceinline__ float up(T v) { return v; }
  static __device__ __forceinline__ T down(float v) { return v; }
};

// N consecutive elements as floats, and back.  VEC: the address is aligned to min(16, N * size) bytes and all N exist;
// otherwise element by element, those from `have` on read as 0 / are not written.
template <int DT, int N>
__device__ __forceinline__ void load_run(const typename Elem<DT>::T* p, bool vec, int have, float (&v)[N]) {
  using E = Elem<DT>;
  constexpr int kBytes = N * (int)sizeof(typename E::T);
  if (vec) {
    if constexpr (kBytes % 16 == 0) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 w = *(reinterpret_cast<const uint4*>(p) + i);
        constexpr int kPer = 16 / (int)sizeof(typename E::T);
        const typename E::T* t = reinterpret_cast<const typename E::T*>(&w);
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[i * kPer + j] = E::up(t[j]);
      }
    } else {
      static_assert(kBytes == 8, "a run is 8 bytes or a multiple of 16");
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      const typename E::T* t = reinterpret_cast<const typename E::T*>(&w);
#pragma unroll
      for (int j = 0; j < N; ++j) v[j] = E::up(t[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < have ? E::up(p[j]) : 0.f;
  }
}
// Two neighbouring elements of a 16-bit type in one word.
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  if constexpr (DT == LQSGD_BF16) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
  } else {
    const __half2 t = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
  }
}
template <int DT>
__device__ __forceinline__ float2 open_pair(uint32_t w) {
  if constexpr (DT == LQSGD_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int DT, int N>
__device__ __forceinline__ void store_run(typename Elem<DT>::T* p, bool vec, int have, const float (&v)[N]) {
  if constexpr (DT != LQSGD_F32 && N % 8 == 0) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < N / 8; ++i)
        reinterpret_cast<uint4*>(p)[i] = make_uint4(pack_pair<DT>(v[8 * i], v[8 * i + 1]), pack_pair<DT>(v[8 * i + 2], v[8 * i + 3]),
                                                    pack_pair<DT>(v[8 * i + 4], v[8 * i + 5]), pack_pair<DT>(v[8 * i + 6], v[8 * i + 7]));
      return;
    }
  }
  using E = Elem<DT>;
  constexpr int kBytes = N * (int)sizeof(typename E::T);
  if (vec) {
    if constexpr (kBytes % 16 == 0) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        uint4 w;
        constexpr int kPer = 16 / (int)sizeof(typename E::T);
        typename E::T* t = reinterpret_cast<typename E::T*>(&w);
#pragma unroll
        for (int j = 0; j < kPer; ++j) t[j] = E::down(v[i * kPer + j]);
        *(reinterpret_cast<uint4*>(p) + i) = w;
      }
    } else {
      uint2 w;
      typename E::T* t = reinterpret_cast<typename E::T*>(&w);
#pragma unroll
      for (int j = 0; j < N; ++j) t[j] = E::down(v[j]);
      *reinterpret_cast<uint2*>(p) = w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < have) p[j] = E::down(v[j]);
  }
}
// ---- arithmetic on two values at a time (one instruction for both; each rounded by itself)
__device__ __forceinline__ void fma2(float& a0, float& a1, float b0, float b1, float c0, float c1, float d0, float d1) {
  asm("{\n .reg .b64 b, c, d;\n mov.b64 b, {%2, %3};\n mov.b64 c, {%4, %5};\n mov.b64 d, {%6, %7};\n fma.rn.f32x2 d, b, c, d;\n mov.b64 {%0, %1}, d;\n}"
      : "=f"(a0), "=f"(a1) : "f"(b0), "f"(b1), "f"(c0), "f"(c1), "f"(d0), "f"(d1));
}
__device__ __forceinline__ void mul2(float& a0, float& a1, float b0, float b1, float c0, float c1) {
  asm("{\n .reg .b64 b, c;\n mov.b64 b, {%2, %3};\n mov.b64 c, {%4, %5};\n mul.rn.f32x2 b, b, c;\n mov.b64 {%0, %1}, b;\n}"
      : "=f"(a0), "=f"(a1) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1, float c0, float c1) {
  asm("{\n .reg .b64 b, c;\n mov.b64 b, {%2, %3};\n mov.b64 c, {%4, %5};\n add.rn.f32x2 b, b, c;\n mov.b64 {%0, %1}, b;\n}"
      : "=f"(a0), "=f"(a1) : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

// ---- largest magnitudes; an infinity or a NaN comes out as one
__device__ __forceinline__ float larger(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
template <int N>
__device__ __forceinline__ float largest(float top, const float (&v)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += 2) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(top) : "f"(top), "f"(v[j]), "f"(v[j + 1]));
  return top;
}

// Rounds to the element type and back: the value a later reader of the stored output sees.
template <int DT> __device__ __forceinline__ float as_stored(float v) { return Elem<DT>::up(Elem<DT>::down(v)); }

// ---- the 8-bit form
// Exponent byte of a group whose largest magnitude is `top` (not negative; an infinity or NaN gives 255).
// top = f 2^k with 1 <= f < 2: e = k - 6 puts top / 2^e into [64, 128), one more where that rounds to 128; never below -126
// (then top / 2^e < 64, whatever top is, subnormal numbers included).
__device__ __forceinline__ int exp_byte(float top) {
  const uint32_t b = __float_as_uint(top);
  if (b >= 0x7f800000u) return kExpNonFinite;
  const int k = (int)(b >> 23) - 127;                                  // -127 for subnormal numbers and 0
  const int e = max(k - 6, -126);
  // top / 2^e >= 127.5 exactly when the significand is >= 127.5 / 64 = 1.9921875 (and e was not raised to -126)
  const bool up = (b & 0x007fffffu) >= 0x007f0000u && k - 6 >= -126;
  return e + (up ? 1 : 0) + kExpBias;
}
// 2^-e of an exponent byte as a float (e <= 122, so it is a normal number); 255 gives 0: the codes of such a group are 0.
__device__ __forceinline__ float inv_step(int eb) {
  return eb == kExpNonFinite ? 0.f : __uint_as_float((uint32_t)(127 + kExpBias - eb) << 23);
}
// 2^e as a float; NaN for 255.
__device__ __forceinline__ float step_of(int eb) {
  return eb == kExpNonFinite ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(eb + 127 - kExpBias) << 23);
}
// Low byte = rint(|x| * inv), halves to even (adding 1.5 * 2^23 leaves an integer in the significand; |x| * inv is
// exact).  NaN and infinities only meet inv = 0; what they leave in the low byte is masked by the decoder's NaN step.
__device__ __forceinline__ uint32_t mag_bits(float x, float inv) { return __float_as_uint(fmaf(fabsf(x), inv, 12582912.f)); }
// Four codes in one word: magnitudes below, sign bits of the four values on top.
__device__ __forceinline__ uint32_t code_word(float a, float b, float c, float d, float inv) {
  const uint32_t m = __byte_perm(__byte_perm(mag_bits(a, inv), mag_bits(b, inv), 0x0040), __byte_perm(mag_bits(c, inv), mag_bits(d, inv), 0x0040), 0x5410);
  const uint32_t s = __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0073), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0073), 0x5410);
  return (m & 0x7f7f7f7fu) | (s & 0x80808080u);
}
__device__ __forceinline__ float decode8(uint32_t code, float step) {
  const float m = (float)(code & 127u) * step;
  const float sat = m > 3.402823466e38f ? 3.402823466e38f : m;          // a NaN stays
  return __uint_as_float(__float_as_uint(sat) | ((code & 128u) << 24));
}

// Four codes of a word at once, without conversions: 0x4b000000 | m is 2^23 + m, and (2^23 + m) 2^e - 2^23 2^e is m 2^e exactly.
// For exponent bytes up to 230 (2^23 2^e is in range); the others take decode8().
constexpr int kQuickByte = 230;
__device__ __forceinline__ void decode4(uint32_t w, float step, float off, float* v) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float m = fmaf(__uint_as_float(((w >> (8 * j)) & 127u) | 0x4b000000u), step, off);
    v[j] = __uint_as_float(__float_as_uint(m) | ((w << (24 - 8 * j)) & 0x80000000u));
  }
}
__device__ __forceinline__ void decode_run(uint2 w, int eb, float (&v)[8]) {
  const float step = step_of(eb);
  if (eb <= kQuickByte) {
    decode4(w.x, step, step * -8388608.f, v);
    decode4(w.y, step, step * -8388608.f, v + 4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = decode8((j < 4 ? w.x : w.y) >> (8 * (j & 3)) & 255u, step);
  }
}

// ---- activations, all in fp32, without branches: two special-function instructions each
__device__ __forceinline__ float exp2_approx(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp_approx(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// The normal distribution function, and e^(-z^2/2) by the way.  With x = |z| / sqrt 2, erfc(x) e^(x^2) / 2 is a polynomial in
// t = 1 / (1 + 0.431 x) to 9.2e-8 of its value for x <= 10 (fitted here by reweighted least squares on the relative
// error, t^1 .. t^8); beyond, e^(-x^2) is 0.  In fp32: |error| < 2.0e-7, relative error of the small tail < 1.6e-6 for |z| < 5.
__device__ __forceinline__ float normal_cdf(float z, float& gauss) {
  const float t = rcp_approx(fmaf(0.30476302f, fabsf(z), 1.f));
  float r = fmaf(0.036738604f, t, -0.15354006f);
  r = fmaf(r, t, 0.18724863f);
  r = fmaf(r, t, -0.039188605f);
  r = fmaf(r, t, 0.12161422f);
  r = fmaf(r, t, 0.10318742f);
  r = fmaf(r, t, 0.12239605f);
  r = fmaf(r, t, 0.12154379f);
  gauss = exp2_approx(z * z * -0.72134752f);                            // 0.5 log2 e
  const float q = gauss * (r * t);
  return z < 0.f ? q : 1.f - q;                                         // a NaN stays
}
__device__ __forceinline__ float logistic(float z) { return rcp_approx(1.f + exp2_approx(z * -1.44269504f)); }

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == LQSGD_ACT_RELU) return z < 0.f ? 0.f : z;        // keeps NaN
  if constexpr (ACT == LQSGD_ACT_GELU) { float g; return z * normal_cdf(z, g); }
  if constexpr (ACT == LQSGD_ACT_SILU) return z * logistic(z);
  return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == LQSGD_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);    // keeps NaN
  if constexpr (ACT == LQSGD_ACT_GELU) { float g; const float c = normal_cdf(z, g); return fmaf(z * 0.39894228f, g, c); }
  if constexpr (ACT == LQSGD_ACT_SILU) { const float s = logistic(z); return s * fmaf(z, 1.f - s, 1.f); }
  return 1.f;
}
// Calls f with the activation as a compile-time constant: one branch outside a loop instead of one per value.
template <int A> struct ActTag { static constexpr int value = A; };
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  if (act == LQSGD_ACT_RELU) f(ActTag<LQSGD_ACT_RELU>());
  else if (act == LQSGD_ACT_GELU) f(ActTag<LQSGD_ACT_GELU>());
  else if (act == LQSGD_ACT_SILU) f(ActTag<LQSGD_ACT_SILU>());
  else f(ActTag<LQSGD_ACT_NONE>());
}
// The same for runs of values, the choice made once.
template <int N>
__device__ __forceinline__ void act_run(int act, float (&v)[N]) {
  if (act == LQSGD_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<LQSGD_ACT_RELU>(v[i]);
  } else if (act == LQSGD_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<LQSGD_ACT_GELU>(v[i]);
  } else if (act == LQSGD_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<LQSGD_ACT_SILU>(v[i]);
  }
}
// The same two values at a time: where a product is over sooner than its epilogue.  Every operation's rounding is its own, so that a value comes out
// the same wherever these are used.
__device__ __forceinline__ void gelu2(float& z0, float& z1) {
  float t0, t1, r0, r1, g0, g1;
  const float n0 = -fabsf(fminf(z0, 3.402823466e38f)), n1 = -fabsf(fminf(z1, 3.402823466e38f));
  fma2(t0, t1, n0, n1, -0.30476302f, -0.30476302f, 1.f, 1.f);
  t0 = rcp_approx(t0);
  t1 = rcp_approx(t1);
  fma2(r0, r1, t0, t1, 0.036738604f, 0.036738604f, -0.15354006f, -0.15354006f);
  fma2(r0, r1, r0, r1, t0, t1, 0.18724863f, 0.18724863f);
  fma2(r0, r1, r0, r1, t0, t1, -0.039188605f, -0.039188605f);
  fma2(r0, r1, r0, r1, t0, t1, 0.12161422f, 0.12161422f);
  fma2(r0, r1, r0, r1, t0, t1, 0.10318742f, 0.10318742f);
  fma2(r0, r1, r0, r1, t0, t1, 0.12239605f, 0.12239605f);
  fma2(r0, r1, r0, r1, t0, t1, 0.12154379f, 0.12154379f);
  mul2(r0, r1, r0, r1, t0, t1);
  mul2(g0, g1, z0, z1, z0, z1);
  mul2(g0, g1, g0, g1, -0.72134752f, -0.72134752f);
  g0 = exp2_approx(g0);
  g1 = exp2_approx(g1);
  // z (z < 0 ? q : 1 - q), q = gauss r: max(z, 0) - |z| q.  q is 0 from 14 on; plus infinity counts as the largest value there, minus infinity
  // does not: infinity times 0, NaN, as act_value() has it.
  mul2(r0, r1, r0, r1, g0, g1);
  fma2(z0, z1, n0, n1, r0, r1, act_value<LQSGD_ACT_RELU>(z0), act_value<LQSGD_ACT_RELU>(z1));
}
__device__ __forceinline__ void silu2(float& z0, float& z1) {
  float e0, e1;
  mul2(e0, e1, z0, z1, -1.44269504f, -1.44269504f);
  e0 = exp2_approx(e0);
  e1 = exp2_approx(e1);
  add2(e0, e1, e0, e1, 1.f, 1.f);
  mul2(z0, z1, z0, z1, rcp_approx(e0), rcp_approx(e1));
}
template <int N>
__device__ __forceinline__ void act_pairs(int act, float (&v)[N]) {
  if (act == LQSGD_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<LQSGD_ACT_RELU>(v[i]);
  } else if (act == LQSGD_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; i += 2) gelu2(v[i], v[i + 1]);
  } else if (act == LQSGD_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; i += 2) silu2(v[i], v[i + 1]);
  }
}
template <int N>
__device__ __forceinline__ void slope_run(int act, float (&v)[N]) {
  if (act == LQSGD_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_slope<LQSGD_ACT_RELU>(v[i]);
  } else if (act == LQSGD_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_slope<LQSGD_ACT_GELU>(v[i]);
  } else if (act == LQSGD_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_slope<LQSGD_ACT_SILU>(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 1.f;
  }
}

}  // namespace
}  // namespace lqsgd
