// Device pieces shared by the operators that work on whole rows: the random bits of dropout, signed 8-bit codes, and how a row is
// dealt out to the threads that hold it.
#pragma once
#include <atomic>

#include "lqsgd_runs_dev.cuh"

namespace lqsgd {

// Dropout as the kernels take it: threshold T in the upper half of a word, 65536 / (65536 - T), the generator's keys of every round (a
// third of its instructions would be adding them up; from the kernel's arguments they are operands).
struct Drop {
  uint64_t offset;
  const uint64_t* dev_seed;                  // NULL: keys and offset are complete
  uint32_t threshold;                        // 0: nothing is dropped
  float scale;
  uint32_t keys[20];
};
inline Drop make_drop(const lqsgd_drop& d) {
  const int t = std::min((int)rint(65536.0 * (double)d.p), 65535);
  Drop o = {d.offset, d.dev_seed, (uint32_t)t << 16, (float)(65536.0 / (65536 - t)), {}};
  for (uint32_t r = 0; r < 10; ++r) {
    o.keys[2 * r] = (uint32_t)d.seed + r * 0x9E3779B9u;
    o.keys[2 * r + 1] = (uint32_t)(d.seed >> 32) + r * 0xBB67AE85u;
  }
  return o;
}

namespace {

// How the rows of a call's matrices are read and written.
//   kWhole  every row of every matrix starts on 16 bytes and is a whole number of runs (8-bit copies: on 8 bytes)
//   kShift  any alignment.  A run is taken from the 16-byte pieces around it, which lie inside the row for all but its first and last
//           runs, and moved into place in registers; it is written as the piece that begins in the run of the lane in front.  Element by
//           element a run would touch as many places as it has elements; turned in shared memory, as the 8-bit streams do it, a
//           row of 16-bit values still goes through 2-byte accesses (the norm of 1021 x 25087 fp16 into codes, before later steps: 87 us element by
//           element or turned, 73 so; now 58, rows of 25088 37).
enum RowAccess { kWhole = 0, kShift = 1 };

// Philox4x32, 10 rounds: a product of each even word by a constant, its high half mixed with a neighbour and the round's key.
__device__ __forceinline__ uint4 philox(uint64_t block, uint64_t offset, const uint32_t* keys) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ keys[2 * r];
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ keys[2 * r + 1];
    c3 = (uint32_t)a;
  }
  return make_uint4(c0, c1, c2, c3);
}
// Where the caller keeps the seed on the device, a block makes the keys and the offset in shared memory.
constexpr int kDropRoom = 22;
__device__ __forceinline__ void open_drop(const Drop& d, uint32_t (&room)[kDropRoom]) {
  if (!d.threshold || !d.dev_seed) return;                 // the same for all threads
  if (threadIdx.x < 20) {
    const uint64_t seed = d.dev_seed[0];
    const uint32_t r = threadIdx.x >> 1;
    room[threadIdx.x] = (threadIdx.x & 1) ? (uint32_t)(seed >> 32) + r * 0xBB67AE85u : (uint32_t)seed + r * 0x9E3779B9u;
  } else if (threadIdx.x < kDropRoom) {
    room[threadIdx.x] = (uint32_t)((d.offset + d.dev_seed[1]) >> (threadIdx.x == 20 ? 0 : 32));
  }
  __syncthreads();
}
// Random bits of a thread's N runs (32 blocks apart); block = row * ceil(cols / 8) + column / 8 of the first.  All at once: the rounds of one
// run depend on one another, those of several fill the gaps.
template <int N>
__device__ __forceinline__ void drop_bits(const Drop& d, const uint32_t (&room)[kDropRoom], uint64_t block, uint4 (&bits)[N]) {
  if (d.dev_seed) {
#pragma unroll
    for (int i = 0; i < N; ++i) bits[i] = philox(block + 32 * i, (uint64_t)room[21] << 32 | room[20], room);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) bits[i] = philox(block + 32 * i, d.offset, d.keys);
  }
}
// r += dropout(v) for a run.  A half word's bits are compared in the upper half of a word, where what lies below them does not count.  One
// rounding, the same in every kernel that drops.
__device__ __forceinline__ void drop_run(const Drop& d, const uint4& bits, const float (&v)[kRun], float (&r)[kRun]) {
  const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if ((w[j] << 16) >= d.threshold) r[2 * j] = __fmaf_rn(v[2 * j], d.scale, r[2 * j]);
    if (w[j] >= d.threshold) r[2 * j + 1] = __fmaf_rn(v[2 * j + 1], d.scale, r[2 * j + 1]);
  }
}

// ---- arithmetic on runs, two values at a time
// a = b c + d and the like, of a run
__device__ __forceinline__ void fma_run(float (&a)[kRun], const float (&b)[kRun], const float (&c)[kRun], const float (&d)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) fma2(a[j], a[j + 1], b[j], b[j + 1], c[j], c[j + 1], d[j], d[j + 1]);
}
__device__ __forceinline__ void fma_run(float (&a)[kRun], const float (&b)[kRun], float c, const float (&d)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) fma2(a[j], a[j + 1], b[j], b[j + 1], c, c, d[j], d[j + 1]);
}
__device__ __forceinline__ void mul_run(float (&a)[kRun], const float (&b)[kRun], const float (&c)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) mul2(a[j], a[j + 1], b[j], b[j + 1], c[j], c[j + 1]);
}
__device__ __forceinline__ void mul_run(float (&a)[kRun], const float (&b)[kRun], float c) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) mul2(a[j], a[j + 1], b[j], b[j + 1], c, c);
}
__device__ __forceinline__ void add_run(float (&a)[kRun], const float (&b)[kRun], const float (&c)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) add2(a[j], a[j + 1], b[j], b[j + 1], c[j], c[j + 1]);
}
__device__ __forceinline__ void clear_run(float (&a)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; ++j) a[j] = 0.f;
}
// sum += the run's products, even and odd columns apart
__device__ __forceinline__ void dot_run(float (&sum)[2], const float (&b)[kRun], const float (&c)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun; j += 2) fma2(sum[0], sum[1], b[j], b[j + 1], c[j], c[j + 1], sum[0], sum[1]);
}

// ---- rows of signed 8-bit codes
constexpr float kRowStepLow = 7.52316385e-37f, kRowInvHigh = 1.32922800e36f;      // 2^-120, 2^120
// Scale of a row, and what its values are multiplied by (0: the row is not finite, its codes are 0).
__device__ __forceinline__ void row_scale(float top, float& scale, float& inv) {
  const bool finite = __float_as_uint(top) < 0x7f800000u;
  scale = finite ? fmaxf(__fdiv_rn(top, 127.f), kRowStepLow) : __uint_as_float(0x7fc00000u);
  inv = finite ? fminf(__fdiv_rn(127.f, top), kRowInvHigh) : 0.f;
}
// Eight codes rint(v inv), |v inv| <= 127 (1 + 2^-23): adding 1.5 * 2^23 to the rounded product leaves an integer in two's complement below.  v inv is rounded by
// itself, as the definition has it (one at a time: of two at a time, product and sum come out fused).
__device__ __forceinline__ uint2 signed_codes(const float (&v)[kRun], float inv) {
  float t[kRun];
#pragma unroll
  for (int j = 0; j < kRun; ++j) t[j] = __fmul_rn(v[j], inv);
#pragma unroll
  for (int j = 0; j < kRun; j += 2) add2(t[j], t[j + 1], t[j], t[j + 1], 12582912.f, 12582912.f);
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    w[k] = __byte_perm(__byte_perm(__float_as_uint(t[4 * k]), __float_as_uint(t[4 * k + 1]), 0x0040),
                       __byte_perm(__float_as_uint(t[4 * k + 2]), __float_as_uint(t[4 * k + 3]), 0x0040), 0x5410);
  return inv == 0.f ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
}

// ---- a run as it is stored: of 16-bit types half the registers that its values take
template <int DT>
__device__ __forceinline__ void open_words(const Piece<DT>& in, float (&v)[kRun]) {
#pragma unroll
  for (int j = 0; j < kRun / 2; ++j) {
    if constexpr (DT == LQSGD_F32) {
      v[2 * j] = __uint_as_float(in.w[2 * j]);
      v[2 * j + 1] = __uint_as_float(in.w[2 * j + 1]);
    } else {
      const float2 f = open_pair<DT>(in.w[j]);
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
  }
}
template <int DT>
__device__ __forceinline__ void close_words(const float (&v)[kRun], Piece<DT>& out) {
#pragma unroll
  for (int j = 0; j < kRun / 2; ++j) {
    if constexpr (DT == LQSGD_F32) {
      out.w[2 * j] = __float_as_uint(v[2 * j]);
      out.w[2 * j + 1] = __float_as_uint(v[2 * j + 1]);
    } else {
      out.w[j] = pack_pair<DT>(v[2 * j], v[2 * j + 1]);
    }
  }
}

// ---- a thread's runs of a row
// Up to N of them, kWarpCols apart, so that whatever a thread touches of a matrix's row is one address and constants; neighbouring lanes hold
// neighbouring runs.  `left`: columns from the thread's first run to the row's end.
constexpr int kWarpCols = 32 * kRun;
template <int DT> constexpr int kRunBytes = kRun * (int)sizeof(typename Elem<DT>::T);
struct Lanes {
  int col, left;                             // the thread's first run
  int lane, lanes;                           // this lane among those that hold neighbouring runs of the row
  bool on;                                   // the row exists
  __device__ __forceinline__ int have(int i) const { return left - i * kWarpCols; }
  __device__ __forceinline__ bool has(int i) const { return on && have(i) > 0; }
};
// Where a thread's first run of a matrix's row lies.  With kShift: the 16-byte piece that it begins in, how far into it, how many columns a
// run must have in front of the row's end to be taken from whole pieces of the row (its first run in no case, if it is shifted).
template <int DT, int HOW>
struct Cursor {
  char* p;
  uint32_t shift;
  int need;
  bool head;
  __device__ __forceinline__ Cursor(const void* matrix, int64_t at, const Lanes& l) {
    constexpr int kSize = (int)sizeof(typename Elem<DT>::T);
    p = static_cast<char*>(const_cast<void*>(matrix)) + (at + l.col) * kSize;
    shift = 0;
    need = kRun;
    head = false;
    if (HOW == kShift) {
      shift = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
      p -= shift;
      if (shift) {
        need = kRun + (int)(16 - shift) / kSize;
        head = l.col == 0;
      }
    }
  }
  __device__ __forceinline__ char* at(int i) const { return p + i * (32 * kRunBytes<DT>); }
  __device__ __forceinline__ bool pieces(const Lanes& l, int i) const { return l.have(i) >= need && !(i == 0 && head); }
};
// N words that begin `shift` bytes into in, at any shift of a thread's own, and at one of Q words and `bits` bits.
template <int N, int M>
__device__ __forceinline__ void shift_words(const uint32_t (&in)[M], uint32_t shift, uint32_t (&out)[N]) {
  static_assert(M >= N + 4, "room to shift");
  uint32_t t[N + 3], u[N + 1];
#pragma unroll
  for (int k = 0; k < N + 3; ++k) t[k] = shift & 4 ? in[k + 1] : in[k];
#pragma unroll
  for (int k = 0; k < N + 1; ++k) u[k] = shift & 8 ? t[k + 2] : t[k];
#pragma unroll
  for (int k = 0; k < N; ++k) out[k] = __funnelshift_r(u[k], u[k + 1], (shift & 3) * 8);
}
template <int Q, int N, int M>
__device__ __forceinline__ void shift_words_by(const uint32_t (&in)[M], uint32_t bits, uint32_t (&out)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) out[k] = __funnelshift_r(in[k + Q], in[k + Q + 1 < M ? k + Q + 1 : k + Q], bits);
}
// f with the number of whole words in a shift below 16 bytes as a constant.
template <int Q> struct WordsTag { static constexpr int value = Q; };
template <typename F>
__device__ __forceinline__ void by_words(uint32_t shift, F&& f) {
  switch (shift >> 2) {
    case 0: f(WordsTag<0>()); break;
    case 1: f(WordsTag<1>()); break;
    case 2: f(WordsTag<2>()); break;
    default: f(WordsTag<3>()); break;
  }
}

// A run as it is fetched: with kShift 16 bytes more, the run beginning c.shift into them (at the row's ends one element to a word).
template <int DT, int HOW>
struct Raw {
  static constexpr int kPieces = kRunBytes<DT> / 16 + (HOW == kShift ? 1 : 0);
  uint32_t w[4 * kPieces];
};
// Run i, zeros where there is none: what follows then needs no branch, and the work on a thread's runs interleaves.
template <int DT, int HOW>
__device__ __forceinline__ void fetch(const Cursor<DT, HOW>& c, const Lanes& l, int i, Raw<DT, HOW>& out) {
  using T = typename Elem<DT>::T;
  constexpr int kPieces = Raw<DT, HOW>::kPieces;
#pragma unroll
  for (int k = 0; k < 4 * kPieces; ++k) out.w[k] = 0u;
  if (!l.has(i)) return;
  if (HOW == kWhole || c.pieces(l, i)) {
    const uint4* p = reinterpret_cast<const uint4*>(c.at(i));
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      if (k < kRunBytes<DT> / 16 || c.shift) reinterpret_cast<uint4*>(out.w)[k] = p[k];
  } else if constexpr (HOW == kShift) {                       // the row's ends: an element to a word (nothing here waits for a load)
    const T* e = reinterpret_cast<const T*>(c.at(i) + c.shift);
#pragma unroll
    for (int j = 0; j < kRun; ++j)
      if (j < l.have(i)) {
        if constexpr (DT == LQSGD_F32) out.w[j] = __float_as_uint(e[j]);
        else out.w[j] = reinterpret_cast<const uint16_t*>(e)[j];
      }
  }
}
// A run at the row's ends as it is stored.
template <int DT, int M>
__device__ __forceinline__ void gather_words(const uint32_t (&in)[M], Piece<DT>& out) {
#pragma unroll
  for (int k = 0; k < kRunBytes<DT> / 4; ++k) {
    if constexpr (DT == LQSGD_F32) out.w[k] = in[k];
    else out.w[k] = in[2 * k] | (in[2 * k + 1] << 16);
  }
}
// What fetch brought as a thread's N runs.  Where a warp holds one row the shift is the warp's.
template <int DT, int HOW, int N>
__device__ __forceinline__ void settle(const Raw<DT, HOW> (&in)[N], const Cursor<DT, HOW>& c, const Lanes& l, Piece<DT> (&out)[N]) {
  if constexpr (HOW == kWhole) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < kRunBytes<DT> / 4; ++k) out[i].w[k] = in[i].w[k];
  } else if (N > 1 || l.lanes == 32) {
    by_words(__shfl_sync(0xffffffffu, c.shift, 0), [&](auto q) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        shift_words_by<decltype(q)::value>(in[i].w, (c.shift & 3) * 8, out[i].w);
        if (!c.pieces(l, i)) gather_words<DT>(in[i].w, out[i]);
      }
    });
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      shift_words(in[i].w, c.shift, out[i].w);
      if (!c.pieces(l, i)) gather_words<DT>(in[i].w, out[i]);
    }
  }
}
// Writes a thread's N runs.  With kShift the whole warp calls it: a run is written as the 16-byte pieces that begin in the run in front, with
// that run's end from the neighbouring lane.
template <int DT, int HOW, int N>
__device__ __forceinline__ void put(const Cursor<DT, HOW>& c, const Lanes& l, const Piece<DT> (&p)[N]) {
  using T = typename Elem<DT>::T;
  constexpr int kWords = kRunBytes<DT> / 4;
  if constexpr (HOW == kWhole) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!l.has(i)) continue;
      uint4* o = reinterpret_cast<uint4*>(c.at(i));
#pragma unroll
      for (int k = 0; k < kWords / 4; ++k) o[k] = reinterpret_cast<const uint4*>(p[i].w)[k];
    }
  } else {
    const int me = threadIdx.x & 31;
    // run i as pieces in w; the ends of the row and of the warp's part of it element by element
    auto write = [&](int i, const uint32_t (&w)[kWords]) {
      const int have = l.have(i);
      if (!l.has(i)) return;
      const bool whole = have >= kRun && (l.lane > 0 || i > 0 || c.shift == 0), next = have >= 2 * kRun && (l.lane + 1 < l.lanes || i + 1 < N);
      if (whole) {
        uint4* o = reinterpret_cast<uint4*>(c.at(i));
#pragma unroll
        for (int k = 0; k < kWords / 4; ++k) o[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
      }
      if (!whole || (c.shift && !next)) {
        T* o = reinterpret_cast<T*>(c.at(i) + c.shift);
        const int head = (kRunBytes<DT> - (int)c.shift) / (int)sizeof(T);
#pragma unroll
        for (int j = 0; j < kRun; ++j)
          if (j < have && (j < head ? !whole : !next)) o[j] = reinterpret_cast<const T*>(p[i].w)[j];
      }
    };
    // the last FROM .. 3 of the four words in front of run i, and the run
    auto both = [&](int i, int from, uint32_t (&b)[kWords + 4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        b[k] = k < from ? 0u : __shfl_sync(0xffffffffu, i > 0 && me == 31 ? p[i > 0 ? i - 1 : 0].w[kWords - 4 + k] : p[i].w[kWords - 4 + k], (me + 31) & 31);
#pragma unroll
      for (int k = 0; k < kWords; ++k) b[4 + k] = p[i].w[k];
    };
    if (N > 1 || l.lanes == 32) {
      const uint32_t shift = __shfl_sync(0xffffffffu, c.shift, 0);
      if (shift == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) write(i, p[i].w);
      } else {
        by_words(16 - shift, [&](auto q) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            uint32_t b[kWords + 4], w[kWords];
            both(i, decltype(q)::value, b);
            shift_words_by<decltype(q)::value>(b, ((16 - shift) & 3) * 8, w);
            write(i, w);
          }
        });
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint32_t b[kWords + 4], w[kWords];
        both(i, 0, b);
        shift_words(b, 16 - c.shift & 15, w);
        if (c.shift) write(i, w);
        else write(i, p[i].w);
      }
    }
  }
}
// A thread's N runs of one step over a long row in shared memory, for itself: 16-byte pieces a block's width apart.
template <int DT, int N>
__device__ __forceinline__ void keep_runs(uint4* room, int step, const Piece<DT> (&p)[N]) {
  constexpr int kPieces = kRunBytes<DT> / 16;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < kPieces; ++k) room[((step * N + i) * kPieces + k) * blockDim.x + threadIdx.x] = reinterpret_cast<const uint4*>(p[i].w)[k];
}
template <int DT, int N>
__device__ __forceinline__ void kept_runs(const uint4* room, int step, Piece<DT> (&p)[N]) {
  constexpr int kPieces = kRunBytes<DT> / 16;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 0; k < kPieces; ++k) reinterpret_cast<uint4*>(p[i].w)[k] = room[((step * N + i) * kPieces + k) * blockDim.x + threadIdx.x];
}
// Run i of a vector of floats, from its element l.col on.
template <int HOW>
__device__ __forceinline__ void fetch_vector(const float* p, bool vec, const Lanes& l, int i, float (&v)[kRun]) {
  const int have = l.have(i);
  if (HOW == kWhole ? have > 0 : vec && have >= kRun) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p + i * kWarpCols)), b = __ldg(reinterpret_cast<const float4*>(p + i * kWarpCols) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int j = 0; j < kRun; ++j) v[j] = HOW != kWhole && j < have ? __ldg(p + i * kWarpCols + j) : 0.f;
  }
}
// Codes of run i at p, the row's from column l.col on.
template <int HOW>
__device__ __forceinline__ void put_codes(uint8_t* p, bool vec, const Lanes& l, int i, uint2 w) {
  const int have = l.have(i);
  if (!l.has(i)) return;
  if (HOW == kWhole || (vec && have >= kRun)) *reinterpret_cast<uint2*>(p + i * kWarpCols) = w;
  else store_codes(p + i * kWarpCols, false, min(have, kRun), w);
}
// The 8-bit form of run i: four neighbouring lanes hold a group of 32.  codes and exps: the row's from column l.col on.  The whole warp calls
// it, with zeros in lanes that have no run.
template <int HOW>
__device__ __forceinline__ void put_packed_run(uint8_t* codes, uint8_t* exps, bool vec, const Lanes& l, int i, const float (&v)[kRun]) {
  float top = largest(0.f, v);
  top = larger(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = larger(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int eb = exp_byte(top);
  const float inv = inv_step(eb);
  put_codes<HOW>(codes, vec, l, i, make_uint2(code_word(v[0], v[1], v[2], v[3], inv), code_word(v[4], v[5], v[6], v[7], inv)));
  if (l.has(i) && (l.lane & 3) == 0) exps[i * (kWarpCols / kGroup)] = (uint8_t)eb;
}

// Asks L2 for the whole 16-byte pieces of `bytes` from p on: one instruction.
__device__ __forceinline__ void ahead(const void* p, int64_t bytes) {
  const uintptr_t from = (reinterpret_cast<uintptr_t>(p) + 15) & ~(uintptr_t)15, to = (reinterpret_cast<uintptr_t>(p) + bytes) & ~(uintptr_t)15;
  if (to > from) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((uint32_t)(to - from)) : "memory");
}

// ---- a row and its threads
// NARROW: 4, 8, 16 or 32 lanes of a warp hold a row, a block of 256 threads several rows.  Otherwise a block holds one.  A warp's columns lie
// side by side.  N runs per thread (one where fewer than 32 lanes hold a row).
template <bool NARROW, int N>
struct Team {
  int warps, shift;
  int64_t row, rows_per_grid;
  __device__ __forceinline__ explicit Team(int lane_shift) : warps(blockDim.x >> 5), shift(NARROW ? lane_shift : 5) {
    const int each = NARROW ? (int)blockDim.x >> shift : 1;
    row = NARROW ? (int64_t)blockIdx.x * each + (threadIdx.x >> shift) : blockIdx.x;
    rows_per_grid = (int64_t)gridDim.x * each;
  }
  // step: how many times over the team's columns the row was walked before (rows longer than the team)
  __device__ __forceinline__ Lanes lanes(int cols, bool on, int step = 0) const {
    Lanes l;
    l.lanes = 1 << shift;
    l.lane = threadIdx.x & (l.lanes - 1);
    l.col = NARROW ? l.lane * kRun : (step * warps + (int)(threadIdx.x >> 5)) * N * kWarpCols + l.lane * kRun;
    l.left = cols - l.col;
    l.on = on;
    return l;
  }
  __device__ __forceinline__ bool first() const { return (threadIdx.x & (NARROW ? (1 << shift) - 1 : 0xffff)) == 0; }
  // Sum and, where TOP, largest of the team's values, in every thread of it.  `slots`: shared memory (unused by NARROW); of two calls in
  // a row the second takes other slots.
  template <bool TOP>
  __device__ __forceinline__ void join(float& sum, float& top, float2 (&slots)[16]) const {
    if constexpr (NARROW) {
      for (int o = 1; o < 1 << shift; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (TOP)
        for (int o = 1; o < 1 << shift; o <<= 1) top = larger(top, __shfl_xor_sync(0xffffffffu, top, o));
    } else {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (TOP) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) top = larger(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      if (warps > 1) {
        if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = make_float2(sum, top);
        __syncthreads();
        sum = 0.f;
#pragma unroll 4
        for (int w = 0; w < warps; ++w) {
          const float2 s = slots[w];
          sum += s.x;
          if (TOP) top = larger(top, s.y);
        }
      }
    }
  }
};

// ---- host side
// How the matrices of a call are read and written: all rows start on 16 bytes, all 8-bit copies' rows on 8, vectors on 16.
static inline int access_of(bool rows, bool others, int32_t cols) { return rows && others && cols % kRun == 0 ? kWhole : kShift; }

// How rows are dealt out.  Up to `narrow` columns: 4 to 32 lanes each.  Longer: a block each, n runs per thread, if `threads` threads hold them;
// else not held, and walked in several steps.
struct RowShape {
  bool narrow, held;
  int lane_shift, threads, n;
  int64_t teams;                             // rows per block
};
static inline RowShape shape_of(int32_t cols, int n, int narrow, int threads) {
  RowShape s = {};
  const int64_t runs = ceil_div64(cols, kRun);
  s.teams = 1;
  if (cols <= narrow) {
    s.narrow = s.held = true;
    s.lane_shift = 2;
    s.n = 1;
    while (s.lane_shift < 5 && (1 << s.lane_shift) < runs) ++s.lane_shift;
    while ((s.n << s.lane_shift) < runs) s.n *= 2;
    s.threads = 256;
    s.teams = 256 >> s.lane_shift;
    return s;
  }
  s.n = n;
  s.threads = (int)std::min<int64_t>(ceil_div64(ceil_div64(runs, n), 32) * 32, 1 << 20);
  s.held = s.threads <= threads;
  return s;
}

// Threads of a block that walks a longer row in as few steps of equal length as `most` threads allow.
static inline int long_threads(int64_t runs, int n, int64_t steps) { return (int)(ceil_div64(ceil_div64(runs, n * steps), 32) * 32); }
static inline int long_threads(int32_t cols, int n, int most) {
  const int64_t runs = ceil_div64(cols, kRun);
  return long_threads(runs, n, ceil_div64(runs, (int64_t)n * most));
}
// Shared memory in which a long row stays between two passes; 0 if two blocks of an SM have not enough (the second pass then reads L2).
constexpr size_t kKeepMost = 112 * 1024;
static inline size_t long_keep(int32_t cols, int n, int elem, int threads) {
  const size_t bytes = (size_t)ceil_div64(ceil_div64(cols, kRun), (int64_t)n * threads) * n * threads * kRun * elem;
  return bytes <= kKeepMost ? bytes : 0;
}
// Lets a kernel have kKeepMost; `ready`: the devices on which it may already.
static inline cudaError_t allow_keep(const void* kernel, std::atomic<uint64_t>& ready) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (ready.load(std::memory_order_acquire) >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kKeepMost);
  if (e == cudaSuccess && dev < 64) ready.fetch_or(1ull << dev, std::memory_order_release);
  return e;
}

}  // namespace
}  // namespace lqsgd

// f<type, access>(...) for a type and an access known at run time
#define BY_ACCESS(DT, how, f, ...) ((how) == kWhole ? f<DT, kWhole>(__VA_ARGS__) : f<DT, kShift>(__VA_ARGS__))
#define BY_TYPE(dtype, how, f, ...)                                  \
  ((dtype) == LQSGD_BF16  ? BY_ACCESS(LQSGD_BF16, how, f, __VA_ARGS__) \
   : (dtype) == LQSGD_F16 ? BY_ACCESS(LQSGD_F16, how, f, __VA_ARGS__)  \
                          : BY_ACCESS(LQSGD_F32, how, f, __VA_ARGS__))
