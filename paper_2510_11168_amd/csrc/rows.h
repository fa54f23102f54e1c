// Rows of BF16 / FP32 matrices as the row-wise kernels (norm, sampling, distillation) read and write them: octets of consecutive
// elements, one 16-byte access in BF16 and two in FP32.  Rows may begin at any element: gfx950 serves a 16-byte global access at
// any address, so there is one form for every stride and offset, and only an octet that a row's end cuts goes element by element.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "numerics.h"
#include "tiles.h"

namespace elmo {

typedef u32x4 __attribute__((aligned(2))) u32x4_any2;      // 16 bytes at the address of any BF16 element
typedef f32x4 __attribute__((aligned(4))) f32x4_any4;
typedef i32x2 __attribute__((aligned(1))) i32x2_any1;

// An octet as it lies in memory, and its values.
template <class T> struct Octet;
template <> struct Octet<uint16_t> {
  u32x4 v;
  __device__ inline float operator[](int i) const { return (i & 1) ? u2f(v[i >> 1] & 0xFFFF0000u) : u2f(v[i >> 1] << 16); }
};
template <> struct Octet<float> {
  f32x4 a, b;
  __device__ inline float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

// valid = elements of the row from p on; those beyond it read as `fill`.
__device__ inline Octet<uint16_t> load_octet(const uint16_t* __restrict__ p, int64_t valid, uint16_t fill = 0) {
  Octet<uint16_t> o;
  if (valid >= 8) {
    o.v = *reinterpret_cast<const u32x4_any2*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 2 * i < valid ? p[2 * i] : fill, hi = 2 * i + 1 < valid ? p[2 * i + 1] : fill;
      o.v[i] = lo | (hi << 16);
    }
  }
  return o;
}
__device__ inline Octet<float> load_octet(const float* __restrict__ p, int64_t valid, float fill = 0.0f) {
  Octet<float> o;
  if (valid >= 8) {
    o.a = *reinterpret_cast<const f32x4_any4*>(p);
    o.b = *reinterpret_cast<const f32x4_any4*>(p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o.a[i] = i < valid ? p[i] : fill;
      o.b[i] = i + 4 < valid ? p[i + 4] : fill;
    }
  }
  return o;
}

// FP32 pair -> BF16, round to nearest even (v_cvt_pk_bf16_f32); infinities and NaN stay what they are.
__device__ inline uint32_t pack_bf16(float a, float b) {
  union { bf16x2 h; uint32_t u; } p;
  p.h[0] = (__bf16)a;
  p.h[1] = (__bf16)b;
  return p.u;
}
// NT: past the caches, for what nothing reads again soon.
template <bool NT = false> __device__ inline void store_octet(uint16_t* __restrict__ p, int64_t valid, const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  if (valid >= 8) {
    if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any2*>(p));
    else *reinterpret_cast<u32x4_any2*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
  }
}
template <bool NT = false> __device__ inline void store_octet(float* __restrict__ p, int64_t valid, const float (&f)[8]) {
  if (valid >= 8) {
    const f32x4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
    if constexpr (NT) {
      __builtin_nontemporal_store(a, reinterpret_cast<f32x4_any4*>(p));
      __builtin_nontemporal_store(b, reinterpret_cast<f32x4_any4*>(p + 4));
    } else {
      *reinterpret_cast<f32x4_any4*>(p) = a;
      *reinterpret_cast<f32x4_any4*>(p + 4) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = f[i];
  }
}
// Eight bytes.
__device__ inline void store_bytes(uint8_t* __restrict__ p, int64_t valid, i32x2 v) {
  if (valid >= 8) {
    *reinterpret_cast<i32x2_any1*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = (uint8_t)((uint32_t)v[i >> 2] >> (8 * (i & 3)));
  }
}

// exp and log in FP64, to a few units of 2^-53, from their series: exp(r) with |r| <= ln(2) / 2 behind a power of two (thirteen terms: the first one
// left out is below 2^-57), log(f) = 2 atanh((f - 1) / (f + 1)) with f in [sqrt(1/2), sqrt(2)] (|quotient| <= 0.172: eleven terms, 2^-60).  The
// coefficients lie in memory, so that they are scalar operands: the library's functions, inlined into a loop, have theirs
// kept in vector registers, which the kernels that hold a row there do not have (and a call would cost them as many).
__constant__ double kExpSeries[14] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880,
                                             1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600, 1.0 / 6227020800.0};
__constant__ double kLogSeries[11] = {2.0, 2.0 / 3, 2.0 / 5, 2.0 / 7, 2.0 / 9, 2.0 / 11, 2.0 / 13, 2.0 / 15, 2.0 / 17, 2.0 / 19, 2.0 / 21};
constexpr double kLn2 = 0.6931471805599453, kLn2Rest = 2.3190468138462996e-17, kLog2e = 1.4426950408889634;
__device__ inline double exp_series(double x) {          // NaN stays NaN; beyond FP64's range 0 or infinity
  x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;
  const double n = __builtin_rint(x * kLog2e);
  const double r = __builtin_fma(-n, kLn2Rest, __builtin_fma(-n, kLn2, x));
  double p = kExpSeries[13];
#pragma unroll
  for (int i = 12; i >= 0; --i) p = __builtin_fma(p, r, kExpSeries[i]);
  return __builtin_ldexp(p, (int)n);
}
__device__ inline double log_series(double x) {          // of a number that is not negative: 0 -> -infinity, infinity and NaN stay
  int e;
  double f = __builtin_frexp(x, &e);                     // [1/2, 1)
  if (f < 0.7071067811865476) { f += f; --e; }
  const double q = (f - 1.0) / (f + 1.0), q2 = q * q;
  double p = kLogSeries[10];
#pragma unroll
  for (int i = 9; i >= 0; --i) p = __builtin_fma(p, q2, kLogSeries[i]);
  p = __builtin_fma((double)e, kLn2, __builtin_fma(p, q, (double)e * kLn2Rest));
  return x == 0.0 ? -__builtin_inf() : x < __builtin_inf() ? p : x;
}

template <class T> __device__ inline float load_one(const T* p, int64_t i);
template <> __device__ inline float load_one<uint16_t>(const uint16_t* p, int64_t i) { return bf16_decode(p[i]); }
template <> __device__ inline float load_one<float>(const float* p, int64_t i) { return p[i]; }
__device__ inline void store_one(uint16_t* p, int64_t i, float f) { p[i] = (uint16_t)pack_bf16(f, f); }
__device__ inline void store_one(float* p, int64_t i, float f) { p[i] = f; }

// Values of other lanes, word by word, by the vector ALU's own exchanges: through LDS (__shfl) each is a trip of some 60 clocks on a pipe that the CU's
// waves share.  All lanes of the wave take part.
template <class T, class F> __device__ inline T by_words(T v, F f) {
  static_assert(sizeof(T) % 4 == 0, "whole words");
  union { T t; uint32_t w[sizeof(T) / 4]; } x = {v}, y = {v};
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 4); ++i) y.w[i] = f(x.w[i]);
  return y.t;
}
// Lanes M apart; for M = 4 and 8 a mirrored lane of the neighbouring M, which has the same once the steps below are done.
template <int M, class T, class Op> __device__ inline T reduce_step(T v, Op op) {
  if constexpr (M <= 8) {
    return op(v, by_words(v, [](uint32_t w) {
      constexpr int ctrl = M == 1 ? 0xB1 : M == 2 ? 0x4E : M == 4 ? 0x141 : 0x140;  // quad_perm 1 0 3 2, 2 3 0 1, row_half_mirror, row_mirror
      return (uint32_t)__builtin_amdgcn_mov_dpp((int)w, ctrl, 0xF, 0xF, true);
    }));
  } else {                                               // (both halves of a swap of a value with itself: the even rows twice, the odd ones twice)
    const auto swap = [](uint32_t w) { return M == 16 ? __builtin_amdgcn_permlane16_swap(w, w, false, false) : __builtin_amdgcn_permlane32_swap(w, w, false, false); };
    return op(by_words(v, [&](uint32_t w) { return (uint32_t)swap(w)[0]; }), by_words(v, [&](uint32_t w) { return (uint32_t)swap(w)[1]; }));
  }
}
// Reductions over a wave, or over each N of its lanes: every lane gets the result.
template <int N = 64, class T, class Op> __device__ inline T wave_reduce(T v, Op op) {
  if constexpr (N >= 2) v = reduce_step<1>(v, op);
  if constexpr (N >= 4) v = reduce_step<2>(v, op);
  if constexpr (N >= 8) v = reduce_step<4>(v, op);
  if constexpr (N >= 16) v = reduce_step<8>(v, op);
  if constexpr (N >= 32) v = reduce_step<16>(v, op);
  if constexpr (N >= 64) v = reduce_step<32>(v, op);
  return v;
}
// One lane's value, for all; `lane` the same in all lanes.
template <class T> __device__ inline T of_lane(T v, int lane) {
  return by_words(v, [&](uint32_t w) { return (uint32_t)__builtin_amdgcn_readlane((int)w, lane); });
}
// Inclusive sums over a wave.
template <class U> __device__ inline U wave_scan(U v) {
#define ELMO_SCAN_STEP(ctrl, rows) v += by_words(v, [](uint32_t w) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, ctrl, rows, 0xF, false); })
  ELMO_SCAN_STEP(0x111, 0xF);                            // row_shr 1, 2, 4, 8: nothing comes in at a row's begin
  ELMO_SCAN_STEP(0x112, 0xF);
  ELMO_SCAN_STEP(0x114, 0xF);
  ELMO_SCAN_STEP(0x118, 0xF);
  ELMO_SCAN_STEP(0x142, 0xA);                            // row_bcast 15: a row's sum to the next, odd ones
  ELMO_SCAN_STEP(0x143, 0xC);                            // row_bcast 31
#undef ELMO_SCAN_STEP
  return v;
}
// The waves' results of a workgroup, one a wave in `slots` behind a barrier (a lane reads one of them: sixteen held at once cost a kernel
// that is short of registers more than the exchange between lanes does).
template <int NW, class T, class Op> __device__ inline T slots_reduce(const T* slots, int lane, Op op) {
  return wave_reduce<NW>(slots[lane & (NW - 1)], op);
}
__device__ inline float wave_sum(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; });
}
__device__ inline double wave_sum64(double v) {
  return wave_reduce(v, [](double a, double b) { return a + b; });
}
// max of FP32 values without NaN, by their order
__device__ inline float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace elmo
