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
__device__ inline void store_octet(uint16_t* __restrict__ p, int64_t valid, const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
  if (valid >= 8) {
    *reinterpret_cast<u32x4_any2*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) p[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
  }
}
__device__ inline void store_octet(float* __restrict__ p, int64_t valid, const float (&f)[8]) {
  if (valid >= 8) {
    *reinterpret_cast<f32x4_any4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4_any4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
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

template <class T> __device__ inline float load_one(const T* p, int64_t i);
template <> __device__ inline float load_one<uint16_t>(const uint16_t* p, int64_t i) { return bf16_decode(p[i]); }
template <> __device__ inline float load_one<float>(const float* p, int64_t i) { return p[i]; }
__device__ inline void store_one(uint16_t* p, int64_t i, float f) { p[i] = (uint16_t)pack_bf16(f, f); }
__device__ inline void store_one(float* p, int64_t i, float f) { p[i] = f; }

// Reductions over a wave: every lane gets the result.
template <class T, class Op> __device__ inline T wave_reduce(T v, Op op) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v = op(v, __shfl_xor(v, m));
  return v;
}
__device__ inline float wave_sum(float v) {
  return wave_reduce(v, [](float a, float b) { return a + b; });
}
// max of FP32 values without NaN, by their order
__device__ inline float wave_max(float v) {
  return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace elmo
