// 8-bit integer product with a scale for each row of either operand:
//   out[m, n] = (sum_k a[m, k] b[n, k]) sa[m] sb[n] + bias[n],   a [M, K], b [N, K] int8, the sum exact in 32 bits.
#pragma once
#include "rows.h"

namespace elmo {

struct Int8Args {
  const char *a, *b;
  const float *sa, *sb, *bias;
  void* out;
  int64_t as, bs, os;                // row strides in elements
  int M, N, K;
};

typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef i32x4 __attribute__((aligned(1))) i32x4_any1;

// 16 bytes of a row from k on, zeros beyond K.
__device__ inline i32x4 load_k16(const char* __restrict__ row, int k, int K) {
  i32x4 v = {0, 0, 0, 0};
  if (k + 16 <= K) return *reinterpret_cast<const i32x4_any1*>(row + k);
  for (int i = 0; i < 16; ++i)
    if (k + i < K) v[i >> 2] |= (int)(uint32_t)(uint8_t)row[k + i] << (8 * (i & 3));
  return v;
}

template <class O> __device__ inline void store_out(const Int8Args& p, int m, int n, int acc) {
  const float v = (float)acc * p.sa[m] * p.sb[n];
  store_one((O*)p.out + (int64_t)m * p.os, n, p.bias ? v + p.bias[n] : v);
}

// 64 x 64 outputs a workgroup, 32 x 32 a wave; slabs of 64 bytes of K through LDS.
constexpr int kInt8Row = 80;         // bytes of an LDS row: 64 of K, 16 of padding
template <class O>
__global__ __launch_bounds__(kThreads) void k_int8_plain(Int8Args p) {
  __shared__ __align__(16) char sa[64 * kInt8Row], sb[64 * kInt8Row];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_n = (p.N + 63) / 64;
  const int m0 = (int)(blockIdx.x / tiles_n) * 64, n0 = (int)(blockIdx.x % tiles_n) * 64;
  const int r = tid >> 2, c = (tid & 3) * 16;
  const char* a = p.a + (int64_t)min(m0 + r, p.M - 1) * p.as;
  const char* b = p.b + (int64_t)min(n0 + r, p.N - 1) * p.bs;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  i32x16 acc = {};
  for (int k0 = 0; k0 < p.K; k0 += 64) {
    *reinterpret_cast<i32x4*>(sa + r * kInt8Row + c) = load_k16(a, k0 + c, p.K);
    *reinterpret_cast<i32x4*>(sb + r * kInt8Row + c) = load_k16(b, k0 + c, p.K);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int at = ks * 32 + 16 * (lane >> 5);
      const i32x4 fa = *reinterpret_cast<const i32x4*>(sa + (wm + (lane & 31)) * kInt8Row + at);
      const i32x4 fb = *reinterpret_cast<const i32x4*>(sb + (wn + (lane & 31)) * kInt8Row + at);
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa, fb, acc, 0, 0, 0);
    }
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int m = m0 + wm + acc_row(v, lane), n = n0 + wn + (lane & 31);
    if (m < p.M && n < p.N) store_out<O>(p, m, n, acc[v]);
  }
}

}  // namespace elmo
