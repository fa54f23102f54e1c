// Root-mean-square norm behind the residual's addition, and its backward pass.
//
//   h = x + r,  R = 1 / sqrt(mean(h^2) + eps),  y = w h R
//
// 8-bit rows: with p = w h and m = max |p| the quotient y / (max |y| / 127) is 127 p / m -- R cancels -- so the whole numbers depend
// on p and m alone.  Both are exact in FP64 (24 x 24 bits), the maximum does not depend on an order, and what is left is 127 (1 / m), two FP64 roundings a row,
// and one product an element: the same numbers whichever way a row is split over lanes.  The scale is m R / 127 (448 for E4M3).
//
// Squares are summed in FP32.  A row whose sum leaves that type's range while its elements are inside is summed once more, times a power of two
// (out_of_range, scale_into_range): the same row as any other but for that.
//
// Bound: memory.  A row is read once and stays in registers, S octets a lane, spread over WPR waves.
#pragma once
#include "rows.h"

namespace elmo {

enum : int { OUT_BF16 = 0, OUT_E4M3 = 1, OUT_FP32 = 2, OUT_INT8 = 3 };

constexpr int norm_threads(int wpr) { return wpr > 4 ? 64 * wpr : kThreads; }

struct NormArgs {
  const void *x, *res, *w;
  void *sum, *y;
  float* scale;
  int64_t rows, xs, rs, ss, ys;      // strides in elements
  int d;
  float eps;
  bool w32;                          // FP32 weights
};

// Mean square `ms` (NaN among them) of a row that has to be summed again.  2^-100: what lies below has lost more than the last bit of squares below 2^-126;
// with that much eps it does not matter.
__device__ inline bool out_of_range(float ms, float eps, bool large) { return !(ms + eps >= 0x1p-100f && (ms < __builtin_inff() || !large)); }
// Elements up to 2^-43 come to 2^53, the least ones (2^-149) to 2^-53; elements up to 2^128 to 2^48.  Squares and their sums stay inside either way.
__device__ inline float scale_into_range(float ms) { return ms < 1.0f ? 0x1p96f : 0x1p-80f; }

// Octet of the weights; 1 without weights.
__device__ inline void load_weights(const void* w, bool w32, int c, int valid, float (&f)[8]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.0f;
  } else if (w32) {
    const Octet<float> o = load_octet((const float*)w + c, valid);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = o[i];
  } else {
    const Octet<uint16_t> o = load_octet((const uint16_t*)w + c, valid);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = o[i];
  }
}

// Sum / maximum over the WPR waves of a row; `slots` are WPR entries of the row's own.
template <int WPR, class T, class Op> __device__ inline T row_reduce(T v, T* slots, int wave_in_row, int lane, Op op) {
  v = wave_reduce(v, op);
  if constexpr (WPR > 1) {
    if (lane == 0) slots[wave_in_row] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int i = 1; i < WPR; ++i) v = op(v, slots[i]);
  }
  return v;
}

template <class T, int OUT, int WPR, int S>
__global__ __launch_bounds__(norm_threads(WPR)) void k_rms_norm(NormArgs a) {
  constexpr int RPG = norm_threads(WPR) / (64 * WPR);     // rows of a workgroup
  constexpr bool EIGHT = OUT == OUT_INT8 || OUT == OUT_E4M3;
  __shared__ float s_sum[RPG][WPR];
  __shared__ double s_max[RPG][WPR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_row = wave % WPR, slot = wave / WPR;
  const int64_t row = (int64_t)blockIdx.x * RPG + slot;
  if (WPR == 1 && row >= a.rows) return;                  // (WPR 4 and more: one row a workgroup, always a valid one)
  const T* x = (const T*)a.x + row * a.xs;
  const T* res = a.res ? (const T*)a.res + row * a.rs : nullptr;
  const int c0 = (in_row * 64 + lane) * 8;
  constexpr int STEP = WPR * 512;

  float h[S][8];
  Octet<T> xo[S], ro[S];
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (c0 + s * STEP < a.d) {
      xo[s] = load_octet(x + c0 + s * STEP, a.d - c0 - s * STEP);
      if (res) ro[s] = load_octet(res + c0 + s * STEP, a.d - c0 - s * STEP);
    }
  float sq = 0.0f;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int c = c0 + s * STEP;
    if (c < a.d) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[s][i] = res ? xo[s][i] + ro[s][i] : xo[s][i];
        sq = __builtin_fmaf(h[s][i], h[s][i], sq);
      }
      if (a.sum) store_octet((T*)a.sum + row * a.ss + c, a.d - c, h[s]);
    }
  }
  sq = row_reduce<WPR>(sq, s_sum[slot], in_row, lane, [](float p, float q) { return p + q; });
  float ms = sq / (float)a.d, eps = a.eps;
  if (out_of_range(ms, eps, !EIGHT)) {                    // (the same for all lanes of a row; 8-bit rows of too large squares have no scale)
    const float up = scale_into_range(ms);
    sq = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (c0 + s * STEP < a.d) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[s][i] *= up;
          sq = __builtin_fmaf(h[s][i], h[s][i], sq);
        }
      }
    if (WPR > 1) __syncthreads();                         // (the slots have been read)
    ms = row_reduce<WPR>(sq, s_sum[slot], in_row, lane, [](float p, float q) { return p + q; }) / (float)a.d;
    eps = eps * up * up;
  }
  const float rstd = 1.0f / sqrtf(ms + eps);

  if constexpr (!EIGHT) {
    using O = typename std::conditional<OUT == OUT_BF16, uint16_t, float>::type;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = c0 + s * STEP;
      if (c < a.d) {
        float w[8], f[8];
        load_weights(a.w, a.w32, c, a.d - c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = h[s][i] * rstd * w[i];
        store_octet((O*)a.y + row * a.ys + c, a.d - c, f);
      }
    }
  } else {
    constexpr double MOST = OUT == OUT_INT8 ? 127.0 : 448.0;
    double m = 0.0;
    float odd = 0.0f;                                     // NaN once a weight is NaN or infinite (the maximum would pass over a NaN)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = c0 + s * STEP;
      if (c < a.d) {
        float w[8];
        load_weights(a.w, a.w32, c, a.d - c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          m = __builtin_fmax(m, __builtin_fabs((double)h[s][i] * (double)w[i]));
          odd = __builtin_fmaf(w[i], 0.0f, odd);
        }
      }
    }
    if (!(odd == 0.0f)) m = __builtin_inf();
    m = row_reduce<WPR>(m, s_max[slot], in_row, lane, [](double p, double q) { return __builtin_fmax(p, q); });
    const bool bad = !(ms < __builtin_inff()) || m == __builtin_inf();
    const bool live = m > 0.0 && !bad;                    // a row of zeros: zeros with scale 0
    const double inv = 1.0 / m * MOST;                    // the order of these roundings decides exact ties
    if (in_row == 0 && lane == 0) a.scale[row] = bad ? __builtin_nanf("") : live ? (float)(m * (double)rstd / MOST) : 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = c0 + s * STEP;
      if (c < a.d) {
        float w[8];
        load_weights(a.w, a.w32, c, a.d - c, w);
        i32x2 q = {0, 0};
        if (live) {
          if constexpr (OUT == OUT_INT8) {
            int n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = (int)__builtin_rint((double)h[s][i] * (double)w[i] * inv);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              q[i] = (n[4 * i] & 255) | ((n[4 * i + 1] & 255) << 8) | ((n[4 * i + 2] & 255) << 16) | (n[4 * i + 3] << 24);
          } else {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)((double)h[s][i] * (double)w[i] * inv);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
              q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], q[i], true);
            }
          }
        }
        store_bytes((uint8_t*)a.y + row * a.ys + c, a.d - c, q);
      }
    }
  }
}

// Backward pass.  With g = w dy:
//   dh = R (g - h R^2 mean(g h)) + dsum,   dw = sum over rows of R dy h.
// A team of WPR waves keeps its columns' share of dw in registers over the rows that it takes; a workgroup's teams add theirs, and the workgroups' shares
// go to `part` ([shares, d] FP32) and are summed in a fixed order by k_norm_dweight: no atomics, the same bits every time.
struct NormBackArgs {
  const void *dy, *h, *w, *dsum;
  void* dh;
  float* part;                       // NULL: no weight gradient
  int64_t rows, dys, hs, dss, dhs;
  int d, shares;                     // shares: workgroups
  float eps;
  bool w32;
};

template <class T, int WPR, int S>
__global__ __launch_bounds__(norm_threads(WPR)) void k_rms_norm_back(NormBackArgs a) {
  constexpr int RPG = norm_threads(WPR) / (64 * WPR);
  __shared__ f32x2 s_red[2][RPG][WPR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in_row = wave % WPR, slot = wave / WPR;
  const int team = blockIdx.x * RPG + slot, teams = a.shares * RPG;
  const int c0 = (in_row * 64 + lane) * 8;
  constexpr int STEP = WPR * 512;
  float w[S][8], dw[S][8];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    load_weights(a.w, a.w32, c0 + s * STEP, a.d - c0 - s * STEP, w[s]);   // (nothing is read beyond d)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[s][i] = 0.0f;
  }
  int phase = 0;
  for (int64_t row = team; row < a.rows; row += teams, phase ^= 1) {
    const T* dy = (const T*)a.dy + row * a.dys;
    const T* h = (const T*)a.h + row * a.hs;
    Octet<T> go[S], ho[S], so[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = c0 + s * STEP;
      if (c < a.d) {
        ho[s] = load_octet(h + c, a.d - c);
        go[s] = load_octet(dy + c, a.d - c);
        if (a.dsum) so[s] = load_octet((const T*)a.dsum + row * a.dss + c, a.d - c);
      }
    }
    const auto means = [&](float up) {               // of h^2 and g h, with h times `up`
      f32x2 both = {0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (c0 + s * STEP < a.d) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float hi = ho[s][i] * up;
            both[0] = __builtin_fmaf(hi, hi, both[0]);
            both[1] = __builtin_fmaf(go[s][i] * w[s][i], hi, both[1]);
          }
        }
      both[0] = wave_sum(both[0]);
      both[1] = wave_sum(both[1]);
      if constexpr (WPR > 1) {
        // two sets of slots: a wave that is a row ahead writes the other one, and two rows ahead lies behind the next barrier
        if (lane == 0) s_red[phase][slot][in_row] = both;
        __syncthreads();
        both = s_red[phase][slot][0];
#pragma unroll
        for (int i = 1; i < WPR; ++i) {
          both[0] += s_red[phase][slot][i][0];
          both[1] += s_red[phase][slot][i][1];
        }
      }
      return f32x2{both[0] / (float)a.d, both[1] / (float)a.d};
    };
    f32x2 mean = means(1.0f);
    float eps = a.eps, up = 1.0f;
    if (out_of_range(mean[0], eps, true)) {
      up = scale_into_range(mean[0]);
      if (WPR > 1) __syncthreads();  // (the slots have been read)
      mean = means(up);
      eps = eps * up * up;
    }
    // (R^3 leaves FP32 long before the gradient does: each factor R stands beside one that it brings back into range)
    const float Rup = 1.0f / sqrtf(mean[0] + eps), along = Rup * mean[1], R = Rup * up;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = c0 + s * STEP;
      if (c < a.d) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = go[s][i] * w[s][i], hR = ho[s][i] * R;
          f[i] = R * (g - hR * along);
          if (a.dsum) f[i] += so[s][i];
          dw[s][i] = __builtin_fmaf(go[s][i], hR, dw[s][i]);
        }
        store_octet((T*)a.dh + row * a.dhs + c, a.d - c, f);
      }
    }
  }
  if (!a.part) return;
  if constexpr (RPG > 1) {           // (WPR 1: lane for lane the same columns)
    __shared__ float s_dw[RPG - 1][S * 8][64];
    if (slot) {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) s_dw[slot - 1][8 * s + i][lane] = dw[s][i];
    }
    __syncthreads();
    if (slot) return;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int t = 0; t < RPG - 1; ++t) dw[s][i] += s_dw[t][8 * s + i][lane];
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int c = c0 + s * STEP;
    if (c < a.d) store_octet(a.part + (int64_t)blockIdx.x * a.d + c, a.d - c, dw[s]);
  }
}

// dw[c] = sum of the workgroups' shares: 16 columns a workgroup, 64 threads for each of them that take every 64th share, then their sums in order.
constexpr int kDweightCols = 16, kDweightLanes = 64, kDweightThreads = kDweightCols * kDweightLanes;
__global__ __launch_bounds__(kDweightThreads) static void k_norm_dweight(const float* __restrict__ part, int shares, int d, float* __restrict__ dw) {
  __shared__ float s[kDweightLanes][kDweightCols + 1];
  const int col = threadIdx.x % kDweightCols, from = threadIdx.x / kDweightCols, c = blockIdx.x * kDweightCols + col;
  float v = 0.0f;
  if (c < d)
#pragma unroll 4
    for (int t = from; t < shares; t += kDweightLanes) v += part[(int64_t)t * d + c];
  s[from][col] = v;
  __syncthreads();
#pragma unroll
  for (int n = kDweightLanes / 2; n >= 1; n /= 2) {
    if (from < n) s[from][col] = v += s[from + n][col];
    __syncthreads();
  }
  if (from == 0 && c < d) dw[c] = v;
}

}  // namespace elmo
