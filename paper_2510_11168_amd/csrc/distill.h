// Distillation from a teacher's top logits.  With p = softmax(z / T) over the V student logits of a row and q = softmax(t / T) over the
// teacher's tokens:
//   loss = v T^2 sum_j q_j (log q_j - log p_{i_j}),   dloss / dz_i = v T (p_i - sum_{j : i_j = i} q_j),   v = the row's weight.
//
// exp is taken as exp2(z c - m c) with c = log2(e) / T: c and m c are rounded once and enter every term of a row alike, so that what m c lost
// cancels; the sums over V are FP32, the loss's own terms (K of them) FP64.  A token at -infinity has p = 0; a row of weight 0 is not read.
#pragma once
#include "rows.h"

namespace elmo {

constexpr int kDistillMaxK = 1024;
constexpr int kDistillThreads = 1024;
constexpr double kLn2 = 0.6931471805599453;

struct DistillArgs {
  const void* z;
  const int32_t* ti;
  const void* tz;
  const float* v;                    // NULL: every row counts 1
  float* loss;
  void* grad;                        // NULL: none
  int64_t zs, gs;                    // row strides in elements
  int64_t V;
  int K;
  float T, c;                        // c = log2(e) / T
  bool t32;                          // FP32 teacher logits
};

// (maximum, sum of exp2((z - m) c)) of two parts of a row.  A part without a finite logit has m = -infinity and no sum.
struct MaxSum { float m, s; };
__device__ inline float shift(float m, float c) { return m == -__builtin_inff() ? 0.0f : m * c; }
__device__ inline MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m), mc = shift(m, c);
  return {m, a.s * __builtin_amdgcn_exp2f(__builtin_fmaf(a.m, c, -mc)) + b.s * __builtin_amdgcn_exp2f(__builtin_fmaf(b.m, c, -mc))};
}

template <class T>
__global__ __launch_bounds__(kDistillThreads) void k_distill_plain(DistillArgs a) {
  constexpr int NW = kDistillThreads / 64;
  __shared__ float s_m[NW], s_s[NW];
  __shared__ double s_d[NW];
  __shared__ float s_q[kDistillMaxK], s_z[kDistillMaxK];
  __shared__ int s_i[kDistillMaxK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const T* z = (const T*)a.z + row * a.zs;
  T* g = a.grad ? (T*)a.grad + row * a.gs : nullptr;
  const float v = a.v ? a.v[row] : 1.0f;
  // ---- teacher: q over the tokens that are there
  int idx = -1;
  float t = -__builtin_inff();
  if (tid < a.K) {
    idx = a.ti[row * a.K + tid];
    if (idx < 0 || idx >= a.V) idx = -1;
    else t = a.t32 ? ((const float*)a.tz)[row * a.K + tid] : bf16_decode(((const uint16_t*)a.tz)[row * a.K + tid]);
    if (!(t == t)) t = __builtin_inff();   // NaN teacher: NaN loss and gradient, by inf - inf
  }
  float m = wave_max(t);
  if (lane == 0) s_m[wave] = m;
  __syncthreads();
  m = s_m[0];
  for (int i = 1; i < NW; ++i) m = fmaxf(m, s_m[i]);
  if (m == -__builtin_inff() || v == 0.0f) {       // no teacher, or a row that does not count
    if (g)
      for (int64_t c = tid; c < a.V; c += kDistillThreads) store_one(g, c, 0.0f);
    if (tid == 0) a.loss[row] = 0.0f;
    return;
  }
  const double x = ((double)t - (double)m) / (double)a.T;
  double e = t == -__builtin_inff() ? 0.0 : exp(x);
  double sum = wave_reduce(e, [](double p, double q) { return p + q; });
  if (lane == 0) s_d[wave] = sum;
  __syncthreads();
  sum = 0.0;
  for (int i = 0; i < NW; ++i) sum += s_d[i];
  const double q = e / sum, logq = x - log(sum);
  // ---- student: maximum and sum
  float mine = -__builtin_inff(), part = 0.0f;
  for (int64_t c = tid; c < a.V; c += kDistillThreads) mine = fmaxf(mine, load_one(z, c));
  mine = wave_max(mine);
  __syncthreads();
  if (lane == 0) s_m[wave] = mine;
  __syncthreads();
  mine = s_m[0];
  for (int i = 1; i < NW; ++i) mine = fmaxf(mine, s_m[i]);
  const float mc = shift(mine, a.c);
  for (int64_t c = tid; c < a.V; c += kDistillThreads) part += __builtin_amdgcn_exp2f(__builtin_fmaf(load_one(z, c), a.c, -mc));
  part = wave_sum(part);
  if (lane == 0) s_s[wave] = part;
  const float zi = idx >= 0 ? load_one(z, idx) : 0.0f;
  s_i[tid] = idx;
  s_q[tid] = (float)q;
  s_z[tid] = zi;
  __syncthreads();
  part = 0.0f;
  for (int i = 0; i < NW; ++i) part += s_s[i];
  // ---- loss
  double term = 0.0;
  if (idx >= 0 && q != 0.0) term = q * (logq - kLn2 * ((double)zi * (double)a.c - (double)mc) + log((double)part));
  if (mine == -__builtin_inff()) term = idx >= 0 && q != 0.0 ? (double)__builtin_inff() : 0.0;
  term = wave_reduce(term, [](double p, double q) { return p + q; });
  __syncthreads();
  if (lane == 0) s_d[wave] = term;
  __syncthreads();
  if (tid == 0) {
    double l = 0.0;
    for (int i = 0; i < NW; ++i) l += s_d[i];
    a.loss[row] = (float)(l * (double)a.T * (double)a.T * (double)v);
  }
  if (!g) return;
  // ---- gradient
  const float scale = v * a.T, inv = part > 0.0f ? scale / part : part == 0.0f ? 0.0f : part;
  for (int64_t c = tid; c < a.V; c += kDistillThreads) store_one(g, c, __builtin_amdgcn_exp2f(__builtin_fmaf(load_one(z, c), a.c, -mc)) * inv);
  __syncthreads();
  if (idx >= 0) {
    float all = 0.0f;
    int first = tid;
    for (int j = 0; j < a.K; ++j)
      if (s_i[j] == idx) {
        first = min(first, j);
        all += s_q[j];
      }
    if (first == tid) store_one(g, idx, __builtin_amdgcn_exp2f(__builtin_fmaf(zi, a.c, -mc)) * inv - scale * all);
  }
}

}  // namespace elmo
