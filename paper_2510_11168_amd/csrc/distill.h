// Distillation from a teacher's top logits.  With p = softmax(z / T) over the V student logits of a row and q = softmax(t / T) over the
// teacher's tokens:
//   loss = v T^2 sum_j q_j (log q_j - log p_{i_j}),   dloss / dz_i = v T (p_i - sum_{j : i_j = i} q_j),   v = the row's weight.
//
// exp((z - m) / T) is taken as exp2((z - m) c) with c = log2(e) / T; the difference first, so that rows of the type's lowest value, whose product with c
// overflows, are rows like others.  The exponentials are FP32 and summed in octets, the octets' sums and the loss's own terms (K of them) FP64: a
// loss is a small difference where student and teacher agree.  A token at -infinity has p = 0; a row of weight 0 is not read.
#pragma once
#include "rows.h"

namespace elmo {

constexpr int kDistillMaxK = 1024;
constexpr int kDistillThreads = 512;

struct DistillArgs {
  const void* z;
  const int32_t* ti;
  const void* tz;
  const float* v;                    // NULL: every row counts 1
  float* loss;
  void* grad;                        // NULL: none
  int64_t zs, gs;                    // row strides in elements
  int64_t rows, V;
  int K;
  float T, c;                        // c = log2(e) / T
  bool t32;                          // FP32 teacher logits
  int parts;                         // workgroups of a row
  void* ws;                          // of split rows: [rows, parts] MaxSum, [rows, kDistillMaxK] logits of the teacher's tokens
};

// (maximum, sum of exp2((z - base(m)) c)) of a part of a row.  A part without a finite logit has m = -infinity and no sum.
struct MaxSum { double s; float m; };
__device__ inline float base(float m) { return m == -__builtin_inff() ? 0.0f : m; }
__device__ inline float power(float z, float from, float c) { return __builtin_amdgcn_exp2f((z - from) * c); }
__device__ inline double rescale(float m, float to, float c) { return m == -__builtin_inff() ? 0.0 : (double)power(m, base(to), c); }

// The exponentials of an octet, summed.
template <class T> __device__ inline float octet_sum(const Octet<T>& o, float from, float c) {
  float e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = power(o[i], from, c);
  return ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
}
template <class T> __device__ inline float octet_max(const Octet<T>& o) {
  return fmaxf(fmaxf(fmaxf(o[0], o[1]), fmaxf(o[2], o[3])), fmaxf(fmaxf(o[4], o[5]), fmaxf(o[6], o[7])));
}
// Octets [lo, hi) of part `part` of `parts`, in whole rounds of a workgroup.
struct Range { int64_t lo, hi; };
__device__ inline Range part_of(int64_t octets, int part, int parts) {
  const int64_t rounds = (octets + kDistillThreads - 1) / kDistillThreads, per = (rounds + parts - 1) / parts;
  const int64_t lo = min(octets, per * part * kDistillThreads);
  return {lo, min(octets, lo + per * kDistillThreads)};
}

// WHOLE: a row a workgroup.  It is read twice -- 256 rows of a large vocabulary that are worked on at a time fit the memory-side cache, from
// which the second reading comes -- and the gradient goes past the caches.  4096 x 131072 BF16: 498 to 527 us, 4.1 to 4.3 TB/s of what has
// to move (a copy: 4.8); rows held in registers, with the next one's loads under way as the gradient is written: 559 to 652.
// SUMS, GRADIENT: few rows, in `parts` workgroups each: the parts' maxima and sums with the teacher's tokens' logits, then the gradient with them.  (The
// second launch takes no logit that another part may already have overwritten.)  One row of 131072: see the launch.
enum : int { DISTILL_WHOLE = 0, DISTILL_SUMS = 1, DISTILL_GRADIENT = 2 };
template <class T, int MODE>
__global__ __launch_bounds__(kDistillThreads) void k_distill(DistillArgs a) {
  constexpr int NT = kDistillThreads, NW = NT / 64, PER = kDistillMaxK / NT;
  __shared__ float s_m[NW], s_t[NW], s_q[kDistillMaxK], s_z[kDistillMaxK];
  __shared__ double s_s[NW], s_d[NW], s_l[NW], s_x[kDistillMaxK], s_e[kDistillMaxK];
  __shared__ int s_i[kDistillMaxK], s_seen[2 * kDistillMaxK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = MODE == DISTILL_WHOLE ? blockIdx.x : blockIdx.x / a.parts;
  const int part = MODE == DISTILL_WHOLE ? 0 : (int)(blockIdx.x % a.parts);
  const T* z = (const T*)a.z + row * a.zs;
  T* g = a.grad ? (T*)a.grad + row * a.gs : nullptr;
  // whole octets; the up to seven elements behind them go to as many threads of the last part, one each
  const int64_t octets = a.V >> 3, rest = octets * 8;
  const Range r = MODE == DISTILL_WHOLE ? Range{0, octets} : part_of(octets, part, a.parts);
  const int tail = part == a.parts - 1 ? (int)(a.V - rest) : 0;
  MaxSum* partials = (MaxSum*)a.ws + row * a.parts;
  float* token_z = (float*)((MaxSum*)a.ws + a.rows * a.parts) + row * kDistillMaxK;
  const float v = a.v ? a.v[row] : 1.0f;
  const auto zeros = [&]() {                             // of a row without a teacher, or one that does not count
    if (MODE == DISTILL_SUMS) return;
    if (g) {
      const float zero[8] = {};
      for (int64_t o = r.lo + tid; o < r.hi; o += NT) store_octet<true>(g + o * 8, 8, zero);
      if (tid < tail) store_one(g, rest + tid, 0.0f);
    }
    if (tid == 0 && part == 0) a.loss[row] = 0.0f;
  };
  if (v == 0.0f) return zeros();
  // a table of the teacher's tokens, at least twice as large as they are many: which of them come more than once
  int bits = 6;
  while ((1 << bits) < 2 * a.K) ++bits;
  const auto first_slot = [&](int token) { return (int)(((uint32_t)token * 2654435761u) >> (32 - bits)); };
  constexpr int kTwice = (int)0x80000000;
  if (MODE != DISTILL_SUMS)
    for (int i = tid; i < 1 << bits; i += NT) s_seen[i] = -1;
  // ---- the teacher's tokens go out first, their logits of the student behind its row: two trips to memory that nothing waits for
  int at[PER];
  float t[PER], zi[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = i * NT + tid;
    at[i] = -1;
    t[i] = -__builtin_inff();
    if (j < a.K) {
      at[i] = a.ti[row * a.K + j];
      t[i] = a.t32 ? ((const float*)a.tz)[row * a.K + j] : bf16_decode(((const uint16_t*)a.tz)[row * a.K + j]);
    }
  }
  // ---- student: maximum and sum in one pass
  const float last = tid < tail ? load_one(z, rest + tid) : -__builtin_inff();
  MaxSum ms = {0.0, -__builtin_inff()};
  if constexpr (MODE != DISTILL_GRADIENT) {
    if (tid < tail) {
      if (last == last) ms.m = last;                     // (a NaN is in the sum)
      ms.s = power(last, base(ms.m), a.c);
    }
#pragma unroll 4
    for (int64_t o = r.lo + tid; o < r.hi; o += NT) {
      const Octet<T> oc = load_octet(z + o * 8, 8);
      const float top = octet_max(oc);
      if (top > ms.m) ms = {ms.s * rescale(ms.m, top, a.c), top};
      ms.s += (double)octet_sum(oc, base(ms.m), a.c);
    }
  }
  float m = -__builtin_inff();                           // the teacher's largest logit
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = i * NT + tid;
    if (!(t[i] == t[i])) t[i] = __builtin_inff();        // a NaN teacher makes the row NaN, by inf - inf
    if (at[i] < 0 || at[i] >= a.V) { at[i] = -1; t[i] = -__builtin_inff(); }
    zi[i] = 0.0f;
    if (MODE == DISTILL_GRADIENT) zi[i] = j < a.K ? token_z[j] : 0.0f;
    else if (at[i] >= 0) zi[i] = load_one(z, at[i]);
    if (MODE == DISTILL_SUMS && part == 0 && j < a.K) token_z[j] = zi[i];
    m = fmaxf(m, t[i]);
  }
  if constexpr (MODE != DISTILL_GRADIENT) {
    const float top = wave_max(ms.m);
    ms = {wave_sum64(ms.s * rescale(ms.m, top, a.c)), top};
    if (lane == 0) {
      s_m[wave] = ms.m;
      s_s[wave] = ms.s;
    }
  }
  m = wave_max(m);
  if (lane == 0) s_t[wave] = m;
  if (MODE != DISTILL_SUMS) {
    __syncthreads();                                     // (the table is empty)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = i * NT + tid;
      if (j < a.K) {
        s_i[j] = at[i];
        s_x[j] = (double)t[i];
        s_z[j] = zi[i];
      }
      if (at[i] >= 0)
        for (int h = first_slot(at[i]);; h = (h + 1) & ((1 << bits) - 1)) {     // (ends: half of the table stays empty)
          const int there = atomicCAS(&s_seen[h], -1, at[i]);
          if (there == -1) break;
          if ((there & ~kTwice) == at[i]) {
            atomicOr(&s_seen[h], kTwice);
            break;
          }
        }
    }
  }
  __syncthreads();
  m = slots_reduce<NW>(s_t, lane, [](float p, float q) { return fmaxf(p, q); });
  if constexpr (MODE != DISTILL_GRADIENT) {
    ms.m = slots_reduce<NW>(s_m, lane, [](float p, float q) { return fmaxf(p, q); });
    ms.s = wave_reduce<NW>(s_s[lane & (NW - 1)] * rescale(s_m[lane & (NW - 1)], ms.m, a.c), [](double p, double q) { return p + q; });
    if (MODE == DISTILL_SUMS) {
      if (tid == 0) partials[part] = ms;
      return;
    }
  } else {
    const MaxSum mine = lane < a.parts ? partials[lane] : ms;    // (at most 64 parts)
    ms.m = wave_max(mine.m);
    ms.s = wave_sum64(mine.s * rescale(mine.m, ms.m, a.c));
  }
  if (m == -__builtin_inff()) return zeros();
  const float from_z = base(ms.m);
  // ---- gradient: p everywhere
  const float vT = v * a.T, inv = ms.s == 0.0 ? 0.0f : vT / (float)ms.s;
  const auto p_of = [&](float f) { return power(f, from_z, a.c) * inv; };
  if (g) {
    if (tid < tail) store_one(g, rest + tid, p_of(last));
#pragma unroll 4
    for (int64_t o = r.lo + tid; o < r.hi; o += NT) {
      const Octet<T> oc = load_octet(z + o * 8, 8);
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = p_of(oc[i]);
      store_octet<true>(g + o * 8, 8, f);
    }
  }
  // ---- loss: the teacher's q, and log p of its tokens
  double sum = 0.0;
#pragma unroll 1
  for (int j = tid; j < a.K; j += NT) {
    const double x = (s_x[j] - (double)m) / (double)a.T, e = s_x[j] == -__builtin_inf() ? 0.0 : exp_series(x);
    s_x[j] = x;
    s_e[j] = e;
    sum += e;
  }
  sum = wave_reduce(sum, [](double p, double q) { return p + q; });
  if (lane == 0) s_d[wave] = sum;
  __syncthreads();
  sum = slots_reduce<NW>(s_d, lane, [](double p, double q) { return p + q; });
  const double logsum = log_series(sum), lognorm = log_series(ms.s);
  double loss = 0.0;
#pragma unroll 1
  for (int j = tid; j < a.K; j += NT) {
    const double q = s_e[j] / sum;
    if (s_i[j] >= 0 && !(q == 0.0))
      loss += ms.m == -__builtin_inff() ? (double)__builtin_inff() : q * (s_x[j] - logsum - ((double)s_z[j] - (double)from_z) / (double)a.T + lognorm);
    s_q[j] = (float)q;
  }
  loss = wave_reduce(loss, [](double p, double q) { return p + q; });
  if (lane == 0) s_l[wave] = loss;
  __syncthreads();                                       // also orders the octets' stores before the ones below
  loss = slots_reduce<NW>(s_l, lane, [](double p, double q) { return p + q; });
  if (tid == 0 && part == 0) a.loss[row] = (float)(loss * (double)a.T * (double)a.T * (double)v);
  if (!g) return;
  // ---- the teacher's tokens once more, each by the part that wrote it; of equal ones the first, for all
  const int64_t from = r.lo * 8, to = r.hi * 8 + tail;
#pragma unroll 1
  for (int k = tid; k < a.K; k += NT) {
    const int token = s_i[k];
    if (token < 0 || token < from || token >= to) continue;
    int h = first_slot(token);
    while ((s_seen[h] & ~kTwice) != token) h = (h + 1) & ((1 << bits) - 1);
    float all = s_q[k];
    if (s_seen[h] < 0) {
      int first = k;
      all = 0.0f;
#pragma unroll 8
      for (int j = 0; j < a.K; ++j) {                    // (without branches: the reads of several tokens are under way together)
        const bool same = s_i[j] == token;
        first = same ? min(first, j) : first;
        all += same ? s_q[j] : 0.0f;
      }
      if (first != k) continue;
    }
    store_one(g, token, p_of(s_z[k]) - vT * all);
  }
}

}  // namespace elmo
