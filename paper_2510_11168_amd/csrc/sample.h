// One token a row by temperature, top-k, top-p and min-p, from a given random number.
//
// Tokens are ordered by (logit falling, index rising), as 64-bit places: an order-preserving key of the logit above the complement of the index.
// Every filter keeps a beginning of that order, so the kept set is what lies at or above one place (`edge`), and for min-p has at least a
// smallest weight.  The token is the first one in order of index at which the kept weight so far exceeds u times the kept weight.
//
// Which token a number falls on is decided next to borders, so the weights are whole numbers, W = round(2^F exp((z - max z) / t)) from FP64, with
// F such that a row's sum stays below 2^63: sums are exact in any order and any split of a row gives the same token.
//
// Bound: a row is read two to four times, by one workgroup, and stays in the caches for the second time on; where many tokens are kept it is the
// weights' arithmetic (some twenty FP64 and integer instructions each).  What is done, by the row's settings:
//   top_k <= 512   the k-th largest of the threads' maxima bounds the k-th token from below; the few tokens above it go to a list in LDS,
//                  which is sorted, filtered and drawn from: two readings, no weights but the list's;
//   top_p, top_k   counts and weights over bins of 1/32 octave of weight, then the tokens of the bin in which the filter ends, sorted (a bin
//                  that holds too many: a radix search over their places); three readings, four with both;
//   always         sums of the kept weights over segments of the row, and the token inside the segment on which the number falls.
#pragma once
#include "rows.h"

namespace elmo {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kSampleShortK = 512;             // largest top_k that goes by the threads' maxima
constexpr int kSampleList = 4096;              // places of the list in LDS; segments of a row
constexpr int kSampleBins = 2048;              // 1/32 octave each: 64 octaves, more than weights have
constexpr uint32_t kKeyNone = 0x007FFFFFu;     // key of -infinity: never kept

struct SampleArgs {
  const void* z;
  int64_t zs, V;
  const float *u, *t, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* prob;
  int F;
};

// Rises with the logit; -0 counts as +0, NaN as -infinity.
__device__ inline uint32_t key_of(float z) {
  const uint32_t b = f2u(z + 0.0f);
  const uint32_t k = (int32_t)b < 0 ? ~b : b | 0x80000000u;
  return z == z ? k : kKeyNone;
}
__device__ inline float of_key(uint32_t k) { return u2f((int32_t)k < 0 ? k & 0x7FFFFFFFu : ~k); }
__device__ inline uint64_t place_of(float z, int64_t index) { return (uint64_t)key_of(z) << 32 | (uint32_t)~(uint32_t)index; }

// Weight of a logit: y = (z - M) 256 log2(e) / t = n + r, 2^(n / 256) by a table of the 256 roots and the exponent, 2^(r / 256) by its series up to
// r^3 (the next term is below 2^-42).  NaN and -infinity end at the lower bound, which rounds to no weight.
struct Weigh {
  const double* roots;                         // 2^(i / 256), in LDS
  double M, k, least;                          // maximum, 256 log2(e) / t, lower bound of y
  int F;
  __device__ inline int steps(double y, double& r) const {       // n
    constexpr double magic = 6755399441055744.0;                 // 1.5 2^52: its sum's low bits are the nearest whole number
    const double s = y + magic;
    r = y - (s - magic);
    return (int)(uint32_t)__double_as_longlong(s);
  }
  __device__ inline uint64_t operator()(float z, int& n) const {
    constexpr double c = 0.6931471805599453 / 256;
    double r;
    n = steps(__builtin_fmax(((double)z - M) * k, least), r);
    const double p = __builtin_fma(__builtin_fma(__builtin_fma(c * c * c / 6, r, c * c / 2), r, c), r, 1.0);
    const double w = __builtin_ldexp(p * roots[n & 255], (n >> 8) + F);
    return (uint64_t)__double_as_longlong(w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;   // + 2^52: rounded to a whole number
  }
  __device__ inline uint64_t operator()(float z) const { int n; return (*this)(z, n); }
  __device__ inline int bin(int n) const { return min(-n >> 3, kSampleBins - 1); }        // 0: the largest weights
};

template <class T> __device__ inline T lowest();                       // -infinity
template <> __device__ inline uint16_t lowest<uint16_t>() { return 0xFF80u; }
template <> __device__ inline float lowest<float>() { return -__builtin_inff(); }

struct RowSettings {
  int64_t k;
  double p, mp, u, t;
};
__device__ inline RowSettings settings_of(const SampleArgs& a, int64_t row) {
  RowSettings s;
  const float t = a.t ? a.t[row] : 1.0f;
  const int32_t k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.0f, mp = a.min_p ? a.min_p[row] : 0.0f, u = a.u[row];
  const bool greedy = !(t > 0.0f);
  s.t = greedy ? 1.0 : (double)t;
  s.k = greedy ? 1 : k > 0 && k < a.V ? k : a.V;
  s.p = p < 1.0f ? (double)p : 1.0;            // NaN: off
  s.mp = mp > 0.0f ? (mp < 1.0f ? (double)mp : 1.0) : 0.0;
  s.u = u > 0.0f ? (double)u : 0.0;
  return s;
}
__device__ inline uint64_t share_of(double part, uint64_t whole) {   // ceil(part whole), at least 1 and at most the whole
  return min(whole, max((uint64_t)1, (uint64_t)__builtin_ceil(part * (double)whole)));
}

template <class U> __device__ inline U wave_scan(U v, int lane) {    // inclusive
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const U other = __shfl_up(v, o);
    if (lane >= o) v += other;
  }
  return v;
}
// Inclusive sums over the workgroup's threads, and their total.  Barriers before and behind the use of `slots`.
template <class U> __device__ inline U block_scan(U v, U* slots, int wave, int lane, U& total) {
  v = wave_scan(v, lane);
  __syncthreads();
  if (lane == 63) slots[wave] = v;
  __syncthreads();
  const U mine = lane < kSampleWaves ? slots[lane] : 0, upto = wave_scan(mine, lane);
  total = __shfl(upto, kSampleWaves - 1);
  return v + __shfl(upto - mine, wave);
}
// Falling order; `n` a power of two, by the whole workgroup.  Barriers before and behind.
__device__ inline void sort_falling(uint64_t* s, int n, int tid) {
  for (int k = 2; k <= n; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      __syncthreads();
      for (int i = tid; i < n / 2; i += kSampleThreads) {
        const int lo = 2 * i - (i & (j - 1)), hi = lo + j;       // lo: bit j clear
        const uint64_t x = s[lo], y = s[hi];
        if ((x < y) == ((lo & k) == 0)) {
          s[lo] = y;
          s[hi] = x;
        }
      }
    }
  __syncthreads();
}

// The list in falling order, s_list[0, n) with n <= kSampleCount: every place's rank is the number of larger ones, counted by as many threads as there are
// for it (64 places: 0.3 us; the exchanges of a sort are a barrier each).  `rank` has kSampleCount entries.  Barriers before and behind.
constexpr int kSampleCount = 256;
template <class F> __device__ inline void for_pairs(int n, int tid, F&& f) {     // f(i, a stretch [from, to) of the others), all of them once
  int size = 1;
  while (size < n) size *= 2;
  const int i = tid & (size - 1), parts = kSampleThreads / size, per = (n + parts - 1) / parts, from = tid / size * per;
  if (i < n && from < n) f(i, from, min(n, from + per));
}
__device__ inline void rank_falling(uint64_t* list, uint32_t* rank, int n, int tid) {
  if (tid < kSampleCount) rank[tid] = 0;
  __syncthreads();
  const uint64_t mine = tid < n ? list[tid] : 0;
  for_pairs(n, tid, [&](int i, int from, int to) {
    const uint64_t x = list[i];
    uint32_t larger = 0;
    for (int j = from; j < to; ++j) larger += list[j] > x;
    if (larger) atomicAdd(&rank[i], larger);
  });
  __syncthreads();
  if (tid < n) list[rank[tid]] = mine;
  __syncthreads();
}

template <class T>
__global__ __launch_bounds__(kSampleThreads) void k_sample(SampleArgs a) {
  constexpr int NT = kSampleThreads;
  __shared__ uint64_t s_list[kSampleList], s_mass[kSampleBins], s_sum[kSampleWaves];
  __shared__ uint32_t s_count[kSampleBins], s_sum32[kSampleWaves];
  __shared__ double s_root[256];
  __shared__ float s_max[kSampleWaves];
  __shared__ uint64_t s_found[3];
  __shared__ int s_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x, octets = (a.V + 7) >> 3;
  const T* z = (const T*)a.z + row * a.zs;
  const RowSettings rs = settings_of(a, row);
  // an octet's logits; beyond the row -infinity.  Where the largest is +infinity only that has a weight: 0 stands for it, -infinity for the others.
  bool infinite = false;
  const auto load8 = [&](int64_t o, float (&f)[8]) {
    const Octet<T> oc = load_octet(z + o * 8, a.V - o * 8, lowest<T>());
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = oc[i];
    if (infinite) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = f[i] == __builtin_inff() ? 0.0f : -__builtin_inff();
    }
  };
  const auto max8 = [](const float (&f)[8]) { return fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7]))); };
  // ---- largest logit, and each thread's
  if (tid < 256) s_root[tid] = exp_series(tid * (kLn2 / 256));
  float mine = -__builtin_inff();
#pragma unroll 8
  for (int64_t o = tid; o < octets; o += NT) {
    float f[8];
    load8(o, f);
    mine = fmaxf(mine, max8(f));
  }
  float M = wave_max(mine);
  if (lane == 0) s_max[wave] = M;
  if (tid == 0) s_n = 0;
  __syncthreads();
  M = slots_reduce<kSampleWaves>(s_max, lane, [](float p, float q) { return fmaxf(p, q); });
  const auto answer = [&](int64_t token, float prob) {
    a.token[row] = (int32_t)token;
    if (a.prob) a.prob[row] = prob;
  };
  if (M == -__builtin_inff()) {
    if (tid == 0) answer(-1, 0.0f);
    return;
  }
  if (M == __builtin_inff()) {
    infinite = true;
    M = 0.0f;
    mine = mine == __builtin_inff() ? 0.0f : -__builtin_inff();
  }
  const Weigh weigh{s_root, (double)M, 256.0 * kLog2e / rs.t, -256.0 * (a.F + 2), a.F};
  const uint64_t one = 1ull << a.F, least = rs.mp > 0.0 ? share_of(rs.mp, one) : 1;
  uint64_t edge = (uint64_t)(kKeyNone + 1) << 32;        // kept: places from here on
  float low = -__builtin_inff();                         // no kept logit lies below this
  // appends what keep(logit, octet's first index + i) names among the octets whose largest logit is at least `from` to the list
  const auto collect = [&](float from, auto&& keep) {
#pragma unroll 4
    for (int64_t o = tid; o < octets; o += NT) {
      float f[8];
      load8(o, f);
      if (max8(f) >= from) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (f[i] >= from && keep(f[i])) {
            const int at = atomicAdd(&s_n, 1);
            if (at < kSampleList) s_list[at] = place_of(f[i], o * 8 + i);
          }
      }
    }
    __syncthreads();
  };
  const auto pad_and_sort = [&](int n) {                 // the list, to the next power of two
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) s_list[i] = 0;
    sort_falling(s_list, size, tid);
  };

  if (rs.k <= kSampleShortK) {
    // ---- few tokens stay: bound, list, sort, filter, draw
    float from = M;
    if (rs.k > 1) {
      // 16 bits of the k-th largest of the threads' maxima, 8 at a time
      uint32_t prefix = 0, left = (uint32_t)rs.k;
      const uint32_t key = key_of(mine);
      for (int sh = 24; sh >= 16; sh -= 8) {
        if (tid < 256) s_count[tid] = 0;
        __syncthreads();
        if (key > kKeyNone && (sh == 24 || key >> 24 == prefix >> 24)) atomicAdd(&s_count[(key >> sh) & 255], 1u);
        __syncthreads();
        if (wave == 0) {                                 // four bins a lane, the largest first
          uint32_t c[4], sum = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += c[i] = s_count[255 - 4 * lane - i];
          uint32_t before = wave_scan(sum, lane) - sum;
          if (lane == 63) s_found[0] = before + sum < left ? ~0ull : 0;      // fewer maxima than k: every token is taken
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (before < left && before + c[i] >= left) { s_found[1] = 255 - 4 * lane - i; s_found[2] = before; }
            before += c[i];
          }
        }
        __syncthreads();
        if (s_found[0]) { prefix = 0; break; }
        prefix |= (uint32_t)s_found[1] << sh;
        left -= (uint32_t)s_found[2];
        __syncthreads();
      }
      from = of_key(max(prefix, kKeyNone + 1));
    }
    if (rs.k == 1) {
      // the largest logit's first place
      uint32_t first = ~0u;
      for (int64_t o = tid; o < octets; o += NT) {
        float f[8];
        load8(o, f);
#pragma unroll
        for (int i = 7; i >= 0; --i)
          if (f[i] == M) first = min(first, (uint32_t)(o * 8 + i));
      }
      first = wave_reduce(first, [](uint32_t p, uint32_t q) { return min(p, q); });
      if (lane == 0) s_sum32[wave] = first;
      __syncthreads();
      first = slots_reduce<kSampleWaves>(s_sum32, lane, [](uint32_t p, uint32_t q) { return min(p, q); });
      if (tid == 0) answer(first, 1.0f);
      return;
    }
    collect(from, [](float f) { return f > -__builtin_inff(); });
    const int n = s_n;
    if (n <= kSampleList) {
      if (n <= kSampleCount) rank_falling(s_list, s_count, n, tid);
      else pad_and_sort(n);
      const int nk = (int)min((int64_t)n, rs.k);         // at most 512: one a thread
      const uint64_t place = tid < nk ? s_list[tid] : 0, w = tid < nk ? weigh(of_key(place >> 32)) : 0;
      uint64_t total;
      const uint64_t upto = block_scan(w, s_sum, wave, lane, total);
      const bool kept = w >= least && (rs.p >= 1.0 || upto - w < share_of(rs.p, total));
      uint64_t all;
      block_scan(kept ? w : 0, s_sum, wave, lane, all);
      uint64_t want = (uint64_t)(rs.u * (double)all);
      if (want >= all) want = all - 1;
      // what is kept before a token by index: of few by pairs, else along the list sorted by index
      if (tid < kSampleShortK) {
        s_mass[tid] = kept ? w : 0;
        s_mass[kSampleShortK + tid] = 0;
        if (nk > kSampleCount) s_list[tid] = kept ? place << 32 | (uint32_t)tid : 0;
      }
      __syncthreads();
      if (nk <= kSampleCount) {
        for_pairs(nk, tid, [&](int i, int from, int to) {
          const uint32_t x = (uint32_t)s_list[i];        // the complement of the index
          uint64_t sum = 0;
          for (int j = from; j < to; ++j) sum += (uint32_t)s_list[j] > x ? s_mass[j] : 0;
          if (sum) atomicAdd((unsigned long long*)&s_mass[kSampleShortK + i], (unsigned long long)sum);
        });
        __syncthreads();
        const uint64_t before = tid < nk ? s_mass[kSampleShortK + tid] : 0;
        if (kept && before <= want && before + w > want) answer((int64_t)(uint32_t)~(uint32_t)place, (float)((double)w / (double)all));
        return;
      }
      sort_falling(s_list, kSampleShortK, tid);
      const uint64_t entry = tid < kSampleShortK ? s_list[tid] : 0;
      // (an entry of 0 would be index 2^32 - 1, which no row has)
      const uint64_t wi = entry ? s_mass[(uint32_t)entry] : 0;
      const uint64_t by_index = block_scan(wi, s_sum, wave, lane, all);
      if (wi && by_index > want && by_index - wi <= want) answer((int64_t)(uint32_t)~(uint32_t)(entry >> 32), (float)((double)wi / (double)all));
      return;
    }
    __syncthreads();
    if (tid == 0) s_n = 0;
  }

  if (rs.k < a.V || rs.p < 1.0) {
    // ---- weights, and with top-k counts, over bins
    const bool by_count = rs.k < a.V;
    for (int i = tid; i < kSampleBins; i += NT) {
      s_mass[i] = 0;
      s_count[i] = 0;
    }
    __syncthreads();
    for (int64_t o = tid; o < octets; o += NT) {
      float f[8];
      load8(o, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int n;
        const uint64_t w = weigh(f[i], n);
        if (w) {
          atomicAdd((unsigned long long*)&s_mass[weigh.bin(n)], (unsigned long long)w);
          if (by_count) atomicAdd(&s_count[weigh.bin(n)], 1u);
        }
      }
    }
    __syncthreads();
    uint64_t total;
    const uint64_t m0 = s_mass[2 * tid], m1 = s_mass[2 * tid + 1];
    uint64_t mass_before = block_scan(m0 + m1, s_sum, wave, lane, total) - m0 - m1;
    // The place at which a filter ends: the smallest beginning of the order with `want` tokens or weight.  Returns the weight from it on.
    const auto end_in = [&](bool mass, uint64_t want, uint64_t before, uint64_t c0, uint64_t c1, uint64_t above_mass) {
      __syncthreads();
      if (before < want && before + c0 >= want) { s_found[0] = 2 * tid; s_found[1] = before; s_found[2] = above_mass; }
      if (before + c0 < want && before + c0 + c1 >= want) { s_found[0] = 2 * tid + 1; s_found[1] = before + c0; s_found[2] = above_mass + m0; }
      if (tid == 0) s_n = 0;
      __syncthreads();
      const int bin = (int)s_found[0];
      uint64_t above = s_found[1], mass_above = s_found[2];
      __syncthreads();
      const auto in_bin = [&](float f) { int n; return weigh(f, n) != 0 && weigh.bin(n) == bin; };
      // (bounds of the bin's logits with room for y's rounding, so that the other octets are passed over)
      collect((float)((double)M + (-8.0 * bin - 9.0) / weigh.k) - 1e-5f * fabsf(M), in_bin);
      const int n = s_n;
      __syncthreads();
      if (n <= kSampleList) {
        pad_and_sort(n);
        // four a thread
        uint64_t w[4], sum = 0, whole;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += w[i] = 4 * tid + i < n ? weigh(of_key(s_list[4 * tid + i] >> 32)) : 0;
        uint64_t upto = mass_above + block_scan(sum, s_sum, wave, lane, whole) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = 4 * tid + i;
          const bool here = at < n && (mass ? upto < want && upto + w[i] >= want : above + at + 1 == want);
          upto += w[i];
          if (here) { s_found[0] = s_list[at]; s_found[1] = upto; }
        }
      } else {
        // too many for the list: a radix search over the bin's places, 8 bits at a time
        uint64_t prefix = 0;
        for (int sh = 56; sh >= 0; sh -= 8) {
          __syncthreads();
          if (tid < 256) { s_list[tid] = 0; s_list[256 + tid] = 0; }
          __syncthreads();
          for (int64_t o = tid; o < octets; o += NT) {
            float f[8];
            load8(o, f);
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
              const uint64_t p = place_of(f[i], o * 8 + i);
              if (in_bin(f[i]) && (sh == 56 || p >> (sh + 8) == prefix >> (sh + 8))) {
                atomicAdd((unsigned long long*)&s_list[(p >> sh) & 255], (unsigned long long)weigh(f[i]));
                atomicAdd((unsigned long long*)&s_list[256 + ((p >> sh) & 255)], 1ull);
              }
            }
          }
          __syncthreads();
          if (tid == 0) {
            int b = 255;
            for (; b > 0; --b) {
              if ((mass ? mass_above + s_list[b] : above + s_list[256 + b]) >= want) break;
              above += s_list[256 + b];
              mass_above += s_list[b];
            }
            s_found[0] = b; s_found[1] = above; s_found[2] = mass_above;
            if (sh == 0) s_list[0] = mass_above + s_list[b];
          }
          __syncthreads();
          prefix |= s_found[0] << sh;
          above = s_found[1];
          mass_above = s_found[2];
        }
        if (tid == 0) { s_found[0] = prefix; s_found[1] = s_list[0]; }
      }
      __syncthreads();
      edge = s_found[0];
      low = of_key(edge >> 32);
      return s_found[1];
    };
    if (by_count) {
      uint64_t live;
      const uint64_t n0 = s_count[2 * tid], n1 = s_count[2 * tid + 1];
      const uint64_t before = block_scan(n0 + n1, s_sum, wave, lane, live) - n0 - n1;
      if ((uint64_t)rs.k < live) total = end_in(false, (uint64_t)rs.k, before, n0, n1, mass_before);
    }
    if (rs.p < 1.0) end_in(true, share_of(rs.p, total), mass_before, m0, m1, mass_before);
  }

  // ---- kept weight by segments of the row, each a wave's: 512 elements, or as many times that as the list has places for
  __syncthreads();
  const int64_t rounds = (octets + 63) / 64, per = (rounds + kSampleList - 1) / kSampleList;
  const int segments = (int)((rounds + per - 1) / per);
  const auto kept8 = [&](int64_t o, uint64_t (&w)[8]) {  // weights of an octet's kept tokens; their sum
    uint64_t sum = 0;
    float f[8];
    const bool in = o < octets;
    if (in) load8(o, f);
    if (in && max8(f) >= low) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = weigh(f[i]);
        if (w[i] < least || place_of(f[i], o * 8 + i) < edge) w[i] = 0;
        sum += w[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 0;
    }
    return sum;
  };
  for (int s = wave; s < segments; s += kSampleWaves) {
    uint64_t sum = 0, w[8];
    for (int64_t i = 0; i < per; ++i) sum += kept8((s * per + i) * 64 + lane, w);
    sum = wave_reduce(sum, [](uint64_t p, uint64_t q) { return p + q; });
    if (lane == 0) s_list[s] = sum;
  }
  __syncthreads();
  uint64_t w4[4], sum = 0, all;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum += w4[i] = 4 * tid + i < segments ? s_list[4 * tid + i] : 0;
  uint64_t before = block_scan(sum, s_sum, wave, lane, all) - sum;
  uint64_t want = (uint64_t)(rs.u * (double)all);
  if (want >= all) want = all - 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (before <= want && before + w4[i] > want) { s_found[0] = 4 * tid + i; s_found[1] = before; }
    before += w4[i];
  }
  __syncthreads();
  if (wave != 0) return;
  // ---- and the token inside its segment
  before = s_found[1];
  for (int64_t i = 0; i < per; ++i) {
    const int64_t o = ((int64_t)s_found[0] * per + i) * 64 + lane;
    uint64_t w[8];
    const uint64_t mine8 = kept8(o, w), upto = wave_scan(mine8, lane);
    uint64_t at = before + upto - mine8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (at <= want && at + w[j] > want) answer(o * 8 + j, (float)((double)w[j] / (double)all));
      at += w[j];
    }
    before += __shfl(upto, 63);
  }
}

}  // namespace elmo
