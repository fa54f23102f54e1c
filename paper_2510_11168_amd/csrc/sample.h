// One token a row by temperature, top-k, top-p and min-p, from a given random number.
//
// Tokens are ordered by (logit falling, index rising), as 64-bit places: an order-preserving key of the logit above the complement of the index.
// Every filter keeps a beginning of that order, so the kept set is what lies at or above one place (`edge`), and for min-p has at least a
// smallest weight.  The token is the first one in order of index at which the kept weight so far exceeds u times the kept weight.
//
// Which token a number falls on is decided next to borders, so the weights are whole numbers, W = round(2^F exp((z - max z) / t)) from FP64, with
// F such that a row's sum stays below 2^63: sums are exact in any order and any split of a row gives the same token.  A token's share is its FP64
// weight over that sum: few bits of a light token's W are left.
//
// Bound: a row is read two to four times, by one workgroup, and stays in the caches for the second time on; where many tokens are kept it is the
// weights' arithmetic (some twenty FP64 and integer instructions each).  256 x 131072 in us, BF16 and FP32: greedy (two plain readings) 23 and 41, top-k
// 50 with top-p 29 and 44, top-k 2000 53 and 124, top-p 55 and 131, no filter (BF16, no counts) 39.  What is done, by the row's settings:
//   top_k <= 512   the k-th largest of the threads' maxima bounds the k-th token from below; the few tokens above it go to a list in LDS,
//                  which is sorted, filtered and drawn from: two readings, no weights but the list's;
//   top_p, top_k   counts and weights over bins of 1/64 octave of weight, then the tokens of the bin in which the filter ends, sorted (a bin
//                  that holds too many: a radix search over their places); three readings, four with both;
//   BF16           in place of the bins, counts of the logits' codes: a weight is computed once a code, and the place at which a filter ends
//                  is a code and a number of tokens that have it;
//   otherwise      sums of the kept weights over segments of the row, and the token inside the segment on which the number falls.
// Few long rows without top-k go over several workgroups each, in four launches: maxima; bins; sums of the segments without the bin in which top-p ends,
// whose tokens go to a list; and by one workgroup the list, its kept tokens added to their segments, and the draw.
#pragma once
#include "rows.h"

namespace elmo {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kSampleShortK = 512;             // largest top_k that goes by the threads' maxima
constexpr int kSampleList = 4096;              // places of the list in LDS; segments of a row
constexpr int kSampleBins = 2048;              // 1/64 octave each, the last one everything below 2^-32 of the largest weight
constexpr uint32_t kKeyNone = 0x007FFFFFu;     // key of -infinity: never kept

struct SampleArgs {
  const void* z;
  int64_t zs, V;
  const float *u, *t, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* prob;
  int F;
  int parts;                         // workgroups of a row
  char* ws;                          // of split rows: kSampleRowBytes each
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
// r^4 (the next term is below 2^-54; roundings of y, root, series and product: 2^-51 of the weight together).  NaN and -infinity end at the lower bound,
// which rounds to no weight.
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
  __device__ inline double unrounded(float z, int& n) const {
    constexpr double c = 0.6931471805599453 / 256;
    double r;
    n = steps(__builtin_fmax(((double)z - M) * k, least), r);
    const double p = __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(c * c * c * c / 24, r, c * c * c / 6), r, c * c / 2), r, c), r, 1.0);
    return __builtin_ldexp(p * roots[n & 255], (n >> 8) + F);
  }
  __device__ inline double unrounded(float z) const { int n; return unrounded(z, n); }
  static __device__ inline uint64_t whole(double w) {
    return (uint64_t)__double_as_longlong(w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;         // + 2^52: rounded to a whole number
  }
  __device__ inline uint64_t operator()(float z, int& n) const { return whole(unrounded(z, n)); }
  __device__ inline uint64_t operator()(float z) const { int n; return (*this)(z, n); }
  __device__ inline int bin(int n) const { return min(-n >> 2, kSampleBins - 1); }        // 0: the largest weights
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
  s.p = p < 1.0f ? fmax((double)p, 0.0) : 1.0; // NaN: off
  s.mp = mp > 0.0f ? (mp < 1.0f ? (double)mp : 1.0) : 0.0;
  s.u = u > 0.0f ? (double)u : 0.0;
  return s;
}
__device__ inline uint64_t share_of(double part, uint64_t whole) {   // ceil(part whole), at least 1 and at most the whole
  return min(whole, max((uint64_t)1, (uint64_t)__builtin_ceil(part * (double)whole)));
}

// Inclusive sums over the workgroup's threads, and their total.  Barriers before and behind the use of `slots`.
template <class U> __device__ inline U block_scan(U v, U* slots, int wave, int lane, U& total) {
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) slots[wave] = v;
  __syncthreads();
  const U mine = lane < kSampleWaves ? slots[lane] : 0, upto = wave_scan(mine);
  total = of_lane(upto, kSampleWaves - 1);
  return v + of_lane(upto - mine, __builtin_amdgcn_readfirstlane(wave));
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

struct SampleLds {
  uint64_t list[kSampleList], mass[kSampleBins], sum[kSampleWaves], found[3];
  double root[256];
  uint32_t count[kSampleBins], sum32[kSampleWaves];
  float max[kSampleWaves];
  int n;
};

// What a split row's workgroups hand on.
struct SampleWs {
  uint64_t mass[kSampleBins], list[kSampleList], segment[kSampleList];
  float max[64];
  uint32_t n;
};
constexpr size_t kSampleRowBytes = (sizeof(SampleWs) + 255) / 256 * 256;

// A BF16 row has few logits that carry weight: the codes of both signs over 21 octaves below the larger end of [smallest logit with a weight, largest
// logit].  Slots in falling order.  (Logits nearer to zero than that, should there be any, send a row the other way.)
constexpr int kCodeOctaves = 21, kCodeHalf = kCodeOctaves * 128, kCodes = 2 * kCodeHalf, kCodesEach = (kCodes + kSampleThreads - 1) / kSampleThreads;
struct SampleCodes {
  uint64_t weight[kCodesEach * kSampleThreads];              // (behind the slots: no weight)
  uint32_t count[kCodesEach * kSampleThreads];
};
static_assert(kCodes < kCodesEach * kSampleThreads, "an entry of no weight");
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// One row in the hands of a workgroup.  Everything inlined into the kernels: called, its state would lie in scratch memory and LDS would be reached through flat addresses.
// (A build in which the compiler called whole, end_in_bin and draw ended in a memory aperture violation.  Every index of that form is in its array and nothing
// is raced for, as here -- tests/test_sample_host.py runs this file with checked memory -- so the cause is not known, and the form stays out.)
template <class T> struct Sampler {
  static constexpr int NT = kSampleThreads;
  const SampleArgs& a;
  SampleLds& l;
  const int64_t row, octets, per;              // per: rounds of 64 octets in a segment, which is a wave's
  const int segments, tid, lane, wave;
  const T* z;
  const RowSettings rs;
  bool infinite = false;                       // the largest logit is +infinity: only such have a weight; 0 stands for it, -infinity for the others
  Weigh weigh;
  uint64_t least = 1;                                            // smallest kept weight
  float low = -__builtin_inff();                                 // smallest kept logit,
  uint32_t last = ~0u;                                           // and of those equal to it the last kept index

  __device__ __forceinline__ Sampler(const SampleArgs& args, SampleLds& lds, int64_t r)
      : a(args), l(lds), row(r), octets((args.V + 7) >> 3), per(((octets + 63) / 64 + kSampleList - 1) / kSampleList),
        segments((int)(((octets + 63) / 64 + per - 1) / per)), tid(threadIdx.x), lane(threadIdx.x & 63), wave(threadIdx.x >> 6),
        z((const T*)args.z + r * args.zs), rs(settings_of(args, r)) {}

  __device__ __forceinline__ void load8(int64_t o, float (&f)[8]) const {
    const Octet<T> oc = load_octet(z + o * 8, a.V - o * 8, lowest<T>());
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = oc[i];
    if (infinite) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = f[i] == __builtin_inff() ? 0.0f : -__builtin_inff();
    }
  }
  static __device__ __forceinline__ float max8(const float (&f)[8]) {
    return fmaxf(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])), fmaxf(fmaxf(f[4], f[5]), fmaxf(f[6], f[7])));
  }
  __device__ __forceinline__ void answer(int64_t token, float prob) const {
    a.token[row] = (int32_t)token;
    if (a.prob) a.prob[row] = prob;
  }
  __device__ __forceinline__ void drawn(int64_t token, double weight, uint64_t all) const { answer(token, (float)(weight / (double)all)); }
  __device__ __forceinline__ float logit_of(int64_t token) const {        // of one that has a weight
    return infinite ? 0.0f : load_one(z, token);
  }
  __device__ __forceinline__ uint64_t number(uint64_t all) const {        // u of the kept weight
    const uint64_t want = (uint64_t)(rs.u * (double)all);
    return want >= all ? all - 1 : want;
  }
  // A thread's largest logit among the octets [from, to).
  __device__ __forceinline__ float largest(int64_t from, int64_t to) const {
    float m = -__builtin_inff();
#pragma unroll 8
    for (int64_t o = from + tid; o < to; o += NT) {
      float f[8];
      load8(o, f);
      m = fmaxf(m, max8(f));
    }
    return m;
  }
  // The row's weights, once its largest logit is known (> -infinity).  Holds a barrier.
  __device__ __forceinline__ void set_max(float M) {
    infinite = M == __builtin_inff();
    if (tid < 256) l.root[tid] = exp_series(tid * (kLn2 / 256));
    if (tid == 0) l.n = 0;
    weigh = Weigh{l.root, infinite ? 0.0 : (double)M, 256.0 * kLog2e / rs.t, -256.0 * (a.F + 2), a.F};
    if (rs.mp > 0.0) least = share_of(rs.mp, 1ull << a.F);
    __syncthreads();
  }
  // Appends the logits >= from that keep() names to the list.
  template <class F> __device__ __forceinline__ void collect(float from, F&& keep) {
#pragma unroll 4
    for (int64_t o = tid; o < octets; o += NT) {
      float f[8];
      load8(o, f);
      if (max8(f) >= from) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (f[i] >= from && keep(f[i])) {
            const int at = atomicAdd(&l.n, 1);
            if (at < kSampleList) l.list[at] = place_of(f[i], o * 8 + i);
          }
      }
    }
    __syncthreads();
  }
  __device__ __forceinline__ void order_list(int n) {
    if (n <= kSampleCount) return rank_falling(l.list, l.count, n, tid);
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) l.list[i] = 0;
    sort_falling(l.list, size, tid);
  }
  // found[0] = the place at which the list's n tokens, behind `above` tokens of weight mass_above, first make up `want` tokens or weight; found[1]
  // = the weight down to it.  Changes count.
  __device__ __forceinline__ void cut_list(int n, bool by_mass, uint64_t want, uint64_t above, uint64_t mass_above) {
    order_list(n);
    uint64_t w[4], sum = 0, whole;                       // four a thread
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += w[i] = 4 * tid + i < n ? weigh(of_key(l.list[4 * tid + i] >> 32)) : 0;
    uint64_t upto = mass_above + block_scan(sum, l.sum, wave, lane, whole) - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 4 * tid + i;
      const bool here = at < n && (by_mass ? upto < want && upto + w[i] >= want : above + at + 1 == want);
      upto += w[i];
      if (here) { l.found[0] = l.list[at]; l.found[1] = upto; }
    }
    __syncthreads();
  }
  // Into found: the bin in which tokens or weight, `before` ahead of this thread's two bins with c0 and c1, first make up `want`; what lies ahead of it; the
  // weight ahead of it.
  __device__ __forceinline__ void find_bin(uint64_t want, uint64_t before, uint64_t c0, uint64_t c1, uint64_t mass_before, uint64_t m0) {
    __syncthreads();
    if (before < want && before + c0 >= want) { l.found[0] = 2 * tid; l.found[1] = before; l.found[2] = mass_before; }
    if (before + c0 < want && before + c0 + c1 >= want) { l.found[0] = 2 * tid + 1; l.found[1] = before + c0; l.found[2] = mass_before + m0; }
    __syncthreads();
  }
  // A bound below a bin's logits, with room for the rounding of y, so that octets below it are passed over.
  __device__ __forceinline__ float bin_floor(int bin) const {
    return bin == kSampleBins - 1 ? -__builtin_inff() : (float)(weigh.M + (-4.0 * bin - 5.0) / weigh.k) - 1e-5f * fabsf((float)weigh.M);
  }

  // ---- top_k <= 512: bound, list, filters, draw.  False: the list does not hold what lies above the bound.
  __device__ __forceinline__ bool short_list(float mine) {
    const float M = (float)weigh.M;
    if (rs.k == 1) {
      uint32_t first = ~0u;                              // the largest logit's first place
      for (int64_t o = tid; o < octets; o += NT) {
        float f[8];
        load8(o, f);
#pragma unroll
        for (int i = 7; i >= 0; --i)
          if (f[i] == M) first = min(first, (uint32_t)(o * 8 + i));
      }
      first = wave_reduce(first, [](uint32_t p, uint32_t q) { return min(p, q); });
      if (lane == 0) l.sum32[wave] = first;
      __syncthreads();
      first = slots_reduce<kSampleWaves>(l.sum32, lane, [](uint32_t p, uint32_t q) { return min(p, q); });
      if (tid == 0) answer(first, 1.0f);
      return true;
    }
    // 16 bits of the k-th largest of the threads' maxima, 8 at a time
    uint32_t prefix = 0, left = (uint32_t)rs.k;
    const uint32_t key = key_of(mine);
    for (int sh = 24; sh >= 16; sh -= 8) {
      if (tid < 256) l.count[tid] = 0;
      __syncthreads();
      if (key > kKeyNone && (sh == 24 || key >> 24 == prefix >> 24)) atomicAdd(&l.count[(key >> sh) & 255], 1u);
      __syncthreads();
      if (wave == 0) {                                   // four bins a lane, the largest first
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = l.count[255 - 4 * lane - i];
        uint32_t before = wave_scan(sum) - sum;
        if (lane == 63) l.found[0] = before + sum < left ? ~0ull : 0;      // fewer maxima than k: every token is taken
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && before + c[i] >= left) { l.found[1] = 255 - 4 * lane - i; l.found[2] = before; }
          before += c[i];
        }
      }
      __syncthreads();
      if (l.found[0]) { prefix = 0; break; }
      prefix |= (uint32_t)l.found[1] << sh;
      left -= (uint32_t)l.found[2];
      __syncthreads();
    }
    collect(of_key(max(prefix, kKeyNone + 1)), [](float f) { return f > -__builtin_inff(); });
    const int n = l.n;
    __syncthreads();
    if (n > kSampleList) return false;
    order_list(n);
    const int nk = (int)min((int64_t)n, rs.k);           // at most 512: one a thread
    const uint64_t place = tid < nk ? l.list[tid] : 0;
    const double exact = tid < nk ? weigh.unrounded(of_key(place >> 32)) : 0.0;
    const uint64_t w = Weigh::whole(exact);
    uint64_t total, all;
    const uint64_t upto = block_scan(w, l.sum, wave, lane, total);
    const bool kept = w >= least && (rs.p >= 1.0 || upto - w < share_of(rs.p, total));
    block_scan(kept ? w : 0, l.sum, wave, lane, all);
    const uint64_t want = number(all);
    // what is kept before a token by index: of few by pairs, else along the list sorted by index
    if (tid < kSampleShortK) {
      l.mass[tid] = kept ? w : 0;
      l.mass[kSampleShortK + tid] = 0;
      if (nk > kSampleCount) l.list[tid] = kept ? place << 32 | (uint32_t)tid : 0;
    }
    __syncthreads();
    if (nk <= kSampleCount) {
      for_pairs(nk, tid, [&](int i, int from, int to) {
        const uint32_t x = (uint32_t)l.list[i];          // the complement of the index
        uint64_t sum = 0;
        for (int j = from; j < to; ++j) sum += (uint32_t)l.list[j] > x ? l.mass[j] : 0;
        if (sum) atomicAdd((unsigned long long*)&l.mass[kSampleShortK + i], (unsigned long long)sum);
      });
      __syncthreads();
      const uint64_t before = tid < nk ? l.mass[kSampleShortK + tid] : 0;
      if (kept && before <= want && before + w > want) drawn((int64_t)(uint32_t)~(uint32_t)place, exact, all);
      return true;
    }
    sort_falling(l.list, kSampleShortK, tid);
    const uint64_t entry = tid < kSampleShortK ? l.list[tid] : 0;
    // (an entry of 0 would be index 2^32 - 1, which no row has)
    const uint64_t wi = entry ? l.mass[(uint32_t)entry] : 0;
    const uint64_t by_index = block_scan(wi, l.sum, wave, lane, all);
    const int64_t token = (int64_t)(uint32_t)~(uint32_t)(entry >> 32);
    if (wi && by_index > want && by_index - wi <= want) drawn(token, weigh.unrounded(logit_of(token)), all);
    return true;
  }

  // ---- weights (and counts) over bins, of the octets [from, to)
  __device__ __forceinline__ void fill_bins(int64_t from, int64_t to, bool by_count) {
    for (int i = tid; i < kSampleBins; i += NT) {
      l.mass[i] = 0;
      l.count[i] = 0;
    }
    __syncthreads();
    for (int64_t o = from + tid; o < to; o += NT) {
      float f[8];
      load8(o, f);
      uint64_t w[8];
      int n[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = weigh(f[i], n[i]);      // (all of them before the first branch: eight chains side by side)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (w[i]) {
          atomicAdd((unsigned long long*)&l.mass[weigh.bin(n[i])], (unsigned long long)w[i]);
          if (by_count) atomicAdd(&l.count[weigh.bin(n[i])], 1u);
        }
    }
    __syncthreads();
  }

  __device__ __forceinline__ void set_edge(uint64_t place) {
    low = of_key(place >> 32);
    last = ~(uint32_t)place;
  }
  // The filter's end, from the bin in found.  Returns the weight down to it.
  __device__ __forceinline__ uint64_t end_in_bin(bool by_mass, uint64_t want) {
    const int bin = (int)l.found[0];
    uint64_t above = l.found[1], mass_above = l.found[2];
    if (tid == 0) l.n = 0;
    __syncthreads();
    const auto in_bin = [&](float f) { int n; return weigh(f, n) != 0 && weigh.bin(n) == bin; };
    collect(bin_floor(bin), in_bin);
    const int n = l.n;
    __syncthreads();
    if (n <= kSampleList) {
      cut_list(n, by_mass, want, above, mass_above);
    } else {
      // too many for the list: a radix search over the bin's places, 8 bits at a time
      uint64_t prefix = 0;
      for (int sh = 56; sh >= 0; sh -= 8) {
        __syncthreads();
        if (tid < 256) { l.list[tid] = 0; l.list[256 + tid] = 0; }
        __syncthreads();
        for (int64_t o = tid; o < octets; o += NT) {
          float f[8];
          load8(o, f);
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            const uint64_t p = place_of(f[i], o * 8 + i);
            if (in_bin(f[i]) && (sh == 56 || p >> (sh + 8) == prefix >> (sh + 8))) {
              atomicAdd((unsigned long long*)&l.list[(p >> sh) & 255], (unsigned long long)weigh(f[i]));
              atomicAdd((unsigned long long*)&l.list[256 + ((p >> sh) & 255)], 1ull);
            }
          }
        }
        __syncthreads();
        if (tid == 0) {
          int b = 255;
          for (; b > 0; --b) {
            if ((by_mass ? mass_above + l.list[b] : above + l.list[256 + b]) >= want) break;
            above += l.list[256 + b];
            mass_above += l.list[b];
          }
          l.found[0] = b; l.found[1] = above; l.found[2] = mass_above;
          if (sh == 0) l.list[0] = mass_above + l.list[b];
        }
        __syncthreads();
        prefix |= l.found[0] << sh;
        above = l.found[1];
        mass_above = l.found[2];
      }
      __syncthreads();
      if (tid == 0) { l.found[0] = prefix; l.found[1] = l.list[0]; }
      __syncthreads();
    }
    set_edge(l.found[0]);
    return l.found[1];
  }

  // Weights of an octet's kept tokens, and their sum.
  __device__ __forceinline__ uint64_t kept8(int64_t o, uint64_t (&w)[8]) const {
    uint64_t sum = 0;
    float f[8];
    const bool in = o < octets;
    if (in) load8(o, f);
    if (in && max8(f) >= low) {
      const uint32_t at = (uint32_t)o * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = weigh(f[i]);
        const bool kept = f[i] > low || (f[i] == low && at + i <= last);
        w[i] = kept && w[i] >= least ? w[i] : 0;
        sum += w[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 0;
    }
    return sum;
  }
  // ---- the token, from the segments' kept weight in list
  __device__ __forceinline__ void draw() {
    uint64_t w4[4], sum = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += w4[i] = 4 * tid + i < segments ? l.list[4 * tid + i] : 0;
    uint64_t before = block_scan(sum, l.sum, wave, lane, all) - sum;
    const uint64_t want = number(all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before <= want && before + w4[i] > want) { l.found[0] = 4 * tid + i; l.found[1] = before; }
      before += w4[i];
    }
    __syncthreads();
    if (wave != 0) return;
    before = l.found[1];
    for (int64_t i = 0; i < per; ++i) {
      const int64_t o = ((int64_t)l.found[0] * per + i) * 64 + lane;
      uint64_t w[8];
      const uint64_t mine = kept8(o, w), upto = wave_scan(mine);
      uint64_t at = before + upto - mine;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (at <= want && at + w[j] > want) drawn(o * 8 + j, weigh.unrounded(logit_of(o * 8 + j)), all);
        at += w[j];
      }
      before += of_lane(upto, 63);
    }
  }

  // ---- BF16, by codes.  False: not this row.
  static constexpr int kNoEnd = 1 << 16;       // beyond what slots_of gives
  static constexpr int kFlight = 4;            // octets of a thread on their way at a time
  __device__ __forceinline__ Octet<uint16_t> load_codes(int64_t o) const {            // (beyond the row: -infinity)
    constexpr uint32_t none = 0xFF80FF80u;
    if (o >= octets) return {{none, none, none, none}};
    return load_octet((const uint16_t*)z + o * 8, a.V - o * 8, 0xFF80u);
  }
  static __device__ __forceinline__ bool has_small(const Octet<uint16_t>& oc, int base) {
    const auto sizes = [&](int i) { return __builtin_bit_cast(u16x2, oc.v[i] & 0x7FFF7FFFu); };
    const u16x2 m = __builtin_elementwise_min(__builtin_elementwise_min(sizes(0), sizes(1)), __builtin_elementwise_min(sizes(2), sizes(3)));
    return min(m[0], m[1]) < base;
  }
  // Adds an octet's logits nearer to zero than the slots go, of at least a weight.
  __device__ __forceinline__ void next_to_zero(int64_t o, int base, uint64_t from, uint64_t& mass, uint64_t& tokens) const {
#pragma unroll 1
    for (int64_t i = o * 8; i < min(a.V, o * 8 + 8); ++i) {
      const float f = load_one((const uint16_t*)z, i);
      if ((int)(f2u(f) >> 16 & 0x7FFF) >= base) continue;
      const uint64_t w = weigh(f);
      mass += w >= from ? w : 0;
      tokens += w >= from;
    }
  }
  // The slots of two codes at a time, in packed 16-bit arithmetic (three instructions a code).  kCodes and more: none.
  static __device__ __forceinline__ u16x2 slots_of(uint32_t codes, int base) {
    const u16x2 from = {(uint16_t)base, (uint16_t)base}, half = {kCodeHalf, kCodeHalf};
    const u16x2 i = __builtin_elementwise_min(__builtin_bit_cast(u16x2, codes & 0x7FFF7FFFu) - from, half);     // (below base: 2^15 and more)
    const uint32_t sign = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, codes) >> 15);
    return __builtin_bit_cast(u16x2, ~(__builtin_bit_cast(uint32_t, i) ^ sign)) + half;
  }
  __device__ __forceinline__ bool by_code(SampleCodes* c) {
    if (infinite) return false;
    const float bottom = (float)(weigh.M + weigh.least / weigh.k);       // (-infinity at a temperature of infinity)
    const uint32_t wide = f2u(fmaxf(fabsf((float)weigh.M), fminf(fabsf(bottom), 3.3e38f))) >> 23;   // exponents up to this one
    const int base = max(0, (int)wide - (kCodeOctaves - 1)) * 128;
    if (base == 0) return false;                                         // (both zeros would have codes)
    const int s0 = kCodesEach * tid;
#pragma unroll
    for (int i = 0; i < kCodesEach; ++i) {
      const int s = s0 + i;
      const uint32_t code = s < kCodeHalf ? base + kCodeHalf - 1 - s : 0x8000u + base + s - kCodeHalf;
      const float f = u2f(code << 16);
      c->weight[s] = s < kCodes && f <= (float)weigh.M ? weigh(f) : 0;
      c->count[s] = 0;
    }
    __syncthreads();
    int end = kNoEnd;                                    // slots before this one are kept, of its own tokens the first `ties`
    uint64_t ties = 0;
    if (rs.k < a.V || rs.p < 1.0) {
      uint64_t zero_mass = 0, zero_tokens = 0;           // of the logits nearer to zero
      for (int64_t o0 = tid; o0 < octets; o0 += kFlight * NT) {
        Octet<uint16_t> oc[kFlight];
#pragma unroll
        for (int q = 0; q < kFlight; ++q) oc[q] = load_codes(o0 + q * NT);
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
          u16x2 most = {0, 0};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const u16x2 s = slots_of(oc[q].v[i], base);
            most = __builtin_elementwise_max(most, s);
            if (s[0] < kCodes) atomicAdd(&c->count[s[0]], 1u);
            if (s[1] < kCodes) atomicAdd(&c->count[s[1]], 1u);
          }
          if (max(most[0], most[1]) >= kCodes && has_small(oc[q], base)) next_to_zero(o0 + q * NT, base, 1, zero_mass, zero_tokens);
        }
      }
      block_scan(zero_mass, l.sum, wave, lane, zero_mass);
      block_scan(zero_tokens, l.sum, wave, lane, zero_tokens);
      __syncthreads();
      // a thread's six slots
      uint64_t w[kCodesEach], n[kCodesEach], mass = 0, tokens = 0, total, live;
#pragma unroll
      for (int i = 0; i < kCodesEach; ++i) {
        w[i] = c->weight[s0 + i];
        n[i] = w[i] ? c->count[s0 + i] : 0;
        mass += w[i] * n[i];
        tokens += n[i];
      }
      static_assert(kCodeHalf % kCodesEach == 0, "a thread has slots of one sign");
      const bool negative = s0 >= kCodeHalf;             // behind the logits next to zero
      const uint64_t mass_before = block_scan(mass, l.sum, wave, lane, total) - mass + (negative ? zero_mass : 0);
      const uint64_t before = block_scan(tokens, l.sum, wave, lane, live) - tokens + (negative ? zero_tokens : 0);
      total += zero_mass;
      live += zero_tokens;
      const auto find = [&](bool by_mass, uint64_t want) {
        uint64_t at_n = before, at_m = mass_before;
        __syncthreads();
        if (tid < 3) l.found[tid] = tid == 0 ? kNoEnd : 0;   // (stays so if the filter ends next to zero)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCodesEach; ++i) {
          const uint64_t at = by_mass ? at_m : at_n, step = by_mass ? w[i] * n[i] : n[i];
          if (at < want && at + step >= want) {
            const uint64_t some = by_mass ? (want - at + w[i] - 1) / w[i] : want - at;
            l.found[0] = s0 + i;
            l.found[1] = some;
            l.found[2] = at_m + some * w[i];
          }
          at_n += n[i];
          at_m += w[i] * n[i];
        }
        __syncthreads();
        end = (int)l.found[0];
        ties = l.found[1];
        return l.found[2];
      };
      if ((uint64_t)rs.k < live) {
        total = find(false, (uint64_t)rs.k);
        if (end == kNoEnd) return false;
      }
      if (rs.p < 1.0) {
        find(true, share_of(rs.p, total));
        if (end == kNoEnd) return false;
      }
    }
    const bool keep_zero = end >= kCodeHalf;
    // what is not kept has no weight from here on; the last code's tokens count apart
    uint64_t we = end != kNoEnd ? c->weight[end] : 0;
    if (we < least) we = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kCodesEach; ++i)
      if (s0 + i >= end || c->weight[s0 + i] < least) c->weight[s0 + i] = 0;
    __syncthreads();
    // an octet's weights without the last code's, and which of it are that.  (What is not kept reads one entry, all lanes the same: no bank conflicts.)
    const uint16_t none = (uint16_t)min(end, kCodes);
    const auto octet = [&](const Octet<uint16_t>& oc, uint64_t (&w)[8], uint32_t& mask, bool& others) {
      uint64_t sum = 0;
      mask = 0;
      u16x2 most = {0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u16x2 s = slots_of(oc.v[i], base), in = __builtin_elementwise_min(s, (u16x2){none, none});
        most = __builtin_elementwise_max(most, s);
        w[2 * i] = c->weight[in[0]];
        w[2 * i + 1] = c->weight[in[1]];
        mask |= (s[0] == end ? 1u << (2 * i) : 0) | (s[1] == end ? 2u << (2 * i) : 0);
        sum += w[2 * i] + w[2 * i + 1];
      }
      others = keep_zero && max(most[0], most[1]) >= kCodes && has_small(oc, base);
      return sum;
    };
    for (int s = wave; s < segments; s += kFlight * kSampleWaves) {      // (beyond the last segment: no octets)
      uint64_t sum[kFlight], w[8], unused = 0;
      uint32_t count[kFlight], mask;
      bool others;
#pragma unroll
      for (int q = 0; q < kFlight; ++q) sum[q] = count[q] = 0;
      for (int64_t i = 0; i < per; ++i) {
        Octet<uint16_t> oc[kFlight];
#pragma unroll
        for (int q = 0; q < kFlight; ++q) oc[q] = load_codes(((s + q * kSampleWaves) * per + i) * 64 + lane);
#pragma unroll
        for (int q = 0; q < kFlight; ++q) {
          sum[q] += octet(oc[q], w, mask, others);
          count[q] += __popc(mask);
          if (others) next_to_zero(((s + q * kSampleWaves) * per + i) * 64 + lane, base, least, sum[q], unused);
        }
      }
#pragma unroll
      for (int q = 0; q < kFlight; ++q) {
        sum[q] = wave_reduce(sum[q], [](uint64_t p, uint64_t r) { return p + r; });
        count[q] = wave_reduce(count[q], [](uint32_t p, uint32_t r) { return p + r; });
      }
#pragma unroll
      for (int q = 0; q < kFlight; ++q)
        if (lane == 0 && s + q * kSampleWaves < segments) {
          l.list[s + q * kSampleWaves] = sum[q];
          c->count[s + q * kSampleWaves] = count[q];
        }
    }
    __syncthreads();
    // the segments' last-code tokens that are kept are the first `ties` of all of them
    uint32_t n4[4], some = 0, whole_count;
#pragma unroll
    for (int i = 0; i < 4; ++i) some += n4[i] = 4 * tid + i < segments ? c->count[4 * tid + i] : 0;
    uint32_t seen = block_scan(some, l.sum32, wave, lane, whole_count) - some;
    uint64_t w4[4], sum = 0, all;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t left = ties > seen ? ties - seen : 0;
      w4[i] = 4 * tid + i < segments ? l.list[4 * tid + i] + min((uint64_t)n4[i], left) * we : 0;
      sum += w4[i];
      seen += n4[i];
    }
    seen -= some;
    uint64_t at = block_scan(sum, l.sum, wave, lane, all) - sum;
    const uint64_t want = number(all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at <= want && at + w4[i] > want) { l.found[0] = 4 * tid + i; l.found[1] = at; l.found[2] = seen; }
      at += w4[i];
      seen += n4[i];
    }
    __syncthreads();
    if (wave != 0) return true;
    at = l.found[1];
    uint64_t ranked = l.found[2];
    for (int64_t i = 0; i < per; ++i) {
      const int64_t o = ((int64_t)l.found[0] * per + i) * 64 + lane;
      const Octet<uint16_t> oc = load_codes(o);
      uint64_t w[8], mine = 0;
      uint32_t mask;
      bool others;
      octet(oc, w, mask, others);
      if (others) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if ((int)(f2u(oc[j]) >> 16 & 0x7FFF) < base) {
            w[j] = weigh(oc[j]);
            if (w[j] < least) w[j] = 0;
          }
      }
      const uint32_t own = __popc(mask), upto_n = wave_scan(own);
      uint64_t rank = ranked + upto_n - own;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (mask >> j & 1) w[j] = rank++ < ties ? we : 0;
        mine += w[j];
      }
      const uint64_t upto = wave_scan(mine);
      uint64_t here = at + upto - mine;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (here <= want && here + w[j] > want) drawn(o * 8 + j, weigh.unrounded(oc[j]), all);
        here += w[j];
      }
      at += of_lane(upto, 63);
      ranked += of_lane(upto_n, 63);
    }
    return true;
  }

  // ---- a row by one workgroup
  __device__ __forceinline__ void whole(SampleCodes* codes) {
    float mine = largest(0, octets), M = wave_max(mine);
    if (lane == 0) l.max[wave] = M;
    __syncthreads();
    M = slots_reduce<kSampleWaves>(l.max, lane, [](float p, float q) { return fmaxf(p, q); });
    if (M == -__builtin_inff()) {
      if (tid == 0) answer(-1, 0.0f);
      return;
    }
    set_max(M);
    if (infinite) mine = mine == __builtin_inff() ? 0.0f : -__builtin_inff();
    if (rs.k <= kSampleShortK && short_list(mine)) return;
    if constexpr (sizeof(T) == 2) {
      __syncthreads();
      if (by_code(codes)) return;
    }
    if (rs.k < a.V || rs.p < 1.0) {
      __syncthreads();
      fill_bins(0, octets, rs.k < a.V);
      uint64_t total;
      const uint64_t m0 = l.mass[2 * tid], m1 = l.mass[2 * tid + 1], n0 = l.count[2 * tid], n1 = l.count[2 * tid + 1];
      const uint64_t mass_before = block_scan(m0 + m1, l.sum, wave, lane, total) - m0 - m1;
      if (rs.k < a.V) {
        uint64_t live;
        const uint64_t before = block_scan(n0 + n1, l.sum, wave, lane, live) - n0 - n1;
        if ((uint64_t)rs.k < live) {
          find_bin((uint64_t)rs.k, before, n0, n1, mass_before, m0);
          total = end_in_bin(false, (uint64_t)rs.k);
        }
      }
      if (rs.p < 1.0) {
        const uint64_t want = share_of(rs.p, total);
        find_bin(want, mass_before, m0, m1, mass_before, m0);
        end_in_bin(true, want);
      }
    }
    __syncthreads();
    for (int s = wave; s < segments; s += kSampleWaves) {
      uint64_t sum = 0, w[8];
      for (int64_t i = 0; i < per; ++i) sum += kept8((s * per + i) * 64 + lane, w);
      sum = wave_reduce(sum, [](uint64_t p, uint64_t q) { return p + q; });
      if (lane == 0) l.list[s] = sum;
    }
    __syncthreads();
    draw();
  }

  // ---- a row by several: this workgroup's segments [s0, s1)
  __device__ __forceinline__ SampleWs* shared_state() const { return (SampleWs*)(a.ws + row * kSampleRowBytes); }
  __device__ __forceinline__ void my_segments(int& s0, int& s1) const {
    const int each = (segments + a.parts - 1) / a.parts, part = (int)(blockIdx.x % a.parts);
    s0 = min(segments, part * each);
    s1 = min(segments, s0 + each);
  }
  // The row's largest logit from its parts'; false where there is nothing for the split form to do.
  __device__ __forceinline__ bool split_max() {
    const float M = wave_max(lane < a.parts ? shared_state()->max[lane] : -__builtin_inff());
    if (M == -__builtin_inff() || rs.k < a.V) return false;       // (a greedy row has k = 1: the last launch takes it whole)
    set_max(M);
    return true;
  }
  __device__ __forceinline__ void part_max() {
    SampleWs* ws = shared_state();
    const int part = (int)(blockIdx.x % a.parts);
    int s0, s1;
    my_segments(s0, s1);
    const float M = wave_max(largest(s0 * per * 64, min(octets, s1 * per * 64)));
    if (lane == 0) l.max[wave] = M;
    for (int i = part * NT + tid; i < kSampleBins; i += a.parts * NT) ws->mass[i] = 0;
    __syncthreads();
    if (wave == 0) {
      const float top = slots_reduce<kSampleWaves>(l.max, lane, [](float p, float q) { return fmaxf(p, q); });
      if (lane == 0) ws->max[part] = top;
      if (lane == 0 && part == 0) ws->n = 0;
    }
  }
  __device__ __forceinline__ void part_bins() {
    if (rs.p >= 1.0 || !split_max()) return;
    int s0, s1;
    my_segments(s0, s1);
    fill_bins(s0 * per * 64, min(octets, s1 * per * 64), false);
    for (int i = tid; i < kSampleBins; i += NT)
      if (l.mass[i]) atomicAdd((unsigned long long*)&shared_state()->mass[i], (unsigned long long)l.mass[i]);
  }
  // Into found: the bin in which top-p ends.  Returns the weight that it asks for.
  __device__ __forceinline__ uint64_t split_bin() {
    const SampleWs* ws = shared_state();
    uint64_t total;
    const uint64_t m0 = ws->mass[2 * tid], m1 = ws->mass[2 * tid + 1];
    const uint64_t mass_before = block_scan(m0 + m1, l.sum, wave, lane, total) - m0 - m1, want = share_of(rs.p, total);
    find_bin(want, mass_before, m0, m1, mass_before, m0);
    return want;
  }
  __device__ __forceinline__ void part_sums() {
    if (!split_max()) return;
    SampleWs* ws = shared_state();
    int bin = kSampleBins, s0, s1;
    if (rs.p < 1.0) {
      split_bin();
      bin = (int)l.found[0];
      low = bin_floor(bin);
    }
    my_segments(s0, s1);
    for (int s = s0 + wave; s < s1; s += kSampleWaves) {
      uint64_t sum = 0;
      for (int64_t i = 0; i < per; ++i) {
        const int64_t o = (s * per + i) * 64 + lane;
        float f[8];
        if (o < octets) load8(o, f);
        if (o < octets && max8(f) >= low) {
          uint64_t w[8];
          int n[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            w[j] = weigh(f[j], n[j]);
            n[j] = weigh.bin(n[j]);
            sum += n[j] < bin && w[j] >= least ? w[j] : 0;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (n[j] == bin && w[j]) {
              const uint32_t at = atomicAdd(&ws->n, 1u);
              if (at < (uint32_t)kSampleList) ws->list[at] = place_of(f[j], o * 8 + j);
            }
        }
      }
      sum = wave_reduce(sum, [](uint64_t p, uint64_t q) { return p + q; });
      if (lane == 0) ws->segment[s] = sum;
    }
  }
  __device__ __forceinline__ void split_draw(SampleCodes* codes) {
    const SampleWs* ws = shared_state();
    const int n = (int)min(ws->n, (uint32_t)kSampleList + 1);
    if (n > kSampleList || !split_max()) return whole(codes);
    if (rs.p < 1.0) {
      const uint64_t want = split_bin(), above = l.found[1], mass_above = l.found[2];
      for (int i = tid; i < n; i += NT) l.list[i] = ws->list[i];
      __syncthreads();
      cut_list(n, true, want, above, mass_above);
      const uint64_t edge = l.found[0];
      set_edge(edge);
      uint64_t place[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) place[i] = i * NT + tid < n ? l.list[i * NT + tid] : 0;
      __syncthreads();
      for (int i = tid; i < segments; i += NT) l.list[i] = ws->segment[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (place[i] >= edge) {                          // (no place is 0)
          const uint64_t w = weigh(of_key(place[i] >> 32));
          if (w >= least) atomicAdd((unsigned long long*)&l.list[(uint32_t)~(uint32_t)place[i] / (uint32_t)(per * 512)], (unsigned long long)w);
        }
    } else {
      for (int i = tid; i < segments; i += NT) l.list[i] = ws->segment[i];
    }
    __syncthreads();
    draw();
  }
};

enum : int { SAMPLE_WHOLE = 0, SAMPLE_MAX = 1, SAMPLE_BINS = 2, SAMPLE_SUMS = 3, SAMPLE_DRAW = 4 };
// Dynamic LDS of a launch: the codes, where a row may be taken whole.
template <class T, int STEP> constexpr int sample_smem() { return sizeof(T) == 2 && (STEP == SAMPLE_WHOLE || STEP == SAMPLE_DRAW) ? (int)sizeof(SampleCodes) : 0; }
template <class T, int STEP>
__global__ __launch_bounds__(kSampleThreads) void k_sample(SampleArgs a) {
  __shared__ SampleLds lds;
  extern __shared__ __align__(16) char dynamic[];
  SampleCodes* codes = reinterpret_cast<SampleCodes*>(dynamic);
  Sampler<T> s(a, lds, STEP == SAMPLE_WHOLE || STEP == SAMPLE_DRAW ? blockIdx.x : blockIdx.x / a.parts);
  if constexpr (STEP == SAMPLE_WHOLE) s.whole(codes);
  else if constexpr (STEP == SAMPLE_MAX) s.part_max();
  else if constexpr (STEP == SAMPLE_BINS) s.part_bins();
  else if constexpr (STEP == SAMPLE_SUMS) s.part_sums();
  else s.split_draw(codes);
}

}  // namespace elmo
