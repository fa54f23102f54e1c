// One token a row by temperature, top-k, top-p and min-p, from a given random number.
//
// Tokens are ordered by (logit falling, index rising).  Every filter keeps a beginning of that order, so the kept set is one logit
// (as an order-preserving 32-bit key) and the number of tokens equal to it that still belong (lowest indices first), and min-p a smallest weight.
// The token is the first one in order of index at which the kept weight so far exceeds u times the kept weight.
//
// Which token a number falls on is decided next to borders, so the weights are whole numbers, W = round(2^F exp((z - max z) / t)) from FP64, with
// F such that a row's sum stays below 2^63: sums are exact in any order and any split of a row gives the same token.
#pragma once
#include "rows.h"

namespace elmo {

constexpr int kSampleThreads = 1024;
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

// The row's weights: 2^F exp((z - M) / t) as a whole number.
struct Weigh {
  uint32_t top;                                // key of the maximum
  double M, rt;                                // maximum, 1 / temperature
  double one;                                  // 2^F
  __device__ inline uint64_t operator()(uint32_t key) const {
    if (key == top) return (uint64_t)one;
    if (key <= kKeyNone) return 0;
    return (uint64_t)(exp(((double)of_key(key) - M) * rt) * one + 0.5);
  }
};

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

__device__ inline uint64_t add64(uint64_t a, uint64_t b) { return a + b; }
template <int NW> __device__ inline uint64_t block_sum64(uint64_t v, uint64_t* s, int wave, int lane) {
  v = wave_reduce(v, add64);
  __syncthreads();
  if (lane == 0) s[wave] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < NW; ++i) v += s[i];
  return v;
}

template <class T>
__global__ __launch_bounds__(kSampleThreads) void k_sample_plain(SampleArgs a) {
  constexpr int NW = kSampleThreads / 64, LEVELS = sizeof(T) == 2 ? 2 : 4;
  __shared__ uint32_t s_key[NW], s_count[256];
  __shared__ uint64_t s_sum[NW], s_mass[256];
  __shared__ uint64_t s_found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const T* z = (const T*)a.z + row * a.zs;
  const RowSettings rs = settings_of(a, row);
  uint32_t top = kKeyNone;
  for (int64_t c = tid; c < a.V; c += kSampleThreads) top = max(top, key_of(load_one(z, c)));
  top = wave_reduce(top, [](uint32_t p, uint32_t q) { return max(p, q); });
  if (lane == 0) s_key[wave] = top;
  __syncthreads();
  for (int i = 0; i < NW; ++i) top = max(top, s_key[i]);
  if (top == kKeyNone) {
    if (tid == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.0f;
    }
    return;
  }
  const Weigh weigh{top, (double)of_key(top), 1.0 / rs.t, __builtin_ldexp(1.0, a.F)};
  // ---- the end of the kept order: key `edge` and how many of its tokens belong
  uint32_t edge = kKeyNone + 1;
  uint64_t ties = ~0ull;
  auto descend = [&](bool by_mass, uint64_t want) {       // smallest beginning of the order with count / weight >= want; returns the weight above the edge
    uint32_t prefix = 0;
    uint64_t above = 0, mass_above = 0;
    for (int l = 0; l < LEVELS; ++l) {
      const int sh = 24 - 8 * l;
      __syncthreads();
      if (tid < 256) { s_count[tid] = 0; s_mass[tid] = 0; }
      __syncthreads();
      for (int64_t c = tid; c < a.V; c += kSampleThreads) {
        const uint32_t key = key_of(load_one(z, c));
        if (key > kKeyNone && (l == 0 || (key >> (sh + 8)) == (prefix >> (sh + 8)))) {
          atomicAdd(&s_count[(key >> sh) & 255], 1u);
          atomicAdd((unsigned long long*)&s_mass[(key >> sh) & 255], (unsigned long long)weigh(key));
        }
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t n = above, m = mass_above;
        int b = 255;
        for (; b > 0; --b) {
          if ((by_mass ? m + s_mass[b] : n + s_count[b]) >= want) break;
          n += s_count[b];
          m += s_mass[b];
        }
        s_found[0] = b; s_found[1] = n; s_found[2] = m;
      }
      __syncthreads();
      prefix |= (uint32_t)s_found[0] << sh;
      above = s_found[1];
      mass_above = s_found[2];
    }
    edge = LEVELS == 2 && (prefix & 0x80000000u) == 0 ? prefix | 0xFFFFu : prefix;    // a negative BF16 value's key ends in ones
    const uint64_t w = weigh(edge);
    ties = by_mass ? (w ? (want - mass_above + w - 1) / w : ~0ull) : want - above;
    return mass_above;
  };
  uint64_t total = 0, below = 0;
  bool cut = false;
  uint64_t live = 0, mass = 0;                             // tokens above -infinity and their weight
  for (int64_t c = tid; c < a.V; c += kSampleThreads) {
    const uint32_t key = key_of(load_one(z, c));
    if (key > kKeyNone) { ++live; mass += weigh(key); }
  }
  live = block_sum64<NW>(live, s_sum, wave, lane);
  total = block_sum64<NW>(mass, s_sum, wave, lane);
  if ((uint64_t)rs.k < live) {
    below = descend(false, rs.k);
    total = below + ties * weigh(edge);
    cut = true;
  }
  if (rs.p < 1.0) {
    const uint64_t want = max((uint64_t)1, (uint64_t)__builtin_ceil(rs.p * (double)total));
    below = descend(true, min(want, total));
    total = below + ties * weigh(edge);
    cut = true;
  }
  const uint64_t least = rs.mp > 0.0 ? max((uint64_t)1, (uint64_t)__builtin_ceil(rs.mp * weigh.one)) : 1;
  // ---- kept weight (min-p may end it earlier), then the token, tile by tile in order of index
  uint64_t want = 0;
  __shared__ uint64_t s_scan[NW], s_tie[NW];
  for (int pass = 0; pass < 2; ++pass) {
    uint64_t before = 0, seen = 0;                         // kept weight and tokens at the edge in the tiles before
    for (int64_t c0 = 0; c0 < a.V; c0 += kSampleThreads) {
      const int64_t c = c0 + tid;
      const uint32_t key = c < a.V ? key_of(load_one(z, c)) : kKeyNone;
      uint64_t w = key > kKeyNone && key >= edge ? weigh(key) : 0;
      if (w < least) w = 0;
      const bool tie = cut && key == edge;
      const uint64_t votes = __ballot(tie);
      __syncthreads();
      if (lane == 0) s_tie[wave] = __popcll(votes);
      __syncthreads();
      uint64_t rank = seen + __popcll(votes & ((1ull << lane) - 1));
      for (int i = 0; i < NW; ++i) {
        if (i < wave) rank += s_tie[i];
        seen += s_tie[i];
      }
      if (tie && rank >= ties) w = 0;
      uint64_t upto = w;                                   // inclusive scan of the tile
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t other = __shfl_up(upto, o);
        if (lane >= o) upto += other;
      }
      if (lane == 63) s_scan[wave] = upto;
      __syncthreads();
      uint64_t tile = 0;
      for (int i = 0; i < NW; ++i) {
        if (i < wave) upto += s_scan[i];
        tile += s_scan[i];
      }
      upto += before;
      if (pass == 1 && w && upto > want && upto - w <= want) {
        a.token[row] = (int32_t)c;
        if (a.prob) a.prob[row] = (float)((double)w / (double)total);
      }
      before += tile;
    }
    if (pass == 0) {
      total = before;
      want = (uint64_t)(rs.u * (double)total);
      if (want >= total) want = total - 1;
    }
  }
}

}  // namespace elmo
