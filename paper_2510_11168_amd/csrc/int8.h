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

// ---------------------------------------------------------------------------------------------
// The product in tiles of TM x TN outputs (waves of 32 FM x 32 FN) over slabs of 128 bytes of K.
// ASYNC, for operands whose rows are 16-byte aligned: slabs go to LDS by asynchronous loads, NST stages; as in ring_stream_pp half of the waves
// issue behind the barrier (all of A and half of B) and half in the middle of the slab, so that one wave of every SIMD multiplies while the other is
// held by its loads.
// Otherwise a slab goes through registers, its loads in flight while the one before is multiplied, to the other of two stages.
// v_mfma_i32_32x32x32_i8: lane i holds row i % 32 of an operand, 16 bytes of K from 16 (i / 32) on.
// Tile row 32 j + l of a wave's columns holds weight row FN l + j: a lane then has FN neighbouring outputs of a row, and a wave stores 32 FN of them next
// to each other.  8192 x 14336 x 4096 in tiles of 256 x 256: 404 to 444 us, 2.2 to 2.4 POP/s (the library's product of that size, without scales: 442);
// bound by the matrix cores, 64 % busy, and their clock, which falls under random values.  Through registers: 574.
// ---------------------------------------------------------------------------------------------
template <int FN> struct Interleave {
  __device__ inline int operator()(int r) const { return (r & ~(32 * FN - 1)) + (r & 31) * FN + ((r >> 5) & (FN - 1)); }
};
template <int TM, int TN, int FM, int FN> constexpr int int8_threads() { return TM / FM * TN / FN / 16; }   // 64 a wave of 32 FM x 32 FN
template <int TM, int TN, int NST> constexpr int int8_smem() { return NST * (TM + TN) * 128 + (TM + 2 * TN) * 4; }

// Order of the tiles: strips of 8 tiles of rows, in each all columns, so that the workgroups of an XCD share operands in its L2.
__device__ inline void int8_tile(int id, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int strip = id / (8 * tiles_n), first = strip * 8, height = min(8, tiles_m - first);
  const int in = id - strip * 8 * tiles_n;
  tm = first + in % height;
  tn = in / height;
}

// FN neighbouring outputs, the first `valid` of them.
template <class O, int FN> __device__ inline void store_columns(O* p, int valid, const float (&f)[FN]) {
  if (valid >= FN) {
    if constexpr (sizeof(O) == 4) {
      typedef float vec __attribute__((ext_vector_type(FN)));
      typedef vec any __attribute__((aligned(4)));
      vec v;
#pragma unroll
      for (int j = 0; j < FN; ++j) v[j] = f[j];
      *reinterpret_cast<any*>(p) = v;
    } else if constexpr (FN > 1) {
      typedef uint32_t vec __attribute__((ext_vector_type(FN / 2)));
      typedef vec any __attribute__((aligned(2)));
      vec v;
#pragma unroll
      for (int j = 0; j < FN / 2; ++j) v[j] = pack_bf16(f[2 * j], f[2 * j + 1]);
      *reinterpret_cast<any*>(p) = v;
    } else {
      store_one(p, 0, f[0]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < FN; ++j)
      if (j < valid) store_one(p, j, f[j]);
  }
}

template <class O, int TM, int TN, int FM, int FN, int NST, bool ASYNC>
__global__ __launch_bounds__((int8_threads<TM, TN, FM, FN>())) void k_int8_tiles(Int8Args p, int tiles_m, int tiles_n) {
  constexpr int NT = int8_threads<TM, TN, FM, FN>(), NH = NT / 128, WGN = TN / 32 / FN, ABYTES = TM * 128, SBYTES = ABYTES + TN * 128, BH = TN / 2;
  constexpr int LPS_LATE = dma_loads_per_wave<BH, 128, NH>(), LPS_EARLY = dma_loads_per_wave<TM, 128, NH>() + LPS_LATE;
  static_assert((NST - 2) * LPS_EARLY <= 63, "ring depth");
  extern __shared__ __align__(256) char smem[];
  float* s_sa = reinterpret_cast<float*>(smem + NST * SBYTES);
  float* s_sb = s_sa + TM;
  float* s_bias = s_sb + TN;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WGN, wn = wave % WGN;
  const bool late = wave >= NH;
  int tm, tn;
  int8_tile(xcd_logical_id(blockIdx.x, gridDim.x), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * TM, n0 = tn * TN, mv = min(TM, p.M - m0), nv = min(TN, p.N - n0);
  const char* a = p.a + (int64_t)m0 * p.as;
  const char* b = p.b + (int64_t)n0 * p.bs;
  i32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x16{};

  const auto half_slab = [&](const char* __restrict__ sa, const char* __restrict__ sb, int h) {
#pragma unroll
    for (int kk = 2 * h; kk < 2 * h + 2; ++kk) {
      i32x4 fa[FM], fb[FN];
      const int c = 2 * kk + (lane >> 5), r = lane & 31;
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = *reinterpret_cast<const i32x4*>(sa + tile_off<128>(wm * 32 * FM + 32 * i + r, c));
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = *reinterpret_cast<const i32x4*>(sb + tile_off<128>(wn * 32 * FN + 32 * j + r, c));
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fa[i], fb[j], acc[i][j], 0, 0, 0);
    }
  };
  const int nk = p.K >> 7;
  // chunk id of a slab: tile row, place in it, and its row of the operand
  const auto chunk_row = [&](int id) {
    const int r = id >> 3;
    return r < TM ? a + (int64_t)min(r, mv - 1) * p.as : b + (int64_t)min(Interleave<FN>{}(r - TM), nv - 1) * p.bs;
  };
  const auto chunk_at = [&](int id) {
    const int r = id >> 3, c = id & 7;
    return r < TM ? tile_off<128>(r, c) : ABYTES + tile_off<128>(r - TM, c);
  };
  const auto run = [&](const char* __restrict__ ga, const char* __restrict__ gb, char* __restrict__ ring) {
    const auto issue = [&](int ks) {
      char* st = ring + (ks % NST) * SBYTES;
      const size_t at = (size_t)ks * 128;
      if (!late) {
        dma_tile<TM, 128, NH>(ga + at, p.as, mv, st, wave, lane);
        dma_tile<BH, 128, NH>(gb + at, p.bs, nv, st + ABYTES, wave, lane, 1 << 20, Interleave<FN>{});
      } else {
        dma_tile<BH, 128, NH>(gb + at, p.bs, nv, st + ABYTES + BH * 128, wave - NH, lane, 1 << 20, [](int r) { return BH + Interleave<FN>{}(r); });
      }
    };
    for (int s = 0; s < NST - 1; ++s)
      if (s < nk) issue(s);
    for (int ks = 0; ks < nk; ++ks) {
      if (late) wait_slabs<LPS_LATE, NST - 2>(nk - 1 - ks);
      else wait_slabs<LPS_EARLY, NST - 2>(nk - 1 - ks);
      barrier_nofence();
      const bool more = ks + NST - 1 < nk;
      if (more && !late) issue(ks + NST - 1);
      const char* st = ring + (ks % NST) * SBYTES;
      __builtin_amdgcn_sched_barrier(0);
      half_slab(st, st + ABYTES, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (more && late) issue(ks + NST - 1);
      __builtin_amdgcn_sched_barrier(0);
      half_slab(st, st + ABYTES, 1);
    }
  };
  if constexpr (ASYNC) {
    run(a, b, smem);
  } else {
    static_assert(NST == 2, "two stages");
    constexpr int NC = (TM + TN) * 8 / NT;
    const char* row[NC];
    i32x4 v[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) row[i] = chunk_row(i * NT + tid) + 16 * (tid & 7);
    const auto fetch = [&](int ks) {
#pragma unroll
      for (int i = 0; i < NC; ++i) v[i] = *reinterpret_cast<const i32x4_any1*>(row[i] + (size_t)ks * 128);
    };
    const auto lay = [&](int ks) {
#pragma unroll
      for (int i = 0; i < NC; ++i) *reinterpret_cast<i32x4*>(smem + (ks & 1) * SBYTES + chunk_at(i * NT + tid)) = v[i];
    };
    if (nk > 0) {
      fetch(0);
      lay(0);
    }
    for (int ks = 0; ks < nk; ++ks) {
      barrier_lds();
      if (ks + 1 < nk) fetch(ks + 1);
      const char* st = smem + (ks & 1) * SBYTES;
      half_slab(st, st + ABYTES, 0);
      half_slab(st, st + ABYTES, 1);
      if (ks + 1 < nk) lay(ks + 1);                        // (its stage was last read before this round's barrier)
    }
  }
  __syncthreads();
  // the last K % 128 bytes through registers, zeros behind them; the scales beside them
  if (p.K & 127) {
#pragma unroll 1
    for (int id = tid; id < (TM + TN) * 8; id += NT)
      *reinterpret_cast<i32x4*>(smem + chunk_at(id)) = load_k16(chunk_row(id), nk * 128 + 16 * (id & 7), p.K);
  }
  for (int i = tid; i < TM; i += NT) s_sa[i] = p.sa[m0 + min(i, mv - 1)];
  for (int i = tid; i < TN; i += NT) {
    s_sb[i] = p.sb[n0 + min(i, nv - 1)];
    s_bias[i] = p.bias ? p.bias[n0 + min(i, nv - 1)] : 0.0f;
  }
  __syncthreads();
  if (p.K & 127) {
    half_slab(smem, smem + ABYTES, 0);
    half_slab(smem, smem + ABYTES, 1);
  }
  // ---- scales, bias, output
  const int n = wn * 32 * FN + (lane & 31) * FN;
  float sb[FN], bias[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    sb[j] = s_sb[n + j];
    bias[j] = s_bias[n + j];
  }
  if (n < nv) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int m = wm * 32 * FM + 32 * i + acc_row(v, lane);
        if (m < mv) {
          const float sa = s_sa[m];
          float f[FN];
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            f[j] = (float)acc[i][j][v] * sa * sb[j];
            if (p.bias) f[j] += bias[j];
          }
          store_columns<O, FN>((O*)p.out + (int64_t)(m0 + m) * p.os + n0 + n, nv - n, f);
        }
      }
  }
}

// ---------------------------------------------------------------------------------------------
// Few tokens (at most 16 FM): the stream of the weights is the work (1 x 28672 x 8192: 37.6 us, 6.3 TB/s).  A workgroup has 16 weight rows, its eight
// waves take every eighth 256 bytes of K, and their sums are added in LDS.  Both operands go from memory to registers as v_mfma_i32_16x16x64_i8 takes them (lane i: row
// i % 16, 16 bytes from 16 (i / 16) on), four loads of each in flight; rows may begin anywhere.
// ---------------------------------------------------------------------------------------------
constexpr int kSkinnyThreads = 512, kSkinnySlab = 256;
template <class O, int FM>
__global__ __launch_bounds__(kSkinnyThreads) void k_int8_skinny(Int8Args p) {
  constexpr int NW = kSkinnyThreads / 64;
  __shared__ int s_acc[NW][FM * 4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, c = 16 * (lane >> 4), n0 = blockIdx.x * 16;
  const char* b = p.b + (int64_t)min(n0 + r, p.N - 1) * p.bs + c;
  const char* a[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) a[i] = p.a + (int64_t)min(16 * i + r, p.M - 1) * p.as + c;
  i32x4 acc[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) acc[i] = i32x4{0, 0, 0, 0};
  int k = wave * kSkinnySlab;
#pragma unroll 2
  for (; k + kSkinnySlab <= p.K; k += NW * kSkinnySlab) {
    i32x4 fb[4], fa[FM][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) fb[s] = *reinterpret_cast<const i32x4_any1*>(b + k + 64 * s);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int s = 0; s < 4; ++s) fa[i][s] = *reinterpret_cast<const i32x4_any1*>(a[i] + k + 64 * s);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i][s], fb[s], acc[i], 0, 0, 0);
  }
#pragma unroll 1
  for (int s = 0; s < 4 && k + 64 * s < p.K; ++s) {        // the row's end, for the wave whose turn it is
    const i32x4 fb = load_k16(b - c, k + 64 * s + c, p.K);
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_k16(a[i] - c, k + 64 * s + c, p.K), fb, acc[i], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int v = 0; v < 4; ++v) s_acc[wave][4 * i + v][lane] = acc[i][v];
  __syncthreads();
  // accumulator v of lane i: token 4 (i / 16) + v, weight row i % 16
  for (int id = tid; id < FM * 256; id += kSkinnyThreads) {
    const int n = n0 + (id & 15), v = (id >> 4) & 3, i = id >> 8, q = (id >> 6) & 3, from = q * 16 + (id & 15);
    int sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += s_acc[w][4 * i + v][from];
    const int m = 16 * i + 4 * q + v;
    if (m < p.M && n < p.N) store_out<O>(p, m, n, sum);
  }
}

}  // namespace elmo
