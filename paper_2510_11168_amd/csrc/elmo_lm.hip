// C ABI of the operators at the output end of a language model (see include/elmo_head.h): norm, 8-bit integer product, sampling,
// distillation.
#include "../../include/elmo_head.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "distill.h"
#include "errors.h"
#include "int8.h"
#include "norm.h"
#include "sample.h"

namespace {

using elmo::check_launch;
using elmo::fail;

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;
constexpr int kNormMostD = 16384;                          // what a workgroup's registers hold

int check_rows(const char* what, int64_t rows, int64_t n, int64_t most) {
  if (rows < 0 || rows > kMostRows) return fail(-1, "%s: rows = %lld outside [0, 2^31)", what, (long long)rows);
  if (n < 1 || n > most) return fail(-1, "%s: row length %lld outside [1, %lld]", what, (long long)n, (long long)most);
  return 0;
}
int check_stride(const char* what, int64_t stride, int64_t n, int64_t rows) {
  if (rows > 1 && stride < n) return fail(-1, "%s = %lld is less than a row's %lld elements", what, (long long)stride, (long long)n);
  if (stride < 0 || stride > ((int64_t)1 << 40)) return fail(-1, "%s = %lld outside [0, 2^40]", what, (long long)stride);
  return 0;
}
bool is_real(int dtype) { return dtype == ELMO_BF16 || dtype == ELMO_FP32; }
int check_aligned(const char* what, const void* p, int dtype) {
  const uintptr_t size = dtype == ELMO_FP32 ? 4 : dtype == ELMO_BF16 ? 2 : 1;
  if ((uintptr_t)p & (size - 1)) return fail(-1, "%s must be aligned to its elements", what);
  return 0;
}
// Work-items of a launch are counted in 32 bits.
constexpr bool fits(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }
int check_grid(const char* what, int64_t workgroups, int threads) {
  if (!fits(workgroups, threads)) return fail(-1, "%s: more rows than one launch takes", what);
  return 0;
}
// Opt in to more than 64 KiB of LDS, once for each kernel and device, whichever host thread comes first.
constexpr int kMostDevices = 64;
template <class Kernel> int raise_lds(Kernel* kernel, int bytes, std::once_flag (&once)[kMostDevices], hipError_t (&rc)[kMostDevices]) {
  int dev = -1;
  ELMO_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMostDevices) return fail(-3, "device ordinal %d outside [0, %d)", dev, kMostDevices);
  std::call_once(once[dev], [&] { rc[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
  if (rc[dev] != hipSuccess) return fail(-3, "hipFuncSetAttribute failed: %s", hipGetErrorString(rc[dev]));
  return 0;
}
#define ELMO_TRY(call) do { if (int rc_ = (call)) return rc_; } while (0)

// ---- norm: waves of a row and octets of a lane.  Short rows a wave each, without a barrier; longer ones four waves, with as much in flight in fewer
// registers (replayed in a graph, 16384 rows of 1024 BF16 -> INT8: 25.4 us with one wave, 31.4 with four; of 4096: 107 and 95, and 88 on buffers that take turns; 1 row of 4096:
// 8.8 and 4.1).
struct RowShape { int wpr, steps; };
RowShape norm_shape(int d) {
  if (d <= 1024) return {1, (d + 511) / 512};
  if (d <= 8192) return {4, (d + 2047) / 2048};
  return {16, 2};
}
int pow2_at_least(int n) { int p = 1; while (p < n) p *= 2; return p; }

template <class T, int OUT, int WPR, int S> int launch_norm(const elmo::NormArgs& a, hipStream_t st) {
  constexpr int threads = elmo::norm_threads(WPR), rpg = threads / (64 * WPR);
  ELMO_TRY(check_grid("elmo_rms_norm", (a.rows + rpg - 1) / rpg, threads));
  elmo::k_rms_norm<T, OUT, WPR, S><<<(unsigned)((a.rows + rpg - 1) / rpg), threads, 0, st>>>(a);
  return check_launch("k_rms_norm");
}
template <class T, int OUT> int launch_norm_shape(const elmo::NormArgs& a, hipStream_t st) {
  const RowShape r = norm_shape(a.d);
  const int s = pow2_at_least(r.steps);
#define ELMO_NORM(W, S) if (r.wpr == W && s == S) return launch_norm<T, OUT, W, S>(a, st)
  ELMO_NORM(1, 1); ELMO_NORM(1, 2);
  ELMO_NORM(4, 1); ELMO_NORM(4, 2); ELMO_NORM(4, 4);
#undef ELMO_NORM
  return launch_norm<T, OUT, 16, 2>(a, st);
}
template <class T> int launch_norm_out(const elmo::NormArgs& a, int out, hipStream_t st) {
  if (out == ELMO_BF16) return launch_norm_shape<T, elmo::OUT_BF16>(a, st);
  if (out == ELMO_FP32) return launch_norm_shape<T, elmo::OUT_FP32>(a, st);
  if (out == ELMO_FP8_E4M3) return launch_norm_shape<T, elmo::OUT_E4M3>(a, st);
  return launch_norm_shape<T, elmo::OUT_INT8>(a, st);
}

// Backward: a team of waves keeps its columns' share of the weight gradient over all rows it takes, and a workgroup leaves one share: 512 of them (16384 x
// 4096 BF16, replayed in a graph: 105 us; 256 of them 127, 1024 of them 113).
constexpr int kNormShares = 512;
int back_shares(int64_t rows, int64_t d) {
  const int64_t teams = d <= 1024 ? 4 : 1;               // of a workgroup
  return (int)std::min<int64_t>((rows + teams - 1) / teams, kNormShares);
}
template <class T, int WPR, int S> void launch_back(const elmo::NormBackArgs& a, hipStream_t st) {
  elmo::k_rms_norm_back<T, WPR, S><<<a.shares, elmo::norm_threads(WPR), 0, st>>>(a);
}
template <class T> void launch_back_shape(const elmo::NormBackArgs& a, hipStream_t st) {
  const RowShape r = norm_shape(a.d);
  const int s = pow2_at_least(r.steps);
#define ELMO_BACK(W, S) if (r.wpr == W && s == S) return launch_back<T, W, S>(a, st)
  ELMO_BACK(1, 1); ELMO_BACK(1, 2);
  ELMO_BACK(4, 1); ELMO_BACK(4, 2); ELMO_BACK(4, 4);
  ELMO_BACK(16, 2);
#undef ELMO_BACK
}

}  // namespace

extern "C" int elmo_rms_norm(const void* x, int64_t x_stride, int dtype, int64_t rows, int64_t d, const void* residual, int64_t residual_stride,
                             const void* weight, int weight_dtype, float eps, void* sum_out, int64_t sum_stride, void* y, int64_t y_stride,
                             int y_dtype, float* scale_out, void* hip_stream) {
  if (!is_real(dtype)) return fail(-2, "dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", dtype);
  if (weight && !is_real(weight_dtype)) return fail(-2, "weight_dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", weight_dtype);
  if (!is_real(y_dtype) && y_dtype != ELMO_FP8_E4M3 && y_dtype != ELMO_INT8) return fail(-2, "unsupported y_dtype %d", y_dtype);
  ELMO_TRY(check_rows("elmo_rms_norm", rows, d, kNormMostD));
  if (!(eps >= 0.0f) || eps > 1e30f) return fail(-1, "eps must be >= 0 and finite (got %g)", (double)eps);
  if (rows == 0) return 0;
  if (!x || !y) return fail(-1, "x and y must not be NULL");
  if (sum_out && !residual) return fail(-1, "sum_out needs a residual");
  if (!is_real(y_dtype) && !scale_out) return fail(-1, "8-bit rows need scale_out");
  if (is_real(y_dtype) && scale_out) return fail(-1, "scale_out goes with 8-bit rows only");
  ELMO_TRY(check_stride("x_stride", x_stride, d, rows));
  ELMO_TRY(check_stride("y_stride", y_stride, d, rows));
  if (residual) ELMO_TRY(check_stride("residual_stride", residual_stride, d, rows));
  if (sum_out) ELMO_TRY(check_stride("sum_stride", sum_stride, d, rows));
  ELMO_TRY(check_aligned("x", x, dtype));
  ELMO_TRY(check_aligned("residual", residual, dtype));
  ELMO_TRY(check_aligned("sum_out", sum_out, dtype));
  ELMO_TRY(check_aligned("weight", weight, weight_dtype));
  ELMO_TRY(check_aligned("y", y, y_dtype));
  ELMO_TRY(check_aligned("scale_out", scale_out, ELMO_FP32));
  const elmo::NormArgs a{x, residual, weight, sum_out, y, scale_out, rows, x_stride, residual_stride, sum_stride, y_stride, (int)d, eps,
                         weight_dtype == ELMO_FP32};
  return dtype == ELMO_BF16 ? launch_norm_out<uint16_t>(a, y_dtype, (hipStream_t)hip_stream) : launch_norm_out<float>(a, y_dtype, (hipStream_t)hip_stream);
}

extern "C" size_t elmo_rms_norm_backward_bytes(int64_t rows, int64_t d) {
  return rows < 1 || d < 1 || d > kNormMostD ? 0 : (size_t)back_shares(rows, d) * (size_t)d * sizeof(float);
}

extern "C" int elmo_rms_norm_backward(const void* dy, int64_t dy_stride, const void* h, int64_t h_stride, int dtype, int64_t rows, int64_t d,
                                      const void* weight, int weight_dtype, float eps, const void* dsum, int64_t dsum_stride, void* dh,
                                      int64_t dh_stride, float* dweight, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!is_real(dtype)) return fail(-2, "dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", dtype);
  if (weight && !is_real(weight_dtype)) return fail(-2, "weight_dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", weight_dtype);
  ELMO_TRY(check_rows("elmo_rms_norm_backward", rows, d, kNormMostD));
  if (!(eps >= 0.0f) || eps > 1e30f) return fail(-1, "eps must be >= 0 and finite (got %g)", (double)eps);
  ELMO_TRY(check_aligned("dweight", dweight, ELMO_FP32));
  hipStream_t st = (hipStream_t)hip_stream;
  const int shares = back_shares(rows, d);
  if (rows > 0) {
    if (!dy || !h || !dh) return fail(-1, "dy, h and dh must not be NULL");
    ELMO_TRY(check_stride("dy_stride", dy_stride, d, rows));
    ELMO_TRY(check_stride("h_stride", h_stride, d, rows));
    ELMO_TRY(check_stride("dh_stride", dh_stride, d, rows));
    if (dsum) ELMO_TRY(check_stride("dsum_stride", dsum_stride, d, rows));
    ELMO_TRY(check_aligned("dy", dy, dtype));
    ELMO_TRY(check_aligned("h", h, dtype));
    ELMO_TRY(check_aligned("dh", dh, dtype));
    ELMO_TRY(check_aligned("dsum", dsum, dtype));
    ELMO_TRY(check_aligned("weight", weight, weight_dtype));
    if (dweight && (!workspace || workspace_bytes < elmo_rms_norm_backward_bytes(rows, d)))
      return fail(-1, "workspace missing or smaller than %zu bytes", elmo_rms_norm_backward_bytes(rows, d));
    if (dweight) ELMO_TRY(check_aligned("workspace", workspace, ELMO_FP32));
    const elmo::NormBackArgs a{dy, h, weight, dsum, dh, dweight ? (float*)workspace : nullptr, rows, dy_stride, h_stride, dsum_stride, dh_stride,
                               (int)d, shares, eps, weight_dtype == ELMO_FP32};
    if (dtype == ELMO_BF16) launch_back_shape<uint16_t>(a, st);
    else launch_back_shape<float>(a, st);
    ELMO_TRY(check_launch("k_rms_norm_back"));
  }
  if (!dweight) return 0;
  elmo::k_norm_dweight<<<(unsigned)((d + elmo::kDweightCols - 1) / elmo::kDweightCols), elmo::kDweightThreads, 0, st>>>((const float*)workspace, shares,
                                                                                                                       (int)d, dweight);
  return check_launch("k_norm_dweight");
}

namespace {
template <class O, int TM, int TN, int FM, int FN, int NST, bool ASYNC> int launch_int8_as(const elmo::Int8Args& p, hipStream_t st) {
  constexpr int smem = elmo::int8_smem<TM, TN, NST>();
  static_assert(smem <= 160 * 1024, "LDS of the tiles");
  const int tiles_m = (p.M + TM - 1) / TM, tiles_n = (p.N + TN - 1) / TN;
  ELMO_TRY(check_grid("elmo_int8_matmul", (int64_t)tiles_m * tiles_n, elmo::int8_threads<TM, TN, FM, FN>()));
  static std::once_flag once[kMostDevices];
  static hipError_t attr[kMostDevices];
  ELMO_TRY(raise_lds(&elmo::k_int8_tiles<O, TM, TN, FM, FN, NST, ASYNC>, smem, once, attr));
  elmo::k_int8_tiles<O, TM, TN, FM, FN, NST, ASYNC><<<tiles_m * tiles_n, elmo::int8_threads<TM, TN, FM, FN>(), smem, st>>>(p, tiles_m, tiles_n);
  return check_launch("k_int8_tiles");
}
template <class O, int TM, int TN, int FM, int FN, int NST> int launch_int8_tiles(const elmo::Int8Args& p, bool aligned, hipStream_t st) {
  return aligned ? launch_int8_as<O, TM, TN, FM, FN, NST, true>(p, st) : launch_int8_as<O, TM, TN, FM, FN, 2, false>(p, st);
}
template <class O, int FM> int launch_int8_skinny(const elmo::Int8Args& p, hipStream_t st) {
  ELMO_TRY(check_grid("elmo_int8_matmul", (p.N + 15) / 16, elmo::kSkinnyThreads));
  elmo::k_int8_skinny<O, FM><<<(unsigned)((p.N + 15) / 16), elmo::kSkinnyThreads, 0, st>>>(p);
  return check_launch("k_int8_skinny");
}
// Which kernel (times in us, MI355X, BF16 outputs):
//  - up to 16 tokens the kernel that streams the weights into registers, where its workgroups have K enough for their eight waves (1 x 4096 x 4096
//    4.9, 64 x 64 tiles 12.4; 16 x 8192 x 8192 18.2 / 23.3) or are few; wide and short it loses (16 x 131072 x 768 33.0 / 23.2).  Up to 32 tokens it reads
//    the tokens as often as that again and pays for one round of workgroups only (32 x 4096 x 4096 8.0 / 13.3; 32 x 32000 x 4096 46 / 23).
//  - else tiles, by the time of the rounds in which they go over the 256 CUs at K = 4096: 256 x 256 63 a round of 256, 128 x 128 40 a round of 512 (two a
//    CU; 26 if there are only 256), 64 x 64 18 a round of 512 (14).  8192 x 14336: 406 in tiles of 256, 502 of 128; 2048 x 4096: 50 / 41;
//    512 x 4096: 42 / 22.5 / 18.8.
//  - of these only what one launch takes: M and N go up to 2^30, which smaller tiles are too many for (and more than 2^27 outputs a token the streaming kernel).
int64_t int8_tiles(int64_t M, int64_t N, int t) { return ((M + t - 1) / t) * ((N + t - 1) / t); }
int int8_tile_of(int64_t M, int64_t N, int64_t K) {        // 0: the streaming kernel
  const auto rounds = [](int64_t n, int64_t slots) { return (n + slots - 1) / slots; };
  if (((M <= 16 && (K >= 2048 || N <= 16384)) || (M <= 32 && N <= 4096)) && fits((N + 15) / 16, elmo::kSkinnyThreads)) return 0;
  const int64_t n256 = int8_tiles(M, N, 256), n128 = int8_tiles(M, N, 128), n64 = int8_tiles(M, N, 64);
  const int64_t t256 = 63 * rounds(n256, 256), t128 = !fits(n128, elmo::int8_threads<128, 128, 1, 2>()) ? INT64_MAX : n128 <= 256 ? 26 : 40 * rounds(n128, 512),
                t64 = !fits(n64, elmo::int8_threads<64, 64, 1, 1>()) ? INT64_MAX : n64 <= 256 ? 14 : 18 * rounds(n64, 512);
  return t256 <= t128 && t256 <= t64 ? 256 : t128 <= t64 ? 128 : 64;
}
template <class O> int launch_int8(elmo::Int8Args p, hipStream_t st) {
  if (p.M == 1) p.as = 0;                                  // (a single row's stride means nothing)
  if (p.N == 1) p.bs = 0;
  // (row offsets within a tile are formed from 24-bit factors)
  const bool aligned = !(((uintptr_t)p.a | (uintptr_t)p.b | (uint64_t)p.as | (uint64_t)p.bs) & 15) && p.as < (1 << 24) && p.bs < (1 << 24);
  switch (int8_tile_of(p.M, p.N, p.K)) {
    case 0: return p.M <= 16 ? launch_int8_skinny<O, 1>(p, st) : launch_int8_skinny<O, 2>(p, st);
    case 256: return launch_int8_tiles<O, 256, 256, 2, 4, 2>(p, aligned, st);
    case 128: return launch_int8_tiles<O, 128, 128, 1, 2, 2>(p, aligned, st);
    default: return launch_int8_tiles<O, 64, 64, 1, 1, 4>(p, aligned, st);
  }
}
constexpr int64_t kInt8Most = (int64_t)1 << 30, kInt8MostK = 131071;      // 131071 products of 128 x 128 stay below 2^31
}  // namespace

extern "C" int elmo_int8_matmul_tile(int64_t M, int64_t N, int64_t K) {
  if (M < 1 || M > kInt8Most || N < 1 || N > kInt8Most || K < 0 || K > kInt8MostK) return fail(-1, "M and N must be in [1, 2^30], K in [0, %lld]", (long long)kInt8MostK);
  const int t = int8_tile_of(M, N, K);
  if (t == 256) ELMO_TRY(check_grid("elmo_int8_matmul", int8_tiles(M, N, 256), elmo::int8_threads<256, 256, 2, 4>()));
  return t;
}

extern "C" int elmo_int8_matmul(const int8_t* a, int64_t a_stride, const float* a_scale, const int8_t* b, int64_t b_stride, const float* b_scale,
                                const float* bias, int64_t M, int64_t N, int64_t K, void* out, int64_t out_stride, int out_dtype,
                                void* hip_stream) {
  if (!is_real(out_dtype)) return fail(-2, "out_dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", out_dtype);
  if (M < 0 || M > kInt8Most || N < 0 || N > kInt8Most) return fail(-1, "M = %lld and N = %lld must be in [0, 2^30]", (long long)M, (long long)N);
  if (K < 0 || K > kInt8MostK) return fail(-1, "K = %lld outside [0, %lld]: longer sums do not fit 32 bits", (long long)K, (long long)kInt8MostK);
  if (M == 0 || N == 0) return 0;
  if ((K > 0 && (!a || !b)) || !a_scale || !b_scale || !out) return fail(-1, "a, b, a_scale, b_scale and out must not be NULL");
  ELMO_TRY(check_stride("a_stride", a_stride, K, M));
  ELMO_TRY(check_stride("b_stride", b_stride, K, N));
  ELMO_TRY(check_stride("out_stride", out_stride, N, M));
  ELMO_TRY(check_aligned("a_scale", a_scale, ELMO_FP32));
  ELMO_TRY(check_aligned("b_scale", b_scale, ELMO_FP32));
  ELMO_TRY(check_aligned("bias", bias, ELMO_FP32));
  ELMO_TRY(check_aligned("out", out, out_dtype));
  const elmo::Int8Args p{(const char*)a, (const char*)b, a_scale, b_scale, bias, out, a_stride, b_stride, out_stride, (int)M, (int)N, (int)K};
  hipStream_t st = (hipStream_t)hip_stream;
  return out_dtype == ELMO_BF16 ? launch_int8<uint16_t>(p, st) : launch_int8<float>(p, st);
}

namespace {
constexpr int64_t kMostV = ((int64_t)1 << 31) - 1;

// Workgroups of a row without top-k: one where the rows fill the chip or are short.  Top-p, us, split and (a row more, or an element less) whole.  FP32:
// 128 rows of 131072 71 and 122, one of 16384 21.8 and 23.5.  BF16, where one workgroup takes a row by codes in about half the time: 32 rows of 131072 37 and
// 44, of 65536 30 and 32, one row of 65536 23 and 28; one of 32768 22.5 and 20.3; 64 rows of 131072 48 and 44.
constexpr int64_t kSampleSplitRows = 128, kSampleSplitV = 16384, kSampleSplitRowsBf16 = 32, kSampleSplitVBf16 = 65536;
int sample_parts(int64_t rows, int64_t V, bool bf16) {
  if (rows > (bf16 ? kSampleSplitRowsBf16 : kSampleSplitRows) || V < (bf16 ? kSampleSplitVBf16 : kSampleSplitV)) return 1;
  return (int)std::min<int64_t>(std::min<int64_t>(64, (V + 4095) / 4096), std::max<int64_t>(2, 256 / rows));
}
template <class T, int STEP> int launch_sample_step(const elmo::SampleArgs& a, unsigned grid, hipStream_t st) {
  constexpr int smem = elmo::sample_smem<T, STEP>();
  static_assert(smem + sizeof(elmo::SampleLds) <= 160 * 1024, "LDS of a row");
  if constexpr (smem > 0) {
    static std::once_flag once[kMostDevices];
    static hipError_t attr[kMostDevices];
    ELMO_TRY(raise_lds(&elmo::k_sample<T, STEP>, smem, once, attr));
  }
  elmo::k_sample<T, STEP><<<grid, elmo::kSampleThreads, smem, st>>>(a);
  return check_launch("k_sample");
}
template <class T> int launch_sample(const elmo::SampleArgs& a, int64_t rows, hipStream_t st) {
  ELMO_TRY(check_grid("elmo_sample", rows * a.parts, elmo::kSampleThreads));
  const unsigned one = (unsigned)rows, all = (unsigned)(rows * a.parts);
  if (a.parts == 1) return launch_sample_step<T, elmo::SAMPLE_WHOLE>(a, one, st);
  ELMO_TRY((launch_sample_step<T, elmo::SAMPLE_MAX>(a, all, st)));
  if (a.top_p) ELMO_TRY((launch_sample_step<T, elmo::SAMPLE_BINS>(a, all, st)));
  ELMO_TRY((launch_sample_step<T, elmo::SAMPLE_SUMS>(a, all, st)));
  return launch_sample_step<T, elmo::SAMPLE_DRAW>(a, one, st);
}
}  // namespace

extern "C" size_t elmo_sample_bytes(int64_t rows, int64_t V) {
  return rows < 1 || rows > kSampleSplitRows || V < kSampleSplitV ? 0 : (size_t)rows * elmo::kSampleRowBytes;
}

extern "C" int elmo_sample(const void* logits, int64_t logits_stride, int dtype, int64_t rows, int64_t V, const float* u, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p, int32_t* idx_out, float* prob_out, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  if (!is_real(dtype)) return fail(-2, "dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", dtype);
  ELMO_TRY(check_rows("elmo_sample", rows, V, kMostV));
  if (rows == 0) return 0;
  if (!logits || !u || !idx_out) return fail(-1, "logits, u and idx_out must not be NULL");
  ELMO_TRY(check_stride("logits_stride", logits_stride, V, rows));
  ELMO_TRY(check_aligned("logits", logits, dtype));
  for (const void* p : {(const void*)u, (const void*)temperature, (const void*)top_k, (const void*)top_p, (const void*)min_p, (const void*)idx_out,
                        (const void*)prob_out})
    ELMO_TRY(check_aligned("u, temperature, top_k, top_p, min_p, idx_out and prob_out", p, ELMO_FP32));
  int bits = 0;
  while (((int64_t)1 << bits) < V) ++bits;
  // (with top-k the few tokens that stay are found faster by one workgroup)
  const int parts = top_k ? 1 : sample_parts(rows, V, dtype == ELMO_BF16);
  const size_t need = parts == 1 ? 0 : elmo_sample_bytes(rows, V);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return fail(-1, "workspace missing, smaller than %zu bytes or not 256-byte aligned", need);
  const elmo::SampleArgs a{logits, logits_stride, V, u, temperature, top_p, min_p, top_k, idx_out, prob_out, std::min(50, 62 - bits),
                           parts, (char*)workspace};
  hipStream_t st = (hipStream_t)hip_stream;
  return dtype == ELMO_BF16 ? launch_sample<uint16_t>(a, rows, st) : launch_sample<float>(a, rows, st);
}

namespace {
// Workgroups of a row: one where the rows fill the chip or are short, else up to 64, each with at least one round of octets (131072 BF16: 1 row 8.7 - 11 us,
// 128 rows 24.0, 129 rows, a workgroup each, 31.0).
int distill_parts(int64_t rows, int64_t V) {
  const int64_t rounds = (V / 8 + elmo::kDistillThreads - 1) / elmo::kDistillThreads;
  if (rows > 128 || rounds < 4) return 1;
  const int64_t parts = std::min<int64_t>(std::min<int64_t>(rounds, 64), 512 / rows);
  const int64_t per = (rounds + parts - 1) / parts;
  return (int)((rounds + per - 1) / per);
}
template <class T> int launch_distill(const elmo::DistillArgs& a, hipStream_t st) {
  ELMO_TRY(check_grid("elmo_distill", a.rows * a.parts, elmo::kDistillThreads));
  const unsigned grid = (unsigned)(a.rows * a.parts);
  if (a.parts == 1) {
    elmo::k_distill<T, elmo::DISTILL_WHOLE><<<grid, elmo::kDistillThreads, 0, st>>>(a);
    return check_launch("k_distill");
  }
  elmo::k_distill<T, elmo::DISTILL_SUMS><<<grid, elmo::kDistillThreads, 0, st>>>(a);
  ELMO_TRY(check_launch("k_distill (sums)"));
  elmo::k_distill<T, elmo::DISTILL_GRADIENT><<<grid, elmo::kDistillThreads, 0, st>>>(a);
  return check_launch("k_distill (gradient)");
}
}  // namespace

extern "C" size_t elmo_distill_bytes(int64_t rows, int64_t V) {
  if (rows < 1 || V < 1) return 0;
  const int parts = distill_parts(rows, V);
  return parts == 1 ? 0 : (size_t)rows * (parts * sizeof(elmo::MaxSum) + elmo::kDistillMaxK * sizeof(float));
}

extern "C" int elmo_distill(const void* logits, int64_t logits_stride, int dtype, int64_t rows, int64_t V, const int32_t* teacher_idx,
                            const void* teacher_logits, int teacher_dtype, int64_t K, float temperature, const float* row_weight, float* loss_out,
                            void* grad_out, int64_t grad_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!is_real(dtype)) return fail(-2, "dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", dtype);
  if (!is_real(teacher_dtype)) return fail(-2, "teacher_dtype must be ELMO_BF16 or ELMO_FP32 (got %d)", teacher_dtype);
  ELMO_TRY(check_rows("elmo_distill", rows, V, kMostV));
  if (K < 1 || K > elmo::kDistillMaxK) return fail(-1, "K = %lld outside [1, %d]", (long long)K, elmo::kDistillMaxK);
  if (!(temperature > 0.0f) || !(temperature <= 1e6f) || temperature < 1e-6f) return fail(-1, "temperature must be in [1e-6, 1e6] (got %g)", (double)temperature);
  if (rows == 0) return 0;
  if (!logits || !teacher_idx || !teacher_logits || !loss_out) return fail(-1, "logits, teacher_idx, teacher_logits and loss_out must not be NULL");
  ELMO_TRY(check_stride("logits_stride", logits_stride, V, rows));
  if (grad_out) ELMO_TRY(check_stride("grad_stride", grad_stride, V, rows));
  ELMO_TRY(check_aligned("logits", logits, dtype));
  ELMO_TRY(check_aligned("grad_out", grad_out, dtype));
  ELMO_TRY(check_aligned("teacher_logits", teacher_logits, teacher_dtype));
  for (const void* p : {(const void*)teacher_idx, (const void*)row_weight, (const void*)loss_out})
    ELMO_TRY(check_aligned("teacher_idx, row_weight and loss_out", p, ELMO_FP32));
  const size_t need = elmo_distill_bytes(rows, V);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return fail(-1, "workspace missing, smaller than %zu bytes or not 256-byte aligned", need);
  const elmo::DistillArgs a{logits, teacher_idx, teacher_logits, row_weight, loss_out, grad_out, logits_stride, grad_stride, rows, V, (int)K, temperature,
                            (float)(1.4426950408889634 / (double)temperature), teacher_dtype == ELMO_FP32, distill_parts(rows, V), workspace};
  hipStream_t st = (hipStream_t)hip_stream;
  return dtype == ELMO_BF16 ? launch_distill<uint16_t>(a, st) : launch_distill<float>(a, st);
}
