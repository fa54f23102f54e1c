// The sampling's workgroup on the host: Sampler of sample.h, its arithmetic and control flow as they are, with a fiber for each of its 1024 threads.  What
// the workgroup shares (LDS, the split rows' workspace) is kept in cells that know who touched them since the last barrier.  Reported are
//   an index outside its array, a load outside the row, a read of what nobody wrote, two threads at one cell between two barriers
//   without an atomic addition, and lanes of a wave or waves of the workgroup that wait for one another in different places.
// The headers are those of the library, but for the declarations that storage and the exchanges between lanes hang on (test_sample_host.py).
#include <math.h>
#include <setjmp.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <memory>
#include <string>
#include <type_traits>
#include <vector>

#define __device__
#define __host__
#define __constant__ static const
#define __forceinline__ inline __attribute__((always_inline))
#define __syncthreads() emu::barrier(__LINE__)
#define __popc __builtin_popcount
#define __builtin_amdgcn_readfirstlane(x) (x)

namespace emu {
constexpr int kThreads = 1024, kStack = 64 << 10;
struct Index { unsigned x; };
static Index thread, block;
static int me;                                   // the running thread, -1 outside of one
static uint32_t epoch;                           // barriers so far, over all launches
static std::string report;
static jmp_buf stop;
[[noreturn]] static void bad(const char* what, long long a = 0, long long b = 0) {
  char text[256];
  snprintf(text, sizeof text, "%s (%lld, %lld), workgroup %u thread %d", what, a, b, block.x, me);
  report = text;
  _longjmp(stop, 1);
}

// ---- cells
template <class T> struct Cell {
  T v;
  uint32_t wrote = 0, read = 0;                  // epochs of the last write and read, 0: never
  int16_t writer = -1, reader = -1;              // reader -2: more than one
  bool atomic = false;
  void reading() {
    if (!wrote) bad("a read of what nobody wrote");
    if (wrote == epoch && writer != me) bad("a read beside a write of the same interval", writer);
    reader = read == epoch && reader != me ? -2 : me;
    read = epoch;
  }
  void writing(bool add) {
    if (read == epoch && reader != me) bad("a write beside a read of the same interval", reader);
    if (wrote == epoch && writer != me && !(add && atomic)) bad("two writes of the same interval", writer);
    if (add && !wrote) bad("an addition to what nobody wrote");
    writer = wrote == epoch && writer != me ? -2 : me;      // -2: several, by additions
    wrote = epoch;
    atomic = add;
  }
  template <class U, class = std::enable_if_t<std::is_same<U, T>::value>> operator U() const { const_cast<Cell*>(this)->reading(); return v; }
  template <class U, class = std::enable_if_t<!std::is_same<U, T>::value>, class = void> explicit operator U() const { const_cast<Cell*>(this)->reading(); return (U)v; }
  Cell& operator=(T x) { writing(false); v = x; return *this; }
  Cell& operator=(const Cell& o) { return *this = (T)o; }
};
template <class T> struct Ptr {
  Cell<T>* c = nullptr;
  int64_t n = 0;
  Cell<T>& operator[](int64_t i) const {
    if (i < 0 || i >= n) bad("an index outside its array", i, n);
    return c[i];
  }
  Cell<T>& operator[](const Cell<uint32_t>& i) const { return (*this)[(int64_t)i]; }
};
template <class T, int N> struct Array {
  Cell<T> c[N];
  operator Ptr<T>() { return {c, N}; }
  Cell<T>& operator[](int64_t i) { return Ptr<T>{c, N}[i]; }
  const Cell<T>& operator[](int64_t i) const { return const_cast<Array*>(this)->operator[](i); }
};
template <class T> struct Same { typedef T type; };
template <class T, class U> T atomicAdd(Cell<T>* c, U x) {
  c->writing(true);
  const T was = c->v;
  c->v += (T)x;
  return was;
}

// ---- the row in memory
static const char *row_begin, *row_end;
static void global(const void* p, int64_t bytes) {
  if ((const char*)p < row_begin || (const char*)p + bytes > row_end) bad("a load outside the row", (const char*)p - row_begin, bytes);
}

// ---- threads
enum State { kRuns, kLane, kBarrier, kEnded };
struct Fiber { ucontext_t start; jmp_buf at; State state; int line; bool started; };
static Fiber fibers[kThreads];
static std::vector<char> stacks;
static ucontext_t origin;
static jmp_buf scheduler;
static const std::function<void()>* body;
static void entry() {
  (*body)();
  fibers[me].state = kEnded;
  _longjmp(scheduler, 1);
}
static void wait(State s, int line) {
  fibers[me].state = s;
  fibers[me].line = line;
  if (!_setjmp(fibers[me].at)) _longjmp(scheduler, 1);
}
static void barrier(int line) { wait(kBarrier, line); }
// What a wave's lanes bring to an exchange; `given` stays until all of them have taken their results.
static char given[kThreads][16], taken[kThreads][16];
typedef void (*Exchange)(int first);
static Exchange exchange[kThreads / 64];
template <class T> T exchanged(T v, Exchange f, int line) {
  static_assert(sizeof(T) <= 16, "a lane's value");
  memcpy(given[me], &v, sizeof v);
  exchange[me / 64] = f;
  wait(kLane, line);
  T r;
  memcpy(&r, taken[me], sizeof r);
  return r;
}
static void run(int t) {
  me = t;
  thread.x = t;
  if (_setjmp(scheduler)) return;
  if (fibers[t].started) _longjmp(fibers[t].at, 1);
  fibers[t].started = true;
  setcontext(&fibers[t].start);
}
static void launch(unsigned workgroup, const std::function<void()>& f) {
  if (stacks.empty()) stacks.resize((size_t)kThreads * kStack);
  block.x = workgroup;
  body = &f;
  ++epoch;
  for (int t = 0; t < kThreads; ++t) {
    getcontext(&fibers[t].start);
    fibers[t].start.uc_stack.ss_sp = stacks.data() + (size_t)t * kStack;
    fibers[t].start.uc_stack.ss_size = kStack;
    fibers[t].start.uc_link = &origin;
    makecontext(&fibers[t].start, entry, 0);
    fibers[t].state = kRuns;
    fibers[t].started = false;
  }
  for (;;) {
    for (int w = 0; w < kThreads / 64; ++w) {
      for (;;) {                                 // a wave as far as it goes
        for (int t = 64 * w; t < 64 * w + 64; ++t)
          if (fibers[t].state == kRuns) run(t);
        me = 64 * w;
        bool all = true, none = true;
        for (int t = 64 * w; t < 64 * w + 64; ++t) {
          const bool here = fibers[t].state == kLane;
          all &= here && fibers[t].line == fibers[64 * w].line;
          none &= !here;
        }
        if (none) break;
        if (!all) bad("lanes of a wave wait in different places", fibers[64 * w].line, w);
        exchange[w](64 * w);
        for (int t = 64 * w; t < 64 * w + 64; ++t) fibers[t].state = kRuns;
      }
      for (int t = 64 * w; t < 64 * w + 64; ++t)
        if (fibers[t].state != fibers[64 * w].state || (fibers[t].state == kBarrier && fibers[t].line != fibers[64 * w].line)) bad("a wave is torn at a barrier", fibers[t].line, w);
    }
    int line = -1;
    for (int t = 0; t < kThreads; ++t)
      if (fibers[t].state == kBarrier) {
        if (line >= 0 && fibers[t].line != line) bad("waves wait at different barriers", fibers[t].line, line);
        line = fibers[t].line;
      }
    if (line < 0) break;                         // all ended
    for (int t = 0; t < kThreads; ++t)
      if (fibers[t].state == kBarrier) fibers[t].state = kRuns;
    ++epoch;
  }
  ++epoch;
  me = -1;
}
}  // namespace emu

#define threadIdx emu::thread
#define blockIdx emu::block
using emu::atomicAdd;
template <class A, class B> inline auto min(const A& a, const B& b) { typedef std::common_type_t<A, B> C; const C x = a, y = b; return x < y ? x : y; }
template <class A, class B> inline auto max(const A& a, const B& b) { typedef std::common_type_t<A, B> C; const C x = a, y = b; return x > y ? x : y; }
static inline long long __double_as_longlong(double d) { return __builtin_bit_cast(long long, d); }

namespace elmo {
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
static inline float u2f(uint32_t u) { return __builtin_bit_cast(float, u); }
static inline uint32_t f2u(float f) { return __builtin_bit_cast(uint32_t, f); }
static inline float bf16_decode(uint16_t h) { return u2f((uint32_t)h << 16); }
}  // namespace elmo

#include "host_rows.h"

namespace elmo {
// The exchanges between a wave's lanes, by value.
template <class T, class Op> struct Reduce {
  static void all(int first) {
    T v[64], r;
    for (int i = 0; i < 64; ++i) memcpy(&v[i], emu::given[first + i], sizeof(T));
    r = v[0];
    for (int i = 1; i < 64; ++i) r = (*op)(r, v[i]);
    for (int i = 0; i < 64; ++i) memcpy(emu::taken[first + i], &r, sizeof(T));
  }
  static inline const Op* op;
};
template <int N = 64, class T, class Op> inline T wave_reduce(T v, Op op, int line = __builtin_LINE()) {
  static_assert(N == 64, "whole waves");
  Reduce<T, Op>::op = &op;
  return emu::exchanged(v, Reduce<T, Op>::all, line);
}
template <class U> inline U wave_scan(U v, int line = __builtin_LINE()) {
  return emu::exchanged(v, [](int first) {
    U sum = 0, x;
    for (int i = 0; i < 64; ++i) {
      memcpy(&x, emu::given[first + i], sizeof x);
      sum += x;
      memcpy(emu::taken[first + i], &sum, sizeof x);
    }
  }, line);
}
template <class T> struct Laned { T v; int lane; };
template <class T> inline T of_lane(T v, int lane, int line = __builtin_LINE()) {
  return emu::exchanged(Laned<T>{v, lane}, [](int first) {
    for (int i = 0; i < 64; ++i) {
      Laned<T> want, have;
      memcpy(&want, emu::given[first + i], sizeof want);
      memcpy(&have, emu::given[first + want.lane], sizeof have);
      memcpy(emu::taken[first + i], &have, sizeof have);
    }
  }, line).v;
}
template <int NW, class A, class Op> inline auto slots_reduce(A& slots, int lane, Op op) {
  auto r = slots[0] + 0;
  for (int i = 1; i < NW; ++i) r = op(r, slots[i] + 0);
  return r;
}
inline float wave_max(float v, int line = __builtin_LINE()) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }, line); }
}  // namespace elmo

#include "host_sample.h"

namespace {
template <class T> void sample_row(elmo::SampleArgs a, int64_t row) {
  using namespace elmo;
  const auto lds = std::make_unique<SampleLds>();
  const auto codes = std::make_unique<SampleCodes>();
  const auto all = [&](int64_t parts, auto step) {
    for (int64_t p = 0; p < parts; ++p) {
      memset((void*)lds.get(), 0, sizeof *lds);              // (nothing is written)
      memset((void*)codes.get(), 0, sizeof *codes);
      emu::launch((unsigned)(row * parts + p), [&] {
        Sampler<T> s(a, *lds, row);
        step(s);
      });
    }
  };
  emu::row_begin = (const char*)((const T*)a.z + row * a.zs);
  emu::row_end = emu::row_begin + a.V * sizeof(T);
  if (a.parts == 1) return all(1, [&](Sampler<T>& s) { s.whole(codes.get()); });
  all(a.parts, [&](Sampler<T>& s) { s.part_max(); });
  if (a.top_p) all(a.parts, [&](Sampler<T>& s) { s.part_bins(); });
  all(a.parts, [&](Sampler<T>& s) { s.part_sums(); });
  all(1, [&](Sampler<T>& s) { s.split_draw(codes.get()); });
}
}  // namespace

// The draws of `rows` rows, each over `parts` workgroups; what was wrong, or NULL.
extern "C" const char* host_sample(const void* z, int64_t stride, int fp32, int64_t rows, int64_t V, const float* u, const float* t, const int32_t* top_k,
                                   const float* top_p, const float* min_p, int32_t* token, float* prob, int parts) {
  int bits = 0;
  while (((int64_t)1 << bits) < V) ++bits;
  emu::report.clear();
  std::vector<char> ws;
  if (!_setjmp(emu::stop)) {
    if (parts > 1) ws.resize(rows * elmo::kSampleRowBytes);  // (zeros: nothing is written)
    elmo::SampleArgs a{z, stride, V, u, t, top_p, min_p, top_k, token, prob, std::min(50, 62 - bits), parts, ws.data()};
    for (int64_t r = 0; r < rows; ++r) {
      if (fp32) sample_row<float>(a, r);
      else sample_row<uint16_t>(a, r);
    }
    return nullptr;
  }
  return emu::report.c_str();
}
