// Runs the typed layers' kernels on the CPU, thread by thread (hip/hip_runtime.h): their results are
// compared, and every array of the caller lies between pages that end the program when they are touched,
// at their beginning and at their end in turn.
// usage: model SCENARIO ARGUMENTS; prints what went wrong and ends with 1 (3: a page was touched).
#include <signal.h>
#include <sys/mman.h>
#include <sys/wait.h>
#include <unistd.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>

#include "../../paper_2411_16025_amd/csrc/groups.h"

dim3 threadIdx, blockIdx, gridDim;

// ---- fibers ------------------------------------------------------------------------

asm(R"(
.text
.globl model_switch
model_switch:
  push %rbp
  push %rbx
  push %r12
  push %r13
  push %r14
  push %r15
  mov %rsp, (%rdi)
  mov %rsi, %rsp
  pop %r15
  pop %r14
  pop %r13
  pop %r12
  pop %rbx
  pop %rbp
  ret
)");
extern "C" void model_switch(void** save, void* to);

namespace model {
namespace {

[[noreturn]] void fail(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vprintf(fmt, ap);
  va_end(ap);
  printf(" (workgroup %u, thread %u)\n", blockIdx.x, threadIdx.x);
  fflush(stdout);
  _exit(1);
}

enum State { kReady, kWave, kBarrier, kDone };
struct Thread {
  void* sp;
  char* stack;
  State state;
  const char* what;
};
struct Wave {
  Given given[2];
  int turn;
};
constexpr size_t kStack = 256 << 10;
std::vector<Thread> g_threads;
std::vector<Wave> g_waves;
void* g_main;
int g_now;
void (*g_go)(void*);
void* g_self;

void leave(State s) {
  Thread& t = g_threads[g_now];
  t.state = s;
  model_switch(&t.sp, g_main);
}

void entry() {
  g_go(g_self);
  leave(kDone);
  abort();
}

void workgroup(unsigned threads) {
  while (g_threads.size() < threads)
    g_threads.push_back({nullptr, (char*)mmap(nullptr, kStack, PROT_READ | PROT_WRITE,
                                              MAP_PRIVATE | MAP_ANONYMOUS, -1, 0),
                         kDone, ""});
  g_waves.resize((threads + 63) / 64);
  for (unsigned t = 0; t < threads; ++t) {
    void** p = (void**)(g_threads[t].stack + kStack - 64);
    *p = (void*)entry;
    for (int i = 1; i <= 6; ++i) p[-i] = nullptr;
    g_threads[t].sp = p - 6;
    g_threads[t].state = kReady;
  }
  for (auto& w : g_waves) w.turn = 0;
  for (;;) {
    bool ran = false, all_at_barrier = true, any = false;
    for (unsigned w = 0; w < g_waves.size(); ++w) {
      const unsigned beg = 64 * w, end = std::min(beg + 64, threads);
      for (;;) {
        // the lanes that wait for each other go on when none is elsewhere
        uint64_t waiting = 0;
        bool barrier = false, ready = false;
        const char* what = nullptr;
        for (unsigned t = beg; t < end; ++t) {
          const Thread& th = g_threads[t];
          if (th.state == kWave) {
            waiting |= 1ull << (t - beg);
            if (what && strcmp(what, th.what)) {
              threadIdx.x = t;
              fail("lanes of a wavefront at different instructions: %s and %s", what, th.what);
            }
            what = th.what;
          }
          barrier |= th.state == kBarrier;
          ready |= th.state == kReady;
        }
        if (waiting && !ready) {
          if (barrier) {
            threadIdx.x = beg;
            fail("lanes of a wavefront at a barrier and at %s", what);
          }
          g_waves[w].given[g_waves[w].turn].lanes = waiting;
          g_waves[w].turn ^= 1;
          for (unsigned t = beg; t < end; ++t)
            if (g_threads[t].state == kWave) g_threads[t].state = kReady;
          ready = true;
        }
        if (!ready) break;
        for (unsigned t = beg; t < end; ++t)
          if (g_threads[t].state == kReady) {
            ran = true;
            g_now = (int)t;
            threadIdx = dim3(t);
            model_switch(&g_main, g_threads[t].sp);
          }
      }
      for (unsigned t = beg; t < end; ++t) {
        any |= g_threads[t].state != kDone;
        all_at_barrier &= g_threads[t].state == kDone || g_threads[t].state == kBarrier;
      }
    }
    if (!any) return;
    if (all_at_barrier)
      for (unsigned t = 0; t < threads; ++t) {
        if (g_threads[t].state == kBarrier) g_threads[t].state = kReady;
      }
    else if (!ran)
      fail("threads wait for ever");
  }
}

}  // namespace

const Given& give(const char* what, const void* v, size_t n) {
  Thread& t = g_threads[g_now];
  Wave& w = g_waves[g_now / 64];
  Given& g = w.given[w.turn];
  if (n > sizeof g.v[0]) fail("too many bytes for a lane");
  memcpy(g.v[g_now & 63], v, n);
  t.what = what;
  leave(kWave);
  return g;
}

void barrier() { leave(kBarrier); }

void run(dim3 grid, dim3 block, void (*go)(void*), void* self) {
  g_go = go;
  g_self = self;
  gridDim = grid;
  const unsigned long blocks = (unsigned long)grid.x * grid.y * grid.z;
  const int jobs = (int)std::min(8ul, blocks);
  fflush(stdout);
  std::vector<pid_t> pids;
  for (int j = 0; j < jobs; ++j) {
    const pid_t pid = jobs > 1 ? fork() : 0;
    if (pid) {
      pids.push_back(pid);
      continue;
    }
    for (unsigned long b = j; b < blocks; b += jobs) {
      blockIdx = dim3(b % grid.x, b / grid.x % grid.y, b / grid.x / grid.y);
      workgroup(block.x);
    }
    if (jobs > 1) _exit(0);
  }
  for (pid_t p : pids) {
    int status = 0;
    waitpid(p, &status, 0);
    if (status) _exit(WIFEXITED(status) ? WEXITSTATUS(status) : 4);
  }
}

// ---- memory ------------------------------------------------------------------------

namespace {

constexpr size_t kPage = 4096, kGuard = 1 << 20;
bool g_at_end = true;
struct Array {
  char* map;
  size_t mapped, bytes;
};
std::map<char*, Array> g_arrays;

// bytes between pages that nothing may touch, up to the last one or from the first one on; shared with the
// processes that run workgroups.
void* array(size_t bytes) {
  const size_t whole = (bytes + kPage - 1) / kPage * kPage;
  char* m = (char*)mmap(nullptr, whole + 2 * kGuard, PROT_NONE, MAP_SHARED | MAP_ANONYMOUS, -1, 0);
  if (m == MAP_FAILED || (whole && mprotect(m + kGuard, whole, PROT_READ | PROT_WRITE))) {
    printf("no memory\n");
    _exit(1);
  }
  memset(m + kGuard, 0xA5, whole);
  char* p = m + kGuard + (g_at_end ? whole - bytes : 0);
  g_arrays[p] = {m, whole + 2 * kGuard, bytes};
  return p;
}

void release(void* p) {
  auto it = g_arrays.find((char*)p);
  munmap(it->second.map, it->second.mapped);
  g_arrays.erase(it);
}

// What lies beside an array in its pages is as it was.
void check_margins() {
  for (auto& [p, a] : g_arrays) {
    for (char* q = a.map + kGuard; q < p; ++q)
      if ((unsigned char)*q != 0xA5) fail("written before an array of %zu bytes", a.bytes);
    for (char* q = p + a.bytes; q < a.map + a.mapped - kGuard; ++q)
      if ((unsigned char)*q != 0xA5) fail("written behind an array of %zu bytes", a.bytes);
  }
}

void on_fault(int, siginfo_t* info, void*) {
  const char* at = (const char*)info->si_addr;
  for (auto& [p, a] : g_arrays)
    if (at >= a.map && at < a.map + a.mapped) {
      printf("%ld bytes from the beginning of an array of %zu (workgroup %u, thread %u)\n",
             (long)(at - p), a.bytes, blockIdx.x, threadIdx.x);
      fflush(stdout);
      _exit(3);
    }
  printf("outside of all arrays (workgroup %u, thread %u)\n", blockIdx.x, threadIdx.x);
  fflush(stdout);
  _exit(3);
}

}  // namespace
}  // namespace model

// ---- the library around the kernels --------------------------------------------------

namespace gcn {

void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vfprintf(stderr, fmt, ap);
  va_end(ap);
  fputc('\n', stderr);
}
void clear_error() {}
gcn_status hip_fail(hipError_t, const char*, const char*, int) { return GCN_EHIP; }
CallScope::CallScope(void* s) : stream((hipStream_t)s), outer(nullptr) {}
CallScope::~CallScope() {}
ProfScope::ProfScope(const char* n, hipStream_t s) : name(n), stream(s) {}
ProfScope::~ProfScope() {}
bool stream_capturing(hipStream_t) { return false; }
gcn_status tmalloc(void** p, size_t bytes, hipStream_t, const char*, const void*) {
  *p = model::array((bytes + 255) / 256 * 256);
  return GCN_OK;
}
void tfree(void* p, hipStream_t) { model::release(p); }
// (of the ungrouped products)
gcn_status sum_partials(int64_t, int64_t, int64_t, const float*, float*, int64_t, hipStream_t) {
  return GCN_EINVAL;
}

}  // namespace gcn

using namespace gcn;

namespace {

#define CHECK(cond, ...)            \
  do {                              \
    if (!(cond)) {                  \
      printf(__VA_ARGS__);          \
      printf("\n");                 \
      fflush(stdout);               \
      exit(1);                      \
    }                               \
  } while (0)

std::mt19937_64 g_rng;

float bf16_up(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
uint16_t bf16_down(float v) {  // to nearest even
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  return (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
}

// A matrix of a type in an array that ends with its last row.
struct Matrix {
  int dtype;
  int64_t n, f, ld;
  char* p;
  Matrix(int t, int64_t n_, int64_t f_, int64_t ld_) : dtype(t), n(n_), f(f_), ld(ld_) {
    p = (char*)model::array(n ? ((n - 1) * ld + f) * size() : 0);
  }
  size_t size() const { return dtype == GCN_DT_F32 ? 4 : 2; }
  double get(int64_t i, int64_t j) const {
    const int64_t at = i * ld + j;
    return dtype == GCN_DT_F32 ? ((float*)p)[at] : bf16_up(((uint16_t*)p)[at]);
  }
  void set(int64_t i, int64_t j, float v) {
    const int64_t at = i * ld + j;
    if (dtype == GCN_DT_F32)
      ((float*)p)[at] = v;
    else
      ((uint16_t*)p)[at] = bf16_down(v);
  }
  // every element, what lies between the rows NaN
  template <class F>
  Matrix& fill(F value) {
    for (int64_t i = 0; i < n; ++i)
      for (int64_t j = 0; j < (i + 1 < n ? ld : f); ++j)
        set(i, j, j < f ? value(i, j) : NAN);
    return *this;
  }
};

int64_t arg(char** v, int i) { return atoll(v[i]); }

// grouped op dtype dtype_c K N pad memory before after sizes...: whole numbers, compared exactly (of large
// products in some rows and columns). memory: 0 the library's, 1 given, 2 given, too little for copies.
void grouped(int c, char** v) {
  const int op = (int)arg(v, 0), dt = (int)arg(v, 1), dc = (int)arg(v, 2);
  const int64_t K = arg(v, 3), N = arg(v, 4), pad = arg(v, 5), memory = arg(v, 6);
  const int64_t before = arg(v, 7), after = arg(v, 8);
  const int G = c - 9;
  int64_t* ends = (int64_t*)model::array((G + 1) * 8);
  ends[0] = before;
  for (int g = 0; g < G; ++g) ends[g + 1] = ends[g] + arg(v, 9 + g);
  const int64_t rows = ends[G] + after;
  if (!model::g_at_end && rows * K * N > 12000000000) return;  // (seconds; the smaller ones do)
  auto number = [&](int64_t, int64_t) { return (float)(int)(g_rng() % 7) - 3.f; };
  auto of_group = [&](int64_t i) { return i >= before && i < ends[G]; };
  const bool tn = op == GCN_GEMM_TN;
  Matrix A(dt, rows, K, K + pad);
  A.fill([&](int64_t i, int64_t j) { return of_group(i) ? number(i, j) : NAN; });
  const int64_t br = op == GCN_GEMM_NT ? N : K, bc = op == GCN_GEMM_NT ? K : N;
  Matrix B(dt, tn ? rows : G * br, tn ? N : bc, (tn ? N : bc) + pad);
  B.fill([&](int64_t i, int64_t j) { return !tn || of_group(i) ? number(i, j) : NAN; });
  Matrix C(dc, tn ? G * K : rows, N, N + pad);
  C.fill([](int64_t, int64_t) { return 7.f; });
  const int64_t stride = tn ? K * C.ld : br * B.ld;
  void* work = nullptr;
  int64_t need = 0;
  auto call = [&](void* w, int64_t* bytes) {
    return gcn_gemm_grouped(op, G, ends, rows, N, K, A.p, A.ld, B.p, B.ld, dt, C.p, C.ld, dc, stride, w,
                            bytes, nullptr);
  };
  if (memory) {
    CHECK(call(nullptr, &need) == GCN_OK, "query");
    if (memory == 2) need = std::max<int64_t>(256, need / 8);
    work = model::array(need + 256);
    work = (void*)(((uintptr_t)work + 255) / 256 * 256);
  }
  const gcn_status st = call(work, memory ? &need : nullptr);
  if (memory == 2 && st == GCN_EINVAL) return;  // too little for the partial sums as well
  CHECK(st == GCN_OK, "call: %d", (int)st);
  model::check_margins();
  const int64_t sr = rows * K * N > 40000000 ? 61 : 1, sc = sr > 1 ? 37 : 1;
  for (int g = 0; g < G; ++g) {
    const int64_t r0 = tn ? 0 : ends[g], r1 = tn ? K : ends[g + 1];
    for (int64_t i = r0; i < r1; i += i + sr < r1 || i == r1 - 1 ? sr : r1 - 1 - i)
      for (int64_t j = 0; j < N; j += j + sc < N || j == N - 1 ? sc : N - 1 - j) {
        double s = 0;
        if (tn)
          for (int64_t k = ends[g]; k < ends[g + 1]; ++k) s += A.get(k, i) * B.get(k, j);
        else
          for (int64_t k = 0; k < K; ++k)
            s += A.get(i, k) * (op == GCN_GEMM_NN ? B.get(g * K + k, j) : B.get(g * N + j, k));
        const double want = dc == GCN_DT_F32 ? s : bf16_up(bf16_down((float)s));
        const double got = C.get(tn ? g * K + i : i, j);
        CHECK(got == want, "group %d, (%ld, %ld): %g instead of %g", g, (long)i, (long)j, got, want);
      }
  }
  for (int64_t i = 0; i < C.n; ++i) {
    if (!tn && !of_group(i))
      for (int64_t j = 0; j < N; ++j) CHECK(C.get(i, j) == 7.0, "row %ld of no group", (long)i);
    for (int64_t j = N; i + 1 < C.n && j < C.ld; ++j)
      CHECK(std::isnan(C.get(i, j)), "between the rows %ld and the next", (long)i);
  }
}

// unordered seed: offsets in any order, beyond the rows and negative: no address leaves the arrays.
void unordered(int, char** v) {
  g_rng.seed(arg(v, 0));
  auto upto = [](int64_t n) { return (int64_t)(g_rng() % (uint64_t)(n + 1)); };
  const int op = (int)upto(2), dt = (int)upto(1), G = 1 + (int)upto(upto(3) ? 8 : 1100);
  const int64_t rows = 1 + upto(upto(1) ? 9000 : 400), K = 1 + upto(140), N = 1 + upto(140);
  int64_t* ends = (int64_t*)model::array((G + 1) * 8);
  for (int g = 0; g <= G; ++g) ends[g] = upto(9) ? upto(rows) : (upto(1) ? -1 : 1) * (int64_t)(g_rng() >> upto(40) >> 1);
  const bool tn = op == GCN_GEMM_TN;
  Matrix A(dt, rows, K, K), B(dt, tn ? rows : G * (op == GCN_GEMM_NT ? N : K), op == GCN_GEMM_NT ? K : N,
                             op == GCN_GEMM_NT ? K : N);
  Matrix C(GCN_DT_F32, tn ? G * K : rows, N, N);
  for (Matrix* m : {&A, &B, &C}) m->fill([](int64_t, int64_t) { return 1.f; });
  CHECK(gcn_gemm_grouped(op, G, ends, rows, N, K, A.p, A.ld, B.p, B.ld, dt, C.p, C.ld, GCN_DT_F32,
                         tn ? K * N : B.n / G * B.ld, nullptr, nullptr, nullptr) == GCN_OK,
        "call");
  model::check_margins();
}

// norm n F dtype pad eps p: forward and backward, within roundings of what the formulas give in 64 bits.
void norm(int, char** v) {
  const int64_t n = arg(v, 0), F = arg(v, 1), pad = arg(v, 3);
  const int dt = (int)arg(v, 2);
  const double eps = atof(v[4]), p = atof(v[5]);
  std::normal_distribution<float> normal;
  auto number = [&](int64_t, int64_t) { return normal(g_rng); };
  Matrix X(dt, n, F, F + pad), dY(dt, n, F, F + pad), Y(dt, n, F, F + pad), dX(dt, n, F, F + pad);
  Matrix gamma(GCN_DT_F32, 1, F, F), beta(GCN_DT_F32, 1, F, F), dg(GCN_DT_F32, 1, F, F), db(GCN_DT_F32, 1, F, F);
  for (Matrix* m : {&X, &dY, &gamma, &beta}) m->fill(number);
  for (Matrix* m : {&Y, &dX, &dg, &db}) m->fill([](int64_t, int64_t) { return 7.f; });
  const gcn_dropout_spec drop{p, 5, 1, nullptr, 0};
  const gcn_dropout_spec* d = p > 0 ? &drop : nullptr;
  Matrix keep(GCN_DT_F32, n, F, F);  // what dropout multiplies by, as dropout of ones
  keep.fill([](int64_t, int64_t) { return 1.f; });
  if (d) CHECK(gcn_dropout(n, F, keep.p, F, GCN_DT_F32, d, keep.p, F, nullptr) == GCN_OK, "dropout");
  CHECK(gcn_layernorm_affine_fwd(n, F, X.p, X.ld, dt, (float*)gamma.p, (float*)beta.p, eps, d, Y.p, Y.ld,
                                 nullptr) == GCN_OK, "forward");
  CHECK(gcn_layernorm_affine_bwd(n, F, X.p, X.ld, dt, (float*)gamma.p, eps, d, dY.p, dY.ld, dX.p, dX.ld,
                                 (float*)dg.p, (float*)db.p, nullptr, nullptr, nullptr) == GCN_OK,
        "backward");
  model::check_margins();
  const double half = dt == GCN_DT_F32 ? 0x1p-24 : 0x1p-8;
  std::vector<double> sg(F), sb(F), mg(F), mb(F);
  for (int64_t i = 0; i < n; ++i) {
    double m = 0, q = 0, t1 = 0, t2 = 0, a1 = 0, a2 = 0;
    for (int64_t f = 0; f < F; ++f) m += X.get(i, f) / F;
    for (int64_t f = 0; f < F; ++f) q += (X.get(i, f) - m) * (X.get(i, f) - m) / F;
    const double rstd = 1 / std::sqrt(q + eps);
    auto h = [&](int64_t f) { return (X.get(i, f) - m) * rstd; };
    auto g = [&](int64_t f) { return dY.get(i, f) * keep.get(i, f); };
    for (int64_t f = 0; f < F; ++f) {
      const double t = g(f) * gamma.get(0, f) / F;
      t1 += t, t2 += t * h(f), a1 += std::fabs(t), a2 += std::fabs(t * h(f));
      sg[f] += g(f) * h(f), sb[f] += g(f);
      mg[f] += std::fabs(g(f) * h(f)), mb[f] += std::fabs(g(f));
      const double a = h(f) * gamma.get(0, f), y = (a + beta.get(0, f)) * keep.get(i, f);
      const double b = (std::fabs(a) + std::fabs(beta.get(0, f))) * keep.get(i, f);
      CHECK(std::fabs(Y.get(i, f) - y) <= 16 * 0x1p-24 * b + half * std::fabs(y), "Y (%ld, %ld)", (long)i,
            (long)f);
    }
    for (int64_t f = 0; f < F; ++f) {
      const double t = g(f) * gamma.get(0, f), x = rstd * (t - t1 - h(f) * t2);
      const double b = rstd * (std::fabs(t) + a1 + std::fabs(h(f)) * a2);
      CHECK(std::fabs(dX.get(i, f) - x) <= 200 * 0x1p-24 * b + half * std::fabs(x), "dX (%ld, %ld)",
            (long)i, (long)f);
    }
  }
  for (int64_t f = 0; f < F; ++f) {
    CHECK(std::fabs(dg.get(0, f) - sg[f]) <= (n + 16) * 0x1p-24 * mg[f], "dgamma %ld", (long)f);
    CHECK(std::fabs(db.get(0, f) - sb[f]) <= (n + 16) * 0x1p-24 * mb[f], "dbeta %ld", (long)f);
  }
}

// dropout n F dtype pad
void dropout(int, char** v) {
  const int64_t n = arg(v, 0), F = arg(v, 1), pad = arg(v, 3);
  const int dt = (int)arg(v, 2);
  Matrix X(dt, n, F, F + pad), Y(dt, n, F, F + pad);
  X.fill([&](int64_t, int64_t) { return 1.f + (float)(g_rng() % 100); });
  Y.fill([](int64_t, int64_t) { return 7.f; });
  const gcn_dropout_spec drop{0.5, 5, 1, nullptr, 0};
  CHECK(gcn_dropout(n, F, X.p, X.ld, dt, &drop, Y.p, Y.ld, nullptr) == GCN_OK, "call");
  model::check_margins();
  for (int64_t i = 0; i < n; ++i)
    for (int64_t f = 0; f < F; ++f)
      CHECK(Y.get(i, f) == 0 || Y.get(i, f) == 2 * X.get(i, f), "(%ld, %ld)", (long)i, (long)f);
}

// One wavefront.
template <class F>
void wavefront(F f) {
  model::launch(dim3(1), dim3(64), f);
}

// tiles seed: the rows that the tiles of random groups have, counted and by slots: each row of a group
// once.
void tiles(int, char** v) {
  g_rng.seed(arg(v, 0));
  const int n = 1 + (int)(g_rng() % (g_rng() % 3 ? 70 : 1024));
  const int R = 16 << g_rng() % 5;
  const int64_t rows = g_rng() % 4000;
  int64_t* ends = (int64_t*)model::array((n + 1) * 8);
  for (int i = 0; i <= n; ++i) ends[i] = rows ? g_rng() % (rows + 1) : 0;
  std::sort(ends, ends + n + 1);
  const Groups by{n, ends, rows};
  const int64_t slots = group_slots(by, R);
  for (int least = 0; least < 2; ++least) {
    std::vector<int> seen(rows), group(n);
    auto have = [&](const GroupTile& t) {
      if (threadIdx.x) return;
      CHECK(t.g >= 0 && t.g < n && t.first == ends[t.g] && t.end == ends[t.g + 1], "the tile's group");
      if (t.beg < t.end || t.beg == t.first) group[t.g] = 1;
      for (int64_t i = t.beg; i < std::min(t.beg + R, t.end); ++i) ++seen[i];
    };
    auto check = [&](const char* how) {
      for (int64_t i = 0; i < rows; ++i)
        CHECK(seen[i] == (i >= ends[0] && i < ends[n]), "%s: row %ld %d times", how, (long)i, seen[i]);
      for (int g = 0; g < n; ++g)
        CHECK(group[g] || (!least && ends[g] == ends[g + 1]), "%s: group %d has no tile", how, g);
      std::fill(seen.begin(), seen.end(), 0);
      std::fill(group.begin(), group.end(), 0);
    };
    wavefront([&] {
      const TileCount c = count_tiles(by, R, least);
      CHECK(c.total <= slots, "%d tiles, %ld slots", c.total, (long)slots);
      for (int t = 0; t < c.total; ++t) have(counted_tile(by, c, t, R, least));
    });
    check("counted");
    wavefront([&] {
      for (int64_t s = 0; s < slots; ++s) {
        const GroupTile t = group_tile(by, s, R);
        if (t.beg < t.end || (least && t.beg == t.first)) have(t);
      }
    });
    check("slots");
  }
}

// bad_offsets n rows R: groups that begin at 0 and end with the last row in turn, so that they
// overlap: whatever tiles are counted, their rows are rows.
void bad_offsets(int, char** v) {
  const int n = (int)arg(v, 0), R = (int)arg(v, 2);
  const int64_t rows = arg(v, 1);
  int64_t* ends = (int64_t*)model::array((n + 1) * 8);
  for (int i = 0; i <= n; ++i) ends[i] = i % 2 ? rows : 0;
  const Groups by{n, ends, rows};
  wavefront([&] {
    const TileCount c = count_tiles(by, R, 0);
    CHECK(c.total >= 0, "%d tiles", c.total);
    std::mt19937_64 rng(7);
    for (int k = 0; k < 2000 && c.total; ++k) {
      const int t = k ? (int)(rng() % c.total) : c.total - 1;
      const GroupTile g = counted_tile(by, c, t, R, 0);
      CHECK(g.beg >= 0 && g.beg < g.end && g.end <= rows, "tile %d: rows %ld to %ld", t, (long)g.beg,
            (long)g.end);
    }
  });
}

}  // namespace

int main(int c, char** v) {
  struct sigaction sa = {};
  static char stack[1 << 16];
  stack_t ss = {};
  ss.ss_sp = stack;
  ss.ss_size = sizeof stack;
  sigaltstack(&ss, nullptr);
  sa.sa_sigaction = model::on_fault;
  sa.sa_flags = SA_SIGINFO | SA_ONSTACK;
  sigaction(SIGSEGV, &sa, nullptr);
  sigaction(SIGBUS, &sa, nullptr);
  const std::string what = c > 1 ? v[1] : "";
  for (int at_end = 1; at_end >= 0; --at_end) {
    model::g_at_end = at_end;
    g_rng.seed(1);
    if (what == "grouped") grouped(c - 2, v + 2);
    else if (what == "unordered") unordered(c - 2, v + 2);
    else if (what == "norm") norm(c - 2, v + 2);
    else if (what == "dropout") dropout(c - 2, v + 2);
    else if (what == "tiles") tiles(c - 2, v + 2);
    else if (what == "bad_offsets") bad_offsets(c - 2, v + 2);
    else return 2;
    for (; !model::g_arrays.empty();) model::release(model::g_arrays.begin()->first);
  }
  printf("ok\n");
  return 0;
}
