// Host threads that make calls at the same time (test infrastructure): the
// host side of the whole library against a fake runtime that records its
// launches.  The kernels of a call that pass results on through the stream's
// workspace must be enqueued without another call's between them.
#include <hip/hip_runtime.h>
#include <stdio.h>
#include <stdlib.h>

#include <chrono>
#include <condition_variable>
#include <functional>
#include <mutex>
#include <thread>
#include <vector>

#include "gdn_tree.h"

static int fails = 0;
#define CHECK(x)                                  \
  do {                                            \
    if (!(x)) {                                   \
      printf("FAIL line %d: %s\n", __LINE__, #x); \
      ++fails;                                    \
    }                                             \
  } while (0)

// ---------------------------------------------------------------------------
// The fake runtime
// ---------------------------------------------------------------------------
static std::mutex g_mu;
static std::condition_variable g_cv;
static std::vector<int> g_launches;  // the launching threads, in order
static bool g_met;                   // a thread saw the other one's launch while it was in its own
static thread_local int t_me = -1;
static thread_local struct {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} t_config;

extern "C" {
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t s) { return t_config = {g, b, lds, s}, hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, hipStream_t* s) {
  *g = t_config.grid, *b = t_config.block, *lds = t_config.lds, *s = t_config.stream;
  return hipSuccess;
}
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, dim3*, dim3*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void**) {}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetDevice(int* dev) { return *dev = 0, hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "fake"; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, const void* s) { return *p = const_cast<void*>(s), hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) { return *p = malloc(n), hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { return *s = hipStreamCaptureStatusNone, hipSuccess; }

hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
  std::unique_lock<std::mutex> lock(g_mu);
  bool first = true;
  for (int t : g_launches) first = first && t != t_me;
  g_launches.push_back(t_me);
  g_cv.notify_all();
  // thread 0 stays in its first launch until thread 1 has launched, or a while
  if (t_me == 0 && first)
    g_met = g_cv.wait_for(lock, std::chrono::milliseconds(500), [] { return g_launches.back() == 1; });
  return hipSuccess;
}
}

// Threads 0 and 1 make a call each, thread 1 once thread 0 is in its first launch.
static void both(const std::function<int()>& a, const std::function<int()>& b) {
  g_launches.clear();
  g_met = false;
  int rc[2] = {-99, -99};
  std::thread one([&] {
    t_me = 0;
    rc[0] = a();
  });
  std::thread two([&] {
    t_me = 1;
    {
      std::unique_lock<std::mutex> lock(g_mu);
      g_cv.wait(lock, [] { return !g_launches.empty(); });
    }
    rc[1] = b();
  });
  one.join();
  two.join();
  CHECK(rc[0] == GDN_OK && rc[1] == GDN_OK);
}

static bool apart() {  // all of one thread's launches, then all of the other's
  int turns = 0;
  for (size_t i = 1; i < g_launches.size(); ++i) turns += g_launches[i] != g_launches[i - 1];
  return g_launches.size() >= 4 && turns == 1;
}

int main() {
  void* p = reinterpret_cast<void*>(0x100000);  // never dereferenced by the host code
  char* at = static_cast<char*>(p);
  const float* f = static_cast<const float*>(p);
  float *fo = reinterpret_cast<float*>(at), *co = reinterpret_cast<float*>(at + (1 << 28));
  int32_t* i = reinterpret_cast<int32_t*>(at);
  const gdn_attn_dims ad = {2, 8, 8, 2, 64, 64, 16, 8, GDN_BF16, 0, 0, 0.0f};
  const gdn_dims small = {2, 60, 2, 4, 64, 64, GDN_BF16, 0.0f}, large = {2, 300, 2, 4, 64, 64, GDN_BF16, 0.0f};
  std::function<int(hipStream_t)> calls[] = {
      [&](hipStream_t s) { return gdn_tree_attend(&ad, nullptr, nullptr, p, p, p, i, i, at + (1 << 28), s); },
      [&](hipStream_t s) { return gdn_tree_verify(&large, p, p, p, p, p, p, f, f, f, fo, s); },
      [&](hipStream_t s) { return gdn_tree_verify_chunked(&small, p, p, p, p, p, p, f, f, f, fo, s); },
      [&](hipStream_t s) { return gdn_tree_step(&large, p, i, p, p, p, p, p, i, p, p, p, p, p, p, f, f, co, fo, fo, s); },
  };
  const hipStream_t streams[] = {nullptr, reinterpret_cast<hipStream_t>(0x2000), reinterpret_cast<hipStream_t>(0x3000)};
  for (auto& a : calls)
    for (auto& b : calls)
      for (hipStream_t s : {streams[0], streams[1]}) {
        if (&a != &b && &a != &calls[0] && &b != &calls[0]) continue;
        both([&] { return a(s); }, [&] { return b(s); });
        CHECK(apart());
      }
  // calls on two streams do not wait for each other
  both([&] { return calls[0](streams[1]); }, [&] { return calls[0](streams[2]); });
  CHECK(g_met);
  both([&] { return calls[0](hipStreamPerThread); }, [&] { return calls[0](hipStreamPerThread); });  // two streams
  CHECK(g_met);
  printf("threads driver: %d failed checks\n", fails);
  return fails != 0;
}
