// Sanitizer driver for the workspace that the library keeps for the kernels of
// a call (test infrastructure): gdn_workspace.hip is linked against a fake
// runtime whose device memory is host memory, so a buffer that was handed out
// and then released is a use after free here.  Built with
// -fsanitize=address,undefined by tests/test_workspace_cpu.py.
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <thread>
#include <vector>

#include "gdn_internal.h"

static int fails = 0;
#define CHECK(x)                                     \
  do {                                               \
    if (!(x)) {                                      \
      printf("FAIL line %d: %s\n", __LINE__, #x);    \
      ++fails;                                       \
    }                                                \
  } while (0)

// ---------------------------------------------------------------------------
// The fake runtime
// ---------------------------------------------------------------------------
static int g_device = 0;
static bool g_capturing = false;
static hipError_t g_last = hipSuccess;
static size_t g_held = 0;          // bytes allocated
static size_t g_limit = SIZE_MAX;  // bytes that there are

extern "C" {
hipError_t hipGetDevice(int* dev) { return *dev = g_device, hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  return *s = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone, hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) {
  if (n > g_limit - g_held) return g_last = hipErrorOutOfMemory;
  g_held += n;
  *p = malloc(n);
  return hipSuccess;
}
hipError_t hipFree(void* p) { return free(p), hipSuccess; }
hipError_t hipGetLastError(void) {
  const hipError_t e = g_last;
  return g_last = hipSuccess, e;
}
}

namespace gdn {
static char g_msg[512];
int set_error(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_msg, sizeof(g_msg), fmt, ap);
  va_end(ap);
  return code;
}
}  // namespace gdn

using gdn::stream_workspace;

static hipStream_t stream(size_t n) { return reinterpret_cast<hipStream_t>(0x1000 * n); }

static void* get(size_t bytes, hipStream_t s) {
  int rc = -99;
  void* p = stream_workspace(bytes, s, &rc);
  CHECK(p && rc == GDN_OK);
  return p;
}

// A captured graph goes on using the buffer that its calls were given, whatever is needed later.
static void buffers_stay() {
  const size_t small = 1 << 10;
  char* first = static_cast<char*>(get(small, stream(1)));
  std::vector<std::pair<char*, size_t>> held = {{first, small}};
  size_t need = small;
  for (int i = 0; i < 40; ++i) {  // a graph for every batch size, in rising order
    need += 777;
    char* p = static_cast<char*>(get(need, stream(1)));
    held.push_back({p, need});
  }
  for (auto& h : held) memset(h.first, 1, h.second);  // replays of all of them
  CHECK(get(small, stream(1)) == get(need, stream(1)));  // a call that fits the last buffer uses it
  CHECK(g_held <= 4 * need);  // what is left behind is bounded
}

static void streams_and_devices_apart() {
  void* a = get(100, stream(2));
  CHECK(a != get(100, stream(3)));
  CHECK(a == get(100, stream(2)));
  g_device = 1;
  CHECK(a != get(100, stream(2)));
  g_device = 0;
  CHECK(a == get(50, stream(2)));
}

static void capture() {
  int rc = 0;
  void* a = get(4096, stream(4));
  g_capturing = true;
  CHECK(stream_workspace(4096, stream(4), &rc) == a && rc == GDN_OK);
  const size_t held = g_held;
  CHECK(!stream_workspace(1 << 20, stream(4), &rc) && rc == GDN_EUNSUPPORTED && strlen(gdn::g_msg));
  CHECK(!stream_workspace(16, stream(5), &rc) && rc == GDN_EUNSUPPORTED);
  CHECK(g_held == held);
  CHECK(stream_workspace(100, stream(4), &rc) == a && rc == GDN_OK);  // the refusal changed nothing
  g_capturing = false;
}

static void out_of_memory() {
  int rc = 0;
  void* a = get(1 << 16, stream(6));
  g_limit = g_held + (3 << 15);
  // no room for more than is asked for: as much as that
  void* b = get(3 << 15, stream(6));
  CHECK(g_last == hipSuccess);  // the next launch's check would report what is left
  CHECK(!stream_workspace(1 << 20, stream(6), &rc) && rc == GDN_EHIP);
  CHECK(g_last == hipSuccess);
  CHECK(get(3 << 15, stream(6)) == b);  // what is there stays in use
  memset(a, 1, 1 << 16);
  memset(b, 1, 3 << 15);
  g_limit = SIZE_MAX;
}

// hipStreamPerThread names another stream in every host thread.
static void streams_per_thread() {
  void *a = get(100, hipStreamPerThread), *b = nullptr, *c = nullptr;
  std::thread([&] { b = get(100, hipStreamPerThread); }).join();
  std::thread([&] { c = get(100, hipStreamPerThread); }).join();  // kernels of the ended thread's may still run
  CHECK(a != b && a != c && b != c);
  CHECK(a == get(100, hipStreamPerThread));
}

int main() {
  buffers_stay();
  streams_and_devices_apart();
  capture();
  out_of_memory();
  streams_per_thread();
  printf("workspace driver: %d failed checks\n", fails);
  return fails != 0;
}
