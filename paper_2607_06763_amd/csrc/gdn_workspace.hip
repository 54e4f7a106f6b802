// gdn_workspace.hip -- device memory that the library keeps for the kernels of
// a call: one buffer per (device, stream), replaced by a larger one on demand;
// none is released before the process ends.
#include <map>
#include <mutex>
#include <utility>

#include "gdn_internal.h"
#include "gdn_workspace.h"

namespace gdn {

void* stream_workspace(size_t bytes, hipStream_t stream, int* rc) {
  static std::mutex mu;
  static std::map<std::pair<int, StreamKey>, std::pair<void*, size_t>> bufs;
  *rc = GDN_OK;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    *rc = set_error(GDN_EHIP, "workspace: hipGetDevice failed");
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(mu);
  auto& e = bufs[{dev, stream_key(stream)}];
  if (e.second >= bytes) return e.first;
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(stream, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone) {
    (void)hipGetLastError();
    *rc = set_error(GDN_EUNSUPPORTED,
                    "workspace: %zu bytes needed while the stream is captured; run the same sizes once "
                    "uncaptured first",
                    bytes);
    return nullptr;
  }
  // A captured graph keeps the address that its calls were given, so a buffer
  // stays when a larger one takes its place.  Each is twice the one before, if
  // there is room: all of them together stay below four times the largest need.
  void* p = nullptr;
  size_t size = bytes > 2 * e.second ? bytes : 2 * e.second;
  hipError_t err = hipMalloc(&p, size);
  if (err != hipSuccess) (void)hipGetLastError();  // or the next launch's check reports it
  if (err != hipSuccess && size > bytes) err = hipMalloc(&p, size = bytes);
  if (err != hipSuccess) {
    (void)hipGetLastError();
    *rc = set_error(GDN_EHIP, "workspace: hipMalloc of %zu bytes failed", bytes);
    return nullptr;
  }
  e = {p, size};
  return p;
}

}  // namespace gdn
