// gdn_workspace.hip -- device memory that the library keeps for the kernels of
// a call: one buffer per (device, stream), grown on demand and kept until the
// process ends.
#include <map>
#include <mutex>
#include <utility>

#include "gdn_internal.h"

namespace gdn {

void* stream_workspace(size_t bytes, hipStream_t stream, int* rc) {
  static std::mutex mu;
  static std::map<std::pair<int, hipStream_t>, std::pair<void*, size_t>> bufs;
  *rc = GDN_OK;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    *rc = set_error(GDN_EHIP, "workspace: hipGetDevice failed");
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(mu);
  auto& e = bufs[{dev, stream}];
  if (e.second >= bytes) return e.first;
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(stream, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone) {
    *rc = set_error(GDN_EUNSUPPORTED,
                    "workspace: %zu bytes needed while the stream is captured; run the same sizes once "
                    "uncaptured first",
                    bytes);
    return nullptr;
  }
  if (e.first) {  // only this stream used it
    if (hipStreamSynchronize(stream) != hipSuccess || hipFree(e.first) != hipSuccess) {
      *rc = set_error(GDN_EHIP, "workspace: release of %zu bytes failed", e.second);
      return nullptr;
    }
    e.first = nullptr;
    e.second = 0;
  }
  if (hipMalloc(&e.first, bytes) != hipSuccess) {
    e.first = nullptr;
    *rc = set_error(GDN_EHIP, "workspace: hipMalloc of %zu bytes failed", bytes);
    return nullptr;
  }
  e.second = bytes;
  return e.first;
}

}  // namespace gdn
