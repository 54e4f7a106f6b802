// gdn_workspace.h -- host threads and the workspaces of streams.
#pragma once

#include <atomic>
#include <map>
#include <mutex>
#include <utility>

#include <hip/hip_runtime_api.h>

namespace gdn {

// A stream, for work of the calling thread: hipStreamPerThread names another
// one in every thread.  Threads are numbered here because the system gives an
// ended thread's identity to a new one, while kernels of the old may still run.
typedef std::pair<hipStream_t, unsigned long long> StreamKey;

inline StreamKey stream_key(hipStream_t stream) {
  static std::atomic<unsigned long long> threads{0};
  if (stream != hipStreamPerThread) return {stream, 0};
  static thread_local const unsigned long long number = ++threads;
  return {stream, number};
}

// Held by a call that passes results from kernel to kernel through the
// workspace of its stream, from before it takes the workspace until all of its
// kernels are enqueued: another thread's kernels on the same stream in between
// would overwrite them.  Calls on different streams do not wait for each other.
class StreamOrder {
 public:
  explicit StreamOrder(hipStream_t stream) : lock_(of(stream)) {}

 private:
  static std::mutex& of(hipStream_t stream) {
    static std::mutex mu;
    static std::map<StreamKey, std::mutex> each;  // its nodes stay where they are
    std::lock_guard<std::mutex> lock(mu);
    return each[stream_key(stream)];
  }
  std::lock_guard<std::mutex> lock_;
};

}  // namespace gdn
