// gdn_workspace.h -- host threads and the workspaces of streams.
#pragma once

#include <map>
#include <mutex>

#include <hip/hip_runtime_api.h>

namespace gdn {

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
    static std::map<hipStream_t, std::mutex> each;  // its nodes stay where they are
    std::lock_guard<std::mutex> lock(mu);
    return each[stream];
  }
  std::lock_guard<std::mutex> lock_;
};

}  // namespace gdn
