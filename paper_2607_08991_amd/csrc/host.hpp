// What the host sides of the library's translation units share.
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>

#include <mutex>

#include "../../include/sats.h"

namespace sats_host {

// Records the text of the calling thread's last error and returns `code`.
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

// Calls on one stream may come from several threads, and a call is several launches that
// hand each other results in the stream's workspace: a call holds the stream's turn from
// before it looks at the workspace until its last launch is enqueued.
typedef std::unique_lock<std::mutex> Turn;

// Workgroups of 256 threads in a row of a launch, at most: HIP takes less than 2^32 threads there.
constexpr int64_t kMaxGrid = ((int64_t)1 << 24) - 1;

// The error of the launch that was just made, if it had one.
inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SATS_OK : fail(SATS_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Takes the turn of (current device, stream), and the serving operators' scratch memory
// of it: at least `bytes`, grown where it is smaller (SATS_ERR_WORKSPACE under stream capture
// or for want of memory; what is there then stays).
int serve_workspace(hipStream_t stream, size_t bytes, char **mem, Turn *turn);

}  // namespace sats_host
