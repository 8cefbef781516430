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

// Takes the turn of (current device, stream), and the serving operators' scratch memory
// of it: at least `bytes`, grown where it is smaller (SATS_ERR_WORKSPACE under stream capture
// or for want of memory; what is there then stays).
int serve_workspace(hipStream_t stream, size_t bytes, char **mem, Turn *turn);

}  // namespace sats_host
