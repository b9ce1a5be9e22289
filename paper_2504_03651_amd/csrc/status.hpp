// status.hpp -- the calling thread's error detail behind echo_last_error(), and checks
// that entry points share.
#pragma once

#include <stddef.h>

#include "echo.h"

namespace echo {

// Records a printf-style detail for echo_last_error() and returns `code`.
int fail(int code, const char *fmt, ...);
// Clears the calling thread's detail (every entry point starts with it).
void clear_error();
// Whether echo_profile(1) is on for the calling thread.
bool profile_enabled();

// For callers of echo_attn_mixed that enqueue work ahead of it: the bytes of both its
// workspaces (host: 0 where it needs none) and its refusals of the batch, from one
// plan; and its check of the host workspace.
int attn_bytes(const echo_kv_pool_t *pool, const echo_batch_t *batch, int32_t num_q_heads, size_t *device,
               size_t *host);
int check_attn_host(void *host_workspace, size_t bytes, size_t need);

}  // namespace echo
