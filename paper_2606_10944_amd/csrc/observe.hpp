// The launch observer of the C ABI's entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/thin.h"

namespace thin {

// The launch observer is a diagnostic of the calling thread (thread-local):
// calls from other threads never see it.
extern thread_local thin_launch_hook_t g_hook;
extern thread_local void* g_hook_ctx;

// Enqueue one launch between the observer's two calls.
template <typename F>
hipError_t observed(int32_t kernel, int32_t round, hipStream_t st, F&& launch) {
  if (g_hook) g_hook(g_hook_ctx, kernel, round, 0, st);
  const hipError_t e = launch();
  if (g_hook) g_hook(g_hook_ctx, kernel, round, 1, st);
  return e;
}

}  // namespace thin
