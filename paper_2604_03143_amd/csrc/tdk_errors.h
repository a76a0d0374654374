// How entry points report errors: a status, and a thread-local reason.
#pragma once

#include <hip/hip_runtime.h>

#include <new>
#include <string>

#include "tdk.h"

namespace tdk {

inline thread_local std::string g_last_error;

inline tdk_status fail(tdk_status st, const std::string& msg) {
  g_last_error = msg;
  return st;
}

inline tdk_status hip_fail(hipError_t e, const char* what) {
  return fail(TDK_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// No exception leaves the library: host allocations that fail become TDK_ERR_NOMEM.
template <typename F>
tdk_status guarded(F&& body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    try { g_last_error = "out of memory"; } catch (...) {}   // short enough to need no allocation
    return TDK_ERR_NOMEM;
  } catch (...) {
    try { g_last_error = "internal error"; } catch (...) {}
    return TDK_ERR_INVALID_ARG;
  }
}

}  // namespace tdk
