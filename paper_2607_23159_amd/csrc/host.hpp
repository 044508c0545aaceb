// Status and error handling shared by the files that implement entry points of
// include/cs.h.
#pragma once

#include <hip/hip_runtime.h>

#include <new>

#include "../../include/cs.h"

namespace cs {

// Stores the message that cs_last_error() returns (thread-local); returns code.
cs_status fail(cs_status code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace cs

#define HIPC(call)                                                                   \
  do {                                                                               \
    hipError_t e_ = (call);                                                          \
    if (e_ != hipSuccess) {                                                          \
      if (e_ == hipErrorOutOfMemory)                                                 \
        return fail(CS_E_NOMEM, "%s: %s", #call, hipGetErrorString(e_));            \
      return fail(CS_E_DEVICE, "%s: %s (%d)", #call, hipGetErrorString(e_), (int)e_); \
    }                                                                                \
  } while (0)

#define CHECK(cond, code, ...)                 \
  do {                                         \
    if (!(cond)) return fail(code, __VA_ARGS__); \
  } while (0)

#define GUARD(...)                                                         \
  try {                                                                    \
    __VA_ARGS__                                                            \
  } catch (const std::bad_alloc&) {                                        \
    return fail(CS_E_NOMEM, "host allocation failed");                     \
  } catch (...) {                                                          \
    return fail(CS_E_DEVICE, "unexpected exception in the runtime");       \
  }

#define TRY(x)                    \
  do {                            \
    cs_status s_ = (x);           \
    if (s_ != CS_OK) return s_;   \
  } while (0)
