// What the sources of the C ABI (api.cpp, api_scaled.cpp) share: error text,
// pointer checks, workspace regions and the launch of one kernel.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mhlmoe.h"

namespace mhl {
namespace api {

// Sets the calling thread's message and returns st.
mhlmoe_status fail(mhlmoe_status st, const char* fmt, ...);
void clear_error();

#define MHL_TRY(expr)                       \
  do {                                      \
    const mhlmoe_status st_ = (expr);       \
    if (st_ != MHLMOE_OK) return st_;       \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline mhlmoe_status maybe(const void* p, const char* name) {
  if (p != nullptr && !aligned16(p)) return fail(MHLMOE_EINVAL, "%s is not 16-byte aligned", name);
  return MHLMOE_OK;
}

inline mhlmoe_status need(const void* p, const char* name) {
  if (p == nullptr) return fail(MHLMOE_EINVAL, "%s is NULL", name);
  return maybe(p, name);
}

// Tensors with a T-sized dimension may be NULL when T == 0.
inline mhlmoe_status need_rows(const void* p, const char* name, int64_t T) {
  return T == 0 ? maybe(p, name) : need(p, name);
}

// Workspace: a list of 256-byte aligned regions.
inline size_t bump(size_t& cur, size_t bytes) {
  const size_t at = cur;
  cur += (bytes + 255) & ~size_t(255);
  return at;
}

template <typename T>
T* at(void* ws, size_t off) {
  return reinterpret_cast<T*>(reinterpret_cast<uint8_t*>(ws) + off);
}

// The optional timing's two events around a launch (NULL when off).
struct TimedLaunch {
  hipEvent_t start, stop;
};
TimedLaunch timing_begin(hipStream_t stream);
void timing_end(const char* name, const TimedLaunch& t, hipStream_t stream);
mhlmoe_status launched(hipError_t e, const char* what, hipStream_t stream);

// Launch one kernel (the callable returns the launch's hipError_t).
template <class F>
mhlmoe_status run_kernel(const char* name, hipStream_t stream, F&& launch) {
  const TimedLaunch t = timing_begin(stream);
  const hipError_t e = launch();
  timing_end(name, t, stream);
  return launched(e, name, stream);
}

}  // namespace api
}  // namespace mhl
