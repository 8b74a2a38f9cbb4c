// What the exported functions share on the host: the thread's error text and the guard that keeps C++
// exceptions inside the library.
#pragma once
#include <cstdint>
#include <new>

#include <cuda_runtime.h>

#include "../../include/rudra_ps.h"

namespace rudra {

// Record the reason of a failure for rudra_last_error() and return `code`.
int fail(int code, const char* fmt, ...);
int cuda_fail(cudaError_t e, const char* what);

// Runs the body of an exported function; a C++ exception (in practice std::bad_alloc from a host
// container) becomes an error code instead of crossing the C boundary.
template <typename F>
auto guarded(F&& body) -> decltype(body()) {
  using R = decltype(body());
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return (R)fail(RUDRA_E_NOMEM, "out of host memory");
  } catch (...) {
    return (R)fail(RUDRA_E_NOMEM, "unexpected C++ exception");
  }
}

constexpr uintptr_t kAlignMask = 31;       // 256-bit vector accesses

inline bool aligned(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & kAlignMask) == 0; }

}  // namespace rudra
