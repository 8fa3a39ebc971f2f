// What every entry point of the C ABI shares (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <new>

#include "../../include/muon.h"

namespace muon {

// Keeps the error for muon_last_hip_error of this thread.
int hip_fail(hipError_t e);

#define MUON_HIP(expr)                                 \
  do {                                                 \
    hipError_t e__ = (expr);                           \
    if (e__ != hipSuccess) return ::muon::hip_fail(e__); \
  } while (0)

// Every entry point runs its body through this: nothing may unwind through the C ABI.
template <typename F>
int guarded(F&& body) noexcept {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return MUON_E_NO_MEMORY;
  } catch (...) {
    return MUON_E_INVALID_ARG;
  }
}

}  // namespace muon
