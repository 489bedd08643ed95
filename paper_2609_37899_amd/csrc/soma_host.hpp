// soma_host.hpp -- what the translation units of the C ABI share on the host:
// the thread's last error and the checks in front of a launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <tuple>

#include "soma.h"

namespace soma {

// Record a description of the error `code` for soma_last_error(); returns code.
int set_error(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Clear it; returns SOMA_OK.
int set_ok();

inline hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// A device call's failure; the runtime's record of it is cleared, for it is told here.
inline int device_error(const char* what, hipError_t e) {
  (void)hipGetLastError();
  return set_error(SOMA_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Launches and reports the launch's own status: the runtime's last error may be of
// a call that the caller made before.
template <class... P, class... A>
int launch(const char* what, void (*kernel)(P...), dim3 grid, dim3 block, unsigned lds, hipStream_t st, const A&... args) {
  std::tuple<P...> values(args...);
  const hipError_t e = std::apply(
      [&](P&... x) {
        void* at[] = {const_cast<void*>(static_cast<const void*>(&x))...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, at, lds, st);
      },
      values);
  return e == hipSuccess ? SOMA_OK : device_error(what, e);
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

inline bool is_type(int32_t t) { return t == SOMA_FLOAT || t == SOMA_BFLOAT; }
inline size_t type_size(int32_t t) { return t == SOMA_BFLOAT ? 2 : 4; }

inline int check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return SOMA_OK;
  if (!ws) return set_error(SOMA_EWORKSPACE, "workspace is NULL");
  if (!is_aligned(ws, 256)) return set_error(SOMA_EWORKSPACE, "workspace must be 256-byte aligned");
  if (have < need) return set_error(SOMA_EWORKSPACE, "workspace too small: %zu < %zu bytes", have, need);
  return SOMA_OK;
}

}  // namespace soma
