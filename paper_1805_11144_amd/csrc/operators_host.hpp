// Host-side helpers of the operators on device arrays: refusals, a failed runtime
// call as an ms::Error, the calling thread's device for the length of a scope,
// workspaces, access widths.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <type_traits>

#include "host.hpp"

#define HIPCHECK(expr)                                                                    \
  do {                                                                                    \
    hipError_t _e = (expr);                                                               \
    if (_e != hipSuccess)                                                                 \
      ms::fail(MS_E_HIP, std::string(#expr) + ": " + hipGetErrorString(_e));              \
  } while (0)

namespace ms {

struct DeviceGuard {
  int prev = 0;
  explicit DeviceGuard(int dev) {
    HIPCHECK(hipGetDevice(&prev));
    if (prev != dev) HIPCHECK(hipSetDevice(dev));
  }
  ~DeviceGuard() {
    int cur = 0;
    if (hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

inline void need(bool ok, const char* what) {
  if (!ok) fail(MS_E_INVALID, what);
}

constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxBlocks = (int64_t)1 << 23;   // workgroups of 256: the grid's threads fit 32 bits

inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

inline size_t size_of(int32_t dtype) { return dtype == MS_DTYPE_BF16 ? 2 : 4; }

inline void need_dtype(int32_t d) { need(d == MS_DTYPE_F32 || d == MS_DTYPE_BF16, "unknown dtype"); }

inline void need_aligned(const void* p, size_t to, const char* what) {
  if ((uintptr_t)p % to != 0) fail(MS_E_INVALID, std::string(what) + " is not aligned to its type");
}

inline void need_workspace(const void* ws, int64_t have, int64_t want) {
  if (want == 0) return;
  need(ws != nullptr, "NULL workspace");
  need((uintptr_t)ws % 256 == 0, "workspace must be 256-byte aligned");
  need(have >= want, "workspace too small");
}

// A piece of the workspace; every piece begins on 256 bytes.
struct Carve {
  char* base;
  int64_t used = 0;
  template <class T>
  T* take(int64_t n) {
    T* p = (T*)(base + used);
    used += up(n * (int64_t)sizeof(T), 256);
    return p;
  }
};

// The widest access, in values, that sizes, strides and pointers allow: at
// most 16 bytes of the narrowest type.
struct Wide {
  int64_t v;
  explicit Wide(size_t elem) : v(16 / (int64_t)elem) {}
  Wide& of(int64_t n) {
    while (n % v != 0) v /= 2;
    return *this;
  }
  Wide& at(const void* p, size_t elem) {
    while ((uintptr_t)p % ((size_t)v * elem) != 0) v /= 2;
    return *this;
  }
};

// Calls f with the access width as a compile-time number.
template <int MAX, class F>
void with_width(int64_t v, F&& f) {
  if constexpr (MAX >= 8)
    if (v == 8) return f(std::integral_constant<int, 8>{});
  if constexpr (MAX >= 4)
    if (v == 4) return f(std::integral_constant<int, 4>{});
  if constexpr (MAX >= 2)
    if (v == 2) return f(std::integral_constant<int, 2>{});
  f(std::integral_constant<int, 1>{});
}

// Calls f with the element type and the access width (at most M16 bf16 or M32
// float32 values).
template <int M16, int M32, class F>
void with_type(int32_t dtype, int64_t v, F&& f) {
  if (dtype == MS_DTYPE_BF16) with_width<M16>(v, [&](auto w) { f((__bf16)0.0f, w); });
  else with_width<M32>(v, [&](auto w) { f(0.0f, w); });
}

inline int32_t threads_per_row(int64_t nv) {
  int32_t t = 1;
  while (t < nv && t < 256) t *= 2;
  return t;
}

inline unsigned row_blocks(int64_t rows, int32_t tpr) {
  const int64_t per = 256 / tpr;
  return (unsigned)std::min<int64_t>((rows + per - 1) / per, kMaxBlocks);
}

}  // namespace ms
