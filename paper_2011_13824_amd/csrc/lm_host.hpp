// Host side shared by the translation units of a language model's operators: checks of arguments,
// types, limits of a launch and the parts of a workspace.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <exception>

#include "host.hpp"
#include "lirpa.h"
#include "lm_types.hpp"

namespace lirpa_host {

constexpr int kMaxWidth = 1 << 20;
constexpr int64_t kMaxLd = (1 << 22) - 1;
constexpr int64_t kMaxRows = (int64_t)1 << 30;

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool is_dtype(int t) { return t == LIRPA_F32 || t == LIRPA_BF16 || t == LIRPA_F16; }
inline size_t bytes_of(int dtype) { return dtype == LIRPA_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A launch has fewer than 2^32 threads.  The most blocks of `threads`:
constexpr int64_t max_blocks(int threads) { return (((int64_t)1 << 32) - 1) / threads; }

// No C++ exception leaves a C entry.
template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(LIRPA_EDEVICE, "%s", e.what());
  } catch (...) {
    return fail(LIRPA_EDEVICE, "unexpected exception");
  }
}

template <typename F>
int by_type(int dtype, F&& f) {
  switch (dtype) {
    case LIRPA_F32: return f(float{});
    case LIRPA_BF16: return f(lm::bf16{});
    default: return f(lm::f16{});
  }
}

inline int check_shape(const char* who, int dtype, int64_t rows, int n) {
  if (!is_dtype(dtype)) return fail(LIRPA_EINVAL, "%s: dtype %d is none of lirpa_dtype", who, dtype);
  if (rows < 0 || rows > kMaxRows)
    return fail(LIRPA_EINVAL, "%s: rows = %lld is outside [0, 2^30]", who, (long long)rows);
  if (n < 1 || n > kMaxWidth) return fail(LIRPA_EINVAL, "%s: width %d is outside [1, 2^20]", who, n);
  return LIRPA_OK;
}

inline int check_rows(const char* who, const char* what, int dtype, const void* p, int64_t ld,
                      int n) {
  if (!p) return fail(LIRPA_EINVAL, "%s: %s is null", who, what);
  if ((uintptr_t)p % bytes_of(dtype))
    return fail(LIRPA_EINVAL, "%s: %s is not aligned to its type", who, what);
  if (ld < n || ld > kMaxLd)
    return fail(LIRPA_EINVAL, "%s: the row distance %lld of %s is outside [%d, 2^22)", who,
                (long long)ld, what, n);
  return LIRPA_OK;
}

// An output in an input's buffer: its rows lie where the input's do, or they would be written over
// rows that are still to be read.
inline int check_in_place(const char* who, const char* out, const void* po, int64_t ldo,
                          const char* in, const void* pi, int64_t ldi, int64_t rows) {
  if (!po || po != pi || ldo == ldi || rows == 1) return LIRPA_OK;
  return fail(LIRPA_EINVAL, "%s: %s is the buffer of %s, with a row distance of %lld, not %lld", who,
              out, in, (long long)ldo, (long long)ldi);
}

inline int check_floats(const char* who, const char* what, const void* p, bool needed = false) {
  if (needed && !p) return fail(LIRPA_EINVAL, "%s: %s is null", who, what);
  if ((uintptr_t)p % 4) return fail(LIRPA_EINVAL, "%s: %s is not aligned to its type", who, what);
  return LIRPA_OK;
}

inline int check_ws(const char* who, const void* ws, size_t ws_bytes, size_t need) {
  if (!ws) return fail(LIRPA_EINVAL, "%s: the workspace is null", who);
  if (!aligned16(ws))
    return fail(LIRPA_EINVAL, "%s: the workspace does not start on 16 bytes", who);
  if (ws_bytes < need)
    return fail(LIRPA_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, ws_bytes,
                need);
  return LIRPA_OK;
}

#define TRY(x)                     \
  do {                             \
    int rc_ = (x);                 \
    if (rc_ != LIRPA_OK) return rc_; \
  } while (0)

// Parts of the workspace, in order, each on 256 bytes.
struct Carver {
  char* base;
  size_t at = 0;
  void* take(size_t bytes) {
    void* p = base ? base + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return p;
  }
};

}  // namespace lirpa_host
