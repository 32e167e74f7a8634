// What the host sides of the operators around the step share: refusals, checks of pointers and sizes, types as constants.
// No state, no allocation, nothing that throws.
#pragma once
#include "../../include/fira.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "fira_error.h"
#include "fira_rows.h"

namespace {

constexpr int64_t kMost = 0x7fffffff, kMostDim = 1 << 24;

__attribute__((format(printf, 2, 3))) fira_status refuse(fira_status st, const char* format, ...) {
  char msg[256];
  va_list args;
  va_start(args, format);
  std::vsnprintf(msg, sizeof msg, format, args);
  va_end(args);
  return fira_fail_without_context(st, msg);
}

fira_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FIRA_OK : refuse(FIRA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <int N>
using Int = std::integral_constant<int, N>;

bool known(int32_t dtype) { return dtype == FIRA_F32 || dtype == FIRA_BF16; }
size_t size_of(int32_t dtype) { return dtype == FIRA_F32 ? 4 : 2; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// A pointer that has to be there and aligned to its elements.
#define FIRA_POINTER(p, bytes)                                                                              \
  do {                                                                                                      \
    if (!(p)) return refuse(FIRA_ERR_INVALID_ARG, #p " is null");                                           \
    if (!aligned(p, bytes)) return refuse(FIRA_ERR_INVALID_ARG, #p " is not aligned to its elements");      \
  } while (0)
#define FIRA_LEADING(ld, width, rows)                                                                       \
  do {                                                                                                      \
    if ((ld) < (width)) return refuse(FIRA_ERR_SHAPE, #ld " is below the width");                           \
    int64_t span_;                                                                                          \
    if (__builtin_mul_overflow((int64_t)(ld), (int64_t)(rows) + 1, &span_) || span_ > INT64_MAX / 4)        \
      return refuse(FIRA_ERR_SHAPE, #ld " is out of range");                                                \
  } while (0)

fira_status check_workspace(const void* p, size_t have, size_t need) {
  if (have < need || (need && !p)) return refuse(FIRA_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", p ? have : (size_t)0, need);
  if (!aligned(p, 256)) return refuse(FIRA_ERR_WORKSPACE, "workspace is not aligned to 256 bytes");
  return FIRA_OK;
}

// Calls f with the types that two fira_dtypes stand for.
template <typename F>
void with_types(int32_t a, int32_t b, F f) {
  if (a == FIRA_F32) { if (b == FIRA_F32) f(FiraStoredF32{}, FiraStoredF32{}); else f(FiraStoredF32{}, FiraStoredBf16{}); }
  else { if (b == FIRA_F32) f(FiraStoredBf16{}, FiraStoredF32{}); else f(FiraStoredBf16{}, FiraStoredBf16{}); }
}

// Calls f with `flag` as a constant.
template <typename F>
void with_flag(bool flag, F f) {
  if (flag) f(std::true_type{});
  else f(std::false_type{});
}

}  // namespace
