// Shared by the C entry points: error reporting and argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "../../include/farskip.h"

namespace fs {
// Detail of the calling thread's last error (fs_last_error_message).
std::string& last_message();
}  // namespace fs

namespace {

[[maybe_unused]] fs_status fail(fs_status st, const std::string& m) {
  fs::last_message() = m;
  return st;
}
[[maybe_unused]] fs_status hip_fail(hipError_t e, const char* where) {
  fs::last_message() = std::string(where) + ": " + hipGetErrorString(e);
  return FS_ERR_HIP;
}
#define FS_HIP(expr, where)                     \
  do {                                          \
    hipError_t e_ = (expr);                     \
    if (e_ != hipSuccess) return hip_fail(e_, where); \
  } while (0)

[[maybe_unused]] bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
[[maybe_unused]] bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

#define NEED(ptr, name)                                                                      \
  do {                                                                                       \
    if (!(ptr)) return fail(FS_ERR_INVALID, std::string(name) + " must not be NULL");        \
    if (!aligned16(ptr)) return fail(FS_ERR_INVALID, std::string(name) + " must be 16-byte aligned"); \
  } while (0)
// int32 index arrays and fp32 gate arrays are read element by element
#define NEED4(ptr, name)                                                                     \
  do {                                                                                       \
    if (!(ptr)) return fail(FS_ERR_INVALID, std::string(name) + " must not be NULL");        \
    if (!aligned4(ptr)) return fail(FS_ERR_INVALID, std::string(name) + " must be 4-byte aligned"); \
  } while (0)
#define OPT4(ptr, name)                                                                      \
  do {                                                                                       \
    if ((ptr) && !aligned4(ptr))                                                             \
      return fail(FS_ERR_INVALID, std::string(name) + " must be 4-byte aligned");            \
  } while (0)
#define OPT(ptr, name)                                                                       \
  do {                                                                                       \
    if ((ptr) && !aligned16(ptr))                                                            \
      return fail(FS_ERR_INVALID, std::string(name) + " must be 16-byte aligned");           \
  } while (0)

[[maybe_unused]] size_t elem(int dtype) { return dtype == FS_F32 ? 4 : 2; }
[[maybe_unused]] size_t align256(size_t b) { return (b + 255) / 256 * 256; }
[[maybe_unused]] hipStream_t S(fs_stream s) { return reinterpret_cast<hipStream_t>(s); }

#define TRY(expr)                 \
  do {                            \
    const fs_status st_ = (expr); \
    if (st_ != FS_OK) return st_; \
  } while (0)

[[maybe_unused]] bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The kernels run on the stream's device, which has to be the current one.
[[maybe_unused]] fs_status check_stream(fs_stream stream) {
  hipStream_t s = S(stream);
  if (!s) return FS_OK;
  int cur = 0;
  hipDevice_t dev = 0;
  FS_HIP(hipGetDevice(&cur), "hipGetDevice");
  FS_HIP(hipStreamGetDevice(s, &dev), "hipStreamGetDevice");
  if ((int)dev != cur)
    return fail(FS_ERR_INVALID, "the stream belongs to device " + std::to_string((int)dev) +
                                    ", not the current device " + std::to_string(cur));
  return FS_OK;
}

[[maybe_unused]] fs_status check_dtype(int32_t dtype) {
  if (dtype != FS_F32 && dtype != FS_BF16) return fail(FS_ERR_INVALID, "dtype must be FS_F32 or FS_BF16");
  return FS_OK;
}

[[maybe_unused]] int dt(int32_t dtype) { return dtype == FS_F32 ? 0 : 1; }

// No exception (a message that finds no memory) leaves a C entry point.
template <typename F>
fs_status entry(F&& f) noexcept {
  try {
    return f();
  } catch (...) {
    return FS_ERR_INVALID;
  }
}

}  // namespace
