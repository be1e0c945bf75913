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

}  // namespace
