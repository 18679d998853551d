// What the C ABI's source files share: argument failures, the calling thread's
// last message, and the wrapper that turns exceptions into a dllm_status.
#pragma once
#include <string>

#include "../../include/dllm.h"
#include "common.h"

namespace dllm {

struct ApiError {
  int code;
  std::string msg;
};

[[noreturn]] inline void fail(int code, const std::string& msg) { throw ApiError{code, msg}; }
inline void require(bool ok, int code, const char* msg) {
  if (!ok) fail(code, msg);
}
inline void require(bool ok, int code, const std::string& msg) {
  if (!ok) fail(code, msg);
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

std::string& last_error();  // of the calling thread

}  // namespace dllm

#define API_BEGIN \
  ::dllm::last_error().clear(); \
  try {
#define API_END                                   \
  }                                               \
  catch (const ::dllm::ApiError& e) {             \
    ::dllm::last_error() = e.msg;                 \
    return e.code;                                \
  }                                               \
  catch (const ::dllm::HipError& e) {             \
    ::dllm::last_error() = e.what();              \
    return DLLM_EHIP;                             \
  }                                               \
  catch (const std::exception& e) {               \
    ::dllm::last_error() = e.what();              \
    return DLLM_EINVAL;                           \
  }                                               \
  return DLLM_OK;
