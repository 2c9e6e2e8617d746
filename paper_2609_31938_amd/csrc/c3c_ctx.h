// The context object and the host helpers that every entry point's
// translation unit uses.  Internal; the public header only names the type.
#pragma once

#include <stdint.h>

#include <string>
#include <vector>

#include "c3c.h"

struct c3c_ctx {
  uint32_t mode = 0;
  c3c_counters ctr{};
  std::vector<c3c_sig_count> shapes;
  std::string last_error;
  void* ws = nullptr;      // caller's workspace (device memory)
  size_t ws_bytes = 0;
};

namespace c3c {

// whether two byte ranges meet (NULL and empty ranges meet nothing)
inline bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  if (!a || !b || abytes <= 0 || bbytes <= 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + static_cast<uintptr_t>(bbytes) && b0 < a0 + static_cast<uintptr_t>(abytes);
}

// sets the context's message and returns the status (the message is lost, and
// nothing is thrown, where there is no memory for it)
inline int fail(c3c_ctx* ctx, int status, const char* msg) noexcept {
  try {
    if (ctx) ctx->last_error = msg;
  } catch (...) {
  }
  return status;
}
inline int fail(c3c_ctx* ctx, int status, const std::string& msg) {
  if (ctx) ctx->last_error = msg;
  return status;
}

}  // namespace c3c
