// Host-side argument checks shared by the C ABI's source files (internal).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>
#include <exception>
#include <vector>

#include "errors.h"
#include "rag_attn.h"

namespace rag {

constexpr int32_t kBlock = 16;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// RAG_ATTN_CHECK=1: device arrays are copied to the host and checked.
inline bool check_mode() {
  static const bool on = [] {
    const char* e = std::getenv("RAG_ATTN_CHECK");
    return e != nullptr && e[0] == '1';
  }();
  return on;
}

// n zeros, if the host has the memory.
template <class T>
inline bool room(std::vector<T>& dst, size_t n) {
  try {
    dst.assign(n, T());
    return true;
  } catch (const std::exception&) {              // (none may leave the C entries)
    return false;
  }
}

// Copies n values from device memory (stream-ordered, synchronous).
template <class T>
inline bool fetch(std::vector<T>& dst, const T* src, size_t n, hipStream_t stream) {
  if (!room(dst, n)) return false;
  if (n == 0) return true;
  if (hipMemcpyAsync(dst.data(), src, n * sizeof(T), hipMemcpyDeviceToHost, stream) != hipSuccess)
    return false;
  return hipStreamSynchronize(stream) == hipSuccess;
}

inline rag_status check_cu(const std::vector<int32_t>& cu, const char* name, int32_t max_len) {
  if (cu[0] != 0) return fail(RAG_ERR_INVALID_ARG, "%s[0] = %d, expected 0", name, cu[0]);
  for (size_t s = 0; s + 1 < cu.size(); ++s) {
    const int64_t n = (int64_t)cu[s + 1] - cu[s];
    if (n < 0) return fail(RAG_ERR_INVALID_ARG, "%s decreases at %zu", name, s);
    if (n > max_len)
      return fail(RAG_ERR_INVALID_ARG, "%s: sequence %zu has %lld > max %d rows", name, s,
                  (long long)n, max_len);
  }
  return RAG_OK;
}

}  // namespace rag
