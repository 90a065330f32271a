// Argument checks that the entry points of the vocabulary head and of the attention block share.
#pragma once

#include <exception>
#include <string>

#include "common.h"

namespace fold {

inline int api_fail(int code, const std::string& msg) {
  set_error(msg);
  return code;
}

// runs an entry point's body; nothing it throws leaves the library
template <class F>
int32_t guarded(F&& body) {
  try {
    clear_error();
    return body();
  } catch (const std::exception& e) {
    return api_fail(FOLD_E_INVALID, std::string("internal error: ") + e.what());
  } catch (...) {
    return api_fail(FOLD_E_INVALID, "internal error");
  }
}

constexpr int64_t kMaxTiles = (1 << 24) - 8;  // workgroups of one launch, rounded up to 8: its threads fit 32 bits

inline bool known_type(int dtype) { return dtype == FOLD_F32 || dtype == FOLD_BF16; }
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline size_t bytes_of(int dtype, int64_t rows, int width) {
  return (size_t)rows * (size_t)row_ld(width) * (dtype == FOLD_BF16 ? 2 : 4);
}

// whether an output shares memory with another buffer (NULL: no)
struct Span {
  const void* p;
  size_t bytes;
};
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x && y && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
// whether an output overlaps another one or one of the others
inline bool any_overlap(const Span* out, int n, const Span* others, int m) {
  for (int i = 0; i < n; ++i) {
    for (int j = i + 1; j < n; ++j)
      if (overlap(out[i], out[j])) return true;
    for (int j = 0; j < m; ++j)
      if (overlap(out[i], others[j])) return true;
  }
  return false;
}

}  // namespace fold
