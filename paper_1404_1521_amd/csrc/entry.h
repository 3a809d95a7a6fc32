// What the entry points of the sequence operators share: the guard around their
// bodies and the checks of their arguments.
#pragma once
#include <initializer_list>

#include "context.h"

namespace pg {

// Kernel ids of these operators among a context's timing marks.
constexpr int kOpKernels = POLYGLOT_NKERNELS;

// Runs an entry point's body; nothing that it throws (a message that finds no
// memory) passes the C boundary.
template <class F>
int entry(F f) noexcept {
  try {
    return f();
  } catch (...) {
    return POLYGLOT_EHIP;
  }
}

inline size_t size_of(int dtype) { return dtype == POLYGLOT_F32 ? 4 : 2; }

inline bool format_ok(int dtype) {
  return dtype == POLYGLOT_F32 || dtype == POLYGLOT_BF16 || dtype == POLYGLOT_F16;
}

inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Rows of `width` elements `ld` apart whose last byte's offset fits 63 bits.
inline bool rows_ok(int64_t ld, int64_t rows, int64_t width) {
  return ld >= width && (rows == 0 || ld <= (INT64_MAX / 8) / rows);
}

// A tensor of [tokens][width] elements of `size` bytes.
struct Rows {
  const void* p;
  int64_t ld;
  int width;
};

inline int check_rows(polyglot_ctx* ctx, int64_t tokens, size_t size, std::initializer_list<Rows> all,
                      const std::string& what, int64_t most_ld = INT64_MAX) {
  if (tokens == 0) return POLYGLOT_OK;
  for (const Rows& r : all) {
    if (!r.p) return fail(ctx, POLYGLOT_ENULL, what + ": NULL pointer");
    if (!rows_ok(r.ld, tokens, r.width) || r.ld > most_ld)
      return fail(ctx, POLYGLOT_EINVAL, what + ": rows closer than their width, or too many");
    if (!aligned(r.p, size)) return fail(ctx, POLYGLOT_EINVAL, what + ": misaligned pointer");
  }
  return POLYGLOT_OK;
}

}  // namespace pg
