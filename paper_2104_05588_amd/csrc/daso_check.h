// What the argument checks of the training operators are made of (host only, no HIP calls).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "daso_train.h"

namespace daso {
namespace host {

constexpr int64_t kMaxElems = DASO_MAX_N;

inline bool known(int32_t type) { return type == DASO_TYPE_F32 || type == DASO_TYPE_BF16; }
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// A buffer of `outer` blocks `outer_stride` apart, each of `rows` rows of `row` elements,
// `stride` apart.
struct Block {
  const void* p;
  int64_t outer, outer_stride, rows, stride, row;
  size_t esz;
};

inline Block rows_of(const void* p, int64_t rows, int64_t stride, int64_t row, size_t esz) {
  return {p, 1, 0, rows, stride, row, esz};
}
inline Block flat(const void* p, int64_t n, size_t esz) { return {p, 1, 0, 1, n, n, esz}; }

inline uintptr_t begin(const Block& b) { return reinterpret_cast<uintptr_t>(b.p); }
inline uintptr_t end(const Block& b) {
  if (b.outer == 0 || b.rows == 0 || b.row == 0) return begin(b);
  return begin(b) + static_cast<uintptr_t>((b.outer - 1) * b.outer_stride + (b.rows - 1) * b.stride + b.row) * b.esz;
}
// Rows the same distance apart, of which one buffer's lie beside the other's: columns of one wider buffer.
inline bool beside(const Block& a, const Block& b) {
  if (a.outer > 1 || b.outer > 1 || a.rows <= 1 || b.rows <= 1) return false;
  const uintptr_t apart = static_cast<uintptr_t>(a.stride) * a.esz;
  if (apart != static_cast<uintptr_t>(b.stride) * b.esz || apart == 0) return false;
  const uintptr_t behind = begin(b) >= begin(a) ? (begin(b) - begin(a)) % apart : (apart - (begin(a) - begin(b)) % apart) % apart;
  return behind >= static_cast<uintptr_t>(a.row) * a.esz && behind + static_cast<uintptr_t>(b.row) * b.esz <= apart;
}
// By their spans, but for such rows.
inline bool overlap(const Block& a, const Block& b) {
  return a.p != nullptr && b.p != nullptr && begin(a) < end(b) && begin(b) < end(a) && !beside(a, b);
}
inline bool same(const Block& a, const Block& b) {
  return a.p == b.p && a.esz == b.esz && (a.rows <= 1 || a.stride == b.stride) &&
         (a.outer <= 1 || a.outer_stride == b.outer_stride);
}

// DASO_OK, or what is wrong with a buffer that is needed (or, with optional, may be null).
inline int need(const Block& b, bool optional = false) {
  if (b.p == nullptr) return optional ? DASO_OK : DASO_EINVAL;
  return aligned(b.p, b.esz) ? DASO_OK : DASO_EALIGN;
}

// The first status that is not DASO_OK.
inline int first(std::initializer_list<int> codes) {
  for (int c : codes)
    if (c != DASO_OK) return c;
  return DASO_OK;
}

inline bool stride_ok(int64_t stride, int64_t row, int64_t rows) {
  return stride >= row && (rows == 0 || stride <= kMaxElems / std::max<int64_t>(rows, 1));
}

inline bool finite_not_negative(float v) { return v >= 0.0f && std::isfinite(v); }

// Outputs against inputs and each other; `in_place` is the one input that outputs[0] may be.  (Lists of the call's own: an
// entry point that only checks its arguments and launches allocates nothing that could throw.)
template <class Inputs>
inline int check_alias(std::initializer_list<Block> outputs, const Inputs& inputs, int in_place) {
  for (const Block* o = outputs.begin(); o != outputs.end(); ++o) {
    int i = 0;
    for (const Block& in : inputs) {
      const bool allowed = i++ == in_place && o == outputs.begin() && same(*o, in);
      if (!allowed && overlap(*o, in)) return DASO_EALIAS;
    }
    for (const Block* k = outputs.begin(); k != o; ++k)
      if (overlap(*o, *k)) return DASO_EALIAS;
  }
  return DASO_OK;
}
inline int check_alias(std::initializer_list<Block> outputs, std::initializer_list<Block> inputs, int in_place) {
  return check_alias<std::initializer_list<Block>>(outputs, inputs, in_place);
}

}  // namespace host
}  // namespace daso
