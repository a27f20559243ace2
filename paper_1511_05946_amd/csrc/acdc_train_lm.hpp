// What the entry points of the language-model operators (acdc_train_lm.h) check on
// the host: that nothing which a call writes shares memory with what it reads, or
// with what else it writes.
#pragma once

#include <initializer_list>

#include "acdc_train.hpp"
#include "acdc_train_lm.h"

namespace acdc {

// Memory from the first value of the first row to the last one of the last row; of a null
// pointer and of no rows: none.
struct Span {
  const char* from = nullptr;
  const char* to = nullptr;
  bool none() const { return from == to; }
};
inline Span span_of(const void* p, int64_t rows, int64_t stride, int64_t width, size_t bytes) {
  if (p == nullptr || rows <= 0) return {};
  const char* a = static_cast<const char*>(p);
  return {a, a + (size_t(rows - 1) * size_t(stride) + size_t(width)) * bytes};
}
inline Span span_of(const void* p, int64_t count, size_t bytes) { return span_of(p, 1, 0, count, bytes); }
inline bool apart(const Span& a, const Span& b) { return a.none() || b.none() || a.to <= b.from || b.to <= a.from; }
// Each of what is written is apart from all that is read and from the others.
inline bool all_apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span* w = written.begin(); w != written.end(); ++w) {
    for (const Span* v = written.begin(); v != w; ++v)
      if (!apart(*v, *w)) return false;
    for (const Span& r : read)
      if (!apart(r, *w)) return false;
  }
  return true;
}

}  // namespace acdc
