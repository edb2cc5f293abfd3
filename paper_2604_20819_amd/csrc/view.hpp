// Checks of strided device tensors (cqsa_view), shared by the operators.
#pragma once

#include <initializer_list>
#include <string>

#include "cqsa.h"
#include "errors.hpp"

namespace cqsa {

inline int64_t elem_bytes(cqsa_dtype dt) { return dt == CQSA_F32 ? 4 : 2; }
inline bool head_dim_ok(int64_t d) { return d >= 32 && d <= 256 && d % 32 == 0; }
inline bool empty(const cqsa_view& v) { return v.B == 0 || v.L == 0 || v.H == 0; }

// Shape, alignment and strides of a view; `written`: its elements must not overlap.
cqsa_status check_view(const cqsa_view* v, const char* name, int64_t d, bool written);
// Whether two views have one shape and dtype.
bool same_shape(const cqsa_view& x, const cqsa_view& y);
// Whether two views of one shape have the same elements' addresses.
bool same_place(const cqsa_view& x, const cqsa_view& y);
// Whether two views that check_view has passed, of one dtype and d, share an element.
// Exact, but for layouts that would take too long to tell apart, which count as sharing.
bool views_share(const cqsa_view& x, const cqsa_view& y);

// The bytes that an array or a view may touch, and its name; empty where an argument is not given.
struct Range {
  const char* name;
  uintptr_t lo, hi;
};
inline Range range_of(const char* name, const void* p, uint64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {name, at, p ? at + bytes : at};
}
// From a view's first element to its last.
Range view_range(const char* name, const cqsa_view& v);
inline cqsa_status check_workspace(const void* p, uint64_t bytes, uint64_t need, const std::string& what) {
  if (need == 0) return CQSA_OK;
  if (!p || bytes < need)
    return fail(CQSA_ERR_INVALID_ARG, what + "the workspace has " + std::to_string(p ? bytes : 0) +
                                          " bytes, the call needs " + std::to_string(need));
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "the workspace must be 16-byte aligned");
  return CQSA_OK;
}

// No range of `written` may meet another of them, or one of `read`.
inline cqsa_status check_apart(std::initializer_list<Range> written, std::initializer_list<Range> read,
                               const std::string& what) {
  auto meet = [](const Range& x, const Range& y) { return x.lo < y.hi && y.lo < x.hi && x.lo < x.hi && y.lo < y.hi; };
  for (const Range* w = written.begin(); w != written.end(); ++w) {
    for (const Range* x = w + 1; x != written.end(); ++x)
      if (meet(*w, *x)) return fail(CQSA_ERR_INVALID_ARG, what + w->name + " overlaps " + x->name);
    for (const Range& x : read)
      if (meet(*w, x)) return fail(CQSA_ERR_INVALID_ARG, what + w->name + " overlaps " + x.name);
  }
  return CQSA_OK;
}

}  // namespace cqsa

// Every entry point reports an exception as a status.
#define CQSA_ENTRY(name, expr)                                          \
  clear_error();                                                        \
  try {                                                                 \
    return expr;                                                        \
  } catch (const std::exception& e) {                                   \
    return fail(CQSA_ERR_INTERNAL, std::string(name ": ") + e.what());  \
  } catch (...) {                                                       \
    return fail(CQSA_ERR_INTERNAL, name ": unknown exception");         \
  }

