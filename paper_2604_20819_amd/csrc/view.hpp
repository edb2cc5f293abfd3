// Checks of strided device tensors (cqsa_view), shared by the operators.
#pragma once

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

}  // namespace cqsa
