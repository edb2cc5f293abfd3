// cqsa_rotary and its plan, and the checks of strided tensors.
#include "rotary.hpp"

#include <algorithm>
#include <cmath>
#include <new>

#include "runtime.hpp"
#include "view.hpp"

namespace cqsa {

cqsa_status check_view(const cqsa_view* v, const char* name, int64_t d, bool written) {
  const std::string n(name);
  if (!v) return fail(CQSA_ERR_INVALID_ARG, n + " is NULL");
  if (v->dtype != CQSA_F32 && v->dtype != CQSA_F16 && v->dtype != CQSA_BF16)
    return fail(CQSA_ERR_INVALID_ARG, n + " has an unknown dtype");
  const int64_t most = int64_t(1) << 31;
  if (v->B < 0 || v->L < 0 || v->H < 0 || v->B >= most || v->L >= most || v->H >= most)
    return fail(CQSA_ERR_INVALID_ARG, n + " has an extent outside [0, 2^31)");
  if (v->d != d) return fail(CQSA_ERR_INVALID_ARG, n + ".d differs from the plan's or the cache's");
  if (empty(*v)) return CQSA_OK;
  if (!v->data) return fail(CQSA_ERR_INVALID_ARG, n + ".data is NULL");
  if (reinterpret_cast<uintptr_t>(v->data) % 16 != 0)
    return fail(CQSA_ERR_INVALID_ARG, n + ".data must be 16-byte aligned");
  struct Axis {
    int64_t n, stride;
  } ax[3] = {{v->B, v->stride_b}, {v->L, v->stride_l}, {v->H, v->stride_h}};
  const int64_t unit = 16 / elem_bytes(v->dtype);
  for (const Axis& a : ax) {
    if (a.n == 1) continue;
    if (a.stride < 0 || a.stride % unit != 0 || a.stride > (int64_t(1) << 42))
      return fail(CQSA_ERR_INVALID_ARG, n + "'s strides must be multiples of 16 bytes, 0 or more");
  }
  if (!written) return CQSA_OK;
  std::sort(ax, ax + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
  __int128 span = v->d;  // elements that the axes so far reach
  for (const Axis& a : ax) {
    if (a.n == 1) continue;
    if (a.stride < span) return fail(CQSA_ERR_INVALID_ARG, n + " is written and overlaps itself");
    span += __int128(a.stride) * (a.n - 1);
  }
  return CQSA_OK;
}

bool same_shape(const cqsa_view& x, const cqsa_view& y) {
  return x.dtype == y.dtype && x.B == y.B && x.L == y.L && x.H == y.H && x.d == y.d;
}

namespace {
// Elements from the first to behind the last one of a view that is not empty.
__int128 extent(const cqsa_view& v) {
  auto reach = [](int64_t n, int64_t s) { return n > 1 ? __int128(n - 1) * s : __int128(0); };
  return reach(v.B, v.stride_b) + reach(v.L, v.stride_l) + reach(v.H, v.stride_h) + v.d;
}
}  // namespace

bool same_place(const cqsa_view& x, const cqsa_view& y) {
  auto same = [](int64_t n, int64_t a, int64_t b) { return n == 1 || a == b; };
  return x.data == y.data && same(x.B, x.stride_b, y.stride_b) && same(x.L, x.stride_l, y.stride_l) &&
         same(x.H, x.stride_h, y.stride_h);
}

namespace {
// Whether a sum of v_t * stride_t, 0 <= v_t <= most_t, lies in [lo, hi]; the strides fall,
// so that few v of each are near enough.
struct Term {
  __int128 stride, most;
};
bool reaches(const Term* t, int n, __int128 lo, __int128 hi, int* steps) {
  if (hi < 0) return false;
  if (lo <= 0) return true;
  if (n == 0) return false;
  if (--*steps < 0) return true;
  __int128 rest = 0;  // the most that the terms behind this one add
  for (int i = 1; i < n; ++i) rest += t[i].stride * t[i].most;
  const __int128 s = t->stride;
  const __int128 first = lo > rest ? (lo - rest + s - 1) / s : 0;
  for (__int128 v = std::min(hi / s, t->most); v >= first; --v)
    if (reaches(t + 1, n - 1, lo - v * s, hi - v * s, steps)) return true;
  return false;
}

// Whether the bytes that two views span meet.
bool views_meet(const cqsa_view& x, const cqsa_view& y) {
  if (empty(x) || empty(y)) return false;
  const __int128 a = reinterpret_cast<uintptr_t>(x.data), b = reinterpret_cast<uintptr_t>(y.data);
  return a < b + extent(y) * elem_bytes(y.dtype) && b < a + extent(x) * elem_bytes(x.dtype);
}
}  // namespace

bool views_share(const cqsa_view& x, const cqsa_view& y) {
  if (!views_meet(x, y)) return false;
  // Rows of d elements: x's at some sum of its strides, y's counted from its last one
  // back, so that every stride adds to their distance, which is below a row's width
  // where two rows meet.
  const int64_t size = elem_bytes(x.dtype);
  Term t[6];
  int n = 0;
  __int128 at = __int128(reinterpret_cast<uintptr_t>(x.data)) - __int128(reinterpret_cast<uintptr_t>(y.data));
  auto add = [&](int64_t count, int64_t stride) {
    if (count < 2 || stride == 0) return;
    for (int i = 0; i < n; ++i)
      if (t[i].stride == __int128(stride) * size) {
        t[i].most += count - 1;
        return;
      }
    t[n++] = {__int128(stride) * size, count - 1};
  };
  add(x.B, x.stride_b), add(x.L, x.stride_l), add(x.H, x.stride_h);
  add(y.B, y.stride_b), add(y.L, y.stride_l), add(y.H, y.stride_h);
  at -= (extent(y) - y.d) * size;
  std::sort(t, t + n, [](const Term& a, const Term& b) { return a.stride > b.stride; });
  const __int128 width = x.d * size;
  int steps = 1 << 16;
  return reaches(t, n, 1 - width - at, width - 1 - at, &steps);
}

namespace {

cqsa_status make_table(const cqsa_rotary_opts& o, cqsa_rotary_s* p) {
  if (!head_dim_ok(o.d))
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: d must be a multiple of 32 in [32, 256]");
  if (o.n_axes < 1 || o.n_axes > CQSA_MAX_AXES)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: n_axes must be in [1, 4]");
  if (o.pairs != CQSA_PAIR_HALF && o.pairs != CQSA_PAIR_ADJACENT)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: unknown order of the pairs");
  if (o.spectrum != CQSA_SPECTRUM_SHARED && o.spectrum != CQSA_SPECTRUM_AXIS)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: unknown spectrum");
  if (o.dealt != 0 && o.dealt != 1)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: dealt must be 0 or 1");
  if (!(o.theta > 1.0) || !std::isfinite(o.theta))
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: theta must be above 1 and finite");
  int64_t n = 0;
  for (int a = 0; a < o.n_axes; ++a) {
    if (o.sections[a] < 1 || o.sections[a] > kMaxPairs)
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: every axis needs 1 pair or more");
    if (!(o.pos_scale[a] > 0.0) || !std::isfinite(o.pos_scale[a]))
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: pos_scale must be positive and finite");
    n += o.sections[a];
  }
  if (n % 8 != 0 || 2 * n > o.d)
    return fail(CQSA_ERR_INVALID_ARG,
                "cqsa_rotary_plan: the sections' sum must be a multiple of 8 and at most d / 2");
  p->opts = o;
  p->n = int32_t(n);
  int used[CQSA_MAX_AXES] = {0, 0, 0, 0};
  int axis = 0;
  for (int i = 0; i < n; ++i) {
    // the axis of pair i: the next one in turn with room, or the first with room
    if (o.dealt && i > 0) axis = (axis + 1) % o.n_axes;
    while (used[axis] == o.sections[axis]) axis = (axis + 1) % o.n_axes;
    const int j = used[axis]++;
    const long double at = o.spectrum == CQSA_SPECTRUM_SHARED ? (long double)i / n
                                                              : (long double)j / o.sections[axis];
    // radians a position, then turns without the whole ones: four roundings to 64 bits
    // of a value of at most pos_scale / 2 pi turns, and that to 2^-64 turns, are under
    // 2^-64 (1 + pos_scale) turns
    const long double f = o.pos_scale[axis] * std::pow((long double)o.theta, -at);
    long double t = f / 6.283185307179586476925286766559006L;
    t -= std::floor(t);
    const long double scaled = std::round(t * 18446744073709551616.0L);
    p->tab.turn[i] = scaled >= 18446744073709551616.0L ? 0 : uint64_t(scaled);
    p->tab.axis[i] = uint8_t(axis);
  }
  for (int i = int(n); i < kMaxPairs; ++i) p->tab.turn[i] = 0, p->tab.axis[i] = 0;
  return CQSA_OK;
}

cqsa_status rotary_impl(const cqsa_rotary_s* p, const int32_t* pos, const cqsa_view* x,
                        const cqsa_view* y, int32_t n, int32_t inverse, hipStream_t s) {
  if (!p) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: plan is NULL");
  if (n != 1 && n != 2) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: n must be 1 or 2");
  if (inverse != 0 && inverse != 1)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: inverse must be 0 or 1");
  if (!x || !y) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: x or y is NULL");
  cqsa_status st;
  bool in_place = true;
  int64_t heads = 0;
  for (int k = 0; k < n; ++k) {
    if ((st = check_view(&x[k], "x", p->opts.d, false)) != CQSA_OK) return st;
    if ((st = check_view(&y[k], "y", p->opts.d, true)) != CQSA_OK) return st;
    if (!same_shape(x[k], y[k]))
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: y differs from x in shape or dtype");
    if (x[k].B != x[0].B || x[k].L != x[0].L || x[k].dtype != x[0].dtype)
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: the tensors must share B, L and the dtype");
    heads += x[k].H;
  }
  for (int k = 0; k < n; ++k) {
    const bool same = empty(x[k]) || same_place(x[k], y[k]);
    in_place = in_place && same;
    if (!same && views_share(x[k], y[k]))
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: y overlaps x without being x");
  }
  if (n == 2) {
    if (views_share(y[0], y[1]))
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: the results are one tensor, or share elements");
    // turned in place, a result meets the other tensor where it meets the other result
    if (!in_place && (views_share(x[0], y[1]) || views_share(x[1], y[0])))
      return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: a result shares elements with the other tensor");
  }
  if (heads > (1 << 20))
    return fail(CQSA_ERR_UNSUPPORTED, "cqsa_rotary: more than 2^20 heads");
  const int64_t rows = x[0].B * x[0].L;
  if (rows == 0 || heads == 0) return CQSA_OK;
  if (!pos) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: pos is NULL");
  if (reinterpret_cast<uintptr_t>(pos) % 4 != 0)
    return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary: pos must be 4-byte aligned");
  RotaryArgs a{};
  for (int k = 0; k < n; ++k)
    a.t[k] = {x[k].data,     y[k].data,     x[k].stride_b, x[k].stride_l,
              x[k].stride_h, y[k].stride_b, y[k].stride_l, y[k].stride_h};
  a.pos = pos;
  a.rows = rows;
  a.L = uint32_t(x[0].L);
  a.H0 = uint32_t(x[0].H);
  a.H = uint32_t(heads);
  a.pairs = uint32_t(p->n);
  const int32_t vec = int32_t(16 / elem_bytes(x[0].dtype));
  a.chunks = uint32_t(p->n / vec);
  a.units = in_place ? a.chunks : uint32_t(p->opts.d / (2 * vec));
  a.inverse = inverse;
  a.tab = p->tab;
  // A thread takes a batch of heads, fewer where that leaves under 2^18 threads
  // (4096 rows of 40 heads, bf16, d = 128: 5 heads each 15.7 us, 1 or 2 24.3;
  // 32768 rows of 32: 8 heads 83, 32 101).
  const int64_t per = rows * a.units;
  a.parts = uint32_t(std::max<int64_t>((a.H + kRotaryBatch - 1) / kRotaryBatch,
                                       std::min<int64_t>(a.H, ((1 << 18) + per - 1) / per)));
  const int64_t per_row = int64_t(a.units) * a.parts;
  const int64_t slab = (int64_t(1) << 30) / per_row;  // rows of a launch; per_row <= 2^24
  for (int64_t r = 0; r < rows; r += slab) {
    a.row0 = r;
    a.n = uint32_t(std::min(slab, rows - r) * per_row);
    CQSA_HIP(launch_rotary(x[0].dtype, p->opts.pairs == CQSA_PAIR_ADJACENT, a, s));
  }
  return CQSA_OK;
}

}  // namespace

}  // namespace cqsa

using namespace cqsa;

extern "C" {

void cqsa_rotary_opts_default(cqsa_rotary_opts* o, int32_t d) {
  if (!o) return;
  *o = cqsa_rotary_opts{};
  o->d = d;
  o->n_axes = 1;
  o->sections[0] = d / 2;
  o->theta = 10000.0;
  for (double& s : o->pos_scale) s = 1.0;
}

cqsa_status cqsa_rotary_plan(const cqsa_rotary_opts* opts, cqsa_rotary_t** out) {
  clear_error();
  try {
    if (!out) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: out is NULL");
    *out = nullptr;
    if (!opts) return fail(CQSA_ERR_INVALID_ARG, "cqsa_rotary_plan: opts is NULL");
    cqsa_rotary_s tmp{};
    const cqsa_status st = make_table(*opts, &tmp);
    if (st != CQSA_OK) return st;
    *out = new cqsa_rotary_s(tmp);
    return CQSA_OK;
  } catch (const std::exception& e) {
    return fail(CQSA_ERR_INTERNAL, std::string("cqsa_rotary_plan: ") + e.what());
  } catch (...) {
    return fail(CQSA_ERR_INTERNAL, "cqsa_rotary_plan: unknown exception");
  }
}

void cqsa_rotary_destroy(cqsa_rotary_t* plan) { delete plan; }

cqsa_status cqsa_rotary(const cqsa_rotary_t* plan, const int32_t* pos, const cqsa_view* x,
                        const cqsa_view* y, int32_t n, int32_t inverse, void* hip_stream) {
  clear_error();
  try {
    return rotary_impl(plan, pos, x, y, n, inverse, (hipStream_t)hip_stream);
  } catch (const std::exception& e) {
    return fail(CQSA_ERR_INTERNAL, std::string("cqsa_rotary: ") + e.what());
  } catch (...) {
    return fail(CQSA_ERR_INTERNAL, "cqsa_rotary: unknown exception");
  }
}

}  // extern "C"
