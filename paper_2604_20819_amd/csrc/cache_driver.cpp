// The entry points of the 4-bit cache: argument checks and launches.
#include "cache.hpp"

#include <algorithm>
#include <cmath>

#include "cache_bound.hpp"
#include "runtime.hpp"
#include "view.hpp"

namespace cqsa {

namespace {

int page_log2_of(int32_t page_size) {
  switch (page_size) {
    case 32: return 5;
    case 64: return 6;
    case 128: return 7;
    case 256: return 8;
    default: return 0;
  }
}

constexpr int32_t kMaxHeads = 65536;
constexpr float kLog2e = 1.4426950408889634f;

cqsa_status check_cache(const cqsa_cache* c, const std::string& what) {
  if (!c) return fail(CQSA_ERR_INVALID_ARG, what + "cache is NULL");
  if (page_log2_of(c->page_size) == 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "page_size must be 32, 64, 128 or 256");
  if (!head_dim_ok(c->d))
    return fail(CQSA_ERR_INVALID_ARG, what + "the cache's d must be a multiple of 32 in [32, 256]");
  if (c->H < 1 || c->H > kMaxHeads)
    return fail(CQSA_ERR_INVALID_ARG, what + "the cache's H must be in [1, 65536]");
  if (c->n_pages < 0 || c->n_pages > (int64_t(1) << 31))
    return fail(CQSA_ERR_INVALID_ARG, what + "n_pages must be in [0, 2^31]");
  return CQSA_OK;
}

cqsa_status check_batch(const cqsa_cache* c, const cqsa_cache_batch* b, const std::string& what) {
  if (!b) return fail(CQSA_ERR_INVALID_ARG, what + "batch is NULL");
  if (b->B < 0 || b->B > (1 << 20)) return fail(CQSA_ERR_INVALID_ARG, what + "batch.B must be in [0, 2^20]");
  if (b->max_pages < 0 || b->pages_stride < b->max_pages)
    return fail(CQSA_ERR_INVALID_ARG, what + "pages_stride must be max_pages or more, and that 0 or more");
  if (b->max_len < 0 || b->max_len > int64_t(b->max_pages) * c->page_size || b->max_len > (1 << 30))
    return fail(CQSA_ERR_INVALID_ARG, what + "max_len must be in [0, max_pages * page_size], at most 2^30");
  return CQSA_OK;
}

// The batch against a tensor of rows.
cqsa_status check_rows(const cqsa_cache_batch* b, const cqsa_view& t, const std::string& what) {
  if (!b->q_start) {
    if (t.B != b->B) return fail(CQSA_ERR_INVALID_ARG, what + "the tensors' B differs from the batch's");
    return CQSA_OK;
  }
  if (t.B != 1) return fail(CQSA_ERR_INVALID_ARG, what + "packed tensors (q_start) have B = 1");
  if (t.L > 0 && (b->max_q < 1 || b->max_q > t.L))
    return fail(CQSA_ERR_INVALID_ARG, what + "max_q must be in [1, rows of the packed tensors]");
  return CQSA_OK;
}

// The device pointers of a call that has work.
cqsa_status check_pointers(const cqsa_cache* c, const cqsa_cache_batch* b, const std::string& what) {
  if (c->n_pages > 0 && !c->data) return fail(CQSA_ERR_INVALID_ARG, what + "the cache's data is NULL");
  if (reinterpret_cast<uintptr_t>(c->data) % 64 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "the cache's data must be 64-byte aligned");
  if (!b->lengths) return fail(CQSA_ERR_INVALID_ARG, what + "batch.lengths is NULL");
  if (b->max_len > 0 && !b->pages) return fail(CQSA_ERR_INVALID_ARG, what + "batch.pages is NULL");
  for (const int32_t* p : {b->pages, b->lengths, b->q_start})
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0)
      return fail(CQSA_ERR_INVALID_ARG, what + "the batch's arrays must be 4-byte aligned");
  return CQSA_OK;
}

CacheArgs args_of(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view& t) {
  CacheArgs a{};
  a.data = (char*)c->data;
  a.pages = b->pages;
  a.lengths = b->lengths;
  a.q_start = b->q_start;
  a.n_pages = c->n_pages;
  a.pages_stride = b->pages_stride;
  a.page_bytes = int64_t(cqsa_cache_page_bytes(c->page_size, c->H, c->d));
  a.page_log2 = page_log2_of(c->page_size);
  a.H = c->H;
  a.d = c->d;
  a.B = b->B;
  a.max_len = b->max_len;
  a.max_q = b->max_q;
  a.rows = int32_t(t.L);
  return a;
}

CacheTensor tensor_of(const cqsa_view& v) { return {v.data, v.stride_b, v.stride_l, v.stride_h}; }

cqsa_status move_impl(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view* K,
                      const cqsa_view* V, bool write, hipStream_t s) {
  const std::string what = write ? "cqsa_cache_write: " : "cqsa_cache_read: ";
  cqsa_status st;
  if ((st = check_cache(c, what)) != CQSA_OK) return st;
  if ((st = check_batch(c, b, what)) != CQSA_OK) return st;
  if ((st = check_view(K, "K", c->d, !write)) != CQSA_OK) return st;
  if ((st = check_view(V, "V", c->d, !write)) != CQSA_OK) return st;
  if (!same_shape(*K, *V)) return fail(CQSA_ERR_INVALID_ARG, what + "K and V differ in shape or dtype");
  if (K->H != c->H) return fail(CQSA_ERR_INVALID_ARG, what + "K's heads differ from the cache's");
  if ((st = check_rows(b, *K, what)) != CQSA_OK) return st;
  if (empty(*K) || b->B == 0) return CQSA_OK;
  if (int64_t(b->B) * c->H > (int64_t(1) << 23))
    return fail(CQSA_ERR_UNSUPPORTED, what + "more sequences and heads than one launch takes");
  if (!write && views_share(*K, *V))
    return fail(CQSA_ERR_INVALID_ARG, what + "K and V are one tensor, or share elements");
  if ((st = check_pointers(c, b, what)) != CQSA_OK) return st;
  CacheMoveArgs a{};
  a.c = args_of(c, b, *K);
  a.k = tensor_of(*K);
  a.v = tensor_of(*V);
  CQSA_HIP(write ? launch_cache_write(K->dtype, a, s) : launch_cache_read(K->dtype, a, s));
  return CQSA_OK;
}

// The launch of a call whose arguments check_attend has passed, and its workspace.
AttendPlan attend_plan(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view& Q) {
  const int64_t n = b->q_start ? b->max_q : Q.L;
  return plan_attend(b->B, c->H, n * (Q.H / c->H), b->max_len, Q.dtype, c->d);
}
uint64_t attend_bytes(const AttendPlan& p, const cqsa_view& Q) {
  if (p.splits == 1) return 0;
  return uint64_t(Q.B) * uint64_t(Q.L) * uint64_t(Q.H) * uint64_t(p.splits) * uint64_t(Q.d + 4) * 4;
}

cqsa_status check_attend(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view* Q,
                         const std::string& what) {
  cqsa_status st;
  if ((st = check_cache(c, what)) != CQSA_OK) return st;
  if ((st = check_batch(c, b, what)) != CQSA_OK) return st;
  if (!Q) return fail(CQSA_ERR_INVALID_ARG, what + "Q is NULL");
  if (Q->H < c->H || Q->H % c->H != 0 || Q->H > kMaxHeads)
    return fail(CQSA_ERR_INVALID_ARG, what + "Q's heads must be a multiple of the cache's, at most 65536");
  if ((st = check_view(Q, "Q", c->d, false)) != CQSA_OK) return st;
  if ((st = check_rows(b, *Q, what)) != CQSA_OK) return st;
  if (empty(*Q) || b->B == 0) return CQSA_OK;
  const int64_t rows = int64_t(b->q_start ? b->max_q : Q->L) * (Q->H / c->H);
  const int64_t heads = int64_t(b->B) * c->H;
  if (rows > (int64_t(1) << 30) || heads > (int64_t(1) << 23) || heads * ((rows + 15) / 16) > kMaxGroups)
    return fail(CQSA_ERR_UNSUPPORTED, what + "more rows than one launch takes");
  return CQSA_OK;
}

cqsa_status attend_impl(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view* Q,
                        const cqsa_view* O, float* LSE, int32_t causal, float scale, void* workspace,
                        uint64_t workspace_bytes, hipStream_t s) {
  const std::string what = "cqsa_cache_attend: ";
  cqsa_status st;
  if ((st = check_attend(c, b, Q, what)) != CQSA_OK) return st;
  if ((st = check_view(O, "O", c->d, true)) != CQSA_OK) return st;
  if (!same_shape(*Q, *O)) return fail(CQSA_ERR_INVALID_ARG, what + "O differs from Q in shape or dtype");
  if (causal != 0 && causal != 1) return fail(CQSA_ERR_INVALID_ARG, what + "causal must be 0 or 1");
  if (!std::isfinite(scale * kLog2e))
    return fail(CQSA_ERR_INVALID_ARG, what + "scale must be finite, in powers of two too");
  if (!empty(*Q) && !same_place(*Q, *O) && views_share(*Q, *O))
    return fail(CQSA_ERR_INVALID_ARG, what + "O overlaps Q without being Q");
  if (empty(*Q) || b->B == 0) return CQSA_OK;
  if ((st = check_pointers(c, b, what)) != CQSA_OK) return st;
  if (reinterpret_cast<uintptr_t>(LSE) % 4 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "LSE must be 4-byte aligned");
  AttendArgs a{};
  a.c = args_of(c, b, *Q);
  a.q = tensor_of(*Q);
  a.o = tensor_of(*O);
  a.lse = LSE;
  a.Hq = int32_t(Q->H);
  a.G = int32_t(Q->H / c->H);
  a.causal = causal;
  a.scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt(float(c->d))) * kLog2e;
  const AttendPlan p = attend_plan(c, b, *Q);
  const uint64_t need = attend_bytes(p, *Q);
  if ((st = check_workspace(workspace, workspace_bytes, need, what)) != CQSA_OK) return st;
  if (need > 0) {
    const int64_t parts = Q->B * Q->L * Q->H * p.splits;
    a.part = (float*)workspace;
    a.part_ml = a.part + parts * c->d;
  }
  CQSA_HIP(launch_cache_attend(Q->dtype, a, p, s));
  return CQSA_OK;
}

Range weights_range(const char* name, const cqsa_weights* w) {
  if (!w || w->B == 0 || w->H == 0 || w->T == 0) return {name, 0, 0};
  const uint64_t last = uint64_t(w->B - 1) * uint64_t(w->stride_b) + uint64_t(w->H - 1) * uint64_t(w->stride_h) +
                        uint64_t(w->T);
  return range_of(name, w->data, last * 4);
}
Range cache_range(const cqsa_cache* c) {
  return range_of("the cache", c->data, uint64_t(c->n_pages) * cqsa_cache_page_bytes(c->page_size, c->H, c->d));
}

// Shape, alignment and strides of numbers for B sequences' tokens; `written`: they must not overlap.
cqsa_status check_weights(const cqsa_weights* w, const char* name, const cqsa_cache* c, const cqsa_cache_batch* b,
                          int64_t tokens, bool written, const std::string& what) {
  auto bad = [&](const std::string& text) { return fail(CQSA_ERR_INVALID_ARG, what + name + text); };
  if (!w) return bad(" is NULL");
  if (w->B != b->B || w->H != c->H)
    return bad("'s B and H differ from the batch's and the cache's");
  if (w->T < tokens || w->T > (int64_t(1) << 31))
    return bad(" must have T = " + std::to_string(tokens) + " or more, below 2^31");
  if (w->B == 0 || w->T == 0) return CQSA_OK;
  if (!w->data || reinterpret_cast<uintptr_t>(w->data) % 4 != 0)
    return bad(".data is NULL or not 4-byte aligned");
  struct Axis {
    int64_t n, stride;
  } ax[2] = {{w->B, w->stride_b}, {w->H, w->stride_h}};
  for (const Axis& a : ax)
    if (a.n > 1 && (a.stride < 0 || a.stride > (int64_t(1) << 40)))
      return bad("'s strides must be in [0, 2^40]");
  if (!written) return CQSA_OK;
  if (ax[0].stride < ax[1].stride) std::swap(ax[0], ax[1]);
  int64_t span = w->T;  // of the tokens, then with the axis of the smaller stride too
  for (int i = 1; i >= 0; --i) {
    if (ax[i].n == 1) continue;
    if (ax[i].stride < span) return bad(" is written and overlaps itself");
    span += ax[i].stride * (ax[i].n - 1);
  }
  return CQSA_OK;
}
bool same_weights(const cqsa_weights& x, const cqsa_weights& y) {
  return x.data == y.data && (x.B == 1 || x.stride_b == y.stride_b) && (x.H == 1 || x.stride_h == y.stride_h);
}
TokenWeights weights_of(const cqsa_weights* w) {
  return w ? TokenWeights{w->data, w->stride_b, w->stride_h} : TokenWeights{nullptr, 0, 0};
}

// The launch of a call whose arguments check_attend has passed, and its workspace.
WeighPlan weigh_plan(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view& Q) {
  const int64_t n = empty(Q) ? 0 : b->q_start ? b->max_q : Q.L;
  return plan_weigh(b->B, c->H, n * (Q.H / c->H), b->max_len, Q.dtype, c->d);
}
uint64_t weigh_bytes(const WeighPlan& p, const cqsa_cache* c, const cqsa_cache_batch* b) {
  return p.splits == 1 ? 0 : uint64_t(p.splits) * uint64_t(b->B) * uint64_t(c->H) * uint64_t(b->max_len) * 4;
}
cqsa_status check_weigh(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view* Q, const std::string& what) {
  const cqsa_status st = check_attend(c, b, Q, what);
  if (st != CQSA_OK) return st;
  // check_rows looks at max_q only where there are rows; without them the tokens' prior is still read
  if (b->q_start && b->max_q < 0) return fail(CQSA_ERR_INVALID_ARG, what + "max_q must be 0 or more");
  const int64_t heads = int64_t(b->B) * c->H, tiles = (int64_t(b->max_len) + 255) / 256;
  if (heads > (int64_t(1) << 23) || heads * tiles > kMaxGroups)
    return fail(CQSA_ERR_UNSUPPORTED, what + "more sequences, heads and tokens than one launch takes");
  return CQSA_OK;
}

Range tables_range(const char* name, const cqsa_cache_batch* b) {
  if (!b || b->B == 0) return {name, 0, 0};
  return range_of(name, b->pages, 4 * (uint64_t(b->B - 1) * uint64_t(b->pages_stride) + uint64_t(b->max_pages)));
}

cqsa_status weigh_impl(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_view* Q, const float* LSE,
                       const int32_t* counts, const cqsa_weights* prior, float decay, const cqsa_weights* W,
                       int32_t causal, float scale, void* workspace, uint64_t workspace_bytes, hipStream_t s) {
  const std::string what = "cqsa_cache_weigh: ";
  cqsa_status st;
  if ((st = check_weigh(c, b, Q, what)) != CQSA_OK) return st;
  if (causal != 0 && causal != 1) return fail(CQSA_ERR_INVALID_ARG, what + "causal must be 0 or 1");
  if (!std::isfinite(scale * kLog2e))
    return fail(CQSA_ERR_INVALID_ARG, what + "scale must be finite, in powers of two too");
  if (!(decay >= 0.f && decay <= 1.f)) return fail(CQSA_ERR_INVALID_ARG, what + "decay must be in [0, 1]");
  if ((st = check_weights(W, "W", c, b, b->max_len, true, what)) != CQSA_OK) return st;
  if (prior && (st = check_weights(prior, "prior", c, b, b->max_len, false, what)) != CQSA_OK) return st;
  if (b->B == 0 || b->max_len == 0) return CQSA_OK;
  if ((st = check_pointers(c, b, what)) != CQSA_OK) return st;
  if (reinterpret_cast<uintptr_t>(counts) % 4 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "counts must be 4-byte aligned");
  if (!empty(*Q) && (!LSE || reinterpret_cast<uintptr_t>(LSE) % 4 != 0))
    return fail(CQSA_ERR_INVALID_ARG, what + "LSE is NULL or not 4-byte aligned");
  const WeighPlan p = weigh_plan(c, b, *Q);
  const uint64_t need = weigh_bytes(p, c, b);
  if ((st = check_workspace(workspace, workspace_bytes, need, what)) != CQSA_OK) return st;
  const Range w = weights_range("W", W);
  const bool in_place = prior && same_weights(*prior, *W);
  const uint64_t four = 4 * uint64_t(b->B);
  if ((st = check_apart({w, range_of("the workspace", workspace, need)},
                        {range_of("LSE", LSE, uint64_t(Q->B) * Q->L * Q->H * 4), cache_range(c),
                         in_place ? Range{"", 0, 0} : weights_range("prior", prior), range_of("counts", counts, four),
                         range_of("the lengths", b->lengths, four), tables_range("the pages", b),
                         range_of("q_start", b->q_start, four + 4), view_range("Q", *Q)},
                        what)) != CQSA_OK)
    return st;
  WeighArgs a{};
  a.c = args_of(c, b, *Q);
  a.q = tensor_of(*Q);
  a.lse = LSE;
  a.counts = counts;
  a.prior = weights_of(decay > 0.f ? prior : nullptr);  // 0 of a NaN is none
  a.w = weights_of(W);
  a.Hq = int32_t(Q->H);
  a.G = int32_t(Q->H / c->H);
  a.causal = causal;
  a.scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt(float(c->d))) * kLog2e;
  a.decay = decay;
  a.part = (float*)workspace;
  CQSA_HIP(launch_cache_weigh(Q->dtype, a, p, s));
  return CQSA_OK;
}

// Parts of an eviction's workspace, each 16-byte aligned, by the sizes of its arguments.
struct EvictSpace {
  int64_t cap, tiles;
  EvictPlan plan;
  uint64_t n_kept, kept, counts, state, chunk_counts, stage, stage_w, bytes;
};
EvictSpace evict_space(const cqsa_cache* c, const cqsa_cache_batch* b, int32_t budget, bool in_place) {
  EvictSpace e{};
  e.cap = std::min(budget, b->max_len);
  e.tiles = (e.cap + 31) / 32;
  const uint64_t heads = uint64_t(b->B) * uint64_t(c->H);
  auto part = [&](uint64_t bytes) {
    const uint64_t at = e.bytes;
    e.bytes += (bytes + 15) / 16 * 16;
    return at;
  };
  e.n_kept = part(4 * uint64_t(b->B));
  e.kept = part(4 * heads * uint64_t(e.cap));
  e.plan = plan_evict(b->B, c->H, b->max_len);
  e.counts = part(4 * uint64_t(e.plan.counts));
  e.state = part(e.plan.chunks ? heads * 3 * sizeof(EvictBorder) : 0);
  e.chunk_counts = part(heads * uint64_t(e.plan.chunks) * sizeof(int2));
  e.stage = part(in_place ? heads * uint64_t(e.tiles) * uint64_t(tile_bytes(c->d)) : 0);
  e.stage_w = part(in_place ? 4 * heads * uint64_t(e.cap) : 0);
  return e;
}

cqsa_status check_evict(const cqsa_cache* c, const cqsa_cache_batch* b, int32_t budget, const std::string& what) {
  cqsa_status st;
  if ((st = check_cache(c, what)) != CQSA_OK) return st;
  if ((st = check_batch(c, b, what)) != CQSA_OK) return st;
  if (budget < 1) return fail(CQSA_ERR_INVALID_ARG, what + "budget must be 1 or more");
  const int64_t heads = int64_t(b->B) * c->H, tiles = (int64_t(std::min(budget, b->max_len)) + 31) / 32;
  if (heads > (int64_t(1) << 23) || heads * tiles > kMaxGroups)
    return fail(CQSA_ERR_UNSUPPORTED, what + "more sequences, heads and tokens than one launch takes");
  return CQSA_OK;
}

cqsa_status evict_impl(const cqsa_cache* c, const cqsa_cache_batch* b, const cqsa_weights* W,
                       const cqsa_evict_opts* o, const cqsa_cache_batch* to, const cqsa_weights* W_to, int32_t* kept,
                       int32_t* new_lengths, void* workspace, uint64_t workspace_bytes, hipStream_t s) {
  const std::string what = "cqsa_cache_evict: ";
  cqsa_status st;
  if (!o) return fail(CQSA_ERR_INVALID_ARG, what + "opts is NULL");
  if ((st = check_evict(c, b, o->budget, what)) != CQSA_OK) return st;
  if (o->first < 0 || o->recent < 0 || int64_t(o->first) + o->recent > o->budget)
    return fail(CQSA_ERR_INVALID_ARG, what + "first and recent must be 0 or more, and budget or less together");
  const EvictSpace e = evict_space(c, b, o->budget, !to);
  if ((st = check_weights(W, "W", c, b, b->max_len, !to, what)) != CQSA_OK) return st;
  if (W_to) {
    if (!to) return fail(CQSA_ERR_INVALID_ARG, what + "W_to must be NULL in place: W is moved");
    if ((st = check_weights(W_to, "W_to", c, b, e.cap, true, what)) != CQSA_OK) return st;
  }
  if (to) {
    if (to->B != b->B) return fail(CQSA_ERR_INVALID_ARG, what + "to.B differs from the batch's");
    if (to->max_pages < 0 || to->pages_stride < to->max_pages)
      return fail(CQSA_ERR_INVALID_ARG, what + "to.pages_stride must be to.max_pages or more, and that 0 or more");
    if (int64_t(to->max_pages) * c->page_size < e.cap)
      return fail(CQSA_ERR_INVALID_ARG, what + "to's tables must have pages for min(budget, max_len) tokens");
  }
  if (b->B == 0) return CQSA_OK;
  if ((st = check_pointers(c, b, what)) != CQSA_OK) return st;
  if (to && e.cap > 0 && (!to->pages || reinterpret_cast<uintptr_t>(to->pages) % 4 != 0))
    return fail(CQSA_ERR_INVALID_ARG, what + "to.pages is NULL or not 4-byte aligned");
  if (!new_lengths || reinterpret_cast<uintptr_t>(new_lengths) % 4 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "new_lengths is NULL or not 4-byte aligned");
  if (reinterpret_cast<uintptr_t>(kept) % 4 != 0)
    return fail(CQSA_ERR_INVALID_ARG, what + "kept must be 4-byte aligned");
  if ((st = check_workspace(workspace, workspace_bytes, e.bytes, what)) != CQSA_OK) return st;
  const uint64_t heads = uint64_t(b->B) * uint64_t(c->H), four = 4 * uint64_t(b->B);
  const Range none{"", 0, 0}, w = weights_range("W", W);
  if ((st = check_apart({range_of("kept", kept, 4 * heads * uint64_t(o->budget)),
                         range_of("new_lengths", new_lengths, four), cache_range(c),
                         range_of("the workspace", workspace, e.bytes), weights_range("W_to", W_to), to ? none : w},
                        {to ? w : none, new_lengths == b->lengths ? none : range_of("the lengths", b->lengths, four),
                         tables_range("the pages", b), tables_range("to's pages", to)},
                        what)) != CQSA_OK)
    return st;
  cqsa_view rows{};  // the call has none
  EvictArgs a{};
  a.c = args_of(c, b, rows);
  a.w = weights_of(W);
  a.w_to = weights_of(W_to);
  a.to_pages = to ? to->pages : nullptr;
  a.to_stride = to ? to->pages_stride : 0;
  a.in_place = !to;
  a.budget = o->budget;
  a.first = o->first;
  a.recent = o->recent;
  a.cap = int32_t(e.cap);
  char* const space = (char*)workspace;
  a.kept = kept ? kept : (int32_t*)(space + e.kept);
  a.kept_stride = kept ? o->budget : e.cap;
  a.pad = kept != nullptr;
  a.n_kept = (int32_t*)(space + e.n_kept);
  a.new_lengths = new_lengths;
  a.chunks = e.plan.chunks;
  a.counts = (uint32_t*)(space + e.counts);
  a.state = (EvictBorder*)(space + e.state);
  a.chunk_counts = (int2*)(space + e.chunk_counts);
  a.stage = space + e.stage;
  a.stage_w = (float*)(space + e.stage_w);
  CQSA_HIP(launch_cache_evict(a, s));
  return CQSA_OK;
}

}  // namespace

}  // namespace cqsa

using namespace cqsa;

extern "C" {

uint64_t cqsa_cache_page_bytes(int32_t page_size, int32_t H, int32_t d) {
  if (page_log2_of(page_size) == 0 || H < 1 || H > kMaxHeads || !head_dim_ok(d)) return 0;
  return uint64_t(H) * uint64_t(page_size / kCacheTile) * uint64_t(tile_bytes(d));
}

cqsa_status cqsa_cache_write(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                             const cqsa_view* K, const cqsa_view* V, void* hip_stream) {
  CQSA_ENTRY("cqsa_cache_write", move_impl(cache, batch, K, V, true, (hipStream_t)hip_stream))
}

cqsa_status cqsa_cache_read(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                            const cqsa_view* K, const cqsa_view* V, void* hip_stream) {
  CQSA_ENTRY("cqsa_cache_read", move_impl(cache, batch, K, V, false, (hipStream_t)hip_stream))
}

cqsa_status cqsa_cache_attend(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                              const cqsa_view* Q, const cqsa_view* O, float* LSE, int32_t causal,
                              float scale, void* workspace, uint64_t workspace_bytes,
                              void* hip_stream) {
  CQSA_ENTRY("cqsa_cache_attend", attend_impl(cache, batch, Q, O, LSE, causal, scale, workspace,
                                              workspace_bytes, (hipStream_t)hip_stream))
}

static cqsa_status workspace_impl(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                                  const cqsa_view* Q, uint64_t* bytes) {
  const std::string what = "cqsa_cache_attend_workspace: ";
  if (!bytes) return fail(CQSA_ERR_INVALID_ARG, what + "bytes is NULL");
  *bytes = 0;
  const cqsa_status st = check_attend(cache, batch, Q, what);
  if (st != CQSA_OK || empty(*Q) || batch->B == 0) return st;
  *bytes = attend_bytes(attend_plan(cache, batch, *Q), *Q);
  return CQSA_OK;
}

cqsa_status cqsa_cache_attend_workspace(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                                        const cqsa_view* Q, uint64_t* bytes) {
  CQSA_ENTRY("cqsa_cache_attend_workspace", workspace_impl(cache, batch, Q, bytes))
}

static cqsa_status launch_impl(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                               const cqsa_view* Q, cqsa_attend_launch* out) {
  const std::string what = "cqsa_cache_attend_launch: ";
  if (!out) return fail(CQSA_ERR_INVALID_ARG, what + "out is NULL");
  *out = cqsa_attend_launch{};
  const cqsa_status st = check_attend(cache, batch, Q, what);
  if (st != CQSA_OK || empty(*Q) || batch->B == 0) return st;
  const AttendPlan p = attend_plan(cache, batch, *Q);
  const bool many = p.row_groups == 0;
  const int rows = many ? attend_many_rows(Q->dtype == CQSA_F16, cache->d) : 16 * p.row_groups;
  *out = {many, rows, many ? rows / 32 : p.waves, p.splits};
  return CQSA_OK;
}

cqsa_status cqsa_cache_attend_launch(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                                     const cqsa_view* Q, cqsa_attend_launch* out) {
  CQSA_ENTRY("cqsa_cache_attend_launch", launch_impl(cache, batch, Q, out))
}

cqsa_status cqsa_cache_weigh(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                             const cqsa_view* Q, const float* LSE, const int32_t* counts,
                             const cqsa_weights* prior, float decay, const cqsa_weights* W,
                             int32_t causal, float scale, void* workspace, uint64_t workspace_bytes,
                             void* hip_stream) {
  CQSA_ENTRY("cqsa_cache_weigh", weigh_impl(cache, batch, Q, LSE, counts, prior, decay, W, causal, scale, workspace,
                                            workspace_bytes, (hipStream_t)hip_stream))
}

static cqsa_status weigh_workspace_impl(const cqsa_cache* cache, const cqsa_cache_batch* batch, const cqsa_view* Q,
                                        uint64_t* bytes) {
  const std::string what = "cqsa_cache_weigh_workspace: ";
  if (!bytes) return fail(CQSA_ERR_INVALID_ARG, what + "bytes is NULL");
  *bytes = 0;
  const cqsa_status st = check_weigh(cache, batch, Q, what);
  if (st != CQSA_OK || batch->B == 0 || batch->max_len == 0) return st;
  *bytes = weigh_bytes(weigh_plan(cache, batch, *Q), cache, batch);
  return CQSA_OK;
}

cqsa_status cqsa_cache_weigh_workspace(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                                       const cqsa_view* Q, uint64_t* bytes) {
  CQSA_ENTRY("cqsa_cache_weigh_workspace", weigh_workspace_impl(cache, batch, Q, bytes))
}

cqsa_status cqsa_cache_evict(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                             const cqsa_weights* W, const cqsa_evict_opts* opts,
                             const cqsa_cache_batch* to, const cqsa_weights* W_to, int32_t* kept,
                             int32_t* new_lengths, void* workspace, uint64_t workspace_bytes,
                             void* hip_stream) {
  CQSA_ENTRY("cqsa_cache_evict", evict_impl(cache, batch, W, opts, to, W_to, kept, new_lengths, workspace,
                                            workspace_bytes, (hipStream_t)hip_stream))
}

static cqsa_status evict_workspace_impl(const cqsa_cache* cache, const cqsa_cache_batch* batch, int32_t budget,
                                        int32_t in_place, uint64_t* bytes) {
  const std::string what = "cqsa_cache_evict_workspace: ";
  if (!bytes) return fail(CQSA_ERR_INVALID_ARG, what + "bytes is NULL");
  *bytes = 0;
  if (in_place != 0 && in_place != 1) return fail(CQSA_ERR_INVALID_ARG, what + "in_place must be 0 or 1");
  const cqsa_status st = check_evict(cache, batch, budget, what);
  if (st != CQSA_OK || batch->B == 0) return st;
  *bytes = evict_space(cache, batch, budget, in_place).bytes;
  return CQSA_OK;
}

cqsa_status cqsa_cache_evict_workspace(const cqsa_cache* cache, const cqsa_cache_batch* batch,
                                       int32_t budget, int32_t in_place, uint64_t* bytes) {
  CQSA_ENTRY("cqsa_cache_evict_workspace", evict_workspace_impl(cache, batch, budget, in_place, bytes))
}

}  // extern "C"
