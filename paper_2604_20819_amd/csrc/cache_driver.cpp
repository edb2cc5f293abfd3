// The entry points of the 4-bit cache: argument checks and launches.
#include "cache.hpp"

#include <cmath>

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
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return fail(CQSA_ERR_INVALID_ARG, what + "the workspace has " + std::to_string(workspace ? workspace_bytes : 0) +
                                            " bytes, the call needs " + std::to_string(need));
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
      return fail(CQSA_ERR_INVALID_ARG, what + "the workspace must be 16-byte aligned");
    const int64_t parts = Q->B * Q->L * Q->H * p.splits;
    a.part = (float*)workspace;
    a.part_ml = a.part + parts * c->d;
  }
  CQSA_HIP(launch_cache_attend(Q->dtype, a, p, s));
  return CQSA_OK;
}

}  // namespace

}  // namespace cqsa

using namespace cqsa;

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

}  // extern "C"
