// cqsa_draft_verify: argument checks and launch.
#include "verify.hpp"

#include "runtime.hpp"
#include "view.hpp"

namespace cqsa {

namespace {

cqsa_status check_probs(const cqsa_probs* p, const char* name, const std::string& what) {
  const std::string n = what + name;
  if (!p) return fail(CQSA_ERR_INVALID_ARG, n + " is NULL");
  if (p->dtype != CQSA_F32 && p->dtype != CQSA_F16 && p->dtype != CQSA_BF16)
    return fail(CQSA_ERR_INVALID_ARG, n + " has an unknown dtype");
  if (p->B < 0 || p->B > (1 << 20)) return fail(CQSA_ERR_INVALID_ARG, n + ".B must be in [0, 2^20]");
  if (p->V < 1 || p->V > (1 << 24)) return fail(CQSA_ERR_INVALID_ARG, n + ".V must be in [1, 2^24]");
  for (int64_t s : {p->B > 1 ? p->stride_b : 0, p->N > 1 ? p->stride_n : 0})
    if (s < 0 || s > (int64_t(1) << 42)) return fail(CQSA_ERR_INVALID_ARG, n + "'s strides must be in [0, 2^42]");
  return CQSA_OK;
}

cqsa_status check_target(const cqsa_probs* p, const std::string& what) {
  const cqsa_status st = check_probs(p, "target", what);
  if (st != CQSA_OK) return st;
  if (p->N < 2 || p->N > 65)
    return fail(CQSA_ERR_INVALID_ARG, what + "target's rows of a sequence are K + 1, K in [1, 64]");
  return CQSA_OK;
}

Range probs_range(const char* name, const cqsa_probs& p) {
  const uint64_t last = uint64_t(p.B - 1) * uint64_t(p.B > 1 ? p.stride_b : 0) +
                        uint64_t(p.N - 1) * uint64_t(p.N > 1 ? p.stride_n : 0) + uint64_t(p.V);
  return range_of(name, p.data, last * uint64_t(elem_bytes(p.dtype)));
}

cqsa_status verify_impl(const cqsa_probs* p, const cqsa_probs* q, const int32_t* tokens, const int32_t* counts,
                        const float* u, int32_t* out, int32_t* n_out, const int32_t* lengths, int32_t* new_lengths,
                        void* workspace, uint64_t workspace_bytes, hipStream_t s) {
  const std::string what = "cqsa_draft_verify: ";
  cqsa_status st;
  if ((st = check_target(p, what)) != CQSA_OK) return st;
  if (q) {
    if ((st = check_probs(q, "draft", what)) != CQSA_OK) return st;
    if (q->dtype != p->dtype || q->B != p->B || q->V != p->V || q->N != p->N - 1)
      return fail(CQSA_ERR_INVALID_ARG, what + "draft must be [B, K, V] of target's dtype");
  }
  if ((lengths == nullptr) != (new_lengths == nullptr))
    return fail(CQSA_ERR_INVALID_ARG, what + "give lengths and new_lengths, or neither");
  if (p->B == 0) return CQSA_OK;
  const uintptr_t unit = uintptr_t(elem_bytes(p->dtype));
  for (const cqsa_probs* x : {p, q})
    if (x && (!x->data || reinterpret_cast<uintptr_t>(x->data) % unit != 0))
      return fail(CQSA_ERR_INVALID_ARG, what + (x == p ? "target" : "draft") + ".data is NULL or not aligned to its elements");
  const void* const needed[] = {tokens, u, out, n_out};
  const char* const names[] = {"tokens", "u", "out", "n_out"};
  for (int i = 0; i < 4; ++i)
    if (!needed[i]) return fail(CQSA_ERR_INVALID_ARG, what + names[i] + " is NULL");
  for (const void* x : {(const void*)tokens, (const void*)counts, (const void*)u, (const void*)out, (const void*)n_out,
                        (const void*)lengths, (const void*)new_lengths})
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0)
      return fail(CQSA_ERR_INVALID_ARG, what + "the arrays must be 4-byte aligned");
  const VerifyPlan plan = plan_verify(p->B, p->V, p->dtype);
  if ((st = check_workspace(workspace, workspace_bytes, plan.bytes, what)) != CQSA_OK) return st;
  const uint64_t B = uint64_t(p->B), K = uint64_t(p->N - 1);
  const Range none{"", 0, 0};
  if ((st = check_apart({range_of("out", out, 4 * B * (K + 1)), range_of("n_out", n_out, 4 * B),
                         range_of("new_lengths", new_lengths, 4 * B), range_of("the workspace", workspace, plan.bytes)},
                        {probs_range("target", *p), q ? probs_range("draft", *q) : none, range_of("tokens", tokens, 4 * B * K),
                         range_of("counts", counts, 4 * B), range_of("u", u, 4 * B * (K + 1)),
                         lengths == new_lengths ? none : range_of("lengths", lengths, 4 * B)},
                        what)) != CQSA_OK)
    return st;
  VerifyArgs a{};
  a.p = p->data;
  a.p_b = p->stride_b;
  a.p_n = p->stride_n;
  if (q) {
    a.q = q->data;
    a.q_b = q->stride_b;
    a.q_n = q->stride_n;
  }
  a.tokens = tokens;
  a.counts = counts;
  a.u = u;
  a.out = out;
  a.n_out = n_out;
  a.lengths = lengths;
  a.new_lengths = new_lengths;
  a.B = int32_t(p->B);
  a.K = int32_t(K);
  a.V = int32_t(p->V);
  a.len = plan.len;
  a.pieces = plan.pieces;
  a.sums = (double*)workspace;
  CQSA_HIP(launch_verify(p->dtype, a, plan.split, s));
  return CQSA_OK;
}

cqsa_status workspace_impl(const cqsa_probs* p, uint64_t* bytes) {
  const std::string what = "cqsa_draft_verify_workspace: ";
  if (!bytes) return fail(CQSA_ERR_INVALID_ARG, what + "bytes is NULL");
  *bytes = 0;
  const cqsa_status st = check_target(p, what);
  if (st == CQSA_OK && p->B > 0) *bytes = plan_verify(p->B, p->V, p->dtype).bytes;
  return st;
}

}  // namespace

}  // namespace cqsa

using namespace cqsa;

extern "C" {

cqsa_status cqsa_draft_verify(const cqsa_probs* target, const cqsa_probs* draft,
                              const int32_t* tokens, const int32_t* counts, const float* u,
                              int32_t* out, int32_t* n_out, const int32_t* lengths,
                              int32_t* new_lengths, void* workspace, uint64_t workspace_bytes,
                              void* hip_stream) {
  CQSA_ENTRY("cqsa_draft_verify", verify_impl(target, draft, tokens, counts, u, out, n_out, lengths, new_lengths,
                                              workspace, workspace_bytes, (hipStream_t)hip_stream))
}

cqsa_status cqsa_draft_verify_workspace(const cqsa_probs* target, uint64_t* bytes) {
  CQSA_ENTRY("cqsa_draft_verify_workspace", workspace_impl(target, bytes))
}

}  // extern "C"
