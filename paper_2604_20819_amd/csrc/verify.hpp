// Verification of drafted tokens (internal).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cqsa.h"

namespace cqsa {

struct VerifyArgs {
  const void *p, *q;  // q or null
  int64_t p_b, p_n, q_b, q_n;
  const int32_t *tokens, *counts;
  const float* u;
  int32_t *out, *n_out;
  const int32_t* lengths;
  int32_t* new_lengths;
  int32_t B, K, V;
  int32_t len, pieces;  // VerifyPlan's
  double* sums;         // with split: [B, pieces], then where each sequence stops, int [B]
};

// How a call's vocabulary is divided; by its sizes alone.
struct VerifyPlan {
  bool split;           // work groups of their own sum the pieces
  int32_t len, pieces;  // elements of a piece, whole loads of a wave
  uint64_t bytes;       // of the workspace
};
VerifyPlan plan_verify(int64_t B, int64_t V, cqsa_dtype dt);

hipError_t launch_verify(cqsa_dtype dt, const VerifyArgs& a, bool split, hipStream_t s);

}  // namespace cqsa
