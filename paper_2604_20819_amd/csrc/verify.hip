// Verification of drafted tokens against the target's probabilities (gfx950).
//
// A token x of the draft's q is accepted where u q(x) < p(x); the first that is not
// is replaced by one drawn from max(0, p - q), which leaves the target's
// distribution.  Of the K + 1 rows of probabilities that a sequence has only the
// one at its first refusal (or behind its last draft) is read.  The draw inverts
// the sum over the vocabulary: sums of pieces first, then the piece where the sum
// passes the drawn share again, element by element.  Everything is in 64 bits: a
// vocabulary has 10^5 borders, and 32 bits would move one of them past the drawn
// share in one draw of a hundred.
#include "hip_common.hpp"
#include "verify.hpp"

namespace cqsa {

namespace {

template <typename T>
__device__ __forceinline__ double prob(T x) {
  const float y = float(x);
  return y > 0.f && y < INFINITY ? double(y) : 0.0;
}

__device__ __forceinline__ double sum_of_wave(double x) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) x += __shfl_xor(x, k);
  return x;
}

}  // namespace

template <typename T>
__global__ void __launch_bounds__(1024) verify_rows(const VerifyArgs a) {
  constexpr int kPieces = 256;
  __shared__ int stop;
  __shared__ double piece_sum[kPieces];
  __shared__ double target;
  __shared__ int piece, token;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* p = (const T*)a.p + b * a.p_b;
  const T* q = a.q ? (const T*)a.q + b * a.q_b : nullptr;
  const int32_t* drafted = a.tokens + int64_t(b) * a.K;
  const float* u = a.u + int64_t(b) * (a.K + 1);
  int n = a.counts ? a.counts[b] : a.K;
  n = n < 0 ? 0 : (n > a.K ? a.K : n);
  if (wave == 0) {
    bool good = false;
    if (lane < n) {
      const int x = drafted[lane];
      const float r = u[lane];
      if (x >= 0 && x < a.V)
        good = double(r != r ? 0.f : r) * (q ? prob(q[lane * a.q_n + x]) : 1.0) < prob(p[lane * a.p_n + x]);
    }
    const uint64_t bad = ~__builtin_amdgcn_ballot_w64(good);
    const int k = bad ? __builtin_ctzll(bad) : 64;
    if (lane == 0) stop = k < n ? k : n;
  }
  __syncthreads();
  const int k = stop;
  p += k * a.p_n;
  if (k == n) q = nullptr;
  else if (q) q += k * a.q_n;
  const int gone = k < n && !a.q ? drafted[k] : -1;  // q without probabilities: 1 here
  const int V = a.V, len = (V + kPieces - 1) / kPieces;
  bool whole = false;  // r = p
  auto rest = [&](int t) -> double {
    const double x = prob(p[t]);
    if (whole) return x;
    const double y = q ? x - prob(q[t]) : x - (t == gone ? 1.0 : 0.0);
    return y > 0.0 ? y : 0.0;
  };
  for (int pass = 0; pass < 2; ++pass) {
    for (int i = wave; i < kPieces; i += 16) {
      const int end = (i + 1) * len < V ? (i + 1) * len : V;
      double x = 0.0;
      for (int t = i * len + lane; t < end; t += 64) x += rest(t);
      x = sum_of_wave(x);
      if (lane == 0) piece_sum[i] = x;
    }
    __syncthreads();
    if (tid == 0) {
      double all = 0.0;
      for (int i = 0; i < kPieces; ++i) all += piece_sum[i];
      const float r = u[a.K];
      const double want = double(r != r ? 0.f : r) * all;
      double before = 0.0;
      int at = -1, last = -1;
      double last_before = 0.0;
      for (int i = 0; i < kPieces; ++i) {
        if (piece_sum[i] > 0.0) last = i, last_before = before;
        const double next = before + piece_sum[i];
        if (next > want) {
          at = i;
          break;
        }
        before = next;
      }
      if (at < 0) at = last, before = last_before;
      piece = at;
      target = want - before;
    }
    __syncthreads();
    if (piece >= 0 || whole) break;
    whole = true;  // nothing beyond the draft: from the target itself
    __syncthreads();
  }
  if (wave == 0) {
    int found = -1;
    if (piece >= 0) {
      const int end = (piece + 1) * len < V ? (piece + 1) * len : V;
      double before = 0.0;
      int last = -1;
      for (int t0 = piece * len; t0 < end && found < 0; t0 += 64) {
        const int t = t0 + lane;
        const double x = t < end ? rest(t) : 0.0;
        double run = x;
#pragma unroll
        for (int j = 1; j < 64; j <<= 1) {
          const double y = __shfl_up(run, j);
          if (lane >= j) run += y;
        }
        const uint64_t some = __builtin_amdgcn_ballot_w64(x > 0.0);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(x > 0.0 && before + run > target);
        if (some) last = t0 + 63 - __builtin_clzll(some);
        if (hit) found = t0 + __builtin_ctzll(hit);
        before += __shfl(run, 63);
      }
      if (found < 0) found = last;
    }
    if (lane == 0) token = found;
  }
  __syncthreads();
  int32_t* out = a.out + int64_t(b) * (a.K + 1);
  if (tid <= a.K) out[tid] = tid < k ? drafted[tid] : tid == k ? token : -1;
  if (tid == 0) {
    a.n_out[b] = k + 1;
    if (a.new_lengths) {
      const int64_t left = int64_t(a.lengths[b]) - (n - k);
      a.new_lengths[b] = left < 0 ? 0 : int32_t(left);
    }
  }
}

hipError_t launch_verify(cqsa_dtype dt, const VerifyArgs& a, hipStream_t s) {
  const dim3 grid(unsigned(a.B)), block(1024);
  if (dt == CQSA_BF16)
    hipLaunchKernelGGL((verify_rows<__bf16>), grid, block, 0, s, a);
  else if (dt == CQSA_F16)
    hipLaunchKernelGGL((verify_rows<_Float16>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((verify_rows<float>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace cqsa
