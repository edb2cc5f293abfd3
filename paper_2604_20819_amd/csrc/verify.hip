// Verification of drafted tokens against the target's probabilities (gfx950).
//
// A token x of the draft's q is accepted where u q(x) < p(x); the first that is not
// is replaced by one drawn from max(0, p - q), which leaves the target's
// distribution.  Of the K + 1 rows of probabilities that a sequence has only the
// one at its first refusal (or behind its last draft) is read, once: that bounds
// it where sequences are many, and some 8 us of dependent loads where they are few.
//
// The draw inverts the sum over the vocabulary: a wave sums each of 64 pieces, and
// the piece in which the sum passes the drawn share is gone through again.
// Everything is in 64 bits: a vocabulary has 10^5 borders, and 32 bits would move
// one of them past the drawn share in one draw of a hundred.
#include "hip_common.hpp"
#include "verify.hpp"

namespace cqsa {

namespace {

constexpr int kPieces = 64;

// Elements of a load of 16 bytes.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

// A piece's elements: whole loads of a wave, so that there are kPieces at most.
template <typename T>
__host__ __device__ constexpr int piece_len(int V) {
  constexpr int row = 64 * kVec<T>;
  return (V + kPieces * row - 1) / (kPieces * row) * row;
}

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
// Inclusive sums over the lanes.
__device__ __forceinline__ double scan_of_wave(double x, int lane) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const double y = __shfl_up(x, k);
    if (lane >= k) x += y;
  }
  return x;
}

// A sequence's row of probabilities that the next token is drawn from.
template <typename T>
struct Rest {
  const T *p, *q;  // q or null
  int gone;        // without q: the token that was refused, or -1
  int n, stop;     // drafted tokens, and those accepted

  __device__ __forceinline__ double at(double p, double q, int t) const {
    const double y = p - (this->q ? q : t == gone ? 1.0 : 0.0);
    return y > 0.0 ? y : 0.0;
  }
};

// Which drafts of sequence b are accepted; every wave finds it by itself.
template <typename T>
__device__ __forceinline__ Rest<T> accept(const VerifyArgs& a, int b, int lane) {
  Rest<T> r;
  r.p = (const T*)a.p + b * a.p_b;
  r.q = a.q ? (const T*)a.q + b * a.q_b : nullptr;
  const int32_t* drafted = a.tokens + int64_t(b) * a.K;
  int n = a.counts ? a.counts[b] : a.K;
  n = n < 0 ? 0 : (n > a.K ? a.K : n);
  bool good = false;
  int x = -1;
  if (lane < n) {
    x = drafted[lane];
    const float u = a.u[int64_t(b) * (a.K + 1) + lane];
    if (x >= 0 && x < a.V)
      good = double(u != u ? 0.f : u) * (r.q ? prob(r.q[lane * a.q_n + x]) : 1.0) < prob(r.p[lane * a.p_n + x]);
  }
  const uint64_t bad = ~__builtin_amdgcn_ballot_w64(good);
  const int k = bad ? __builtin_ctzll(bad) : 64;
  r.n = n;
  r.stop = k < n ? k : n;
  r.gone = r.stop < n && !a.q ? __builtin_amdgcn_readlane(x, r.stop) : -1;
  r.p += r.stop * a.p_n;
  r.q = r.q && r.stop < n ? r.q + r.stop * a.q_n : nullptr;
  return r;
}

// Sums over a piece by a wave, of r = max(0, p - q) and of p.
struct Sums {
  double rest, all;
};
template <typename T>
__device__ __forceinline__ Sums sum_piece(const Rest<T>& r, int V, int piece, int lane) {
  constexpr int VEC = kVec<T>;
  typedef __attribute__((__vector_size__(16))) T vec;
  const int len = piece_len<T>(V), begin = piece * len;
  const int end = begin + len < V ? begin + len : V;
  Sums s = {0.0, 0.0};
#pragma unroll 2
  for (int t0 = begin; t0 < end; t0 += 64 * VEC) {
    const int t = t0 + lane * VEC;
    vec x, y;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = y[i] = T(0.f);
    if (t + VEC <= end) {  // rows begin at any element
      __builtin_memcpy(&x, r.p + t, 16);
      if (r.q) __builtin_memcpy(&y, r.q + t, 16);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (t + i < end) {
          x[i] = r.p[t + i];
          if (r.q) y[i] = r.q[t + i];
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const double p = prob(x[i]);
      s.rest += r.at(p, prob(y[i]), t + i);
      s.all += p;
    }
  }
  s.rest = sum_of_wave(s.rest);
  s.all = sum_of_wave(s.all);
  return s;
}

// The token drawn, by a work group of WAVES: piece sums in `sums` (LDS, behind a barrier).
template <typename T, int WAVES>
__device__ __forceinline__ int draw(const VerifyArgs& a, const Rest<T>& r, int b, const Sums* sums) {
  constexpr int NT = 64 * WAVES;
  __shared__ double wave_sum[WAVES];
  __shared__ int first[WAVES], last[WAVES];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int V = a.V, len = piece_len<T>(V), pieces = (V + len - 1) / len;
  // every wave: the piece, and the share that is left within it
  const Sums mine = lane < pieces ? sums[lane] : Sums{0.0, 0.0};
  const bool beyond = __builtin_amdgcn_ballot_w64(mine.rest > 0.0);
  const double here = beyond ? mine.rest : mine.all;
  const double run = scan_of_wave(here, lane);
  const float u = a.u[int64_t(b) * (a.K + 1) + a.K];
  const double want = double(u != u ? 0.f : u) * __shfl(run, 63);
  const uint64_t some = __builtin_amdgcn_ballot_w64(here > 0.0);
  if (!some) return -1;
  const uint64_t past = __builtin_amdgcn_ballot_w64(here > 0.0 && run > want);
  const int piece = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
  const double left = want - (piece ? __shfl(run, piece - 1) : 0.0);
  // its elements, some in a row for each thread
  const int begin = piece * len, end = begin + len < V ? begin + len : V, per = (len + NT - 1) / NT;
  const int t0 = begin + tid * per, t1 = t0 + per < end ? t0 + per : end;
  auto element = [&](int t) {
    const double p = prob(r.p[t]);
    return beyond ? r.at(p, r.q ? prob(r.q[t]) : 0.0, t) : p;
  };
  double sum = 0.0;
  for (int t = t0; t < t1; ++t) sum += element(t);
  const double upto = scan_of_wave(sum, lane);
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  double before = __shfl_up(upto, 1);  // by every lane: one that sits out has no value to give
  if (lane == 0) before = 0.0;
  for (int i = 0; i < wave; ++i) before += wave_sum[i];
  int hit = -1, end_of = -1;
  for (int t = t0; t < t1; ++t) {
    const double x = element(t);
    before += x;
    if (x > 0.0) {
      end_of = t;
      if (hit < 0 && before > left) hit = t;
    }
  }
  const uint64_t hits = __builtin_amdgcn_ballot_w64(hit >= 0), ends = __builtin_amdgcn_ballot_w64(end_of >= 0);
  const int h = hits ? __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits)) : -1;
  const int e = ends ? __builtin_amdgcn_readlane(end_of, 63 - __builtin_clzll(ends)) : -1;
  if (lane == 0) first[wave] = h, last[wave] = e;
  __syncthreads();
  int token = -1;
  for (int i = 0; i < WAVES; ++i) {
    if (first[i] >= 0) return first[i];
    if (last[i] >= 0) token = last[i];
  }
  return token;
}

template <typename T>
__device__ __forceinline__ void put(const VerifyArgs& a, const Rest<T>& r, int b, int token) {
  const int tid = threadIdx.x, k = r.stop;
  const int32_t* drafted = a.tokens + int64_t(b) * a.K;
  int32_t* out = a.out + int64_t(b) * (a.K + 1);
  if (tid <= a.K) out[tid] = tid < k ? drafted[tid] : tid == k ? token : -1;
  if (tid == 0) {
    a.n_out[b] = k + 1;
    if (a.new_lengths) {
      const int64_t left = int64_t(a.lengths[b]) - (r.n - k);
      a.new_lengths[b] = left < 0 ? 0 : int32_t(left);
    }
  }
}

}  // namespace

// A work group for each sequence.
template <typename T>
__global__ void __launch_bounds__(1024) verify_whole(const VerifyArgs a) {
  __shared__ Sums sums[kPieces];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rest<T> r = accept<T>(a, b, lane);
  const int len = piece_len<T>(a.V);
  for (int i = wave; i < kPieces && int64_t(i) * len < a.V; i += 16) {
    const Sums s = sum_piece(r, a.V, i, lane);
    if (lane == 0) sums[i] = s;
  }
  __syncthreads();
  const int token = draw<T, 16>(a, r, b, sums);
  put(a, r, b, token);
}

// Where sequences are few: 16 work groups for each sum the pieces, a wave each, ...
template <typename T>
__global__ void __launch_bounds__(256) verify_sums(const VerifyArgs a) {
  const int b = blockIdx.x >> 4, lane = threadIdx.x & 63;
  const int piece = (blockIdx.x & 15) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rest<T> r = accept<T>(a, b, lane);
  if (int64_t(piece) * piece_len<T>(a.V) >= a.V) return;
  const Sums s = sum_piece(r, a.V, piece, lane);
  if (lane == 0) ((Sums*)a.sums)[int64_t(b) * kPieces + piece] = s;
}
// ... and one draws.
template <typename T>
__global__ void __launch_bounds__(256) verify_draw(const VerifyArgs a) {
  __shared__ Sums sums[kPieces];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int len = piece_len<T>(a.V);
  if (int(threadIdx.x) < kPieces && int64_t(threadIdx.x) * len < a.V)
    sums[threadIdx.x] = ((const Sums*)a.sums)[int64_t(b) * kPieces + threadIdx.x];
  const Rest<T> r = accept<T>(a, b, lane);
  __syncthreads();
  const int token = draw<T, 4>(a, r, b, sums);
  put(a, r, b, token);
}

bool verify_splits(int64_t B, int64_t V, cqsa_dtype dt) {
  return B < 192 && V * (dt == CQSA_F32 ? 4 : 2) > 160000;
}
uint64_t verify_bytes(int64_t B, int64_t V, cqsa_dtype dt) {
  return verify_splits(B, V, dt) ? uint64_t(B) * kPieces * sizeof(Sums) : 0;
}

namespace {

template <typename T>
void launch(const VerifyArgs& a, bool split, hipStream_t s) {
  if (split) {
    hipLaunchKernelGGL((verify_sums<T>), dim3(unsigned(16 * a.B)), dim3(256), 0, s, a);
    hipLaunchKernelGGL((verify_draw<T>), dim3(unsigned(a.B)), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((verify_whole<T>), dim3(unsigned(a.B)), dim3(1024), 0, s, a);
  }
}

}  // namespace

hipError_t launch_verify(cqsa_dtype dt, const VerifyArgs& a, hipStream_t s) {
  const bool split = verify_splits(a.B, a.V, dt);
  if (dt == CQSA_BF16)
    launch<__bf16>(a, split, s);
  else if (dt == CQSA_F16)
    launch<_Float16>(a, split, s);
  else
    launch<float>(a, split, s);
  return hipGetLastError();
}

}  // namespace cqsa
