// Verification of drafted tokens against the target's probabilities (gfx950).
//
// A token x of the draft's q is accepted where u q(x) < p(x); the first that is not
// is replaced by one drawn from max(0, p - q), which leaves the target's
// distribution.  Of the K + 1 rows of probabilities that a sequence has only the
// one at its first refusal (or behind its last draft) is read, once: that bounds
// it where sequences are many (256 of 100003 tokens in fp32: 102 MB in 21 us, 4.9 TB/s),
// and two kernels of 4 us, chains of loads, where they are few (one of 32000 tokens 8 us).
//
// The draw inverts the sum over the vocabulary: a wave sums each of up to 256 pieces, and
// the piece in which the sum passes the drawn share is gone through again.
// Everything is in 64 bits: a vocabulary has 10^5 borders, and 32 bits would move
// one of them past the drawn share in one draw of a hundred.
#include "hip_common.hpp"
#include "verify.hpp"

namespace cqsa {

namespace {

constexpr int kPieces = 256;  // at most

// Elements of a load of 16 bytes.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

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

// Which drafts of sequence b are accepted; every wave finds it by itself, or takes it from
// `known` (or null).
template <typename T>
__device__ __forceinline__ Rest<T> accept(const VerifyArgs& a, int b, int lane, const int* known) {
  Rest<T> r;
  r.p = (const T*)a.p + b * a.p_b;
  r.q = a.q ? (const T*)a.q + b * a.q_b : nullptr;
  // a lane for each draft; those behind the last one are read but not used
  const int x = lane < a.K ? a.tokens[int64_t(b) * a.K + lane] : -1;
  const float u = lane < a.K ? a.u[int64_t(b) * (a.K + 1) + lane] : 0.f;
  int n = a.counts ? a.counts[b] : a.K;
  r.n = n < 0 ? 0 : (n > a.K ? a.K : n);
  if (known) {
    r.stop = *known;
  } else {
    bool good = false;
    if (lane < r.n && x >= 0 && x < a.V)
      good = double(u != u ? 0.f : u) * (r.q ? prob(r.q[lane * a.q_n + x]) : 1.0) < prob(r.p[lane * a.p_n + x]);
    const uint64_t bad = ~__builtin_amdgcn_ballot_w64(good);
    const int k = bad ? __builtin_ctzll(bad) : 64;
    r.stop = k < r.n ? k : r.n;
  }
  r.gone = r.stop < r.n && !a.q ? __builtin_amdgcn_readlane(x, r.stop) : -1;
  r.p += r.stop * a.p_n;
  r.q = r.q && r.stop < r.n ? r.q + r.stop * a.q_n : nullptr;
  return r;
}

// The largest of the words' elements as unsigned bits: a probability that is negative, NaN or
// infinite lies at the bits of infinity or above.
typedef __attribute__((__vector_size__(4))) unsigned short u16x2;
template <typename T>
struct Bits {
  u16x2 m = {0, 0};
  __device__ __forceinline__ void add(const u32x4& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = w[i];
      m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x));
    }
  }
  __device__ __forceinline__ bool strange() const {
    constexpr unsigned short top = __is_same(T, __bf16) ? 0x7f80 : 0x7c00;
    return m[0] >= top || m[1] >= top;
  }
};
template <>
struct Bits<float> {
  uint32_t m = 0;
  __device__ __forceinline__ void add(const u32x4& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = w[i] > m ? w[i] : m;
  }
  __device__ __forceinline__ bool strange() const { return m >= 0x7f800000u; }
};

// A load's elements; those behind `end` are 0.
template <typename T>
__device__ __forceinline__ u32x4 load_probs(const T* p, int t, int end) {
  constexpr int VEC = kVec<T>;
  u32x4 w = {0u, 0u, 0u, 0u};
  if (t + VEC <= end) {
    __builtin_memcpy(&w, p + t, 16);  // rows begin at any element
  } else if (t < end) {
    typedef __attribute__((__vector_size__(16))) T vec;
    vec x = __builtin_bit_cast(vec, w);
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (t + i < end) x[i] = p[t + i];
    w = __builtin_bit_cast(u32x4, x);
  }
  return w;
}

// The sum over a piece by a wave: of r = max(0, p - q), or of p.  What bounds it where a
// sequence's row has few CUs is the arithmetic, so the elements are looked at for
// strange ones by their bits, 2 (of 16 bits) an instruction, and taken as they are where
// there are none (one sequence, 131072 tokens in bf16, by a work group: 32 us with a check
// of each).
template <typename T, bool REST>
__device__ __forceinline__ double sum_piece(const VerifyArgs& a, const Rest<T>& r, int piece, int lane) {
  constexpr int VEC = kVec<T>, U = 4;
  typedef __attribute__((__vector_size__(16))) T vec;
  const int begin = piece * a.len, end = begin + a.len < a.V ? begin + a.len : a.V;
  const bool two = REST && r.q;
  double s = 0.0;
  for (int t0 = begin; t0 < end; t0 += 64 * VEC * U) {
    u32x4 x[U], y[U];
    Bits<T> bits;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = t0 + 64 * VEC * k + lane * VEC;
      x[k] = load_probs(r.p, t, end);
      y[k] = u32x4{0u, 0u, 0u, 0u};
      if (two) y[k] = load_probs(r.q, t, end);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      bits.add(x[k]);
      if (two) bits.add(y[k]);
    }
    const bool refused = REST && r.gone >= t0 && r.gone < t0 + 64 * VEC * U;
    if (refused || __builtin_amdgcn_ballot_w64(bits.strange())) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (t0 + 64 * VEC * k >= end) break;
        const vec p = __builtin_bit_cast(vec, x[k]), q = __builtin_bit_cast(vec, y[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const double x = prob(p[i]);
          s += REST ? r.at(x, prob(q[i]), t0 + 64 * VEC * k + lane * VEC + i) : x;
        }
      }
    } else if (two) {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (t0 + 64 * VEC * k >= end) break;
        const vec p = __builtin_bit_cast(vec, x[k]), q = __builtin_bit_cast(vec, y[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s += __builtin_fmax(double(float(p[i])) - double(float(q[i])), 0.0);
      }
    } else {
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (t0 + 64 * VEC * k >= end) break;
        const vec p = __builtin_bit_cast(vec, x[k]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s += double(float(p[i]));
      }
    }
  }
  return sum_of_wave(s);
}

// The token drawn, by a work group of WAVES: sums of r over the pieces in `sums` (LDS, behind a barrier).
template <typename T, int WAVES>
__device__ __forceinline__ int draw(const VerifyArgs& a, const Rest<T>& r, int b, double* sums) {
  constexpr int NT = 64 * WAVES;
  __shared__ double wave_sum[WAVES];
  __shared__ int first[WAVES], last[WAVES];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // every wave: the piece, and the share that is left within it; a lane takes up to four in a row
  const int each = (a.pieces + 63) >> 6;
  auto of_lane = [&]() {
    double s = 0.0;
    for (int i = lane * each; i < lane * each + each && i < a.pieces; ++i) s += sums[i];
    return s;
  };
  double here = of_lane();
  const bool beyond = __builtin_amdgcn_ballot_w64(here > 0.0);
  if (!beyond) {  // nothing beyond the draft: from the target itself
    __syncthreads();
    for (int i = wave; i < a.pieces; i += WAVES) {
      const double s = sum_piece<T, false>(a, r, i, lane);
      if (lane == 0) sums[i] = s;
    }
    __syncthreads();
    here = of_lane();
  }
  const double run = scan_of_wave(here, lane);
  const float u = a.u[int64_t(b) * (a.K + 1) + a.K];
  const double want = double(u != u ? 0.f : u) * __shfl(run, 63);
  const uint64_t some = __builtin_amdgcn_ballot_w64(here > 0.0);
  if (!some) return -1;
  const uint64_t past = __builtin_amdgcn_ballot_w64(here > 0.0 && run > want);
  const int from = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
  double left = want - (from ? __shfl(run, from - 1) : 0.0);
  int piece = -1;
  double before_piece = 0.0, upto_piece = 0.0;
  for (int i = from * each; i < from * each + each && i < a.pieces; ++i) {
    const double s = sums[i];
    if (s > 0.0) {
      piece = i, before_piece = upto_piece;
      if (upto_piece + s > left) break;
    }
    upto_piece += s;
  }
  left -= before_piece;
  // its elements, some in a row for each thread
  const int begin = piece * a.len, end = begin + a.len < a.V ? begin + a.len : a.V, per = (a.len + NT - 1) / NT;
  const int t0 = begin + tid * per, t1 = t0 + per < end ? t0 + per : end;
  auto element = [&](int t) {
    const double p = prob(r.p[t]);
    return beyond ? r.at(p, r.q ? prob(r.q[t]) : 0.0, t) : p;
  };
  constexpr int HELD = 8;  // elements that stay in registers in between
  double held[HELD], sum = 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) held[i] = t0 + i < t1 ? element(t0 + i) : 0.0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) sum += held[i];
  for (int t = t0 + HELD; t < t1; ++t) sum += element(t);
  const double upto = scan_of_wave(sum, lane);
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  double before = __shfl_up(upto, 1);  // by every lane: one that sits out has no value to give
  if (lane == 0) before = 0.0;
  for (int i = 0; i < wave; ++i) before += wave_sum[i];
  int hit = -1, end_of = -1;
  auto pass = [&](int t, double x) {
    before += x;
    if (x > 0.0) {
      end_of = t;
      if (hit < 0 && before > left) hit = t;
    }
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) pass(t0 + i, held[i]);
  for (int t = t0 + HELD; t < t1; ++t) pass(t, element(t));
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
  __shared__ double sums[kPieces];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rest<T> r = accept<T>(a, b, lane, nullptr);
  for (int i = wave; i < a.pieces; i += 16) {
    const double s = sum_piece<T, true>(a, r, i, lane);
    if (lane == 0) sums[i] = s;
  }
  __syncthreads();
  const int token = draw<T, 16>(a, r, b, sums);
  put(a, r, b, token);
}

// Where sequences are few: `groups` work groups for each sum the pieces, a wave each, ...
template <typename T>
__global__ void __launch_bounds__(256) verify_sums(const VerifyArgs a, int groups) {
  const int b = blockIdx.x / groups, lane = threadIdx.x & 63;
  const int piece = blockIdx.x % groups * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rest<T> r = accept<T>(a, b, lane, nullptr);
  if (piece == 0 && lane == 0) ((int*)(a.sums + int64_t(a.B) * a.pieces))[b] = r.stop;
  if (piece >= a.pieces) return;
  const double s = sum_piece<T, true>(a, r, piece, lane);
  if (lane == 0) a.sums[int64_t(b) * a.pieces + piece] = s;
}
// ... and one draws.
template <typename T>
__global__ void __launch_bounds__(256) verify_draw(const VerifyArgs a) {
  __shared__ double sums[kPieces];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  static_assert(kPieces <= 256, "a thread each");
  if (int(threadIdx.x) < a.pieces) sums[threadIdx.x] = a.sums[int64_t(b) * a.pieces + threadIdx.x];
  const Rest<T> r = accept<T>(a, b, lane, (const int*)(a.sums + int64_t(a.B) * a.pieces) + b);
  __syncthreads();
  const int token = draw<T, 4>(a, r, b, sums);
  put(a, r, b, token);
}

// Work groups of their own for the sums pay from 16 pieces on and below 128 sequences (us,
// split and whole: one of 2000 tokens in fp32 6.8 and 6.0, of 8000 6.9 and 8.2, of 131072 8.7
// and 13; 64 of 131072 18.8 and 22.2, 128 26.1 and 24.5), and four times the pieces where the
// sequences are too few to fill the GPU with them.
VerifyPlan plan_verify(int64_t B, int64_t V, cqsa_dtype dt) {
  const int64_t row = 64 * 16 / (dt == CQSA_F32 ? 4 : 2);  // a wave's load
  auto piece_len = [&](int64_t pieces) { return (V + pieces * row - 1) / (pieces * row) * row; };
  VerifyPlan p;
  const int64_t split = piece_len(B <= 16 ? 256 : 64), whole = piece_len(64);
  p.split = B < 128 && (V + split - 1) / split > 16;
  p.len = int32_t(p.split ? split : whole);
  p.pieces = int32_t((V + p.len - 1) / p.len);
  p.bytes = p.split ? uint64_t(B) * (uint64_t(p.pieces) * sizeof(double) + sizeof(int)) : 0;
  return p;
}

namespace {

template <typename T>
void launch(const VerifyArgs& a, bool split, hipStream_t s) {
  if (split) {
    const int groups = (a.pieces + 3) / 4;
    hipLaunchKernelGGL((verify_sums<T>), dim3(unsigned(groups * a.B)), dim3(256), 0, s, a, groups);
    hipLaunchKernelGGL((verify_draw<T>), dim3(unsigned(a.B)), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((verify_whole<T>), dim3(unsigned(a.B)), dim3(1024), 0, s, a);
  }
}

}  // namespace

hipError_t launch_verify(cqsa_dtype dt, const VerifyArgs& a, bool split, hipStream_t s) {
  if (dt == CQSA_BF16)
    launch<__bf16>(a, split, s);
  else if (dt == CQSA_F16)
    launch<_Float16>(a, split, s);
  else
    launch<float>(a, split, s);
  return hipGetLastError();
}

}  // namespace cqsa
