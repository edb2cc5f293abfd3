// Rotary positions with several axes (gfx950).
//
// A pair's angle at position p is p * f radians.  The plan holds f / 2 pi as a
// 64-bit fixed-point fraction F of a turn, so the integer product p * F modulo
// 2^64 is the angle modulo one turn with no rounding: positions of a million
// lose nothing, where p * f in fp32 would be off by up to 0.03 radians.  Its
// upper 32 bits, under 2^-32 turns less, split exactly into a quarter turn and a
// rest within an eighth turn, whose sine and cosine are their Taylor sums (x <= pi / 4: the first term
// left out is 2e-9 of the sine and 3e-10 of the cosine).
#include "hip_common.hpp"
#include "rotary.hpp"

namespace cqsa {

namespace {

// What a thread holds of a head: two vectors of 16 bytes.
template <typename T>
struct Pair16 {
  static constexpr int N = 16 / sizeof(T);
  typedef __attribute__((__vector_size__(16))) T vec;
  vec x[2];
  __device__ __forceinline__ void load(const T* p, const T* q) { x[0] = *(const vec*)p, x[1] = *(const vec*)q; }
  template <bool LINES>
  __device__ __forceinline__ void store(T* p, T* q) const {
    if constexpr (LINES) {
      __builtin_nontemporal_store(x[0], (vec*)p);
      __builtin_nontemporal_store(x[1], (vec*)q);
    } else {
      *(vec*)p = x[0];
      *(vec*)q = x[1];
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) f[i] = float(x[i / N][i % N]);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) x[i / N][i % N] = T(f[i]);
  }
};

// Sine and cosine of v * 2^-32 turns.
__device__ __forceinline__ void sin_cos_turns(uint32_t v, float* s, float* c) {
  const uint32_t quarter = (v + 0x20000000u) >> 30;
  const float x = float(int32_t(v - (quarter << 30))) * 1.4629180792671596e-9f;  // 2 pi 2^-32
  const float z = x * x;
  const float sn =
      x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float cs =
      1.f + z * (-.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 - z * (1.f / 3628800)))));
  const float a = (quarter & 1) ? cs : sn, b = (quarter & 1) ? sn : cs;
  *s = (quarter & 2) ? -a : a;
  *c = ((quarter + 1) & 2) ? -b : b;
}

}  // namespace

// One thread turns a chunk of N pairs, N the elements of 16 bytes, of the heads
// part, part + parts, ... of one row; the chunk's angles, some 40 instructions
// each, are computed once for all of them.  A chunk is two vectors, each beside
// its neighbours' in every load and store: N pairs across them, or N / 2 within
// each.  kRotaryBatch heads are read before the first of them is written (32768
// rows of 32 heads, bf16, d = 128: 83 us with 8, 97 with 4).  Where 8 lanes side
// by side write a line of 128 bytes at once, they write it past the caches,
// which it would only pass through (the same rows: 97 and 149 us); written in
// halves, it is better gathered there.
template <typename T, bool ADJACENT, bool LINES>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
  constexpr int BATCH = kRotaryBatch, N = Pair16<T>::N;
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n) return;
  const uint32_t u = i % a.units, part = i / a.units % a.parts;
  const int64_t row = a.row0 + i / (a.units * a.parts);
  const int64_t b = row / a.L, l = row % a.L;
  const bool turned = u < a.chunks;
  float sn[N], cs[N];
  // the first vector's elements, and the second's: of the pairs, or of the rest
  // in its two halves
  const uint32_t e0 = N * u + (turned ? 0 : a.pairs);
  const uint32_t e1 = e0 + (turned ? a.pairs : N * (a.units - a.chunks));
  if (turned) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t pair = ADJACENT ? (j < N / 2 ? e0 / 2 + j : e1 / 2 + j - N / 2) : e0 + j;
      const int64_t p = a.pos[a.tab.axis[pair] * a.rows + row];
      sin_cos_turns(uint32_t((uint64_t(p) * a.tab.turn[pair]) >> 32), &sn[j], &cs[j]);
      if (a.inverse) sn[j] = -sn[j];
    }
  }
  for (uint32_t h0 = part; h0 < a.H; h0 += BATCH * a.parts) {
    Pair16<T> v[BATCH];
    T* y[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const uint32_t hv = h0 + k * a.parts;
      if (hv < a.H) {
        const RotaryArgs::Tensor& t = a.t[hv >= a.H0];
        const int64_t h = hv - (hv >= a.H0 ? a.H0 : 0);
        const T* x = (const T*)t.x + b * t.x_b + l * t.x_l + h * t.x_h;
        y[k] = (T*)t.y + b * t.y_b + l * t.y_l + h * t.y_h;
        v[k].load(x + e0, x + e1);
      }
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (h0 + k * a.parts < a.H) {
        if (turned) {
          float x[2 * N], w[2 * N];
          v[k].get(x);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int p = ADJACENT ? 2 * j : j, q = ADJACENT ? 2 * j + 1 : j + N;
            w[p] = x[p] * cs[j] - x[q] * sn[j];
            w[q] = x[q] * cs[j] + x[p] * sn[j];
          }
          v[k].set(w);
        }
        v[k].template store<LINES>(y[k] + e0, y[k] + e1);
      }
  }
}

hipError_t launch_rotary(cqsa_dtype dt, bool adjacent, const RotaryArgs& a, hipStream_t s) {
  const dim3 grid((a.n + 255) / 256), block(256);
  const bool lines = a.chunks % 8 == 0;
#define CQSA_ROT(T)                                                             \
  if (adjacent && lines)                                                        \
    hipLaunchKernelGGL((rotary_kernel<T, true, true>), grid, block, 0, s, a);   \
  else if (adjacent)                                                            \
    hipLaunchKernelGGL((rotary_kernel<T, true, false>), grid, block, 0, s, a);  \
  else if (lines)                                                               \
    hipLaunchKernelGGL((rotary_kernel<T, false, true>), grid, block, 0, s, a);  \
  else                                                                          \
    hipLaunchKernelGGL((rotary_kernel<T, false, false>), grid, block, 0, s, a);
  if (dt == CQSA_BF16) {
    CQSA_ROT(__bf16)
  } else if (dt == CQSA_F16) {
    CQSA_ROT(_Float16)
  } else {
    CQSA_ROT(float)
  }
#undef CQSA_ROT
  return hipGetLastError();
}

}  // namespace cqsa
