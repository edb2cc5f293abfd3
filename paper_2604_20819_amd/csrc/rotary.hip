// Rotary positions with several axes (gfx950).
//
// A pair's angle at position p is p * f radians.  The plan holds f / 2 pi as a
// 64-bit fixed-point fraction F of a turn, so the integer product p * F modulo
// 2^64 is the angle modulo one turn with no rounding: positions of a million
// lose nothing, where p * f in fp32 would be off by up to 0.03 radians.  Its
// upper 32 bits split exactly into a quarter turn and a rest within an eighth
// turn, whose sine and cosine are their Taylor sums (x <= pi / 4: the first term
// left out is 2e-9 of the sine and 3e-10 of the cosine).
#include "hip_common.hpp"
#include "rotary.hpp"

namespace cqsa {

namespace {

// Two runs of 8 elements.  A run of fp32 is two vectors, `far` elements apart,
// so that every load and store of neighbouring lanes covers whole lines.
template <typename T>
struct Vec16 {
  static constexpr int N = 16 / sizeof(T), V = 8 / N;  // of a 16-byte vector, vectors of a run
  typedef __attribute__((__vector_size__(16))) T vec;
  vec x[2 * V];
  __device__ __forceinline__ void load(const T* p, const T* q, uint32_t far) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = *(const vec*)(p + i * far), x[V + i] = *(const vec*)(q + i * far);
  }
  template <bool LINES>
  __device__ __forceinline__ void store(T* p, T* q, uint32_t far) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      vec* const a = (vec*)(p + i * far);
      vec* const b = (vec*)(q + i * far);
      if constexpr (LINES) {
        __builtin_nontemporal_store(x[i], a);
        __builtin_nontemporal_store(x[V + i], b);
      } else {
        *a = x[i];
        *b = x[V + i];
      }
    }
  }
  __device__ __forceinline__ void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = float(x[i / N][i % N]);
  }
  __device__ __forceinline__ void set(const float* f) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i / N][i % N] = T(f[i]);
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

// One thread turns a chunk of 8 pairs of the heads part, part + parts, ... of
// one row; the chunk's angles, some 300 instructions, are computed once for
// all of them.  rotary_batch heads are read before the first of them is written:
// 8 of 16 bits, 4 of 32 (32768 rows of 32 heads, bf16, d = 128: 83 us with 8, 97
// with 4; 131072 of 16, fp32, d = 64: 222 and 216).  Where 8 lanes side by side
// write a line of 128 bytes at once, they write it past the caches, which it
// would only pass through (the same rows: 97 and 149 us); written in halves, it
// is better gathered there (fp32, d = 64: 216 and 197).
template <typename T, bool ADJACENT, bool LINES>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
  constexpr int BATCH = rotary_batch(sizeof(T));
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n) return;
  const uint32_t u = i % a.units, part = i / a.units % a.parts;
  const int64_t row = a.row0 + i / (a.units * a.parts);
  const int64_t b = row / a.L, l = row % a.L;
  const bool turned = u < a.chunks;
  float sn[8], cs[8];
  // The chunk's two runs of 8 elements: 8 pairs across the runs, or 4 within each.
  constexpr uint32_t N = Vec16<T>::N;
  const uint32_t e0 = turned ? N * u : 16 * u, e1 = e0 + (turned ? a.pairs : 8);
  const uint32_t far = turned ? a.pairs / 2 : N;
  if (turned) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // of the run's elements e (and of those in the other run that are its like)
      const uint32_t k = ADJACENT ? 2 * (j % 4) : j, e = N * u + k / N * far + k % N;
      const uint32_t pair = ADJACENT ? (j / 4 * a.pairs + e) / 2 : e;
      const int64_t p = a.pos[a.tab.axis[pair] * a.rows + row];
      sin_cos_turns(uint32_t((uint64_t(p) * a.tab.turn[pair]) >> 32), &sn[j], &cs[j]);
      if (a.inverse) sn[j] = -sn[j];
    }
  }
  for (uint32_t h0 = part; h0 < a.H; h0 += BATCH * a.parts) {
    Vec16<T> v[BATCH];
    T* y[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const uint32_t hv = h0 + k * a.parts;
      if (hv < a.H) {
        const RotaryArgs::Tensor& t = a.t[hv >= a.H0];
        const int64_t h = hv - (hv >= a.H0 ? a.H0 : 0);
        const T* x = (const T*)t.x + b * t.x_b + l * t.x_l + h * t.x_h;
        y[k] = (T*)t.y + b * t.y_b + l * t.y_l + h * t.y_h;
        v[k].load(x + e0, x + e1, far);
      }
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (h0 + k * a.parts < a.H) {
        if (turned) {
          float x[16], w[16];
          v[k].get(x);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int p = ADJACENT ? 2 * j : j, q = ADJACENT ? 2 * j + 1 : j + 8;
            w[p] = x[p] * cs[j] - x[q] * sn[j];
            w[q] = x[q] * cs[j] + x[p] * sn[j];
          }
          v[k].set(w);
        }
        v[k].template store<LINES>(y[k] + e0, y[k] + e1, far);
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
