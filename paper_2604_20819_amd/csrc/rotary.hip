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

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
  typedef __attribute__((__vector_size__(8 * sizeof(T)))) T vec;
  const vec x = *(const vec*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = float(x[i]);
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* v) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const f32x4 x = ((const f32x4*)p)[j];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * j + i] = x[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v) {
  typedef __attribute__((__vector_size__(8 * sizeof(T)))) T vec;
  vec x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = T(v[i]);
  *(vec*)p = x;
}
template <>
__device__ __forceinline__ void store8<float>(float* p, const float* v) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[4 * j + i];
    ((f32x4*)p)[j] = x;
  }
}

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
// one row; the chunk's angles are computed once for all of them.
template <typename T, bool ADJACENT>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n) return;
  const uint32_t u = i % a.units, part = i / a.units % a.parts;
  const int64_t row = a.row0 + i / (a.units * a.parts);
  const int64_t b = row / a.L, l = row % a.L;
  const bool turned = u < a.chunks;
  float sn[8], cs[8];
  // elements of the chunk's first and second eight
  const uint32_t e0 = turned && !ADJACENT ? 8 * u : 16 * u;
  const uint32_t e1 = turned && !ADJACENT ? 8 * u + a.pairs : 16 * u + 8;
  if (turned) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t p = a.pos[a.tab.axis[8 * u + j] * a.rows + row];
      sin_cos_turns(uint32_t((uint64_t(p) * a.tab.turn[8 * u + j]) >> 32), &sn[j], &cs[j]);
      if (a.inverse) sn[j] = -sn[j];
    }
  }
  for (uint32_t hv = part; hv < a.H; hv += a.parts) {
    const int k = hv >= a.H0;
    const RotaryArgs::Tensor& t = a.t[k];
    const int64_t h = hv - (k ? a.H0 : 0);
    const T* x = (const T*)t.x + b * t.x_b + l * t.x_l + h * t.x_h;
    T* y = (T*)t.y + b * t.y_b + l * t.y_l + h * t.y_h;
    float v[16], w[16];
    load8<T>(x + e0, v);
    load8<T>(x + e1, v + 8);
    if (turned) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int p = ADJACENT ? 2 * j : j, q = ADJACENT ? 2 * j + 1 : j + 8;
        w[p] = v[p] * cs[j] - v[q] * sn[j];
        w[q] = v[q] * cs[j] + v[p] * sn[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = v[j];
    }
    store8<T>(y + e0, w);
    store8<T>(y + e1, w + 8);
  }
}

hipError_t launch_rotary(cqsa_dtype dt, bool adjacent, const RotaryArgs& a, hipStream_t s) {
  const dim3 grid((a.n + 255) / 256), block(256);
#define CQSA_ROT(T)                                                             \
  if (adjacent)                                                                 \
    hipLaunchKernelGGL((rotary_kernel<T, true>), grid, block, 0, s, a);         \
  else                                                                          \
    hipLaunchKernelGGL((rotary_kernel<T, false>), grid, block, 0, s, a);
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
