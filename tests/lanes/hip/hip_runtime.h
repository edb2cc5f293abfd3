// The part of HIP that the attention weights' kernels use, for the CPU: a lane is a fiber, and what passes between
// the lanes of a wave is a meeting of them (lanes.cpp).  With it a kernel's own source compiles for the
// host, where every access is checked.
#pragma once
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#define __device__
#define __global__
#define __host__
#define __constant__
#define __forceinline__ inline
#define __shared__ static  // one work group runs at a time
#define __launch_bounds__(...)
#define __amdgpu_buffer_rsrc_t uint64_t

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
struct int2 { int x, y; };
struct int4 { int x, y, z, w; };
struct uint2 { unsigned x, y; };
struct float2 { float x, y; };
struct float4 { float x, y, z, w; };
extern dim3 blockIdx, threadIdx, gridDim, blockDim;
typedef int hipError_t;
typedef void* hipStream_t;
inline hipError_t hipGetLastError() { return 0; }

namespace lanes {

// What the lanes of a wave bring to a meeting.
struct Brought {
  char bytes[64][32];
  uint64_t mask;  // the lanes that came
};
const Brought& meet(const void* p, int bytes, int site);
void barrier();
int lane();
void launch(dim3 grid, dim3 block, void (*kernel)(void*), void* args);

template <typename T>
T of(const Brought& r, int l) {
  T x;
  if (r.mask >> l & 1)
    memcpy(&x, r.bytes[l], sizeof x);
  else
    memset(&x, 0x7f, sizeof x);  // a lane that sits out has no value to give
  return x;
}
template <typename T>
T from(T x, int l, int site) {
  return of<T>(meet(&x, sizeof x, site), l & 63);
}
inline uint64_t ballot(bool p, int site) {
  const char c = p;
  const Brought& r = meet(&c, 1, site);
  uint64_t m = 0;
  for (int i = 0; i < 64; ++i)
    if (r.mask >> i & 1 && r.bytes[i][0]) m |= uint64_t(1) << i;
  return m;
}
struct Pair {
  uint32_t v[2];
  uint32_t operator[](int i) const { return v[i]; }
};
// The upper half of a and the lower half of b change places.
inline Pair swap32(uint32_t a, uint32_t b, int site) {
  const uint32_t x[2] = {a, b};
  const Brought& r = meet(x, 8, site);
  const int l = lane();
  return l < 32 ? Pair{{a, of<Pair>(r, l + 32).v[0]}} : Pair{{of<Pair>(r, l - 32).v[1], b}};
}
// Matrix products, M x M with 8 elements of each operand a lane, summed in fp32.
template <int M, typename A, typename C>
C mfma(const A& a, const A& b, const C& sum, int site) {
  struct Both {
    A a, b;
  } x = {a, b};
  static_assert(sizeof x == 32, "");
  C c = sum;
  const Brought& r = meet(&x, 32, site);
  const int l = lane();
  for (int e = 0; e < int(sizeof(C) / 4); ++e) {
    const int row = M == 32 ? 8 * (e / 4) + 4 * (l / 32) + e % 4 : 4 * (l / 16) + e;
    float s = 0.f;
    for (int q = 0; q < 64 / M; ++q) {
      const A u = of<Both>(r, row + M * q).a, v = of<Both>(r, l % M + M * q).b;
      for (int i = 0; i < 8; ++i) s += float(u[i]) * float(v[i]);
    }
    c[e] += s;
  }
  return c;
}
// Two e2m1 values of byte k, times the power of two in the scale's exponent bits.
typedef __attribute__((__vector_size__(4))) __bf16 bf16x2;
inline bf16x2 fp4(uint32_t code, float scale, int k) {
  static const float level[8] = {0.f, .5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  uint32_t e;
  memcpy(&e, &scale, 4);
  e = e >> 23 & 255;
  bf16x2 r;
  for (int i = 0; i < 2; ++i) {
    const uint32_t c = code >> (8 * k + 4 * i) & 15;
    const float x = e == 255 ? NAN : ldexpf(level[c & 7], int(e) - 127);
    r[i] = (__bf16)(c & 8 ? -x : x);
  }
  return r;
}

}  // namespace lanes

inline void __syncthreads() { lanes::barrier(); }

#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...)                      \
  do {                                                                                 \
    auto call = [&]() { (kernel)(__VA_ARGS__); };                                      \
    lanes::launch(grid, block, [](void* x) { (*(decltype(call)*)x)(); }, &call);       \
  } while (0)

#define __shfl(x, l) lanes::from(x, l, __LINE__)
#define __shfl_xor(x, k) lanes::from(x, lanes::lane() ^ (k), __LINE__)
#define __shfl_up(x, k) lanes::from(x, lanes::lane() < (k) ? lanes::lane() : lanes::lane() - (k), __LINE__)
#define __builtin_amdgcn_readlane(x, l) lanes::from(x, l, __LINE__)
#define __builtin_amdgcn_readfirstlane(x) (x)
#define __builtin_amdgcn_ballot_w64(p) lanes::ballot(p, __LINE__)
#define __builtin_amdgcn_permlane32_swap(a, b, c, d) lanes::swap32(a, b, __LINE__)
#define __builtin_amdgcn_mbcnt_lo(m, n) \
  ((n) + __builtin_popcount((m) & (lanes::lane() < 32 ? (1u << lanes::lane()) - 1 : ~0u)))
#define __builtin_amdgcn_mbcnt_hi(m, n) \
  ((n) + __builtin_popcount((m) & (lanes::lane() < 32 ? 0u : (1u << (lanes::lane() - 32)) - 1)))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) lanes::mfma<32>(a, b, c, __LINE__)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) lanes::mfma<16>(a, b, c, __LINE__)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, k) lanes::fp4(code, scale, k)

// Named by headers, used by other kernels.
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) (c)
#define __builtin_amdgcn_perm(a, b, c) ((a) ^ (b) ^ (c))
#define __builtin_amdgcn_fdot2_f32_bf16(a, b, c, d) (c)
#define __builtin_amdgcn_fdot2(a, b, c, d) (c)
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) (i16x4{})
#define __builtin_amdgcn_make_buffer_rsrc(a, b, c, d) 0
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(...) ((void)0)
