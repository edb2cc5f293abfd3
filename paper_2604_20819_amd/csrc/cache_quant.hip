// Writing keys and values into the 4-bit cache, and reading them back (gfx950).
//
// A block's power comes from its largest magnitude's fp32 bits by integer
// operations, (bits + 2^21) >> 23, which is the exponent or, from 1.75 times its
// power on, the next one; codes are v_cvt_scalef32_pk_fp4_f32's (to nearest
// even, ending at 6), values v_cvt_scalef32_pk_f32_fp4's, which are exact.
#include "cache.hpp"
#include "hip_common.hpp"

namespace cqsa {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

template <typename T>
__device__ __forceinline__ void load32(const T* p, float* v) {
  constexpr int N = 16 / sizeof(T);
  typedef __attribute__((__vector_size__(16))) T vec;
#pragma unroll
  for (int j = 0; j < 32 / N; ++j) {
    const vec x = ((const vec*)p)[j];
#pragma unroll
    for (int i = 0; i < N; ++i) v[N * j + i] = float(x[i]);
  }
}
template <typename T>
__device__ __forceinline__ void store32(T* p, const float* v) {
  constexpr int N = 16 / sizeof(T);
  typedef __attribute__((__vector_size__(16))) T vec;
#pragma unroll
  for (int j = 0; j < 32 / N; ++j) {
    vec x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = T(v[N * j + i]);
    ((vec*)p)[j] = x;
  }
}

// Exponent byte and 32 codes of a block.
__device__ __forceinline__ uint32_t quantise32(const float* v, u32x4* codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t m = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  if (top >= 0x7f800000u) {  // an infinity or a NaN
    *codes = u32x4{0u, 0u, 0u, 0u};
    return kNanExponent;
  }
  const uint32_t up = (top + 0x200000u) >> 23;
  const uint32_t e = up <= 2 ? 0 : (up - 2 < kMaxExponent ? up - 2 : kMaxExponent);
  const float scale = __builtin_bit_cast(float, e << 23);  // its exponent alone is used
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[8 * j + 0], v[8 * j + 1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[8 * j + 2], v[8 * j + 3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[8 * j + 4], v[8 * j + 5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[8 * j + 6], v[8 * j + 7], scale, 3);
    (*codes)[j] = w;
  }
  return e;
}

__device__ __forceinline__ void values32(const u32x4& codes, uint32_t e, float* v) {
  const float scale = __builtin_bit_cast(float, e << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[j], scale, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[j], scale, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[j], scale, 2);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[j], scale, 3);
    v[8 * j + 0] = a[0], v[8 * j + 1] = a[1], v[8 * j + 2] = b[0], v[8 * j + 3] = b[1];
    v[8 * j + 4] = c[0], v[8 * j + 5] = c[1], v[8 * j + 6] = d[0], v[8 * j + 7] = d[1];
  }
}

}  // namespace

// One thread moves one block of 32 elements of K and of V of one row and head;
// a work group takes rows of one sequence.
template <typename T, bool WRITE>
__global__ void __launch_bounds__(256) cache_move_kernel(const CacheMoveArgs a, int per_seq) {
  const CacheArgs& c = a.c;
  const int b = blockIdx.x / per_seq;
  const Seq s = sequence(c, b);
  const int nb = c.d / 32;
  const int64_t units = int64_t(s.n) * c.H * nb;
  for (int64_t i = int64_t(blockIdx.x % per_seq) * 256 + threadIdx.x; i < units;
       i += int64_t(per_seq) * 256) {
    const int blk = int(i % nb), h = int(i / nb % c.H), row = int(i / (nb * int64_t(c.H)));
    const int pos = s.len - s.n + row;
    const int64_t tb = c.q_start ? 0 : b, tl = int64_t(s.row0) + row;
    T* kp = (T*)a.k.p + tb * a.k.b + tl * a.k.l + h * a.k.h + blk * 32;
    T* vp = (T*)a.v.p + tb * a.v.b + tl * a.v.l + h * a.v.h + blk * 32;
    const int64_t page = pos < 0 ? -1 : page_of(c, b, pos >> 5);
    const int t = pos & 31;
    char* tile = c.data + (page < 0 ? 0 : tile_at(c, page, h, pos >> 5));
    float v[32];
    u32x4 codes;
    if (WRITE) {
      if (page < 0) continue;
      load32<T>(kp, v);
      uint32_t e = quantise32(v, &codes);
      *(u32x4*)(tile + k_code_at(c.d, t, blk, 0)) = codes;
      tile[k_exp_at(c.d, t, blk)] = char(e);
      load32<T>(vp, v);
      e = quantise32(v, &codes);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        tile[v_code_at(c.d, t, blk, j)] = char(codes[j / 4] >> (8 * (j % 4)));
      tile[v_exp_at(c.d, t, blk)] = char(e);
    } else {
      codes = u32x4{0u, 0u, 0u, 0u};
      uint32_t e = 0;
      if (page >= 0) {
        codes = *(const u32x4*)(tile + k_code_at(c.d, t, blk, 0));
        e = uint8_t(tile[k_exp_at(c.d, t, blk)]);
      }
      values32(codes, e, v);
      store32<T>(kp, v);
      if (page >= 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w = 0;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            w |= uint32_t(uint8_t(tile[v_code_at(c.d, t, blk, 4 * j + q)])) << (8 * q);
          codes[j] = w;
        }
        e = uint8_t(tile[v_exp_at(c.d, t, blk)]);
      }
      values32(codes, e, v);
      store32<T>(vp, v);
    }
  }
}

namespace {
template <bool WRITE>
hipError_t launch_move(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  const int64_t n = int64_t(a.c.q_start ? a.c.max_q : a.c.rows) * a.c.H * (a.c.d / 32);
  int64_t per = (n + 255) / 256;
  const int64_t most = (int64_t(1) << 23) / a.c.B;
  if (per > most) per = most;
  if (per < 1) per = 1;
  const dim3 grid(unsigned(per * a.c.B)), block(256);
  if (dt == CQSA_BF16)
    hipLaunchKernelGGL((cache_move_kernel<__bf16, WRITE>), grid, block, 0, s, a, int(per));
  else if (dt == CQSA_F16)
    hipLaunchKernelGGL((cache_move_kernel<_Float16, WRITE>), grid, block, 0, s, a, int(per));
  else
    hipLaunchKernelGGL((cache_move_kernel<float, WRITE>), grid, block, 0, s, a, int(per));
  return hipGetLastError();
}
}  // namespace

hipError_t launch_cache_write(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  return launch_move<true>(dt, a, s);
}
hipError_t launch_cache_read(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  return launch_move<false>(dt, a, s);
}

}  // namespace cqsa
