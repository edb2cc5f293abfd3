// Device code shared by the kernels of attention over the 4-bit cache: the
// matrix operands that queries, weights and cached tokens become (internal).
//
// bf16 holds every cached value exactly, so both products are bf16 matrix
// products with fp32 sums; what has more bits than a bf16 enters them in parts
// that add up to it: queries of fp16 in 2, of fp32 in 3, which makes the scores'
// products exact; weights in 2 for fp16 and 3 for fp32, and for bf16 rows in 2
// where there are few and the cache's bytes bound the call (2 to 3 % of its
// time), else in 1, which adds to a result that is rounded to bf16 anyway about
// as much as that rounding (error of the result against 64 bits 2.3e-3 with
// one part, 1.7e-3 with two; two take 10 to 15 % more from 17 rows on); the result
// is then divided by the sum of the weights as rounded (one_part_factor).  v_mfma_scale_f32_16x16x128_f8f6f4 would take
// the keys' codes and exponents as they are and save their decoding, but it
// drops bits of products that lie some 11 binades below a sum's largest (a
// score off by 2^-13 of its largest product, measured), and queries in e4m3
// terms span more.
#pragma once

#include "cache.hpp"
#include "hip_common.hpp"

namespace cqsa {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

// Rows of dtype T: bf16 parts of a query, and of a weight with many and with few
// rows.
template <typename T>
struct RowType;
template <>
struct RowType<__bf16> {
  static constexpr int kQuery = 1, kWeight = 1, kWeightFew = 2;
};
template <>
struct RowType<_Float16> {
  static constexpr int kQuery = 2, kWeight = 2, kWeightFew = 2;
};
template <>
struct RowType<float> {
  static constexpr int kQuery = 3, kWeight = 3, kWeightFew = 3;
};

constexpr int kMaxSplits = 512;
constexpr float kLn2 = 0.69314718055994530942f;
// A tile keeps its row's shift while no score is more than this above it (in
// powers of two): the weights then stay under 2^8, far from fp32's and bf16's
// ends, and the sums lose nothing, since a rounding is relative.
constexpr float kKeptRise = 8.f;

template <typename T>
__device__ __forceinline__ void load_row8(const T* p, float* v) {
  constexpr int N = 16 / sizeof(T);
  typedef __attribute__((__vector_size__(16))) T vec;
#pragma unroll
  for (int j = 0; j < 8 / N; ++j) {
    const vec x = ((const vec*)p)[j];
#pragma unroll
    for (int i = 0; i < N; ++i) v[N * j + i] = float(x[i]);
  }
}

// Two floats rounded to a pair of bf16.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// 8 values as PARTS operands whose sum they are, up to the last one's rounding.
template <int PARTS>
__device__ __forceinline__ void split8(float* p, bf16x8* out) {
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16(p[2 * j], p[2 * j + 1]);
      if (k + 1 < PARTS) {
        p[2 * j] -= __builtin_bit_cast(float, w[j] << 16);
        p[2 * j + 1] -= __builtin_bit_cast(float, w[j] & 0xffff0000u);
      }
    }
    out[k] = __builtin_bit_cast(bf16x8, w);
  }
}

__device__ __forceinline__ uint32_t decode_pair(uint32_t code, float scale, int k) {
  const bf16x2 x = k == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0)
                   : k == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1)
                   : k == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2)
                            : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return __builtin_bit_cast(uint32_t, x);
}

// The conversion takes its scale from a float's exponent bits alone, so an
// exponent byte is only shifted there: byte k of e.
__device__ __forceinline__ float scale_of(uint32_t e, int k) {
  return __builtin_bit_cast(float, k == 3 ? e >> 1 : e << (23 - 8 * k));
}

// 8 consecutive elements of a token.
__device__ __forceinline__ bf16x8 decode8(uint32_t code, float scale) {
  u32x4 w;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = decode_pair(code, scale, k);
  return __builtin_bit_cast(bf16x8, w);
}

// Values of 4 tokens' channel pairs (a byte of codes each, and of exponents):
// the even channels' operand words in even[0..1], the odd ones' in odd[0..1].
__device__ __forceinline__ void decode_quad(uint32_t code, uint32_t exps, uint32_t* even,
                                            uint32_t* odd) {
  const uint32_t a = decode_pair(code, scale_of(exps, 0), 0), b = decode_pair(code, scale_of(exps, 1), 1);
  const uint32_t c = decode_pair(code, scale_of(exps, 2), 2), d = decode_pair(code, scale_of(exps, 3), 3);
  even[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  odd[0] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  even[1] = __builtin_amdgcn_perm(d, c, 0x05040100u);
  odd[1] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// Bit k set where byte k of a word of exponents stands for NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t e) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) m |= ((e >> (8 * k)) & 255u) == kNanExponent ? 1u << k : 0u;
  return m;
}
// The bytes whose bits are set in m as 0xff.
__device__ __forceinline__ uint32_t byte_mask(uint32_t m) {
  return ((m & 1) ? 0xffu : 0u) | ((m & 2) ? 0xff00u : 0u) | ((m & 4) ? 0xff0000u : 0u) |
         ((m & 8) ? 0xff000000u : 0u);
}

// Value of another lane 16 or 32 lanes away in both directions (a butterfly).
__device__ __forceinline__ float max_of_quarters(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_of_quarters(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ float max_of_wave(float x) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) x = fmaxf(x, __shfl_xor(x, k));
  return x;
}
__device__ __forceinline__ float sum_of_wave(float x) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) x += __shfl_xor(x, k);
  return x;
}

// What a row's unnormalised result is multiplied by where its weights enter the
// product in one part: then it goes with the sum of the weights as rounded, lp,
// but is divided by (and joined with others by) their exact sum l, which is LSE's.
// Without it weights that all round the same way, as near-uniform attention has
// them, would put the result off by up to a half step of bf16.  The second sum
// costs 1 to 4 % from d = 96 on (4096 rows over 32768 tokens, d = 128: 1002 us,
// without 976) and 7 to 9 % at d = 64 and 32.
__device__ __forceinline__ float one_part_factor(float l, float lp) { return lp == 0.f ? 1.f : l / lp; }

// Tokens that a row sees.
__device__ __forceinline__ int seen_by(const Seq& s, int causal, int token) {
  const int v = causal ? s.len - s.n + token + 1 : s.len;
  return v < 0 ? 0 : v;
}

}  // namespace cqsa
