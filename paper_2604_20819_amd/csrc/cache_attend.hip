// Attention over the 4-bit cache (gfx950): one pass over a row's tokens with the
// running maximum and sum of the softmax, all in fp32.
#include "cache.hpp"
#include "hip_common.hpp"

namespace cqsa {

// One wave per row and query head.  Lane i scores token i of 64 at a time;
// then the lanes take the channels, and walk the 64 weights.
template <typename T>
__global__ void __launch_bounds__(64) cache_attend_kernel(const AttendArgs a, int per_seq) {
  typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x;
  const int b = blockIdx.x / (per_seq * a.Hq);
  const int hq = int(blockIdx.x / per_seq) % a.Hq, h = hq / a.G;
  const Seq s = sequence(c, b);
  const int nb = c.d / 32;
  __shared__ float qs[256], ps[64];
  __shared__ int64_t at[2];
  for (int row = blockIdx.x % per_seq; row < s.n; row += per_seq) {
    const int64_t tb = c.q_start ? 0 : b, tl = int64_t(s.row0) + row;
    const T* q = (const T*)a.q.p + tb * a.q.b + tl * a.q.l + hq * a.q.h;
    T* o = (T*)a.o.p + tb * a.o.b + tl * a.o.l + hq * a.o.h;
    __syncthreads();
    for (int i = lane; i < c.d; i += 64) qs[i] = float(q[i]);
    int seen = a.causal ? s.len - s.n + row + 1 : s.len;
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < seen; t0 += 64) {
      __syncthreads();
      if (lane < 2 && t0 + 32 * lane < seen) {
        const int64_t page = page_of(c, b, (t0 >> 5) + lane);
        at[lane] = page < 0 ? -1 : tile_at(c, page, h, (t0 >> 5) + lane);
      }
      __syncthreads();
      const bool ok = t0 + lane < seen && at[lane >> 5] >= 0;
      float x = -INFINITY;
      if (ok) {
        const char* tile = c.data + at[lane >> 5];
        float dot = 0.f;
        for (int blk = 0; blk < nb; ++blk) {
          const u32x4 w = *(const u32x4*)(tile + k_code_at(c.d, lane & 31, blk, 0));
          const float sc =
              __builtin_bit_cast(float, uint32_t(uint8_t(tile[k_exp_at(c.d, lane & 31, blk)])) << 23);
          for (int j = 0; j < 4; ++j) {
            const float* qq = qs + 32 * blk + 8 * j;
            f32x2 e;
            e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], sc, 0);
            dot += qq[0] * e[0] + qq[1] * e[1];
            e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], sc, 1);
            dot += qq[2] * e[0] + qq[3] * e[1];
            e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], sc, 2);
            dot += qq[4] * e[0] + qq[5] * e[1];
            e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[j], sc, 3);
            dot += qq[6] * e[0] + qq[7] * e[1];
          }
        }
        x = dot * a.scale_log2;
      }
      float top = x;
      for (int k = 1; k < 64; k <<= 1) {
        const float y = __shfl_xor(top, k);
        top = top != top || y != y ? NAN : (y > top ? y : top);
      }
      if (top == -INFINITY) continue;  // uniform: every lane has the same maximum
      const float mn = top != top || m != m ? NAN : (top > m ? top : m);
      const float keep = m == -INFINITY ? 0.f : fast_exp2(m - mn);
      const float p = ok ? fast_exp2(x - mn) : 0.f;
      m = mn;
      ps[lane] = p;
      float sum = p;
      for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
      l = l * keep + sum;
      __syncthreads();
      for (int j = 0; j < 4; ++j) acc[j] *= keep;
      for (int t = 0; t < 64 && t0 + t < seen; ++t) {
        if (at[t >> 5] < 0) continue;
        const char* tile = c.data + at[t >> 5];
        const float w = ps[t];
        for (int j = 0; j < 4; ++j) {
          const int ch = lane + 64 * j;
          if (ch >= c.d) break;
          const int code = uint8_t(tile[v_code_at(c.d, t & 31, ch >> 5, (ch & 31) >> 1)]) >> (4 * (ch & 1));
          const uint32_t e = uint8_t(tile[v_exp_at(c.d, t & 31, ch >> 5)]);
          const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(
              code & 15, __builtin_bit_cast(float, e << 23), 0);
          acc[j] += w * v[0];
        }
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int j = 0; j < 4; ++j)
      if (lane + 64 * j < c.d) o[lane + 64 * j] = T(acc[j] * inv);
    if (a.lse && lane == 0) {
      const int64_t r = (tb * a.Hq + hq) * int64_t(c.rows) + tl;
      a.lse[r] = m == -INFINITY ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    }
  }
}

hipError_t launch_cache_attend(cqsa_dtype dt, const AttendArgs& a, hipStream_t s) {
  int64_t per = a.c.q_start ? a.c.max_q : a.c.rows;
  const int64_t most = (int64_t(1) << 25) / (int64_t(a.c.B) * a.Hq);
  if (per > most) per = most;
  if (per < 1) per = 1;
  const dim3 grid(unsigned(per * a.c.B * a.Hq)), block(64);
  if (dt == CQSA_BF16)
    hipLaunchKernelGGL((cache_attend_kernel<__bf16>), grid, block, 0, s, a, int(per));
  else if (dt == CQSA_F16)
    hipLaunchKernelGGL((cache_attend_kernel<_Float16>), grid, block, 0, s, a, int(per));
  else
    hipLaunchKernelGGL((cache_attend_kernel<float>), grid, block, 0, s, a, int(per));
  return hipGetLastError();
}

}  // namespace cqsa
