// The attention weights of a call's rows, summed for each token of the 4-bit
// cache (gfx950): W[t] = decay prior[t] + sum over rows of exp(s_t - LSE).
//
// A key head's G query heads of a sequence's n tokens are n G rows of one matrix
// product with its keys; a wave holds 32 tokens' keys and goes through the rows.
// The product's columns are the tokens, so that a lane sums over the rows what it
// holds and four lanes' sums make a token's.
#include "cache_attend.hpp"
#include "cache_bound.hpp"

namespace cqsa {

namespace {
constexpr float kLog2eF = 1.4426950408889634f;
}

template <typename T, int DB>
__global__ void __launch_bounds__(256) cache_weigh_rows(const WeighArgs a, int per_seq) {
  constexpr int D = 32 * DB, QP = RowType<T>::kQuery;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int b = id % c.B, part = id / c.B;
  const Seq s = sequence(c, b);
  int count = a.counts ? a.counts[b] : s.n;
  count = count < 0 ? 0 : (count > s.n ? s.n : count);
  const int rows = count * a.G;
  const int old = s.len - s.n;  // tokens that were there before the rows
  const int64_t tb = c.q_start ? 0 : b;
  const float* prior = a.prior.p ? a.prior.p + b * a.prior.b + h * a.prior.h : nullptr;
  float* out = a.w.p + b * a.w.b + h * a.w.h;

  for (int t = part * 4 + wave; 32 * t < s.len; t += 4 * per_seq) {
    const int64_t page = page_of(c, b, t);
    float sum[2] = {0.f, 0.f};
    if (page >= 0) {
      const char* p = c.data + tile_at(c, page, h, t);
      bf16x8 kk[DB][2];
#pragma unroll
      for (int w = 0; w < DB; ++w) {
        const uint32_t e = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * w);
#pragma unroll
        for (int u = 0; u < 2; ++u)
          kk[w][u] = decode8(*(const uint32_t*)(p + w * 512 + (16 * u + col) * 16 + 4 * quarter), scale_of(e, u));
      }
      for (int r0 = 0; r0 < rows; r0 += 16) {
        const int r = r0 + col;
        const T* q = (const T*)a.q.p + tb * a.q.b + int64_t(s.row0 + r / a.G) * a.q.l +
                     int64_t(h * a.G + r % a.G) * a.q.h + 8 * quarter;
        f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int w = 0; w < DB; ++w) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = 0.f;
          if (r < rows) load_row8<T>(q + 32 * w, v);
          bf16x8 qq[QP];
          split8<QP>(v, qq);
#pragma unroll
          for (int k = QP - 1; k >= 0; --k) {
            x[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qq[k], kk[w][0], x[0], 0, 0, 0);
            x[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qq[k], kk[w][1], x[1], 0, 0, 0);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = r0 + 4 * quarter + e;
          float lse = INFINITY;
          int seen = 0;
          if (row < rows) {
            lse = a.lse[(tb * a.Hq + h * a.G + row % a.G) * int64_t(c.rows) + s.row0 + row / a.G];
            if (__builtin_fabsf(lse) < INFINITY) seen = seen_by(s, a.causal, row / a.G);
          }
          const float shift = lse * kLog2eF;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float y = fast_exp2(__builtin_fmaf(x[u][e], a.scale_log2, -shift));
            sum[u] += 32 * t + 16 * u + col < seen ? y : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float y = sum_of_quarters(sum[u]);
      const int tok = 32 * t + 16 * u + col;
      if (quarter == 0 && tok < s.len) out[tok] = prior && tok < old ? __builtin_fmaf(a.decay, prior[tok], y) : y;
    }
  }
}

namespace {

template <typename T>
hipError_t launch_rows(const WeighArgs& a, hipStream_t s) {
  const int64_t heads = int64_t(a.c.B) * a.c.H;
  int64_t per = (int64_t(a.c.max_len) + 127) / 128;
  const int64_t most = (int64_t(1) << 23) / heads;  // heads are at most 2^23
  if (per > most) per = most;
  const dim3 grid(unsigned(per * heads));
  switch (a.c.d / 32) {
#define CQSA_WEIGH(DB)                                                                              \
  case DB:                                                                                          \
    hipLaunchKernelGGL((cache_weigh_rows<T, DB>), grid, dim3(256), 0, s, a, int(per));              \
    break;
    CQSA_WEIGH(1)
    CQSA_WEIGH(2)
    CQSA_WEIGH(3)
    CQSA_WEIGH(4)
    CQSA_WEIGH(5)
    CQSA_WEIGH(6)
    CQSA_WEIGH(7)
    CQSA_WEIGH(8)
#undef CQSA_WEIGH
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_weigh(cqsa_dtype dt, const WeighArgs& a, hipStream_t s) {
  if (dt == CQSA_BF16) return launch_rows<__bf16>(a, s);
  if (dt == CQSA_F16) return launch_rows<_Float16>(a, s);
  return launch_rows<float>(a, s);
}

}  // namespace cqsa
