// Attention over the 4-bit cache for few rows a sequence (gfx950): decoding.
//
// A key head's G query heads of a sequence's n tokens are n G rows of one matrix
// product with its keys, 16 NQ of them a work group.  The four waves of a work
// group take 32-token tiles in turn and keep a running maximum, sum and
// unnormalised result each, which are joined at the end through LDS; a long
// sequence is split over `splits` work groups, joined by a second kernel.
//
// Per tile, lane (q, c) = (lane / 16, lane % 16) holds for the keys 16 t + c
// (t = 0, 1) the blocks 4 j + q (the sums over d take them in this order), and
// for the values the channels 2 c and 2 c + 1 of every block at the tokens 16 t
// + 4 q + r, which are the tokens whose scores the first product leaves it for
// row c: the weights go from one product to the next in their registers.
#include "cache_attend.hpp"

namespace cqsa {

namespace {

constexpr int kWaves = 4;

// What a wave reads of one tile.
template <int DB>
struct Tile {
  static constexpr int NJ = (DB + 3) / 4;
  u32x4 k[NJ][2];
  uint32_t ke[NJ];
  u32x2 v[DB], ve[DB];
};

}  // namespace

template <typename T, int DB, int NQ>
__global__ void __launch_bounds__(64 * kWaves)
    cache_attend_few(const AttendArgs a, int row_tiles, int splits) {
  constexpr int D = 32 * DB, NJ = (DB + 3) / 4, QP = RowType<T>::kQuery, WP = RowType<T>::kWeight;
  constexpr int ROWS = 16 * NQ, QSTRIDE = 256 * NJ + 16;  // 16: rows on different banks
  constexpr int OSTRIDE = D + 4;
  constexpr int QBYTES = QP * ROWS * QSTRIDE, OBYTES = kWaves * 16 * OSTRIDE * 4;
  __shared__ __attribute__((aligned(16))) char lds[QBYTES > OBYTES ? QBYTES : OBYTES];
  __shared__ float stat[kWaves][ROWS][2];

  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int id = blockIdx.x;
  const int rt = id % row_tiles;
  id /= row_tiles;
  const int sp = id % splits;
  id /= splits;
  const int h = id % c.H, b = id / c.H;
  const Seq s = sequence(c, b);
  const int rows = s.n * a.G, r0 = rt * ROWS;  // at most 2^31: checked on the host
  if (r0 >= rows) return;
  const int rlast = r0 + ROWS < rows ? r0 + ROWS - 1 : rows - 1;
  const int seen_min = seen_by(s, a.causal, r0 / a.G), seen_max = seen_by(s, a.causal, rlast / a.G);
  const int tiles = (seen_max + 31) >> 5;
  const int chunk = (tiles + splits - 1) / splits;
  const int t0 = sp * chunk, t1 = t0 + chunk < tiles ? t0 + chunk : tiles;

  const int64_t tb = c.q_start ? 0 : b;
  // queries, split into operands
  for (int u = tid; u < ROWS * 16 * NJ; u += 64 * kWaves) {
    const int r = u / (16 * NJ), e = 8 * (u % (16 * NJ));
    float v[8];
    if (r0 + r < rows && e < D) {
      const int tok = (r0 + r) / a.G, g = (r0 + r) % a.G;
      load_row8<T>((const T*)a.q.p + tb * a.q.b + int64_t(s.row0 + tok) * a.q.l +
                       int64_t(h * a.G + g) * a.q.h + e, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    bf16x8 part[QP];
    split8<QP>(v, part);
#pragma unroll
    for (int k = 0; k < QP; ++k) *(bf16x8*)(lds + (k * ROWS + r) * QSTRIDE + 2 * e) = part[k];
  }
  __syncthreads();
  bf16x8 qf[NQ][NJ][4][QP];
#pragma unroll
  for (int n = 0; n < NQ; ++n)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int k = 0; k < QP; ++k)
          qf[n][j][w][k] = *(const bf16x8*)(lds + (k * ROWS + 16 * n + col) * QSTRIDE +
                                            2 * (32 * (4 * j + quarter) + 8 * w));
  int seen[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = r0 + 16 * n + col;
    seen[n] = r < rows ? seen_by(s, a.causal, r / a.G) : 0x7fffffff;
  }

  f32x4 o[NQ][DB][2];
  float m[NQ], l[NQ];  // m: the shift (0 before the first tile that is seen, with l = 0)
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int k = 0; k < DB; ++k) o[n][k][0] = o[n][k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // pages of this wave's next 64 tiles, one a lane
  auto window = [&](int t) {
    const int u = t + kWaves * lane;
    return u < t1 ? int32_t(page_of(c, b, u)) : -1;
  };
  int koff[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    // a block past d reads the last one's bytes again; its query is 0
    const int blk = 4 * j + quarter < DB ? 4 * j + quarter : DB - 1;
    koff[j] = blk * 512 + col * 16;
  }
  auto load = [&](Tile<DB>& x, int t, int32_t page) {
    const char* p = c.data + tile_at(c, page, h, t);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      x.k[j][0] = *(const u32x4*)(p + koff[j]);
      x.k[j][1] = *(const u32x4*)(p + koff[j] + 256);
      const int blk = 4 * j + quarter < DB ? 4 * j + quarter : DB - 1;
      x.ke[j] = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * blk);
    }
#pragma unroll
    for (int k = 0; k < DB; ++k) {
      x.v[k] = *(const u32x2*)(p + 16 * D + k * 512 + col * 32 + quarter * 8);
      x.ve[k] = *(const u32x2*)(p + 33 * D + quarter * 8 * DB + 8 * k);
    }
  };
  auto compute = [&](Tile<DB>& x, int t) {
    const bool mixed = 32 * t + 32 > seen_min;  // some row does not see all of the tile
    f32x4 acc[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) acc[n][0] = acc[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 kk = decode8(x.k[j][u][w], scale_of(x.ke[j], u));
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int k = QP - 1; k >= 0; --k)
              acc[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qf[n][j][w][k], acc[n][u], 0, 0, 0);
        }
    float p[NQ][8];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[n][e] = acc[n][e >> 2][e & 3] * a.scale_log2;
      if (mixed) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (32 * t + 16 * (e >> 2) + 4 * quarter + (e & 3) >= seen[n]) p[n][e] = -INFINITY;
      }
      float top = p[n][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, p[n][e]);
      if (__builtin_amdgcn_ballot_w64(top > m[n] + kKeptRise)) {
        const float mn = fmaxf(m[n], max_of_quarters(top));
        const float f = m[n] == -INFINITY ? 0.f : fast_exp2(m[n] - mn);
        m[n] = mn;
        l[n] *= f;
#pragma unroll
        for (int k = 0; k < DB; ++k) o[n][k][0] *= f, o[n][k][1] *= f;
      }
      const float shift = m[n] == -INFINITY ? 0.f : m[n];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[n][e] = fast_exp2(p[n][e] - shift);
        sum += p[n][e];
      }
      l[n] += sum;
    }
    bf16x8 w[NQ][WP];
#pragma unroll
    for (int n = 0; n < NQ; ++n) split8<WP>(p[n], w[n]);
    if (mixed) {
      // Tokens that no row of the work group sees may be any bytes: their
      // exponents become 0, so that they are finite (their weights are 0).  A
      // token that stands for NaN is taken out too, and the rows that see it
      // get their NaN here, since its weight of 0 would give the others one.
      uint32_t off[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int left = seen_max - (32 * t + 16 * u + 4 * quarter);
        off[u] = left <= 0 ? 15u : (left >= 4 ? 0u : (15u << left) & 15u);
      }
#pragma unroll
      for (int k = 0; k < DB; ++k) {
#pragma unroll
        for (int u = 0; u < 2; ++u) x.ve[k][u] &= ~byte_mask(off[u]);
        const uint32_t bad0 = nan_bytes(x.ve[k][0]), bad1 = nan_bytes(x.ve[k][1]);
        if (__builtin_amdgcn_ballot_w64((bad0 | bad1) != 0u)) {
          x.ve[k][0] &= ~byte_mask(bad0);
          x.ve[k][1] &= ~byte_mask(bad1);
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            bool hit = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t is = (e < 4 ? bad0 : bad1) >> (e & 3) & 1u;
              hit = hit || (is && 32 * t + 16 * (e >> 2) + 4 * quarter + (e & 3) < seen[n]);
            }
            if (sum_of_quarters(hit ? 1.f : 0.f) > 0.f) {
              o[n][k][0] = o[n][k][0] + NAN;
              o[n][k][1] = o[n][k][1] + NAN;
            }
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < DB; ++k) {
      u32x4 even, odd;
      uint32_t ev[2], od[2];
      decode_quad(x.v[k][0], x.ve[k][0], ev, od);
      even[0] = ev[0], even[1] = ev[1], odd[0] = od[0], odd[1] = od[1];
      decode_quad(x.v[k][1], x.ve[k][1], ev, od);
      even[2] = ev[0], even[3] = ev[1], odd[2] = od[0], odd[3] = od[1];
      const bf16x8 fe = __builtin_bit_cast(bf16x8, even), fo = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int q = WP - 1; q >= 0; --q) {
          o[n][k][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fe, w[n][q], o[n][k][0], 0, 0, 0);
          o[n][k][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fo, w[n][q], o[n][k][1], 0, 0, 0);
        }
    }
  };

  // Two tiles at a time in registers: one loads while the other is computed.
  int32_t pages = -1;
  int at = 64;  // place in the window
  auto next_page = [&](int t) {
    if (at == 64) {
      pages = window(t);
      at = 0;
    }
    return __builtin_amdgcn_readlane(pages, at++);
  };
  Tile<DB> x0, x1;
  int t = t0 + wave;
  int32_t p0 = -1, p1 = -1;
  if (t < t1) {
    p0 = next_page(t);
    if (p0 >= 0) load(x0, t, p0);
  }
  while (t < t1) {
    const int u = t + kWaves;
    if (u < t1) {
      p1 = next_page(u);
      if (p1 >= 0) load(x1, u, p1);
    }
    if (p0 >= 0) compute(x0, t);
    t = u + kWaves;
    if (t < t1) {
      p0 = next_page(t);
      if (p0 >= 0) load(x0, t, p0);
    }
    if (u < t1 && p1 >= 0) compute(x1, u);
  }

  // join the waves
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l[n] = sum_of_quarters(l[n]);
    if (quarter == 0) {
      stat[wave][16 * n + col][0] = m[n];
      stat[wave][16 * n + col][1] = l[n];
    }
  }
  __syncthreads();  // also: the queries' LDS is free
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w][16 * n + col][0]);
    const float f = m[n] == -INFINITY ? 0.f : fast_exp2(m[n] - top);
    float* dst = (float*)lds + (wave * 16 + col) * OSTRIDE + 8 * quarter;
#pragma unroll
    for (int k = 0; k < DB; ++k) {
      const f32x4 e = o[n][k][0], q = o[n][k][1];
      // m is -inf where every score was (or none was seen): NaN that came by a
      // value or a score stays
      const float g = m[n] == -INFINITY ? 1.f : f;
      *(f32x4*)(dst + 32 * k) = f32x4{e[0] * g, q[0] * g, e[1] * g, q[1] * g};
      *(f32x4*)(dst + 32 * k + 4) = f32x4{e[2] * g, q[2] * g, e[3] * g, q[3] * g};
    }
    __syncthreads();
    for (int u = tid; u < 16 * 4 * DB; u += 64 * kWaves) {
      const int rr = u / (4 * DB), ch = 8 * (u % (4 * DB)), r = r0 + 16 * n + rr;
      if (r < rows) {
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) mt = fmaxf(mt, stat[w][16 * n + rr][0]);
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float mw = stat[w][16 * n + rr][0];
          lt += stat[w][16 * n + rr][1] * (mw == -INFINITY ? 1.f : fast_exp2(mw - mt));
          const float* src = (const float*)lds + (w * 16 + rr) * OSTRIDE + ch;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] += src[e];
        }
        const int tok = r / a.G, hq = h * a.G + r % a.G;
        const int64_t flat = (tb * a.Hq + hq) * int64_t(c.rows) + s.row0 + tok;
        if (splits == 1) {
          const float inv = lt == 0.f ? 1.f : 1.f / lt;
          T* dstp = (T*)a.o.p + tb * a.o.b + int64_t(s.row0 + tok) * a.o.l + int64_t(hq) * a.o.h + ch;
          typedef __attribute__((__vector_size__(8 * sizeof(T)))) T vec;
          vec y;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = T(acc[e] * inv);
          *(vec*)dstp = y;
          if (a.lse && ch == 0) a.lse[flat] = lt == 0.f ? -INFINITY : ((mt == -INFINITY ? 0.f : mt) + __builtin_amdgcn_logf(lt)) * kLn2;
        } else {
          float* part = a.part + (flat * splits + sp) * D + ch;
          *(f32x4*)part = f32x4{acc[0], acc[1], acc[2], acc[3]};
          *(f32x4*)(part + 4) = f32x4{acc[4], acc[5], acc[6], acc[7]};
          if (ch == 0) {
            a.part_ml[2 * (flat * splits + sp)] = mt;
            a.part_ml[2 * (flat * splits + sp) + 1] = lt;
          }
        }
      }
    }
    if (n + 1 < NQ) __syncthreads();
  }
}

// Joins the splits of a row: 16 rows a work group, 16 lanes each.
template <typename T>
__global__ void __launch_bounds__(256) cache_attend_join(const AttendArgs a, int per_seq, int splits) {
  const CacheArgs& c = a.c;
  const int sub = threadIdx.x & 15;
  const int b = blockIdx.x / per_seq;
  const Seq s = sequence(c, b);
  const int64_t tb = c.q_start ? 0 : b;
  const int64_t rows = int64_t(s.n) * a.Hq;
  for (int64_t i = int64_t(blockIdx.x % per_seq) * 16 + (threadIdx.x >> 4); i < rows;
       i += int64_t(per_seq) * 16) {
    const int tok = int(i / a.Hq), hq = int(i % a.Hq);
    const int64_t flat = (tb * a.Hq + hq) * int64_t(c.rows) + s.row0 + tok;
    const float* ml = a.part_ml + 2 * flat * splits;
    float m = -INFINITY, l = 0.f;
    for (int k = 0; k < splits; ++k) m = fmaxf(m, ml[2 * k]);
    for (int k = 0; k < splits; ++k)
      l += ml[2 * k + 1] * (ml[2 * k] == -INFINITY ? 1.f : fast_exp2(ml[2 * k] - m));
    const float inv = l == 0.f ? 1.f : 1.f / l;
    T* o = (T*)a.o.p + tb * a.o.b + int64_t(s.row0 + tok) * a.o.l + int64_t(hq) * a.o.h;
    for (int ch = 4 * sub; ch < c.d; ch += 64) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < splits; ++k) {
        const float f = ml[2 * k] == -INFINITY ? 1.f : fast_exp2(ml[2 * k] - m);
        acc += *(const f32x4*)(a.part + (flat * splits + k) * c.d + ch) * f;
      }
      typedef __attribute__((__vector_size__(4 * sizeof(T)))) T vec;
      *(vec*)(o + ch) = vec{T(acc[0] * inv), T(acc[1] * inv), T(acc[2] * inv), T(acc[3] * inv)};
    }
    if (a.lse && sub == 0)
      a.lse[flat] = l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

namespace {

template <typename T, int NQ>
hipError_t launch_few(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const dim3 grid(unsigned(int64_t(a.c.B) * a.c.H * p.row_tiles * p.splits)), block(64 * kWaves);
  switch (a.c.d) {
#define CQSA_FEW(DB)                                                                             \
  case 32 * DB:                                                                                  \
    hipLaunchKernelGGL((cache_attend_few<T, DB, NQ>), grid, block, 0, s, a, p.row_tiles, p.splits); \
    break;
    CQSA_FEW(1)
    CQSA_FEW(2)
    CQSA_FEW(3)
    CQSA_FEW(4)
    CQSA_FEW(5)
    CQSA_FEW(6)
    CQSA_FEW(7)
    CQSA_FEW(8)
#undef CQSA_FEW
    default:
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_all(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  hipError_t e;
  if constexpr (sizeof(T) == 2)
    e = p.row_groups == 2 ? launch_few<T, 2>(a, p, s) : launch_few<T, 1>(a, p, s);
  else
    e = launch_few<T, 1>(a, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t rows = int64_t(a.c.q_start ? a.c.max_q : a.c.rows) * a.Hq;
  int64_t per = (rows + 15) / 16;
  const int64_t most = (int64_t(1) << 23) / a.c.B;
  if (per > most) per = most;
  hipLaunchKernelGGL((cache_attend_join<T>), dim3(unsigned(per * a.c.B)), dim3(256), 0, s, a, int(per),
                     p.splits);
  return hipGetLastError();
}

}  // namespace

AttendPlan plan_attend(int64_t B, int64_t H, int64_t rows, int64_t max_len, cqsa_dtype dt, int d) {
  AttendPlan p;
  p.row_groups = rows > 16 && dt != CQSA_F32 && d <= 128 ? 2 : 1;
  p.row_tiles = int((rows + 16 * p.row_groups - 1) / (16 * p.row_groups));
  const int64_t tiles = (max_len + 31) / 32, groups = B * H * p.row_tiles;
  int64_t s = 1;
  if (groups < 1024) s = (1024 + groups - 1) / groups;
  if (s > tiles / 8) s = tiles / 8;
  p.splits = int(s < 1 ? 1 : s);
  return p;
}

hipError_t launch_cache_attend(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  if (dt == CQSA_BF16) return launch_all<__bf16>(a, p, s);
  if (dt == CQSA_F16) return launch_all<_Float16>(a, p, s);
  return launch_all<float>(a, p, s);
}

}  // namespace cqsa
