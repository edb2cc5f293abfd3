// Attention over the 4-bit cache for few rows a sequence (gfx950): decoding.
//
// A key head's G query heads of a sequence's n tokens are n G rows of one matrix
// product with its keys, 16 NQ of them a work group.  The W waves of a work group
// take 32-token tiles in turn and keep a running maximum, sum and unnormalised
// result each, which are joined at the end through LDS; a long sequence is split
// over `splits` work groups, joined by a second kernel.
//
// What bounds it: the cache's bytes where they are many (one sequence of 2^20
// tokens, 8 heads, d = 128: 1.14 GB in 207 us, 5.5 TB/s; a copy reaches 4.7),
// some 7 us of start, dependent loads and end where they are few (500 tokens 7.5
// us).  A tile of d = 128 is 300 vector instructions a wave, half of them the
// decoding: about half of the SIMDs' time in the first of these calls.
//
// Per tile, lane (q, c) = (lane / 16, lane % 16) holds keys 16 t + c (t = 0, 1):
// where d is a multiple of 128 the blocks 4 j + q, 16 bytes of codes each (the
// sums over d take their terms in this order), else 8 elements of every block,
// 4 bytes each, since a fourth of the lanes would hold no block.  Of the values
// it holds the channels 2 c and 2 c + 1 of every block at the tokens 16 t + 4 q
// + r, which are the tokens whose scores the first product leaves it for row c:
// the weights go from one product to the next in their registers.
#include "cache_attend.hpp"
#include <algorithm>

namespace cqsa {

namespace {

// Waves a SIMD is to hold (and work groups a CU): as many as the registers
// allow without spilling.  `parts` of the queries, blocks of 32 channels, groups
// of 16 rows.
constexpr int few_waves(int parts, int db, int nq) {
  if (nq == 2) return parts == 1 ? (db == 1 ? 4 : (db == 2 ? 3 : 2)) : (db <= 2 ? 3 : 2);
  if (parts == 1) return db <= 3 ? 4 : (db <= 5 ? 3 : 2);
  if (parts == 2) return db <= 2 ? 4 : (db <= 4 ? 3 : 2);
  return db <= 2 ? 4 : (db == 3 ? 3 : (db <= 6 ? 2 : 1));
}

}  // namespace

template <typename T, int DB, int NQ, int W>
__global__ void __launch_bounds__(64 * W, (few_waves(RowType<T>::kQuery, DB, NQ)))
    cache_attend_few(const AttendArgs a, int row_tiles, int splits, int min_chunk) {
  constexpr bool WIDE = DB % 4 == 0;  // whole blocks a lane
  constexpr int D = 32 * DB, QP = RowType<T>::kQuery, WP = NQ == 1 ? RowType<T>::kWeightFew : RowType<T>::kWeight;
  constexpr int ROWS = 16 * NQ, QSTRIDE = 2 * D + 16;  // 16: rows on different banks
  constexpr int OSTRIDE = D + 4;
  constexpr int QBYTES = QP * ROWS * QSTRIDE, SLOTS = W > 4 ? W / 2 : W, OBYTES = SLOTS * 16 * OSTRIDE * 4;
  __shared__ __attribute__((aligned(16))) char lds[QBYTES > OBYTES ? QBYTES : OBYTES];
  __shared__ float stat[W][ROWS][2];

  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Work groups go round the XCDs in this order: neighbours are other heads and
  // sequences, so that the splits of a sequence, the last of which may be
  // short, do not load one XCD more than another.
  int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int b = id % c.B;
  id /= c.B;
  const int rt = id % row_tiles, sp = id / row_tiles;
  const Seq s = sequence(c, b);
  const int rows = s.n * a.G, r0 = rt * ROWS;  // at most 2^31: checked on the host
  // no such rows, or, where the grid has two dimensions, behind the last work group
  if (r0 >= rows || sp >= splits) return;
  const int rlast = r0 + ROWS < rows ? r0 + ROWS - 1 : rows - 1;
  const int seen_min = seen_by(s, a.causal, r0 / a.G), seen_max = seen_by(s, a.causal, rlast / a.G);
  const int tiles = (seen_max + 31) >> 5;
  const int even = (tiles + splits - 1) / splits, chunk = even > min_chunk ? even : min_chunk;
  const int t0 = sp * chunk, t1 = t0 + chunk < tiles ? t0 + chunk : tiles;
  const int64_t tb = c.q_start ? 0 : b;
  if (splits > 1 && t0 >= t1) {  // nothing here: the join reads no more of it than this
    if (tid < ROWS && r0 + tid < rows) {
      const int r = r0 + tid;
      const int64_t flat = (tb * a.Hq + h * a.G + r % a.G) * int64_t(c.rows) + s.row0 + r / a.G;
      *(f32x2*)(a.part_ml + 2 * (flat * splits + sp)) = f32x2{-INFINITY, 0.f};
    }
    return;
  }

  // pages of this wave's next 64 tiles, one a lane
  auto window = [&](int t) {
    const int u = t + W * lane;
    return u < t1 ? int32_t(page_of(c, b, u)) : -1;
  };
  // What a wave holds of a tile: the keys are used first, so the next tile's are
  // on their way while the values are, and the other way round.
  uint32_t xk[DB][2];               // step w's 8 codes of tokens c and 16 + c
  uint32_t xke[WIDE ? DB / 4 : DB];  // and their exponents
  u32x2 xv[DB], xve[DB];
  auto load_keys = [&](int t, int32_t page) {
    const char* p = c.data + tile_at(c, page, h, t);
    if constexpr (WIDE) {
#pragma unroll
      for (int j = 0; j < DB / 4; ++j) {
        const int blk = 4 * j + quarter;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const u32x4 x = *(const u32x4*)(p + blk * 512 + (16 * u + col) * 16);
#pragma unroll
          for (int w = 0; w < 4; ++w) xk[4 * j + w][u] = x[w];
        }
        xke[j] = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * blk);
      }
    } else {
#pragma unroll
      for (int w = 0; w < DB; ++w) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          xk[w][u] = *(const uint32_t*)(p + w * 512 + (16 * u + col) * 16 + 4 * quarter);
        xke[w] = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * w);
      }
    }
  };
  auto load_values = [&](int t, int32_t page) {
    const char* p = c.data + tile_at(c, page, h, t);
#pragma unroll
    for (int k = 0; k < DB; ++k) {
      xv[k] = *(const u32x2*)(p + 16 * D + k * 512 + col * 32 + quarter * 8);
      xve[k] = *(const u32x2*)(p + 33 * D + quarter * 8 * DB + 8 * k);
    }
  };
  int32_t pages = -1;
  int at = 64;  // place in the window
  auto next_page = [&](int t) {
    if (t >= t1) return -1;
    if (at == 64) {
      pages = window(t);
      at = 0;
    }
    return __builtin_amdgcn_readlane(pages, at++);
  };
  int32_t page = next_page(t0 + wave);  // on its way while the queries come
  if (page >= 0) {
    load_keys(t0 + wave, page);
    load_values(t0 + wave, page);
  }

  // queries, split into operands
  for (int u = tid; u < ROWS * 4 * DB; u += 64 * W) {
    const int r = u / (4 * DB), e = 8 * (u % (4 * DB));
    float v[8];
    if (r0 + r < rows) {
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
  // step w of the scores' product: 8 elements of each of 4 blocks, or a block
  bf16x8 qf[NQ][DB][QP];
#pragma unroll
  for (int n = 0; n < NQ; ++n)
#pragma unroll
    for (int w = 0; w < DB; ++w)
#pragma unroll
      for (int k = 0; k < QP; ++k) {
        const int e = WIDE ? 32 * (4 * (w / 4) + quarter) + 8 * (w % 4) : 32 * w + 8 * quarter;
        qf[n][w][k] = *(const bf16x8*)(lds + (k * ROWS + 16 * n + col) * QSTRIDE + 2 * e);
      }
  int seen[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = r0 + 16 * n + col;
    seen[n] = r < rows ? seen_by(s, a.causal, r / a.G) : 0x7fffffff;
  }

  f32x4 o[NQ][DB][2];
  float m[NQ], l[NQ];  // m: the shift (0 before the first tile that is seen, with l = 0)
  float lp[NQ];        // with weights in one part: their sum as rounded
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    l[n] = lp[n] = 0.f;
#pragma unroll
    for (int k = 0; k < DB; ++k) o[n][k][0] = o[n][k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  f32x4 acc[NQ][2];
  auto score = [&]() {
#pragma unroll
    for (int n = 0; n < NQ; ++n) acc[n][0] = acc[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < DB; ++w)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 kk = decode8(xk[w][u], scale_of(xke[WIDE ? w / 4 : w], u));
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int k = QP - 1; k >= 0; --k)
            acc[n][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, qf[n][w][k], acc[n][u], 0, 0, 0);
      }
  };
  auto weigh = [&](int t) {
    const bool mixed = 32 * t + 32 > seen_min;  // some row does not see all of the tile
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
        if constexpr (WP == 1) lp[n] *= f;
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
    for (int n = 0; n < NQ; ++n) {
      split8<WP>(p[n], w[n]);
      if constexpr (WP == 1) lp[n] = sum8<BF16>(w[n][0], lp[n]);
    }
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
        for (int u = 0; u < 2; ++u) xve[k][u] &= ~byte_mask(off[u]);
        const uint32_t bad0 = nan_bytes(xve[k][0]), bad1 = nan_bytes(xve[k][1]);
        if (__builtin_amdgcn_ballot_w64((bad0 | bad1) != 0u)) {
          xve[k][0] &= ~byte_mask(bad0);
          xve[k][1] &= ~byte_mask(bad1);
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
      decode_quad(xv[k][0], xve[k][0], ev, od);
      even[0] = ev[0], even[1] = ev[1], odd[0] = od[0], odd[1] = od[1];
      decode_quad(xv[k][1], xve[k][1], ev, od);
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

  for (int t = t0 + wave; t < t1; t += W) {
    const int32_t next = next_page(t + W);
    const bool here = page >= 0;
    if (here) score();
    if (next >= 0) load_keys(t + W, next);
    if (here) weigh(t);
    if (next >= 0) load_values(t + W, next);
    page = next;
  }

  // join the waves
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    l[n] = sum_of_quarters(l[n]);
    if constexpr (WP == 1) lp[n] = sum_of_quarters(lp[n]);
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
    for (int w = 0; w < W; ++w) top = fmaxf(top, stat[w][16 * n + col][0]);
    // m is -inf where every score was (or none was seen): NaN that came by a
    // value or a score stays
    float f = m[n] == -INFINITY ? 1.f : fast_exp2(m[n] - top);
    if constexpr (WP == 1) f *= one_part_factor(l[n], lp[n]);
#pragma unroll
    for (int k = 0; k < DB; ++k) o[n][k][0] *= f, o[n][k][1] *= f;
    auto slot = [&](int w) { return (float*)lds + (w * 16 + col) * OSTRIDE + 8 * quarter; };
    auto put = [&](float* dst) {
#pragma unroll
      for (int k = 0; k < DB; ++k) {
        const f32x4 e = o[n][k][0], q = o[n][k][1];
        *(f32x4*)(dst + 32 * k) = f32x4{e[0], q[0], e[1], q[1]};
        *(f32x4*)(dst + 32 * k + 4) = f32x4{e[2], q[2], e[3], q[3]};
      }
    };
    // more than four waves: half of them add the other half's, until four or
    // three are left
    int live = W;
#pragma unroll
    while (live > 4) {
      live /= 2;
      if (wave >= live && wave < 2 * live) put(slot(wave - live));
      __syncthreads();
      if (wave < live) {
        const float* src = slot(wave);
#pragma unroll
        for (int k = 0; k < DB; ++k) {
          const f32x4 x = *(const f32x4*)(src + 32 * k), y = *(const f32x4*)(src + 32 * k + 4);
          o[n][k][0] += f32x4{x[0], x[2], y[0], y[2]};
          o[n][k][1] += f32x4{x[1], x[3], y[1], y[3]};
        }
      }
      __syncthreads();
    }
    if (wave < live) put(slot(wave));
    __syncthreads();
    for (int u = tid; u < 16 * 4 * DB; u += 64 * W) {
      const int rr = u / (4 * DB), ch = 8 * (u % (4 * DB)), r = r0 + 16 * n + rr;
      if (r < rows) {
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) mt = fmaxf(mt, stat[w][16 * n + rr][0]);
        float acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float mw = stat[w][16 * n + rr][0];
          lt += stat[w][16 * n + rr][1] * (mw == -INFINITY ? 1.f : fast_exp2(mw - mt));
        }
        for (int w = 0; w < live; ++w) {
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

// Joins the splits of a row: WPR waves a row, whose lanes share out its splits
// and channels (4 a lane), so that a row of many splits is not a chain of
// loads.
template <typename T, int WPR>
__global__ void __launch_bounds__(WPR > 4 ? 64 * WPR : 256)
    cache_attend_join(const AttendArgs a, int per_seq, int splits) {
  constexpr int W = WPR > 4 ? WPR : 4, RPG = W / WPR;  // waves and rows of a work group
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = wave % WPR;
  const int b = blockIdx.x / per_seq;
  const Seq s = sequence(c, b);
  const int64_t tb = c.q_start ? 0 : b;
  const int64_t rows = int64_t(s.n) * a.Hq;
  const int lanes = c.d / 4, ways = 64 / lanes;  // lanes of a split, splits at a time
  const int way = lane / lanes, ch = 4 * (lane % lanes);
  __shared__ float factor[W][kMaxSplits];
  __shared__ f32x4 part[W][64];
  for (int64_t i0 = int64_t(blockIdx.x % per_seq) * RPG; i0 < rows; i0 += int64_t(per_seq) * RPG) {
    const int64_t i = i0 + wave / WPR;
    const bool live = i < rows;
    const int tok = live ? int(i / a.Hq) : 0, hq = live ? int(i % a.Hq) : 0;
    const int64_t flat = (tb * a.Hq + hq) * int64_t(c.rows) + s.row0 + tok;
    const float* ml = a.part_ml + 2 * flat * splits;
    float m = -INFINITY, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      for (int k = lane; k < splits; k += 64) m = fmaxf(m, ml[2 * k]);
      m = max_of_wave(m);
      for (int k = lane; k < splits; k += 64) {
        // a split that saw nothing wrote no more than these two
        const float x = ml[2 * k], y = ml[2 * k + 1];
        const float f = x == -INFINITY ? (y == 0.f ? 0.f : 1.f) : fast_exp2(x - m);
        l += y * f;
        factor[wave][k] = y == 0.f ? 0.f : f;
      }
      __builtin_amdgcn_wave_barrier();  // other lanes' factors
      l = sum_of_wave(l);
      if (way < ways) {
#pragma unroll 4
        for (int k = sub * ways + way; k < splits; k += WPR * ways)
          if (factor[wave][k] != 0.f)
            acc += *(const f32x4*)(a.part + (flat * splits + k) * c.d + ch) * factor[wave][k];
      }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (live && sub == 0 && lane < lanes) {
      acc = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < WPR; ++w)
        for (int k = 0; k < ways; ++k) acc += part[wave + w][k * lanes + lane];
      const float inv = l == 0.f ? 1.f : 1.f / l;
      T* o = (T*)a.o.p + tb * a.o.b + int64_t(s.row0 + tok) * a.o.l + int64_t(hq) * a.o.h;
      typedef __attribute__((__vector_size__(4 * sizeof(T)))) T vec;
      *(vec*)(o + ch) = vec{T(acc[0] * inv), T(acc[1] * inv), T(acc[2] * inv), T(acc[3] * inv)};
      if (a.lse && lane == 0)
        a.lse[flat] = l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
    }
    __syncthreads();
  }
}

namespace {

template <typename T, int NQ, int DB>
void launch_waves(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const dim3 grid = attend_grid(int64_t(a.c.B) * a.c.H * p.row_tiles * p.splits);
  constexpr int W = 4 * few_waves(RowType<T>::kQuery, DB, 1);
  if constexpr (NQ == 1 && W > 4)
    if (p.waves > 4) {
      hipLaunchKernelGGL((cache_attend_few<T, DB, 1, W>), grid, dim3(64 * W), 0, s, a, p.row_tiles, p.splits,
                         p.min_chunk);
      return;
    }
  hipLaunchKernelGGL((cache_attend_few<T, DB, NQ, 4>), grid, dim3(256), 0, s, a, p.row_tiles, p.splits,
                     p.min_chunk);
}

template <typename T, int NQ>
hipError_t launch_few(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  switch (a.c.d) {
#define CQSA_FEW(DB)                                              \
  case 32 * DB:                                                   \
    if constexpr (NQ == 1 || DB <= 4) launch_waves<T, NQ, DB>(a, p, s); \
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
hipError_t launch_join(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  const int64_t rows = int64_t(a.c.q_start ? a.c.max_q : a.c.rows) * a.Hq;
  // Waves a row: 16 where a wave would go round 64 times (one key head's 8 rows
  // over 262144 tokens, d = 128, 512 splits: the call 25 us, with 4 waves 39; 16384
  // tokens, d = 64, 64 splits: 12.9 and 10.5).
  const int waves = p.splits * a.c.d >= 1 << 14 ? 16 : (p.splits > 8 ? 4 : 1);
  int64_t per = waves > 1 ? rows : (rows + 3) / 4;
  const int64_t most = (int64_t(1) << 21) / a.c.B;  // B is at most 2^20
  if (per > most) per = most;
  const dim3 grid(unsigned(per * a.c.B));
  if (waves == 16)
    hipLaunchKernelGGL((cache_attend_join<T, 16>), grid, dim3(1024), 0, s, a, int(per), p.splits);
  else if (waves == 4)
    hipLaunchKernelGGL((cache_attend_join<T, 4>), grid, dim3(256), 0, s, a, int(per), p.splits);
  else
    hipLaunchKernelGGL((cache_attend_join<T, 1>), grid, dim3(256), 0, s, a, int(per), p.splits);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_all(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  hipError_t e;
  if constexpr (sizeof(T) == 2)
    e = p.row_groups == 0   ? launch_attend_many(dt, a, p, s)
        : p.row_groups == 2 ? launch_few<T, 2>(a, p, s)
                            : launch_few<T, 1>(a, p, s);
  else
    e = launch_few<T, 1>(a, p, s);
  return e != hipSuccess || p.splits == 1 ? e : launch_join<T>(a, p, s);
}

}  // namespace

// Which kernel, and how many work groups over a sequence's tokens.  Everything
// goes by the work of a call, `units` of 16 rows by 32 tokens at the lengths'
// bound, and by how the kernels' work groups fill the GPU.
AttendPlan plan_attend(int64_t B, int64_t H, int64_t rows, int64_t max_len, cqsa_dtype dt, int d) {
  AttendPlan p;
  const int parts = dt == CQSA_F32 ? 3 : (dt == CQSA_F16 ? 2 : 1);
  int64_t tiles = (max_len + 31) / 32;
  const int64_t units = B * H * ((rows + 15) / 16) * tiles;
  // The kernel for many rows decodes a tile once for 256 rows, but walks its tiles
  // with a barrier each, so it has to fill the GPU: unsplit, or with many tiles.  us,
  // few and many, bf16, 8 key heads: 64 sequences of 128 tokens, 512 rows, d = 128, 95
  // and 42, d = 256 195 and 82; 32 of 1000, 128 rows, d = 128 34 and 30, d = 192 69
  // and 43.  With splits, one sequence: d = 32 and 64, 2^17 units (4096 tokens, 2048
  // rows) 36.7 and 33.8, 48.3 and 39.3; d = 128: 2^17 52.0 and 55.4, 53.5 and 65.7
  // (2048, 4096), 5 / 4 of it (5120, 2048) 63.1 and 63.3, 2^18 97.0 and 87.5; d = 192:
  // 2^15 (2048, 1024) 35.2 and 47.9, 2^16 68.3 and 53.6; d = 256: 2^16 68.1 and 69.9,
  // 2^18 227 and 162.
  // Unsplit, a work group that its rows fill in part takes as long as a full one, and
  // sequences too short for that to show are the fewer the narrower the heads: 64
  // sequences of 1000, 70 rows, d = 32 20.9 and 35.6, d = 64 29.1 and 39.7, d = 96 46.7
  // and 53.1, d = 128 45.9 and 55.1, d = 224 97 and 87, d = 256 85 and 106; 100 rows, d =
  // 128 58.1 and 55.8, d = 160 81 and 72; 140 rows, d = 32 30.0 and 41.3, 42.9 and 47.7,
  // 69.8 and 64.3, 69.6 and 68.9, 157 and 107; of 300, 70 rows 13.6 and 16.6, 17.6
  // and 18.5, 21.4 and 25.2, 24.7 and 26.2, 51 and 40; 128 rows 16.0 and 18.0, 21.9
  // and 20.2, 34.7 and 27.3; of 128, 100 rows 13.3 and 11.3, 16.9 and 12.7, 19.7 and
  // 17.6.  fp16, whose work groups have 128 rows at d = 224: of 1000, 140 rows 162 and
  // 226, 100 rows 131 and 137; of 300, 140 rows 84 and 98.
  // In fp16 at d = 256 and in fp32 the queries' parts leave too few registers: fp16
  // takes it only for short sequences that fill the GPU and whose rows fill its work
  // groups to 7/8 (64 sequences of 128 tokens, 4 key heads, 512 rows, 115 and 62; 64 of
  // 256, 128 rows, 40 and 32, but 80 rows 28 and 30; 32 of 512, 8 key heads, 128 rows
  // 52 and 49, 256 rows 86 and 83; 64 of 512, 100 rows 82 and 91; 32 of 1000, 128 rows
  // 75 and 84, 384 rows 173 and 181, 512 rows 211 and 201; 16 of 1000, 512 rows 136 and
  // 147, of 1024, 1024 rows 251 and 241; of 4096 823 and 963; split, 2^18, 257 and 317),
  // and for fp32 it is not built (d = 128 2^20 742 and 727, d = 256 1757 and 2450).
  const int tall = attend_many_rows(dt == CQSA_F16, d);
  const int64_t row_tiles = (rows + tall - 1) / tall;
  const bool fills = B * H * row_tiles >= 256;
  int eighths = 0;  // of the work groups' rows that there have to be, unsplit
  if (dt == CQSA_F16 && d >= 224)
    eighths = d == 256 ? 7 : 6;
  else if (d <= 64)
    eighths = max_len > 384 ? 6 : 4;
  else if (d == 96)
    eighths = 4;
  else if (max_len > 384 && (dt == CQSA_F16 || d <= 160 || d == 256))
    eighths = 3;
  if (max_len <= 128 && d < 256) eighths = 0;
  bool many = dt != CQSA_F32 && rows > 64;
  if (fills)
    many = many && 8 * rows >= eighths * tall * row_tiles;
  else
    many = many && units >= (d <= 64 ? 1 << 17 : (d <= 128 ? 5 << 15 : 1 << 16));
  if (dt == CQSA_F16 && d == 256) many = many && fills && max_len <= (rows >= 512 ? 1024 : 512);
  if (many) {
    p.row_groups = 0;
    p.row_tiles = int(row_tiles);
    // one work group a CU: the number of splits whose rounds of 256 are the
    // shortest in all, with 6 tiles' time for a round's start and end, and for a
    // join its launch's and that of its parts, 4 d bytes a row written and read;
    // more than 16 only to fill one round (one key head, 256 rows over 262144
    // tokens, bf16, d = 128: 58 us, with 16 splits 473)
    const int tokens = attend_many_tokens(d);
    tiles = (max_len + tokens - 1) / tokens;
    const int64_t groups = B * H * p.row_tiles;
    int64_t best = 0;
    p.splits = 1;
    for (int s = 1; (s <= 16 || groups * s <= 256) && (s == 1 || tiles / s >= 8); ++s) {
      int64_t cost = (groups * s + 255) / 256 * ((tiles + s - 1) / s + 6);
      if (s > 1) cost += 2 + B * H * rows * s / (128 * tokens * parts);
      if (s == 1 || cost < best) best = cost, p.splits = s;
    }
    p.min_chunk = 8;
    return p;
  }
  // Two groups of 16 rows a wave share a tile's decoding, one leaves twice the
  // work groups: 2^13 units 13.0 us with one and 13.6 with two, 2^15 27.9 and
  // 25.8, 2^18 126.4 and 97.8 (bf16, d = 128).
  p.row_groups = dt != CQSA_F32 && d <= 128 && rows > 16 && units >= 1 << 15 ? 2 : 1;
  p.row_tiles = int((rows + 16 * p.row_groups - 1) / (16 * p.row_groups));
  const int64_t groups = B * H * p.row_tiles;
  const int64_t slots = 256 * few_waves(parts, d / 32, p.row_groups);
  const int64_t once = (groups * tiles + slots - 1) / slots;  // tiles that fill the GPU once
  // One sequence: equal parts, all at once (2^20 tokens, 8 heads: 96 splits 204
  // us, 64 236, 128 253).  Several: their lengths may differ, so parts of a
  // quarter of that even them out (64 of up to 16384 tokens: 139, in one round
  // 161).  A part is no smaller than what its start, its end and the join cost:
  // 8 tiles for one sequence (1000 tokens: 9.7 us, unsplit 10.7; 4096: 10.0, with
  // 32 tiles 13.6), 16 to 24 for several (16 of up to 8192: 24 tiles 22.6, 16
  // 25.3), and 96 where the work groups without any split fill half of the GPU
  // (64 of up to 2048: unsplit 24.3, 32 tiles 27.5).
  const int64_t least = 2 * groups >= slots ? 96 : (B == 1 ? 8 : std::max<int64_t>(16, std::min<int64_t>(24, once)));
  int64_t chunk = std::max<int64_t>(least, B > 1 ? (once + 3) / 4 : once);
  if (tiles <= 16) chunk = 16;
  // Work groups that fill a CU, where one for each sequence, head and rows keeps
  // more than half of the CUs busy, or where a part would be a wave's few tiles:
  // no join (32 sequences of up to 2500 tokens 18.6 us, split 20.6, 16 of them
  // 16.9 and 16.0; 4 of up to 700 9.6 and 11.0, of 1500 12.7 and 11.2).
  const int wide = p.row_groups == 1 ? 4 * few_waves(parts, d / 32, 1) : 4;
  p.waves = 4;
  if (wide > 4 && groups <= 256 && (groups > 128 ? tiles <= 128 : (wide > 8 && tiles <= 24))) {
    p.waves = wide;
    chunk = tiles + 1;
  }
  p.splits = int(std::min<int64_t>(kMaxSplits, std::max<int64_t>(1, (tiles + chunk - 1) / chunk)));
  p.min_chunk = int(std::min<int64_t>(chunk, 1 << 30));
  return p;
}

hipError_t launch_cache_attend(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  if (dt == CQSA_BF16) return launch_all<__bf16>(dt, a, p, s);
  if (dt == CQSA_F16) return launch_all<_Float16>(dt, a, p, s);
  return launch_all<float>(dt, a, p, s);
}

}  // namespace cqsa
