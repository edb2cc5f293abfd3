// Attention over the 4-bit cache for many rows a sequence (gfx950): chunks of
// prompts.
//
// A work group takes 32 rows a wave of one sequence's and key head's n G rows
// and walks its tokens in tiles of TK.  The tile's codes are decoded once for
// all waves, into LDS, where each operand of the two matrix products lies as
// the 64 lanes read it: 16 bytes a lane, one after the other, so that reads
// and writes are free of bank conflicts.  Two tiles lie there, one being read
// while the next is decoded, and the codes of the one after that are on their
// way into registers: one barrier a tile.
//
// Scores are S^T = K Q^T (32x32x16): a lane holds one row's scores, of half the
// keys.  The rows of K are put in such an order that the scores a lane gets
// are those of the tokens 4 q .. 4 q + 3 and 16 + 4 q .. of each 32, q = 2 s +
// lane / 32 for step s of the weights' product, which is the order in which
// the cache holds values together.
#include "cache_attend.hpp"

namespace cqsa {

namespace {

// Row of the scores' product that token t of 32 takes.
__device__ __forceinline__ int score_row(int t) {
  return 16 * ((t >> 3) & 1) + 8 * (t >> 4) + 4 * ((t >> 2) & 1) + (t & 3);
}
// Token (of 32) of accumulator register r in half `half` of the lanes.
__device__ __forceinline__ int score_token(int r, int half) {
  return 4 * (2 * (r >> 3) + half) + 16 * ((r >> 2) & 1) + (r & 3);
}

}  // namespace

template <typename T, int DB, int WAVES, int TK>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : 1)
    cache_attend_many(const AttendArgs a, int row_tiles, int splits, int min_chunk) {
  constexpr int D = 32 * DB, QP = RowType<T>::kQuery, WP = RowType<T>::kWeight;
  constexpr int NT = 64 * WAVES, ROWS = 32 * WAVES, GROUPS = TK / 32;
  constexpr int KFRAGS = GROUPS * DB * 2;           // of 1 KB: (group, block, step)
  constexpr int UNITS = GROUPS * DB * 64;           // 8-byte pieces of codes of K, of V
  constexpr int NU = (UNITS + NT - 1) / NT;
  __shared__ __attribute__((aligned(16))) char lds[2][2 * KFRAGS * 1024];
  __shared__ uint32_t nan_of[2][GROUPS * DB * 4];   // 8 tokens' bits of each octet's values

  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the rows that see most first
  int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int b = id % c.B;
  id /= c.B;
  const int sp = id % splits, rt = row_tiles - 1 - id / splits;
  const Seq s = sequence(c, b);
  const int rows = s.n * a.G, r0 = rt * ROWS;
  // no such rows, or, where the grid has two dimensions, behind the last work group
  if (r0 >= rows || rt < 0) return;
  const int rlast = r0 + ROWS < rows ? r0 + ROWS - 1 : rows - 1;
  const int seen_max = seen_by(s, a.causal, rlast / a.G);
  const int tiles = (seen_max + TK - 1) / TK;
  const int even = (tiles + splits - 1) / splits, chunk = even > min_chunk ? even : min_chunk;
  const int t0 = sp * chunk, t1 = t0 + chunk < tiles ? t0 + chunk : tiles;
  const int64_t tb = c.q_start ? 0 : b;

  // this lane's row, and what the wave's rows see
  const int w0 = r0 + 32 * wave, myrow = w0 + (lane & 31);
  const bool live = w0 < rows;
  const int wlast = w0 + 31 < rows ? w0 + 31 : rows - 1;
  const int wave_min = live ? seen_by(s, a.causal, w0 / a.G) : 0;
  const int wave_max = live ? seen_by(s, a.causal, wlast / a.G) : 0;
  const int wg_min = seen_by(s, a.causal, r0 / a.G);
  const int seen = myrow < rows ? seen_by(s, a.causal, myrow / a.G) : 0x7fffffff;
  const int tok = myrow / a.G, hq = h * a.G + myrow % a.G;

  bf16x8 qf[DB][2][QP];
#pragma unroll
  for (int k = 0; k < DB; ++k)
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      float v[8];
      if (myrow < rows) {
        load_row8<T>((const T*)a.q.p + tb * a.q.b + int64_t(s.row0 + tok) * a.q.l + int64_t(hq) * a.q.h +
                         32 * k + 16 * st + 8 * half, v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
      }
      split8<QP>(v, qf[k][st]);
    }

  // Codes of a tile on their way: unit u of K is the 16 elements (half `st`) of
  // a block of a token, of V a channel pair's octet of tokens.
  u32x2 kc[NU], vc[NU], ve[NU];
  uint32_t ke[NU];
  int32_t pages = -1;
  int at = 64;
  int32_t page[GROUPS];
  auto next_pages = [&](int t) {  // of tile t's groups; tiles come in order
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      if (at == 64) {
        const int u = t * GROUPS + g + lane;
        pages = 32 * u < seen_max ? int32_t(page_of(c, b, u)) : -1;
        at = 0;
      }
      page[g] = __builtin_amdgcn_readlane(pages, at++);
    }
  };
  auto load = [&](int t) {
    next_pages(t);
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + i * NT;
      const int g = GROUPS == 1 ? 0 : u / (DB * 64);
      const int blk = u / 64 % DB;
      kc[i] = vc[i] = ve[i] = u32x2{0u, 0u};
      ke[i] = 0;
      const int32_t pg = GROUPS == 1 ? page[0] : (g == 0 ? page[0] : page[GROUPS - 1]);
      if ((UNITS % NT != 0 && u >= UNITS) || pg < 0) continue;
      const char* p = c.data + tile_at(c, pg, h, t * GROUPS + g);
      const int key = u & 31, st = (u >> 5) & 1;
      kc[i] = *(const u32x2*)(p + blk * 512 + key * 16 + 8 * st);
      ke[i] = *(const uint8_t*)(p + k_exp_at(D, key, blk));
      const int pair = u & 15, oct = (u >> 4) & 3;
      vc[i] = *(const u32x2*)(p + 16 * D + blk * 512 + pair * 32 + oct * 8);
      ve[i] = *(const u32x2*)(p + 33 * D + oct * 8 * DB + 8 * blk);
    }
  };
  // Decodes the codes of tile t into buffer `buf`.  Tokens that no row sees may
  // be any bytes: their exponents become 0, so that they are finite.  Where
  // some rows see a token and others do not, one that stands for NaN is taken
  // out and its octet's bits say so.
  auto decode = [&](int t, int buf) {
    char* kl = lds[buf];
    char* vl = lds[buf] + KFRAGS * 1024;
    const bool mixed = (t + 1) * TK > wg_min;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + i * NT;
      if (UNITS % NT != 0 && u >= UNITS) continue;
      const int g = GROUPS == 1 ? 0 : u / (DB * 64);
      const int blk = u / 64 % DB, frag = (g * DB + blk) * 2;
      const int key = u & 31, st = (u >> 5) & 1;
      const float sc = scale_of(ke[i], 0);
      char* kd = kl + (frag + st) * 1024 + score_row(key) * 16;
      *(bf16x8*)kd = decode8(kc[i][0], sc);
      *(bf16x8*)(kd + 512) = decode8(kc[i][1], sc);
      const int pair = u & 15, oct = (u >> 4) & 3;
      if (mixed) {
        uint32_t bad = 0;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int left = seen_max - (t * TK + 32 * g + 16 * w + 4 * oct);
          ve[i][w] &= ~byte_mask(left <= 0 ? 15u : (left >= 4 ? 0u : (15u << left) & 15u));
          const uint32_t m = nan_bytes(ve[i][w]);
          bad |= m << (4 * w);
          ve[i][w] &= ~byte_mask(m);
        }
        if (pair == 0) nan_of[buf][(g * DB + blk) * 4 + oct] = bad;
      }
      uint32_t ev[4], od[4];
      decode_quad(vc[i][0], ve[i][0], ev, od);
      decode_quad(vc[i][1], ve[i][1], ev + 2, od + 2);
      char* vd = vl + (frag + (oct >> 1)) * 1024 + ((oct & 1) * 32 + pair) * 16;
      *(u32x4*)vd = u32x4{ev[0], ev[1], ev[2], ev[3]};
      *(u32x4*)(vd + 256) = u32x4{od[0], od[1], od[2], od[3]};
    }
  };

  f32x16 o[DB];
#pragma unroll
  for (int k = 0; k < DB; ++k)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[k][r] = 0.f;
  float m = -INFINITY, l = 0.f;
  float lp = 0.f;  // with weights in one part: their sum as rounded

  auto compute = [&](int t, int buf, int dead) {
    const char* kl = lds[buf] + lane * 16;
    const char* vl = kl + KFRAGS * 1024;
    const bool mixed = (t + 1) * TK > wave_min;
    f32x16 x[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[g][r] = 0.f;
#pragma unroll
      for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const bf16x8 kk = *(const bf16x8*)(kl + ((g * DB + k) * 2 + st) * 1024);
#pragma unroll
          for (int q = QP - 1; q >= 0; --q)
            x[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, qf[k][st][q], x[g], 0, 0, 0);
        }
    }
    if (mixed || dead) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * TK + 32 * g + score_token(r, half) >= seen || ((dead >> g) & 1)) x[g][r] = -INFINITY;
    }
    float top = x[0][0];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, x[g][r]);
    // the scale is positive: the largest score is the largest product's
    top *= a.scale_log2;
    if (__builtin_amdgcn_ballot_w64(top > m + kKeptRise)) {
      const float mn = fmaxf(m, fmaxf(top, swap_halves(top)));
      const float f = m == -INFINITY ? 0.f : fast_exp2(m - mn);
      m = mn;
      l *= f;
      if constexpr (WP == 1) lp *= f;
#pragma unroll
      for (int k = 0; k < DB; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[k][r] *= f;
    }
    const float shift = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[g][r] = fast_exp2(__builtin_fmaf(x[g][r], a.scale_log2, -shift));
        sum += x[g][r];
      }
    l += sum;
    if ((t + 1) * TK > wg_min) {
      const uint32_t bad = lane < GROUPS * DB * 4 ? nan_of[buf][lane] : 0u;
      uint64_t any = __builtin_amdgcn_ballot_w64(bad != 0u);
      while (any) {  // an octet with a NaN: the rows that see it
        const int e = __builtin_ctzll(any);
        any &= any - 1;
        const uint32_t bits = __builtin_amdgcn_readlane(bad, e);
        const int base = t * TK + 32 * (e / (DB * 4)) + 4 * (e & 3);
        bool hit = false;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          hit = hit || ((bits >> k & 1u) && base + 16 * (k >> 2) + (k & 3) < seen);
#pragma unroll
        for (int k = 0; k < DB; ++k)
          if (hit && k == e / 4 % DB) {
#pragma unroll
            for (int r = 0; r < 16; ++r) o[k][r] += NAN;
          }
      }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        float p[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) p[r] = x[g][8 * st + r];
        bf16x8 w[WP];
        split8<WP>(p, w);
        if constexpr (WP == 1) lp = sum8<BF16>(w[0], lp);
#pragma unroll
        for (int k = 0; k < DB; ++k) {
          const bf16x8 vv = *(const bf16x8*)(vl + ((g * DB + k) * 2 + st) * 1024);
#pragma unroll
          for (int q = WP - 1; q >= 0; --q)
            o[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv, w[q], o[k], 0, 0, 0);
        }
      }
  };
  auto dead_groups = [&]() {
    int d = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) d |= page[g] < 0 ? 1 << g : 0;
    return d;
  };

  int dead = 0, dead_next = 0;
  if (t0 < t1) {
    load(t0);
    dead = dead_groups();
    decode(t0, 0);
    if (t0 + 1 < t1) {
      load(t0 + 1);
      dead_next = dead_groups();
    }
  }
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    __syncthreads();
    if (t * TK < wave_max) compute(t, buf, dead);
    dead = dead_next;
    if (t + 1 < t1) {
      decode(t + 1, buf ^ 1);
      if (t + 2 < t1) {
        load(t + 2);
        dead_next = dead_groups();
      }
    }
  }

  l += swap_halves(l);
  const float other = WP == 1 ? swap_halves(lp) : 0.f;
  if (myrow >= rows) return;
  if constexpr (WP == 1) {
    const float f = one_part_factor(l, lp + other);
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[k][r] *= f;
  }
  const int64_t flat = (tb * a.Hq + hq) * int64_t(c.rows) + s.row0 + tok;
  if (splits == 1) {
    const float inv = l == 0.f ? 1.f : 1.f / l;
    T* dst = (T*)a.o.p + tb * a.o.b + int64_t(s.row0 + tok) * a.o.l + int64_t(hq) * a.o.h + 8 * half;
    typedef __attribute__((__vector_size__(8 * sizeof(T)))) T vec;
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        vec y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          y[2 * r] = T(o[k][4 * u + r] * inv);
          y[2 * r + 1] = T(o[k][8 + 4 * u + r] * inv);
        }
        *(vec*)(dst + 32 * k + 16 * u) = y;
      }
    if (a.lse && half == 0)
      a.lse[flat] = l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
  } else if (t0 >= t1) {  // nothing here: the join reads no more of it than this
    if (half == 0) *(f32x2*)(a.part_ml + 2 * (flat * splits + sp)) = f32x2{-INFINITY, 0.f};
  } else {
    float* dst = a.part + (flat * splits + sp) * D + 8 * half;
#pragma unroll
    for (int k = 0; k < DB; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        *(f32x4*)(dst + 32 * k + 16 * u) =
            f32x4{o[k][4 * u], o[k][8 + 4 * u], o[k][4 * u + 1], o[k][9 + 4 * u]};
        *(f32x4*)(dst + 32 * k + 16 * u + 4) =
            f32x4{o[k][4 * u + 2], o[k][10 + 4 * u], o[k][4 * u + 3], o[k][11 + 4 * u]};
      }
    if (half == 0) {
      a.part_ml[2 * (flat * splits + sp)] = m;
      a.part_ml[2 * (flat * splits + sp) + 1] = l;
    }
  }
}

namespace {

template <typename T, int DB>
void launch_one(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  constexpr int W = attend_many_rows(RowType<T>::kQuery == 2, 32 * DB) / 32;
  const dim3 grid = attend_grid(int64_t(a.c.B) * a.c.H * p.row_tiles * p.splits), block(64 * W);
  hipLaunchKernelGGL((cache_attend_many<T, DB, W, attend_many_tokens(32 * DB)>), grid, block, 0, s, a, p.row_tiles,
                     p.splits, p.min_chunk);
}

}  // namespace

template <typename T>
hipError_t launch_many(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  switch (a.c.d) {
#define CQSA_MANY(DB)              \
  case 32 * DB:                    \
    launch_one<T, DB>(a, p, s);    \
    break;
    CQSA_MANY(1)
    CQSA_MANY(2)
    CQSA_MANY(3)
    CQSA_MANY(4)
    CQSA_MANY(5)
    CQSA_MANY(6)
    CQSA_MANY(7)
    CQSA_MANY(8)
#undef CQSA_MANY
    default:
      return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_attend_many(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  if (dt == CQSA_BF16) return launch_many<__bf16>(a, p, s);
  return launch_many<_Float16>(a, p, s);
}

}  // namespace cqsa
