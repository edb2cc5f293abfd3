// The attention weights of a call's rows, summed for each token of the 4-bit
// cache (gfx950): W[t] = decay prior[t] + sum over rows of exp(s_t - LSE).
//
// A key head's G query heads of a sequence's n tokens are n G rows of one matrix
// product with its keys, whose columns are the tokens: a lane sums over the rows
// what it holds of its token, with no maximum to keep, since LSE is known, and
// the lanes of a column are added at the end.
#include <algorithm>

#include "cache_attend.hpp"
#include "cache_bound.hpp"

namespace cqsa {

namespace {

constexpr float kLog2eF = 1.4426950408889634f;

// Rows of sequence s that count.
__device__ __forceinline__ int rows_of(const WeighArgs& a, const Seq& s, int b) {
  int n = a.counts ? a.counts[b] : s.n;
  n = n < 0 ? 0 : (n > s.n ? s.n : n);
  return n * a.G;
}

// What row `tok` of head g is shifted by, in powers of two, and the tokens that it
// sees: none where its LSE is not finite.
struct RowShift {
  float shift;
  int seen;
};
__device__ __forceinline__ RowShift row_shift(const WeighArgs& a, const Seq& s, int64_t tb, int h, int tok, int g) {
  const float lse = a.lse[(tb * a.Hq + h * a.G + g) * int64_t(a.c.rows) + s.row0 + tok];
  const bool ok = __builtin_fabsf(lse) < INFINITY;
  return {ok ? lse * kLog2eF : INFINITY, ok ? seen_by(s, a.causal, tok) : 0};
}
constexpr RowShift kBlindRow = {INFINITY, 0};

// Groups of 16 rows that the kernel for few rows takes in registers.  A second one pays at d = 128
// and 256, with 8 operands a group at most (64 sequences of up to 8192 tokens, 8 heads, 24 and 32
// rows: bf16 d = 128 49 and 53 us, from LDS 56 and 52; fp16 d = 128 63 and 67, 80 and 75; bf16
// d = 256 107 and 110, 113 and 108), not elsewhere (bf16 d = 64 43 and 47, from LDS 39 and 36;
// d = 96 64 and 65, 50 and 46; d = 160 91 and 95, 78 and 74; fp32 d = 64 57 and 63, 53 and 50).
constexpr int weigh_few_groups(int parts, int db) { return db % 4 == 0 && parts * db <= 8 ? 2 : 1; }
// Waves a SIMD is to hold: as many as the registers allow without spilling.
constexpr int weigh_few_waves(int parts, int db, int nq) {
  const int held = parts * db * nq;
  if (nq == 1) return held <= 18 ? 4 : held <= 21 ? 3 : 2;
  return held <= 7 || (held == 8 && parts == 1) ? 4 : held <= 14 ? 3 : 2;
}

}  // namespace

// Few rows, 16 NQ at most: they stay in registers while a wave goes through the
// tokens in tiles of 32, the next tile's keys on their way.  The keys' bytes and the
// weights bound it where they are many (one token of 2^20, 8 heads, d = 128: 637 MB in 126
// us, 5.1 TB/s; a copy reaches 4.9), a chain of loads, 4.4 us, where they are few.  Two
// tiles at a time, for more loads on their way, were 3 % slower for long sequences and as much
// faster for short ones, and spilled from d = 224 on.
template <typename T, int DB, int NQ>
__global__ void __launch_bounds__(256, (weigh_few_waves(RowType<T>::kQuery, DB, NQ))) cache_weigh_few(const WeighArgs a, int per_seq) {
  constexpr bool WIDE = DB % 4 == 0;  // whole blocks a lane
  constexpr int D = 32 * DB, QP = RowType<T>::kQuery;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Work groups go round the XCDs, and there round the shader engines, by their number: those of a
  // sequence are neighbours, so that long sequences load no part of the GPU more than another (16 of
  // up to 8192 tokens, drafts, 13.1 us; with sequences as neighbours 14.5).
  int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int part = id % per_seq, b = id / per_seq;
  if (b >= c.B) return;  // behind the last work group, where the grid has two dimensions
  const Seq s = sequence(c, b);
  const int t1 = (s.len + 31) >> 5, step = 4 * per_seq;
  int t = 4 * part + wave;
  if (t >= t1) return;
  const int rows = rows_of(a, s, b), old = s.len - s.n;
  const int64_t tb = c.q_start ? 0 : b;
  const float* prior = a.prior.p ? a.prior.p + b * a.prior.b + h * a.prior.h : nullptr;
  float* out = a.w.p + b * a.w.b + h * a.w.h;

  uint32_t xk[DB][2], xke[WIDE ? DB / 4 : DB];
  float before = 0.f;
  // lanes 0 .. 15 and 32 .. 47 hold a tile's sums in the end
  const int mine = 16 * (quarter >> 1) + col;
  auto load = [&](int u, int32_t page) {
    if (page >= 0) {
      const char* p = c.data + tile_at(c, page, h, u);
      if constexpr (WIDE) {
#pragma unroll
        for (int j = 0; j < DB / 4; ++j) {
          const int blk = 4 * j + quarter;
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const u32x4 x = *(const u32x4*)(p + blk * 512 + (16 * v + col) * 16);
#pragma unroll
            for (int w = 0; w < 4; ++w) xk[4 * j + w][v] = x[w];
          }
          xke[j] = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * blk);
        }
      } else {
#pragma unroll
        for (int w = 0; w < DB; ++w) {
#pragma unroll
          for (int v = 0; v < 2; ++v) xk[w][v] = *(const uint32_t*)(p + w * 512 + (16 * v + col) * 16 + 4 * quarter);
          xke[w] = *(const uint16_t*)(p + 32 * D + col * 2 * DB + 2 * w);
        }
      }
    }
    const int tok = 32 * u + mine;
    before = prior && tok < old ? prior[tok] : 0.f;
  };
  // pages of the wave's next 64 tiles, one a lane
  int32_t pages = -1;
  int at = 64;
  auto next_page = [&](int u) {
    if (u >= t1) return -1;
    if (at == 64) {
      const int v = u + step * lane;
      pages = v < t1 ? int32_t(page_of(c, b, v)) : -1;
      at = 0;
    }
    return __builtin_amdgcn_readlane(pages, at++);
  };
  int32_t page = next_page(t);
  load(t, page);

  // Row 4 e + q of a group is the product's row 4 q + e: few rows are then few of
  // every lane's four.
  bf16x8 qf[NQ][DB][QP];
  float shift[NQ][4];
  int seen[NQ][4];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = 16 * n + 4 * (col & 3) + (col >> 2);
    const int tok = r / a.G, g = r % a.G;
#pragma unroll
    for (int w = 0; w < DB; ++w) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
      const int e = WIDE ? 32 * (4 * (w / 4) + quarter) + 8 * (w % 4) : 32 * w + 8 * quarter;
      if (r < rows)
        load_row8<T>((const T*)a.q.p + tb * a.q.b + int64_t(s.row0 + tok) * a.q.l + int64_t(h * a.G + g) * a.q.h + e, v);
      split8<QP>(v, qf[n][w]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 16 * n + 4 * e + quarter;
      const RowShift x = i < rows ? row_shift(a, s, tb, h, i / a.G, i % a.G) : kBlindRow;
      shift[n][e] = x.shift, seen[n][e] = x.seen;
    }
  }

  while (t < t1) {
    const int next = t + step;
    const int32_t page2 = next_page(next);
    const bool here = page >= 0;
    f32x4 x[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) x[n][0] = x[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (here) {
#pragma unroll
      for (int w = 0; w < DB; ++w)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const bf16x8 kk = decode8(xk[w][v], scale_of(xke[WIDE ? w / 4 : w], v));
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int k = QP - 1; k >= 0; --k)
              x[n][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[n][w][k], kk, x[n][v], 0, 0, 0);
        }
    }
    const float had = before;
    if (next < t1) load(next, page2);
    float sum[2] = {0.f, 0.f};
    if (here) {
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * n + 4 * e < rows) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const float y = fast_exp2(__builtin_fmaf(x[n][v][e], a.scale_log2, -shift[n][e]));
              sum[v] += 32 * t + 16 * v + col < seen[n][e] ? y : 0.f;
            }
          }
    }
    // the halves' lanes exchange: the lower half gets the first 16 tokens' sums
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, sum[0]),
                                                    __builtin_bit_cast(uint32_t, sum[1]), false, false);
    const uint32_t lo = r[0], hi = r[1];
    float y = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    y += __shfl_xor(y, 16);
    const int tok = 32 * t + mine;
    if ((quarter & 1) == 0 && tok < s.len) out[tok] = __builtin_fmaf(a.decay, had, y);
    t = next, page = page2;
  }
}

// Many rows: a wave keeps 64 tokens' decoded keys in registers, and the work
// group's waves go through the rows together, stage by stage of RS through LDS,
// where a matrix operand lies as the 64 lanes read it.  RESIDENT: all rows fit the two
// stages that LDS holds; they are brought once, and the work group goes on to every
// `tiles`-th of its sequence's 64 W tokens, the next ones' keys on their way.
// Exponentials bound it, beside the products: 3 vector instructions a weight, one of them
// of 16 cycles, and d / 16 products of 32 cycles for 32 x 32 weights (4096 rows of 4 heads over
// 32768 tokens, d = 128: 478 us, 1090 TFLOP/s, vector units 62 % busy, matrix cores 48 %; d = 64:
// 363).  Products issued among the exponentials of the 32 rows before were as fast at d = 128
// (529 us both, with 8 waves) and 30 % slower at d = 64, whose registers then leave half the waves.
template <typename T, int DB, int W, int RS, bool RESIDENT>
__global__ void __launch_bounds__(64 * W, W > 8 ? 4 : 2)
    cache_weigh_many(const WeighArgs a, int tiles, int splits) {
  constexpr int D = 32 * DB, QP = RowType<T>::kQuery, NT = 64 * W, TOKENS = 64 * W;
  constexpr int UNITS = RS * 4 * DB, NU = (UNITS + NT - 1) / NT;  // of 8 elements
  constexpr int FOLD = 1024 / RS;                                 // stages that a lane adds before it folds
  __shared__ __attribute__((aligned(16))) char lds[2][RS * D * 2 * QP];
  __shared__ __attribute__((aligned(16))) float row_of[2][RS];
  __shared__ __attribute__((aligned(16))) int seen_of[2][RS];
  __shared__ __attribute__((aligned(16))) float total_of[RESIDENT ? 1 : NT][4];
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // A sequence's work groups are neighbours here too (239 rows of 64 sequences of up to 35604 tokens, 2
  // heads, d = 128: 639 us, with sequences as neighbours 860), and the tiles begin elsewhere for each,
  // since masks leave the first ones more rows than the last.
  int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int h = id % c.H;
  id /= c.H;
  const int sp = id % splits;
  id /= splits;
  const int b = id / tiles, tile = (id + b) % tiles, first = tile * TOKENS;
  if (b >= c.B) return;  // behind the last work group, where the grid has two dimensions
  const Seq s = sequence(c, b);
  if (first >= s.len) return;
  const int rows = rows_of(a, s, b), old = s.len - s.n, G = a.G;
  const int64_t tb = c.q_start ? 0 : b;

  // the work group's stages: those whose rows see its first token, an equal part of them
  int begin = !RESIDENT && a.causal && first > old ? (first - old) * G / RS : 0;
  const int all = (rows + RS - 1) / RS;
  const int each = all > begin ? (all - begin + splits - 1) / splits : 0;
  begin += sp * each;
  const int end = begin + each < all ? begin + each : all;

  // keys: half the lanes hold elements 0 .. 15 of a block, the others 16 .. 31
  int tok0 = first + 64 * wave;
  u32x2 code[2][DB];
  uint32_t power[2][DB];
  bool there[2];
  float had = 0.f;
  auto prior_at = [&](int tok) {
    return a.prior.p && tok < old ? a.prior.p[b * a.prior.b + h * a.prior.h + tok] : 0.f;
  };
  auto fetch = [&](int t0) {
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int t = (t0 >> 5) + v, key = lane & 31;
      const int64_t page = 32 * t < s.len ? page_of(c, b, t) : -1;
      there[v] = page >= 0;
      const char* p = c.data + tile_at(c, page < 0 ? 0 : page, h, t);
#pragma unroll
      for (int w = 0; w < DB; ++w) {
        code[v][w] = u32x2{0u, 0u};
        power[v][w] = 0;
        if (there[v]) {
          code[v][w] = *(const u32x2*)(p + w * 512 + key * 16 + 8 * half);
          power[v][w] = *(const uint8_t*)(p + k_exp_at(D, key, w));
        }
      }
    }
    if (RESIDENT) had = prior_at(t0 + lane);
  };
  bf16x8 kk[2][DB][2];
  auto decode = [&]() {
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int w = 0; w < DB; ++w)
#pragma unroll
        for (int st = 0; st < 2; ++st) kk[v][w][st] = decode8(code[v][w][st], scale_of(power[v][w], 0));
  };
  fetch(tok0);

  // Rows on their way: unit u is chunk u / 16 % 4 of a block of row u % 16 of 16,
  // so that neighbouring lanes write neighbouring 16 bytes of LDS.
  constexpr int NV = sizeof(T) == 4 ? 2 : 1;
  u32x4 in[NU][NV];
  int tok_of[NU], g_of[NU];
  const int r00 = begin * RS;
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = tid + i * NT, r = r00 + u / 64 / DB * 16 + (u & 15);
    tok_of[i] = r / G, g_of[i] = r % G;
  }
  int my_tok = (r00 + tid) / G, my_g = (r00 + tid) % G;  // of the row whose LSE the thread brings
  RowShift my = kBlindRow;
  const int rs_q = RS / G, rs_r = RS % G;
  auto advance = [&](int& tok, int& g) {
    tok += rs_q, g += rs_r;
    if (g >= G) g -= G, ++tok;
  };
  auto load = [&](int stage) {
    const int r0 = stage * RS;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + i * NT;
      const int v = u >> 6, blk = v % DB, r = r0 + v / DB * 16 + (u & 15), e = 32 * blk + 8 * ((u >> 4) & 3);
#pragma unroll
      for (int k = 0; k < NV; ++k) in[i][k] = u32x4{0u, 0u, 0u, 0u};
      if ((UNITS % NT == 0 || u < UNITS) && r < rows) {
        const T* p = (const T*)a.q.p + tb * a.q.b + int64_t(s.row0 + tok_of[i]) * a.q.l +
                     int64_t(h * G + g_of[i]) * a.q.h + e;
#pragma unroll
        for (int k = 0; k < NV; ++k) in[i][k] = ((const u32x4*)p)[k];
      }
      advance(tok_of[i], g_of[i]);
    }
    if (tid < RS) {
      my = r0 + tid < rows ? row_shift(a, s, tb, h, my_tok, my_g) : kBlindRow;
      advance(my_tok, my_g);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int u = tid + i * NT;
      if (UNITS % NT != 0 && u >= UNITS) continue;
      const int v = u >> 6, blk = v % DB, r = v / DB * 16 + (u & 15), ch = (u >> 4) & 3;
      bf16x8 q[QP];
      if constexpr (QP == 1) {
        q[0] = __builtin_bit_cast(bf16x8, in[i][0]);
      } else {
        float x[8];
        load_row8<T>((const T*)&in[i][0], x);
        split8<QP>(x, q);
      }
      char* p = lds[buf] + (((r >> 5) * DB + blk) * 2 + (ch & 1)) * QP * 1024 + ((ch >> 1) * 32 + (r & 31)) * 16;
#pragma unroll
      for (int k = 0; k < QP; ++k) *(bf16x8*)(p + 1024 * k) = q[k];
    }
    if (tid < RS) row_of[buf][tid] = my.shift, seen_of[buf][tid] = my.seen;
  };

  float sum[2] = {0.f, 0.f};
  auto compute = [&](int buf) {
#pragma unroll
    for (int rt = 0; rt < RS / 32; ++rt) {
      const int see = seen_of[buf][32 * rt + (lane & 31)];
      if (!__builtin_amdgcn_ballot_w64(see > tok0)) continue;
      f32x16 x[2];
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[v][r] = 0.f;
#pragma unroll
      for (int w = 0; w < DB; ++w)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int k = QP - 1; k >= 0; --k) {
            const bf16x8 q = *(const bf16x8*)(lds[buf] + (((rt * DB + w) * 2 + st) * QP + k) * 1024 + lane * 16);
#pragma unroll
            for (int v = 0; v < 2; ++v) x[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, kk[v][w][st], x[v], 0, 0, 0);
          }
      const bool whole = !__builtin_amdgcn_ballot_w64(see < tok0 + 64);
      float part[2][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 sh = *(const f32x4*)&row_of[buf][32 * rt + 8 * i + 4 * half];
        float y[2][4];
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[v][e] = fast_exp2(__builtin_fmaf(x[v][4 * i + e], a.scale_log2, -sh[e]));
        if (!whole) {
          typedef __attribute__((__vector_size__(16))) int i32x4;
          const i32x4 sn = *(const i32x4*)&seen_of[buf][32 * rt + 8 * i + 4 * half];
#pragma unroll
          for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (tok0 + 32 * v + (lane & 31) >= sn[e]) y[v][e] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) part[v][i] = (y[v][0] + y[v][1]) + (y[v][2] + y[v][3]);
      }
#pragma unroll
      for (int v = 0; v < 2; ++v) sum[v] += (part[v][0] + part[v][1]) + (part[v][2] + part[v][3]);
    }
  };

  // A lane's sums go into a total every 1024 rows, which carries what its own additions lose: added one to
  // another, weights that are much alike would all round the same way (131072 of them 3.5e-5 off, so 3.7e-7).
  // It lies in LDS, since the registers of 16 waves are all taken (12 would spill at bf16 d = 128).  It takes
  // 0 to 1 % of a call's time, past d = 128 0 to 2 % (one sequence of 4096 tokens and rows of 4 heads, d = 128,
  // 89.5 and 90.1 us; fp32 d = 256 321 and 324).
  auto fold = [&](bool first) {
    int slot = tid;
    keep_in_register(slot);  // found anew each time: no other register holds its address meanwhile
    const f32x4 old = first ? f32x4{0.f, 0.f, 0.f, 0.f} : *(const f32x4*)total_of[slot];
    f32x4 now;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const float y = sum[v] - old[2 + v], t = old[v] + y;
      now[v] = t, now[2 + v] = t < INFINITY ? (t - old[v]) - y : 0.f;
      sum[v] = 0.f;
    }
    *(f32x4*)total_of[slot] = now;
  };

  auto finish = [&](bool there0, bool there1, float before) {
    // the halves' lanes exchange: the lower half gets the first 32 tokens' sums
    if (!there0) sum[0] = 0.f;
    if (!there1) sum[1] = 0.f;
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, sum[0]),
                                                    __builtin_bit_cast(uint32_t, sum[1]), false, false);
    const uint32_t lo = r[0], hi = r[1];
    const float y = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    const int tok = tok0 + lane;
    if (tok >= s.len) return;
    if (splits > 1)
      a.part[(int64_t(sp) * c.B + b) * c.H * c.max_len + int64_t(h) * c.max_len + tok] = y;
    else
      a.w.p[b * a.w.b + h * a.w.h + tok] = __builtin_fmaf(a.decay, before, y);
  };

  if (begin < end) load(begin);
  if constexpr (RESIDENT) {
    if (begin < end) put(0);
    if (begin + 1 < end) {
      load(begin + 1);
      put(1);
    }
    __syncthreads();
    while (tok0 < s.len) {
      decode();
      const bool there0 = there[0], there1 = there[1];
      const float before = had;
      const int next = tok0 + tiles * TOKENS;
      if (next < s.len) fetch(next);
      sum[0] = sum[1] = 0.f;
      if (there0 || there1) {
        if (begin < end) compute(0);
        if (begin + 1 < end) compute(1);
      }
      finish(there0, there1, before);
      tok0 = next;
    }
    return;
  }
  decode();
  if (begin < end) {
    put(0);
    if (begin + 1 < end) load(begin + 1);
  }
  for (int stage = begin; stage < end; ++stage) {
    const int buf = (stage - begin) & 1;
    __syncthreads();
    if (tok0 < s.len) compute(buf);
    if (((stage - begin) & (FOLD - 1)) == FOLD - 1) fold(stage - begin < FOLD);
    if (stage + 1 < end) {
      put(buf ^ 1);
      if (stage + 2 < end) load(stage + 2);
    }
  }
  if (end - begin >= FOLD) {
    fold(false);
    sum[0] = total_of[tid][0], sum[1] = total_of[tid][1];
  }
  finish(there[0], there[1], splits == 1 ? prior_at(tok0 + lane) : 0.f);
}

// Adds the parts of a split call, in their order.
__global__ void __launch_bounds__(256) cache_weigh_join(const WeighArgs a, int pieces, int splits) {
  const CacheArgs& c = a.c;
  const int64_t bh = blockIdx.x / pieces;
  const int b = int(bh / c.H), h = int(bh % c.H);
  const Seq s = sequence(c, b);
  for (int tok = blockIdx.x % pieces * 256 + threadIdx.x; tok < s.len; tok += 256 * pieces) {
    float y = 0.f;
    for (int i = 0; i < splits; ++i) y += a.part[(int64_t(i) * c.B * c.H + bh) * c.max_len + tok];
    const float had = a.prior.p && tok < s.len - s.n ? a.prior.p[b * a.prior.b + h * a.prior.h + tok] : 0.f;
    a.w.p[b * a.w.b + h * a.w.h + tok] = __builtin_fmaf(a.decay, had, y);
  }
}

namespace {

// Rows of a stage, so that two of them fit LDS.
constexpr int stage_rows(int parts, int db) { return parts * db <= 8 ? 64 : 32; }
// Waves of a work group: 4, or more, which go through more rows a byte of LDS, as many as the
// registers of their keys allow.
constexpr int kShortWaves = 4;
constexpr int long_waves(int db) { return db <= 4 ? 16 : 8; }
// More wherever 4 have no second work group's registers beside them (fp32 past d = 128: 8 sequences of
// 2000 tokens, 4 heads a group, d = 256 338 us, 997 before).  Else where work groups have much of the same
// length: not over many sequences, whose lengths differ, and not over few tokens (1 of 8192 tokens and rows,
// bf16 d = 128 307 us, with 4 waves 333; 4096 rows over 32768 508 and 601; of 3000 72 and 67; 64 of up to 4000,
// 200 rows, 16 heads a group, 387 and 312; fp16 d = 128, 4 of up to 3000, 198 and 230; d = 160, 64 of 200
// over 4000, 638 and 599).  4 waves spill 5 registers at bf16 d = 256 (64 of 200 over 4000 530, with 4 606; of
// 700 180 and 157), 16 waves spill 4 at fp32 d = 128 (1 of 1024 rows over 16384 294 us, with 4 waves 331; 4096
// over 8192 522 and 505; 4 of 300 over up to 16384 256 and 272).  Narrow heads, whose rows take little LDS, have
// no use for more (bf16 d = 64: 1 of 8192 236, with 4 215; d = 32 206 and 169).
constexpr bool has_long(int parts, int db) { return db > 4 || (db > 1 && parts * db > 2); }
constexpr bool has_short(int parts, int db) { return db <= 4 || parts < 3; }
bool takes_long(int parts, int db, int64_t B, int64_t max_len) {
  if (!has_long(parts, db) || !has_short(parts, db)) return has_long(parts, db);
  if (db > 4) return max_len > 1536 && (B <= 4 / parts || parts * db == 8);
  return parts * db == 8 ? B <= 8 && max_len >= 2048 : B <= 4 && max_len >= 8192;
}
// And over resident rows: 4, or 8 where their stages leave LDS for one work group a CU (fp32 d = 256,
// 64 sequences of up to 8192 tokens: 32 rows 161 us, 217 with 4 waves, 64 rows 238 and 332; over 4
// sequences of 1000 16 and 13; d = 192 191 and 177).
constexpr int resident_waves(int parts, int db) { return parts * db > 18 ? 8 : 4; }

template <typename T, int DB>
void launch_d(const WeighArgs& a, const WeighPlan& p, hipStream_t s) {
  constexpr int QP = RowType<T>::kQuery, NQ = weigh_few_groups(QP, DB), RS = stage_rows(QP, DB), LW = long_waves(DB),
                RW = resident_waves(QP, DB);
  const dim3 grid = attend_grid(p.groups), block(64 * p.waves);
  if (p.row_groups == 0) {
    if (p.resident)
      hipLaunchKernelGGL((cache_weigh_many<T, DB, RW, RS, true>), grid, block, 0, s, a, p.tiles, 1);
    if constexpr (has_long(QP, DB))
      if (!p.resident && p.waves == LW)
        hipLaunchKernelGGL((cache_weigh_many<T, DB, LW, RS, false>), grid, block, 0, s, a, p.tiles, p.splits);
    if constexpr (has_short(QP, DB))
      if (!p.resident && p.waves == kShortWaves)
        hipLaunchKernelGGL((cache_weigh_many<T, DB, kShortWaves, RS, false>), grid, block, 0, s, a, p.tiles, p.splits);
  } else if (p.row_groups == 1) {
    hipLaunchKernelGGL((cache_weigh_few<T, DB, 1>), grid, block, 0, s, a, p.tiles);
  } else if constexpr (NQ == 2) {
    hipLaunchKernelGGL((cache_weigh_few<T, DB, 2>), grid, block, 0, s, a, p.tiles);
  }
}

template <typename T>
hipError_t launch_rows(const WeighArgs& a, const WeighPlan& p, hipStream_t s) {
  switch (a.c.d / 32) {
#define CQSA_WEIGH(DB)        \
  case DB:                    \
    launch_d<T, DB>(a, p, s); \
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
  if (p.splits > 1) {
    const int64_t heads = int64_t(a.c.B) * a.c.H;
    const int64_t pieces = std::min<int64_t>((int64_t(a.c.max_len) + 255) / 256, (int64_t(1) << 23) / heads);
    hipLaunchKernelGGL(cache_weigh_join, dim3(unsigned(pieces * heads)), dim3(256), 0, s, a, int(pieces), p.splits);
  }
  return hipGetLastError();
}

}  // namespace

WeighPlan plan_weigh(int64_t B, int64_t H, int64_t rows, int64_t max_len, cqsa_dtype dt, int d) {
  WeighPlan p{};
  const int parts = dt == CQSA_F32 ? 3 : (dt == CQSA_F16 ? 2 : 1), db = d / 32, stage = stage_rows(parts, db);
  const int64_t heads = B * H;
  p.splits = 1;
  p.waves = 4;
  if (rows <= 16 * weigh_few_groups(parts, db)) {
    p.row_groups = rows > 16 ? 2 : 1;
    // Work groups a sequence and head: as many as the GPU holds at once, or of several
    // sequences, whose lengths differ, one for every 8 tiles of its waves with one group
    // of rows and 16 with two, so that the long ones' parts even out (64 of up to
    // 16384 tokens, 8 heads, d = 128: 67 us, with as many as fit 81; 16 of them 20 and 20;
    // one of 2^20 126, in parts of 8 tiles 138; 64 of up to 16384, two groups of rows, 98 and 101).
    const int64_t tiles = (max_len + 31) / 32, most = (tiles + 3) / 4;
    const int held = parts * db * p.row_groups;
    const int64_t fit = (held <= 4 ? 1536 : held <= 12 ? 1024 : 768) / heads;
    const int64_t even = B == 1 ? 0 : tiles / (32 * p.row_groups);
    p.tiles = int(std::max<int64_t>(1, std::min(most, std::max(fit, even))));
    p.groups = heads * p.tiles;
    return p;
  }
  if (rows <= 2 * stage) {
    // the same with tiles of 64 tokens a wave, 4 a work group (48 rows, 64 sequences of up to 8192
    // tokens, d = 128: 67 us, one 100; 128 rows, 16 of them 37 and 48)
    p.resident = true;
    p.waves = resident_waves(parts, db);
    const int64_t most = (max_len + 64 * p.waves - 1) / (64 * p.waves), fit = 6144 / p.waves / heads;
    p.tiles = int(std::max<int64_t>(1, std::min(most, std::max<int64_t>(fit, B == 1 ? 0 : most / 4))));
    p.groups = heads * p.tiles;
    return p;
  }
  if (takes_long(parts, db, B, max_len)) p.waves = long_waves(db);
  p.tiles = int((max_len + 64 * p.waves - 1) / (64 * p.waves));
  // The rows are split until the GPU has 8 work groups of 4 waves a CU, which evens out what causal
  // masks leave of them (32 sequences of 300 tokens and rows of 4 heads, d = 128: 31 us in 3 or 4 parts,
  // 54 in one), or as many as their registers allow (d = 256: 32 of 300 56 in 2, 61 in 3), or 2 of more
  // waves; of 128 rows at least.  And into parts of 512 rows up to 8, of 1024 from there on, where the lengths
  // of sequences differ (64 of up to 746 tokens and rows, 16 heads a group, d = 160: 222 us, without 445; fp32
  // 676 and 1281; 64 of up to 700, 4 heads, fp32 d = 256 350, in parts of 1024 529), up to 2^14 work
  // groups, which bounds the workspace by max_len.  One alone is split into parts of 2048 rows by 4 waves (4096
  // rows of 4 heads over 32768, bf16 d = 64: 361 us, of 4096 393) and no further by more (d = 128 483 and 502).
  const int64_t groups = heads * p.tiles;
  const int64_t total = p.waves > 4 ? 512 : db > 4 ? 1024 : 2048;
  const int64_t even = B == 1 ? (p.waves > 4 ? 0 : rows / 2048)
                              : std::max<int64_t>(rows / 1024, std::min<int64_t>(rows / 512, 8));
  const int64_t most = std::min<int64_t>(rows / 128, 64);
  p.splits = int(std::max<int64_t>(1, std::min(most, std::max((total + groups - 1) / groups, std::min(even, 16384 / groups)))));
  p.groups = groups * p.splits;
  return p;
}

hipError_t launch_cache_weigh(cqsa_dtype dt, const WeighArgs& a, const WeighPlan& p, hipStream_t s) {
  if (dt == CQSA_BF16) return launch_rows<__bf16>(a, p, s);
  if (dt == CQSA_F16) return launch_rows<_Float16>(a, p, s);
  return launch_rows<float>(a, p, s);
}

}  // namespace cqsa
