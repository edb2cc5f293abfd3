// Eviction from the 4-bit cache: which tokens a sequence's heads keep, and their
// moving together (gfx950).
//
// A token's rank is a 32-bit key: 0 where its page holds nothing, 1 for a NaN, the
// weight's bits in an order that integers compare by, and 2^32 - 1 for the first and
// the recent tokens.  The n-th largest key is found by its digits of 11, 11 and 10
// bits, from counts of the keys that share its upper ones: integers, whose sums go in
// any order.  A head's tokens up to 32768 are a work group's, which holds their keys in
// registers; longer ones are shared by many, with the counts in memory.
#include <algorithm>

#include "cache_bound.hpp"
#include "hip_common.hpp"

namespace cqsa {

namespace {

constexpr uint32_t kForced = 0xffffffffu;
constexpr int kItems = 16;    // keys of a lane of a work group that shares a head with others
constexpr int kBins = 2048;   // of a digit
constexpr int kChunk = 4096;  // tokens of a work group that shares a head with others
// words of a head in memory: three digits' counts, and how many tokens have no page
constexpr int kHeadWords = 3 * kBins + 4;

__device__ __forceinline__ uint32_t rank_of(float w) {
  uint32_t u = __builtin_bit_cast(uint32_t, w);
  const uint32_t mag = u & 0x7fffffffu;
  if (mag > 0x7f800000u) return 1u;
  if (mag == 0u) u = 0u;  // both zeros
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int length_of(const CacheArgs& c, int b) {
  const int32_t n = c.lengths[b];
  return n < 0 ? 0 : (n > c.max_len ? c.max_len : n);
}

// The key of token t, by its weight and its page (-1 behind the sequence).
__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, float w, int32_t page, int t, int len) {
  const uint32_t k = t < a.first || t >= len - a.recent ? kForced : rank_of(w);
  return page < 0 || page >= a.c.n_pages ? 0u : k;
}

// Keys of a wave's tokens t0 + step i + lane, i < items, by use(i, key).  A work group goes through its code
// once, so that long code costs more than it does: 8 loads at a time, and keys that are looked at
// again lie in LDS.
template <typename F>
__device__ __forceinline__ void each_key(const EvictArgs& a, const float* w, int b, int len, int t0, int step, int items,
                                         F use) {
  constexpr int U = 8;
#pragma unroll 1
  for (int i0 = 0; i0 < items; i0 += U) {
    float x[U];
    int32_t page[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = t0 + step * (i0 + k);
      const bool here = i0 + k < items && t < len;
      x[k] = here ? w[t] : 0.f;
      page[k] = here ? a.c.pages[b * a.c.pages_stride + (t >> a.c.page_log2)] : -1;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (i0 + k >= items) break;
      use(i0 + k, key_of(a, x[k], page[k], t0 + step * (i0 + k), len));
    }
  }
}

// A digit of a key, from the uppermost on: 11, 11 and 10 bits.
__device__ __forceinline__ uint32_t digit_of(uint32_t k, int pass) {
  return pass == 0 ? k >> 21 : pass == 1 ? k >> 10 & 2047u : k & 1023u;
}
// Whether k has the border's upper digits.
__device__ __forceinline__ bool shares(uint32_t k, uint32_t border, int pass) {
  return pass == 0 || (pass == 1 ? k >> 21 == border >> 21 : k >> 10 == border >> 10);
}

// Inclusive sums over the lanes.
__device__ __forceinline__ int scan_of_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // within rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // rows 0 and 2 into 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // the lower half into the upper
  return x;
}

// The digit in which the `left`-th largest of the counted keys lies: counts of kBins in
// `count` (LDS or memory), by the NT threads of a work group.  `scratch`: a word a wave and 3.
// Where all keys that share the digits so far are kept the border is below them, and left is 0:
// no digit has to follow.
template <int NT>
__device__ __forceinline__ EvictBorder next_digit(const uint32_t* count, const EvictBorder& at, int pass, int* scratch) {
  constexpr int PER = kBins / NT, WAVES = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += mine[i] = int(count[kBins - 1 - (tid * PER + i)]);  // from the largest down
  const int run = scan_of_wave(sum);
  if (lane == 63) scratch[wave] = run;
  __syncthreads();
  int above = run - sum;
  for (int i = 0; i < WAVES; ++i) above += i < wave ? scratch[i] : 0;
  if (above < at.left && above + sum >= at.left) {  // one thread's, if left is 1 or more
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (above < at.left && above + mine[i] >= at.left) {
        scratch[WAVES] = kBins - 1 - (tid * PER + i);
        scratch[WAVES + 1] = at.left - above;
        scratch[WAVES + 2] = mine[i];
      }
      above += mine[i];
    }
  }
  __syncthreads();
  const uint32_t d = uint32_t(scratch[WAVES]);
  EvictBorder next = {at.key | (pass == 0 ? d << 21 : pass == 1 ? d << 10 : d), scratch[WAVES + 1]};
  if (next.left == scratch[WAVES + 2]) next = {next.key ? next.key - 1 : 0u, 0};
  return next;
}

__device__ __forceinline__ int lanes_below(uint64_t m) {
  return int(__builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0u)));
}

// Adds a key to its digit's count in LDS where it shares the border's upper ones.  Zeros, of which there
// may be very many, are counted by themselves and added once (512 heads of 16384 of them: 102 us with an
// addition each, which one address takes one after the other).
constexpr uint32_t kZero = 0x80000000u;
__device__ __forceinline__ void count_key(uint32_t* count, uint32_t k, const EvictBorder& at, int pass) {
  if (k != 0u && k != kZero && shares(k, at.key, pass)) atomicAdd(&count[digit_of(k, pass)], 1u);
}
__device__ __forceinline__ void count_zeros(uint32_t* count, int zeros, const EvictBorder& at, int pass) {
  if (zeros > 0 && shares(kZero, at.key, pass)) atomicAdd(&count[digit_of(kZero, pass)], uint32_t(zeros));
}
__device__ __forceinline__ int lanes_of(bool x) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(x)); }

// Places of 64 keys in a row, a lane each: kept are those above the border, and the first `left` that equal
// it; n0 and n1 such keys lie before them.
__device__ __forceinline__ void place(uint32_t k, const EvictBorder& at, int t, int n0, int n1, int32_t* kept) {
  const uint64_t above = __builtin_amdgcn_ballot_w64(k > at.key), equal = __builtin_amdgcn_ballot_w64(k == at.key);
  const int m0 = n0 + lanes_below(above), m1 = n1 + lanes_below(equal);
  if (k > at.key || (k == at.key && m1 < at.left)) kept[m0 + (m1 < at.left ? m1 : at.left)] = t;
}

// A wave's keys above the border, and those that equal it.
struct Counts {
  int above, equal;
  __device__ __forceinline__ void add(uint32_t k, const EvictBorder& at) {
    above += lanes_of(k > at.key);
    equal += lanes_of(k == at.key);
  }
};

constexpr EvictBorder kNothing = {kForced, 0};  // of a sequence that keeps nothing, of 0 tokens

__device__ __forceinline__ int kept_of(const EvictArgs& a, int present) { return present < a.budget ? present : a.budget; }

}  // namespace

// A work group takes all of a head's tokens, 16 waves of 64 ITEMS in a row, whose keys stay in registers.
// What bounds it is issuing the 100 instructions or so that 64 keys cost in all, and a chain of loads and
// barriers where they are few (8 heads of 1000 tokens 8.3 us, of 16384 14.7; 512 heads of 16384 29).
// The fewer keys a lane holds the shorter that chain: 8 heads of 2111 tokens 6.4 us with 4, with 16
// 10.3; 512 heads of 4096 10.5 and 13.6.
template <int ITEMS>
__global__ void __launch_bounds__(1024, ITEMS > 16 ? 4 : 8) cache_evict_select(const EvictArgs a) {
  constexpr int WAVES = 16, NT = 64 * WAVES;
  __shared__ uint32_t count[kBins];
  __shared__ int scratch[WAVES + 3];
  __shared__ int before[2][WAVES];
  const int64_t id = (int64_t(blockIdx.y) << kGridLog2) + blockIdx.x;
  const int h = int(id % a.c.H), b = int(id / a.c.H);
  if (b >= a.c.B) return;  // the grid has two dimensions
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = length_of(a.c, b);
  const float* w = a.w.p + b * a.w.b + h * a.w.h;
  const int t0 = 64 * ITEMS * wave;
  const bool some = t0 < len;  // waves without tokens pass the code by
  for (int i = tid; i < kBins; i += NT) count[i] = 0;
  uint32_t key[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) key[i] = 0u;
  int present = 0, zeros = 0;
  if (some) {
    constexpr int U = ITEMS < 8 ? ITEMS : 8;  // loads at a time
#pragma unroll
    for (int i0 = 0; i0 < ITEMS; i0 += U) {
      float x[U];
      int32_t page[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int t = t0 + 64 * (i0 + i) + lane;
        x[i] = t < len ? w[t] : 0.f;
        page[i] = t < len ? a.c.pages[b * a.c.pages_stride + (t >> a.c.page_log2)] : -1;
      }
#pragma unroll
      for (int i = 0; i < U; ++i) key[i0 + i] = key_of(a, x[i], page[i], t0 + 64 * (i0 + i) + lane, len);
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) present += lanes_of(key[i] != 0u), zeros += lanes_of(key[i] == kZero);
  }
  if (lane == 0) before[0][wave] = present;
  __syncthreads();
  present = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) present += before[0][i];
  const int keep = kept_of(a, present);
  EvictBorder at = {0u, keep};
  if (keep == 0) {
    at = kNothing;
  } else {
#pragma unroll 1
    for (int pass = 0; pass < 3 && at.left > 0; ++pass) {
      if (pass > 0) {  // (a barrier lies behind the last reads of the counts and of scratch)
        for (int i = tid; i < kBins; i += NT) count[i] = 0;
        __syncthreads();
      }
      if (some) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) count_key(count, key[i], at, pass);
      }
      if (lane == 0) count_zeros(count, zeros, at, pass);
      __syncthreads();
      at = next_digit<NT>(count, at, pass, scratch);
    }
  }
  Counts n = {0, 0};
  if (some) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) n.add(key[i], at);
  }
  __syncthreads();
  if (lane == 0) before[0][wave] = n.above, before[1][wave] = n.equal;
  __syncthreads();
  int n0 = 0, n1 = 0;
  for (int i = 0; i < wave; ++i) n0 += before[0][i], n1 += before[1][i];
  int32_t* kept = a.kept + id * a.kept_stride;
  if (some) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      place(key[i], at, t0 + 64 * i + lane, n0, n1, kept);
      n0 += lanes_of(key[i] > at.key), n1 += lanes_of(key[i] == at.key);
    }
  }
  if (a.pad)
    for (int64_t i = keep + tid; i < a.budget; i += NT) kept[i] = -1;
  if (h == 0 && tid == 0) a.n_kept[b] = keep;
}

// ------------------------------------------------- heads that work groups share
// A head has `per` work groups, one for each chunk of kChunk tokens, or fewer where there
// are very many.
__global__ void __launch_bounds__(256) cache_evict_clear(uint32_t* words, int64_t n) {
  for (int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; i < n; i += int64_t(gridDim.x) * 1024)
    *(u32x4*)(words + i) = u32x4{0u, 0u, 0u, 0u};
}

// The border so far: by the counts of the pass before, with the digits that its own work groups
// left in `state`.  The first chunk's work group leaves it there in turn.
template <int PASS>
__device__ __forceinline__ EvictBorder border_of(const EvictArgs& a, int64_t id, int len, bool leave, int* scratch) {
  uint32_t* words = a.counts + id * kHeadWords;
  if (PASS == 0) return {0u, 0};
  EvictBorder at;
  if (PASS == 1) {
    at = {0u, kept_of(a, len - int(words[3 * kBins]))};
    if (at.left == 0) at = kNothing;
  } else {
    at = a.state[id * 3 + PASS - 2];
  }
  if (at.left > 0) at = next_digit<256>(words + (PASS - 1) * kBins, at, PASS - 1, scratch);
  if (leave && threadIdx.x == 0) a.state[id * 3 + PASS - 1] = at;
  return at;
}

template <int PASS>
__global__ void __launch_bounds__(256) cache_evict_count(const EvictArgs a, int per) {
  __shared__ uint32_t count[kBins];
  __shared__ int scratch[7];
  const int64_t id = blockIdx.x / per;
  const int part = blockIdx.x % per;
  const int h = int(id % a.c.H), b = int(id / a.c.H);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = length_of(a.c, b);
  const EvictBorder at = border_of<PASS>(a, id, len, part == 0, scratch);
  if ((PASS == 1 || PASS == 2) && at.left == 0) return;  // known by now
  const float* w = a.w.p + b * a.w.b + h * a.w.h;
  uint32_t* words = a.counts + id * kHeadWords;
  if (PASS < 3) {
    for (int i = tid; i < kBins; i += 256) count[i] = 0;
    __syncthreads();
  }
  int absent = 0, zeros = 0;
  for (int chunk = part; chunk < a.chunks; chunk += per) {
    const int t0 = chunk * kChunk + 1024 * wave;
    const int items = t0 < len ? kItems : 0;
    Counts n = {0, 0};
    each_key(a, w, b, len, t0 + lane, 64, items, [&](int i, uint32_t k) {
      if (PASS == 3) {
        n.add(k, at);
      } else {
        if (PASS == 0) absent += k == 0u && t0 + 64 * i + lane < len;
        zeros += lanes_of(k == kZero);
        count_key(count, k, at, PASS);
      }
    });
    if (PASS == 3) {
      __syncthreads();
      if (lane == 0) scratch[wave] = n.above, count[wave] = uint32_t(n.equal);
      __syncthreads();
      if (tid == 0)
        a.chunk_counts[id * a.chunks + chunk] =
            int2{scratch[0] + scratch[1] + scratch[2] + scratch[3], int(count[0] + count[1] + count[2] + count[3])};
    }
  }
  if (PASS == 3) return;
  if (lane == 0) count_zeros(count, zeros, at, PASS);
  if (PASS == 0 && absent) atomicAdd(&words[3 * kBins], uint32_t(absent));
  __syncthreads();
  for (int i = tid; i < kBins; i += 256)
    if (count[i]) atomicAdd(&words[PASS * kBins + i], count[i]);
}

__global__ void __launch_bounds__(256) cache_evict_place(const EvictArgs a, int per) {
  __shared__ uint32_t keys[kChunk];
  __shared__ int before[2][4], own[2][4];
  const int64_t id = blockIdx.x / per;
  const int part = blockIdx.x % per;
  const int h = int(id % a.c.H), b = int(id / a.c.H);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = length_of(a.c, b);
  const EvictBorder at = a.state[id * 3 + 2];
  const int keep = kept_of(a, len - int(a.counts[id * kHeadWords + 3 * kBins]));
  const float* w = a.w.p + b * a.w.b + h * a.w.h;
  int32_t* kept = a.kept + id * a.kept_stride;
  const int2* chunks = a.chunk_counts + id * a.chunks;
  int from = 0, sum0 = 0, sum1 = 0;  // keys of the chunks before, this thread's part of them
  for (int chunk = part; int64_t(chunk) * kChunk < len; chunk += per) {
    const int t0 = chunk * kChunk + 1024 * wave;
    const int items = t0 < len ? kItems : 0;
    uint32_t* const key = keys + 1024 * wave;
    Counts n = {0, 0};
    each_key(a, w, b, len, t0 + lane, 64, items, [&](int i, uint32_t k) {
      key[64 * i + lane] = k;
      n.add(k, at);
    });
    for (int i = from + tid; i < chunk; i += 256) {
      const int2 x = chunks[i];
      sum0 += x.x, sum1 += x.y;
    }
    from = chunk;
    int m0 = sum0, m1 = sum1;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) m0 += __shfl_xor(m0, k), m1 += __shfl_xor(m1, k);
    __syncthreads();
    if (lane == 0) before[0][wave] = m0, before[1][wave] = m1, own[0][wave] = n.above, own[1][wave] = n.equal;
    __syncthreads();
    int n0 = 0, n1 = 0;
    for (int i = 0; i < 4; ++i) {
      n0 += before[0][i], n1 += before[1][i];
      if (i < wave) n0 += own[0][i], n1 += own[1][i];
    }
    for (int i = 0; i < items; ++i) {
      const uint32_t k = key[64 * i + lane];
      place(k, at, t0 + 64 * i + lane, n0, n1, kept);
      n0 += lanes_of(k > at.key), n1 += lanes_of(k == at.key);
    }
  }
  if (a.pad)
    for (int64_t i = keep + int64_t(part) * 256 + tid; i < a.budget; i += int64_t(per) * 256) kept[i] = -1;
  if (h == 0 && part == 0 && tid == 0) a.n_kept[b] = keep;
}

// --------------------------------------------------------------------- moving
// A wave moves 32 kept tokens of a head.  STAGED: from the stage into the pages, in their
// places; else from the pages into the stage (in place) or the target's pages.  A lane's four
// source tokens are the same for all channel pairs, whose 4 bytes it gathers one by one:
// the cache holds values by channel pairs, so that any token moved touches all of its tile.  The
// bytes bound it (64 sequences of up to 16384 tokens down to 4096, 8 heads, d = 128: 617 MB read and
// 260 written in 187 us, 4.7 TB/s; by work groups of 4 waves for 32 tokens, with barriers, 316).
template <bool STAGED>
__global__ void __launch_bounds__(256) cache_evict_move(const EvictArgs a, int tiles) {
  const CacheArgs& c = a.c;
  const int d = c.d, db = d >> 5, lane = threadIdx.x & 63, low = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = ((int64_t(blockIdx.y) << kGridLog2) + blockIdx.x) * 4 + wave;
  const int tile = int(id % tiles);
  const int64_t bh = id / tiles;
  const int h = int(bh % c.H), b = int(bh / c.H);
  if (b >= c.B) return;  // behind the last tile
  const int keep = a.n_kept[b];
  if (h == 0 && tile == 0 && lane == 0 && (STAGED || !a.in_place)) a.new_lengths[b] = keep;
  const int n = keep - 32 * tile < 32 ? keep - 32 * tile : 32;
  if (n <= 0) return;
  const int t = low < n ? a.kept[bh * a.kept_stride + 32 * tile + low] : -1;
  // in place: tokens that stay where they are
  if (a.in_place && !__builtin_amdgcn_ballot_w64(low < n && t != 32 * tile + low)) return;
  char* const stage = a.stage + (bh * tiles + tile) * tile_bytes(d);
  if (lane < n) {
    const float* w = a.w.p + b * a.w.b + h * a.w.h;
    const int64_t i = bh * a.cap + 32 * tile + lane;
    if (STAGED)
      a.w.p[b * a.w.b + h * a.w.h + 32 * tile + lane] = a.stage_w[i];
    else if (a.in_place)
      a.stage_w[i] = w[t];
    else if (a.w_to.p)
      a.w_to.p[b * a.w_to.b + h * a.w_to.h + 32 * tile + lane] = w[t];
  }
  char* dst = stage;
  if (STAGED || !a.in_place) {
    const int32_t* table = STAGED ? c.pages + b * c.pages_stride : a.to_pages + b * a.to_stride;
    const int32_t p = table[tile >> (c.page_log2 - 5)];
    if (p < 0 || p >= c.n_pages) return;  // no such page: dropped
    dst = c.data + tile_at(c, p, h, tile);
  }
  if (STAGED && n == 32) {
    const int vecs = 34 * d / 16;
    for (int i = lane; i < vecs; i += 64) ((u32x4*)dst)[i] = ((const u32x4*)stage)[i];
    return;
  }
  // this lane's token `low`, as keys have it, and the four of its word of values
  const int src = low < n ? t : 0;
  const int64_t from = STAGED || low >= n ? 0 : tile_at(c, page_of(c, b, src >> 5), h, src >> 5);
  const char* const base = STAGED ? stage : c.data;
  const int at = STAGED ? low : src & 31;
  const int word = lane & 7, first = 16 * (word & 1) + 4 * (word >> 1);
  const char* v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int tok = first + k < n ? first + k : 0;
    const int64_t o = int64_t(uint32_t(__shfl(int(from), tok))) | int64_t(__shfl(int(from >> 32), tok)) << 32;
    v[k] = base + o + 16 * d + v_token_at(__shfl(at, tok)) + 32 * (lane >> 3);
  }
  const char* const k0 = base + from;
#pragma unroll 2
  for (int blk = lane >> 5; blk < db; blk += 2) {
    if (low >= n) continue;
    *(u32x4*)(dst + k_code_at(d, low, blk, 0)) = *(const u32x4*)(k0 + k_code_at(d, at, blk, 0));
    dst[k_exp_at(d, low, blk)] = k0[k_exp_at(d, at, blk)];
    dst[v_exp_at(d, low, blk)] = k0[v_exp_at(d, at, blk)];
  }
  char* const out = dst + 16 * d + 32 * (lane >> 3) + 4 * word;
  const bool full = first + 3 < n;
#pragma unroll 4
  for (int i = 0; i < 2 * db; ++i) {  // 8 of the 16 db channel pairs
    uint32_t x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = uint8_t(v[k][256 * i]);
    if (full) {
      *(uint32_t*)(out + 256 * i) = x[0] | x[1] << 8 | x[2] << 16 | x[3] << 24;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (first + k < n) out[256 * i + k] = char(x[k]);
    }
  }
}

// ------------------------------------------------------------------ launching
EvictPlan plan_evict(int64_t B, int64_t H, int64_t max_len) {
  EvictPlan p{};
  // 8 heads of 32768 tokens: 23 us by a work group each, 32 by shared ones (of 65536 50 and 32);
  // 512 heads 59 and 104 (149 and 169)
  if (max_len <= 32 * 1024) return p;
  p.chunks = int((max_len + kChunk - 1) / kChunk);
  p.counts = B * H * kHeadWords;
  return p;
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t s) {
  const int64_t heads = int64_t(a.c.B) * a.c.H;
  if (a.chunks == 0) {
    if (a.c.max_len <= 4096)
      hipLaunchKernelGGL((cache_evict_select<4>), attend_grid(heads), dim3(1024), 0, s, a);
    else if (a.c.max_len <= 16384)
      hipLaunchKernelGGL((cache_evict_select<16>), attend_grid(heads), dim3(1024), 0, s, a);
    else
      hipLaunchKernelGGL((cache_evict_select<32>), attend_grid(heads), dim3(1024), 0, s, a);
  } else {
    const int64_t words = heads * kHeadWords;
    const int per = int(std::min<int64_t>(a.chunks, std::max<int64_t>(1, (int64_t(1) << 22) / heads)));
    const dim3 grid(unsigned(heads * per));
    hipLaunchKernelGGL(cache_evict_clear, dim3(unsigned(std::min<int64_t>((words + 1023) / 1024, 1 << 16))), dim3(256), 0, s,
                       a.counts, words);
    hipLaunchKernelGGL((cache_evict_count<0>), grid, dim3(256), 0, s, a, per);
    hipLaunchKernelGGL((cache_evict_count<1>), grid, dim3(256), 0, s, a, per);
    hipLaunchKernelGGL((cache_evict_count<2>), grid, dim3(256), 0, s, a, per);
    hipLaunchKernelGGL((cache_evict_count<3>), grid, dim3(256), 0, s, a, per);
    hipLaunchKernelGGL(cache_evict_place, grid, dim3(256), 0, s, a, per);
  }
  const int tiles = a.cap > 0 ? (a.cap + 31) / 32 : 1;
  const dim3 grid = attend_grid((heads * tiles + 3) / 4);
  hipLaunchKernelGGL((cache_evict_move<false>), grid, dim3(256), 0, s, a, tiles);
  if (a.in_place) hipLaunchKernelGGL((cache_evict_move<true>), grid, dim3(256), 0, s, a, tiles);
  return hipGetLastError();
}

}  // namespace cqsa
