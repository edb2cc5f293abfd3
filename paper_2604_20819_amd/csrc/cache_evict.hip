// Eviction from the 4-bit cache: which tokens a sequence's heads keep, and their
// moving together (gfx950).
//
// A token's rank is a 32-bit key: 0 where its page holds nothing, 1 for a NaN, the
// weight's bits in an order that integers compare by, and 2^32 - 1 for the first and
// the recent tokens.  The n-th largest key is found by its digits, from counts of
// the keys that share its upper ones.
#include "cache_bound.hpp"
#include "hip_common.hpp"

namespace cqsa {

namespace {

constexpr uint32_t kForced = 0xffffffffu;

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

__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, const float* w, int b, int len, int t) {
  if (t >= len || page_of(a.c, b, t >> 5) < 0) return 0u;
  return t < a.first || t >= len - a.recent ? kForced : rank_of(w[t]);
}

}  // namespace

// One work group a sequence and head.
__global__ void __launch_bounds__(1024) cache_evict_select(const EvictArgs a) {
  __shared__ uint32_t count[256];
  __shared__ uint32_t found[2];
  __shared__ int per_wave[2][16];
  const int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int h = id % a.c.H, b = id / a.c.H;
  if (b >= a.c.B) return;  // the grid has two dimensions
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = length_of(a.c, b);
  const float* w = a.w.p + b * a.w.b + h * a.w.h;
  uint32_t prefix = 0, left = 0;  // the border's upper digits; keys still to find at it
  int keep = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    uint32_t absent = 0;
    for (int t = tid; t < len; t += 1024) {
      const uint32_t k = key_of(a, w, b, len, t);
      absent += k == 0u;
      if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&count[k >> shift & 255u], 1u);
    }
    if (shift == 24) {
      if (tid == 0) found[0] = 0;
      __syncthreads();
      if (absent) atomicAdd(&found[0], absent);
      __syncthreads();
      const int present = len - int(found[0]);
      keep = present < a.budget ? present : a.budget;
      left = uint32_t(keep);
    }
    __syncthreads();
    if (tid == 0) {
      uint32_t above = 0;
      int d = 255;
      while (d > 0 && above + count[d] < left) above += count[d--];
      found[0] = uint32_t(d), found[1] = above;
    }
    __syncthreads();
    prefix = prefix << 8 | found[0];
    left -= found[1];
    __syncthreads();
  }
  if (keep == 0) prefix = kForced, left = 0;
  // keys above the border are kept, and the first `left` that equal it
  int32_t* kept = a.kept + (int64_t(b) * a.c.H + h) * a.kept_stride;
  int done = 0, ties = 0;
  for (int t0 = 0; t0 < len; t0 += 1024) {
    const int t = t0 + tid;
    const uint32_t k = key_of(a, w, b, len, t);
    const uint64_t above = __builtin_amdgcn_ballot_w64(k > prefix), equal = __builtin_amdgcn_ballot_w64(k == prefix && k != 0u);
    if (lane == 0) per_wave[0][wave] = __builtin_popcountll(above), per_wave[1][wave] = __builtin_popcountll(equal);
    __syncthreads();
    int n0 = done, n1 = ties, all0 = 0, all1 = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) n0 += per_wave[0][i], n1 += per_wave[1][i];
      all0 += per_wave[0][i], all1 += per_wave[1][i];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    n0 += __builtin_popcountll(above & below), n1 += __builtin_popcountll(equal & below);
    const int lim = int(left);
    const bool mine = k > prefix || (k == prefix && k != 0u && n1 < lim);
    if (mine) kept[n0 + (n1 < lim ? n1 : lim)] = t;
    done += all0, ties += all1;
    __syncthreads();
  }
  if (a.pad)
    for (int i = keep + tid; i < a.budget; i += 1024) kept[i] = -1;
  if (h == 0 && tid == 0) a.n_kept[b] = keep;
}

// A work group for each 32 kept tokens.  STAGED: from the stage into the pages, in
// their places; else from the pages into the stage (in place) or the target's pages.
template <bool STAGED>
__global__ void __launch_bounds__(256) cache_evict_move(const EvictArgs a, int tiles) {
  __shared__ const char* from[32];
  __shared__ int at[32];
  const CacheArgs& c = a.c;
  const int d = c.d, db = d >> 5, tid = threadIdx.x;
  const int id = (blockIdx.y << kGridLog2) + blockIdx.x;
  const int tile = id % tiles;
  const int64_t bh = id / tiles;
  const int h = int(bh % c.H), b = int(bh / c.H);
  if (b >= c.B) return;  // the grid has two dimensions
  const int keep = a.n_kept[b];
  if (h == 0 && tile == 0 && tid == 0 && (STAGED || !a.in_place)) a.new_lengths[b] = keep;
  const int n = keep - 32 * tile < 32 ? keep - 32 * tile : 32;
  if (n <= 0) return;
  const int32_t* kept = a.kept + bh * a.kept_stride + 32 * tile;
  char* const stage = a.stage + (bh * tiles + tile) * tile_bytes(d);
  // where the tile goes
  char* dst = stage;
  if (STAGED || !a.in_place) {
    const int32_t* table = STAGED ? c.pages + b * c.pages_stride : a.to_pages + b * a.to_stride;
    const int32_t p = table[tile >> (c.page_log2 - 5)];
    dst = p >= 0 && p < c.n_pages ? c.data + tile_at(c, p, h, tile) : nullptr;
  }
  if (tid < 32) {
    const int t = tid < n ? kept[tid] : 0;
    from[tid] = STAGED ? stage : tid < n ? c.data + tile_at(c, page_of(c, b, t >> 5), h, t >> 5) : nullptr;
    at[tid] = STAGED ? tid : t & 31;
    if (tid < n) {
      const int64_t i = bh * a.cap + 32 * tile + tid;
      if (STAGED)
        a.w.p[b * a.w.b + h * a.w.h + 32 * tile + tid] = a.stage_w[i];
      else if (a.in_place)
        a.stage_w[i] = a.w.p[b * a.w.b + h * a.w.h + t];
      else if (a.w_to.p)
        a.w_to.p[b * a.w_to.b + h * a.w_to.h + 32 * tile + tid] = a.w.p[b * a.w.b + h * a.w.h + t];
    }
  }
  __syncthreads();
  if (!dst) return;
  for (int u = tid; u < 32 * db; u += 256) {  // keys' codes: a token's block
    const int tok = u & 31, blk = u >> 5;
    if (tok < n) *(u32x4*)(dst + k_code_at(d, tok, blk, 0)) = *(const u32x4*)(from[tok] + k_code_at(d, at[tok], blk, 0));
  }
  for (int u = tid; u < 16 * d; u += 256) {  // values' codes: a token's channel pair
    const int tok = u & 31, i = u >> 5;  // i: 16 blk + pair
    if (tok < n) dst[v_code_at(d, tok, i >> 4, i & 15)] = from[tok][v_code_at(d, at[tok], i >> 4, i & 15)];
  }
  for (int u = tid; u < d; u += 256) {
    const int tok = u & 31, blk = u >> 5;
    if (tok < n) {
      dst[k_exp_at(d, tok, blk)] = from[tok][k_exp_at(d, at[tok], blk)];
      dst[v_exp_at(d, tok, blk)] = from[tok][v_exp_at(d, at[tok], blk)];
    }
  }
}

hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t s) {
  const int64_t heads = int64_t(a.c.B) * a.c.H;
  hipLaunchKernelGGL(cache_evict_select, attend_grid(heads), dim3(1024), 0, s, a);
  const int tiles = a.cap > 0 ? (a.cap + 31) / 32 : 1;
  const dim3 grid = attend_grid(heads * tiles);
  hipLaunchKernelGGL((cache_evict_move<false>), grid, dim3(256), 0, s, a, tiles);
  if (a.in_place) hipLaunchKernelGGL((cache_evict_move<true>), grid, dim3(256), 0, s, a, tiles);
  return hipGetLastError();
}

}  // namespace cqsa
