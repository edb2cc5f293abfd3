// The 4-bit key-value cache: layout, arguments and device helpers shared by its
// kernels (internal; the format is in cqsa.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cqsa.h"

namespace cqsa {

constexpr int kCacheTile = 32;   // tokens of a tile
constexpr int kMxBlock = 32;  // elements that share an exponent
constexpr uint32_t kMaxExponent = 252;  // of 2^125: 6 times it is the last finite value
constexpr uint32_t kNanExponent = 255;

constexpr int64_t tile_bytes(int d) { return 34 * int64_t(d); }

// Sequences and cache of a call, as the kernels see them.
struct CacheArgs {
  char* data;
  const int32_t* pages;
  const int32_t* lengths;
  const int32_t* q_start;  // or null
  int64_t n_pages;
  int64_t pages_stride;
  int64_t page_bytes;
  int32_t page_log2;  // log2 of the page's tokens
  int32_t H, d;
  int32_t B;
  int32_t max_len, max_q;
  int32_t rows;       // L of the tensors: rows a sequence, or T when packed
};

struct CacheTensor {
  void* p;
  int64_t b, l, h;  // strides in elements
};

struct CacheMoveArgs {
  CacheArgs c;
  CacheTensor k, v;
};

struct AttendArgs {
  CacheArgs c;
  CacheTensor q, o;
  float* lse;        // [B, Hq, rows] or null
  int32_t Hq, G;     // query heads, and of them for each head of the cache
  int32_t causal;
  float scale_log2;  // softmax scale * log2(e)
  // with splits: every row's (by its place in LSE) and split's unnormalised
  // result, its shift (log2) and sum
  float* part;
  float* part_ml;
};

// How a call's rows and tokens are spread over work groups; by its sizes alone.
struct AttendPlan {
  int row_groups;  // of 16 rows, for each wave; 0: cache_attend_many
  int waves;       // of a work group for few rows: 4, or as many as fill a CU
  int row_tiles;   // work groups over a sequence's and head's rows
  int splits;      // work groups over a sequence's tokens
  int min_chunk;   // tiles that a split takes at least
};
// rows: the most that a sequence and key head has.
AttendPlan plan_attend(int64_t B, int64_t H, int64_t rows, int64_t max_len, cqsa_dtype dt, int d);

// Tiles of 16 rows that a call may have; it is split only where they do not fill the
// GPU, so that its work groups count in 32 bits.
constexpr int64_t kMaxGroups = int64_t(1) << 27;
// They lie over two dimensions of the grid, the first 2^21 wide where there is a second,
// since one has fewer than 2^32 threads.
constexpr int kGridLog2 = 21;
inline dim3 attend_grid(int64_t groups) {
  const int64_t x = int64_t(1) << kGridLog2;
  return groups <= x ? dim3(unsigned(groups)) : dim3(unsigned(x), unsigned((groups + x - 1) / x));
}

// The kernel for many rows (of 16 bits): rows of a work group, 32 a wave, with two
// waves on a SIMD where their registers fit or all but 13 do (bf16 at d = 256 spills
// 13 of them and takes 0.53 ms, with 4 waves 0.81; fp16 at d = 192 13 and 0.63 ms,
// 0.93; at d = 224 47 and 1.00 to 1.02 ms, but 0.23 to 0.13 where sequences have 128
// rows); tokens of a tile (64 KB of LDS for two of them); launch.
constexpr int attend_many_rows(bool f16, int d) { return f16 && d > 192 ? 128 : 256; }
constexpr int attend_many_tokens(int d) { return d <= 128 ? 64 : 32; }
hipError_t launch_attend_many(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s);

hipError_t launch_cache_write(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s);
hipError_t launch_cache_read(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s);
hipError_t launch_cache_attend(cqsa_dtype dt, const AttendArgs& a, const AttendPlan& p, hipStream_t s);

#ifdef __HIPCC__

// One sequence's rows and tokens, from clamped device values: n rows from row0
// of the packed tensors (0 with one sequence a batch element), whose first sits
// at position len - n.
struct Seq {
  int32_t row0, n, len;
};
__device__ __forceinline__ Seq sequence(const CacheArgs& c, int b) {
  Seq s;
  int32_t len = c.lengths[b];
  len = len < 0 ? 0 : len;
  s.len = len > c.max_len ? c.max_len : len;
  if (c.q_start) {
    int32_t lo = c.q_start[b], hi = c.q_start[b + 1];
    lo = lo < 0 ? 0 : (lo > c.rows ? c.rows : lo);
    hi = hi < lo ? lo : (hi > c.rows ? c.rows : hi);
    s.row0 = lo;
    s.n = hi - lo < c.max_q ? hi - lo : c.max_q;
  } else {
    s.row0 = 0;
    s.n = c.rows;
  }
  return s;
}

// Page of the 32 tokens from token 32 t of sequence b, or -1.  The token lies
// below max_len, so the entry is in the table.
__device__ __forceinline__ int64_t page_of(const CacheArgs& c, int b, int32_t t) {
  const int32_t p = c.pages[b * c.pages_stride + (t >> (c.page_log2 - 5))];
  return uint32_t(p) < uint64_t(c.n_pages) && p >= 0 ? p : -1;
}
// Byte offset of head h's tile t of a sequence in its page.
__device__ __forceinline__ int64_t tile_at(const CacheArgs& c, int64_t page, int h, int32_t t) {
  const int per = c.page_log2 - 5;
  return page * c.page_bytes + ((int64_t(h) << per) + (t & ((1 << per) - 1))) * tile_bytes(c.d);
}

// Offsets in a tile of token t (< 32), block b (d / 32 of them), code byte i (< 16).
__device__ __forceinline__ int k_code_at(int d, int t, int b, int i) { return b * 512 + t * 16 + i; }
__device__ __forceinline__ int v_token_at(int t) {
  return ((t >> 2) & 3) * 8 + (t >> 4) * 4 + (t & 3);
}
__device__ __forceinline__ int v_code_at(int d, int t, int b, int i) {
  return 16 * d + b * 512 + i * 32 + v_token_at(t);
}
__device__ __forceinline__ int k_exp_at(int d, int t, int b) {
  return 32 * d + (t & 15) * (d >> 4) + 2 * b + (t >> 4);
}
__device__ __forceinline__ int v_exp_at(int d, int t, int b) {
  return 33 * d + ((t >> 2) & 3) * (d >> 2) + b * 8 + (t >> 4) * 4 + (t & 3);
}

#endif

}  // namespace cqsa
