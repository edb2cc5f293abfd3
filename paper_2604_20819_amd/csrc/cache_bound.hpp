// Arguments of the operators that bound the 4-bit cache: the tokens' attention
// weights and eviction by them (internal).
#pragma once

#include "cache.hpp"

namespace cqsa {

// fp32 [B, H, T], a number for each cached token; strides in elements.
struct TokenWeights {
  float* p;
  int64_t b, h;
};

struct WeighArgs {
  CacheArgs c;
  CacheTensor q;
  const float* lse;       // [B, Hq, rows]
  const int32_t* counts;  // or null
  TokenWeights prior, w;  // prior.p or null
  int32_t Hq, G;
  int32_t causal;
  float scale_log2;
  float decay;
  float* part;  // with splits: [splits][B][H][max_len]
};

// How a call's rows and tokens are spread over work groups; by its sizes alone.
struct WeighPlan {
  int row_groups;  // of 16 rows, in registers; 0: the kernel for many rows
  bool resident;   // which holds them all in LDS
  int waves;       // of a work group
  int tiles;       // work groups over a sequence's tokens
  int splits;      // and over its rows
  int64_t groups;  // work groups in all
};
// rows: the most that a sequence and key head has.
WeighPlan plan_weigh(int64_t B, int64_t H, int64_t rows, int64_t max_len, cqsa_dtype dt, int d);

// The key at which a head's kept tokens end.
struct EvictBorder {
  uint32_t key;  // its digits so far
  int left;      // keys to take among those that share them
};

struct EvictArgs {
  CacheArgs c;  // the cache and the sequences as they are
  TokenWeights w, w_to;
  const int32_t* to_pages;  // not in place
  int64_t to_stride;
  bool in_place;
  int32_t budget, first, recent;
  int32_t cap;          // the most tokens that a sequence keeps
  int32_t* kept;        // [B, H, kept_stride]
  int64_t kept_stride;
  bool pad;             // -1 behind the kept tokens' positions
  int32_t* n_kept;      // [B], workspace
  int32_t* new_lengths;
  // heads that work groups share, chunk by chunk
  int chunks;           // 0: they do not
  uint32_t* counts;     // EvictPlan::counts words
  EvictBorder* state;   // [B, H, 3]
  int2* chunk_counts;   // [B, H, chunks]: keys above the border, and equal to it
  char* stage;          // in place: [B, H, ceil(cap / 32)] tiles,
  float* stage_w;       // and [B, H, cap] weights
};

hipError_t launch_cache_weigh(cqsa_dtype dt, const WeighArgs& a, const WeighPlan& p, hipStream_t s);
struct EvictPlan {
  int chunks;
  int64_t counts;
};
EvictPlan plan_evict(int64_t B, int64_t H, int64_t max_len);
hipError_t launch_cache_evict(const EvictArgs& a, hipStream_t s);

}  // namespace cqsa
