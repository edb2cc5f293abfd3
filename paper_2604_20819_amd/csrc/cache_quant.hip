// Writing keys and values into the 4-bit cache, and reading them back (gfx950).
//
// A block's power comes from its largest magnitude's fp32 bits by integer
// operations, (bits + 2^21) >> 23, which is the exponent or, from 1.75 times its
// power on, the next one; codes are v_cvt_scalef32_pk_fp4_f32's (to nearest
// even, ending at 6), values v_cvt_scalef32_pk_f32_fp4's, which are exact.
//
// Both kernels move bytes: 4 d of 16-bit rows and 34 d / 32 of cache a token and
// head.  A work group takes a tile of 32 tokens of as many heads as make 256
// elements, a thread 8 elements of 4 consecutive tokens: its row accesses are
// 16 bytes beside its neighbours', four lanes hold a block, and the 4 x 4 bytes
// of codes that it has turn from tokens to channel pairs (V's order) in 8
// byte permutations.  The tile's image passes through LDS, so that the cache is
// read and written in whole lines.
#include "cache.hpp"
#include "hip_common.hpp"

namespace cqsa {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

// 8 elements of a row.
template <typename T>
struct Row8 {
  static constexpr int N = sizeof(T) / 2;  // vectors of 16 bytes
  u32x4 v[N];
};
template <typename T>
__device__ __forceinline__ Row8<T> load_row(const T* p) {
  Row8<T> r;
#pragma unroll
  for (int i = 0; i < Row8<T>::N; ++i) r.v[i] = ((const u32x4*)p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ float element(const Row8<T>& r, int i) {
  if constexpr (sizeof(T) == 4) {
    const uint32_t x = r.v[i / 4][i % 4];  // a copy: the cast of a vector's element takes its first
    return __builtin_bit_cast(float, x);
  }
  const uint32_t w = r.v[0][i / 2];
  if constexpr (__is_same(T, __bf16)) return __builtin_bit_cast(float, i % 2 ? w & 0xffff0000u : w << 16);
  return float(__builtin_bit_cast(_Float16, uint16_t(i % 2 ? w >> 16 : w)));
}

__device__ __forceinline__ uint32_t max_of_four(uint32_t x) {  // over lanes 4 k .. 4 k + 3
  uint32_t y = __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true);
  x = y > x ? y : x;
  y = __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true);
  return y > x ? y : x;
}

// 8 codes, and the exponent byte of the block that four lanes hold.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const Row8<T>& r, uint32_t* exponent) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __builtin_bit_cast(uint32_t, element(r, i)) & 0x7fffffffu;
    top = m > top ? m : top;
  }
  top = max_of_four(top);
  const uint32_t up = (top + 0x200000u) >> 23;
  const uint32_t e = up <= 2 ? 0 : (up - 2 < kMaxExponent ? up - 2 : kMaxExponent);
  const float scale = __builtin_bit_cast(float, e << 23);  // its exponent alone is used
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, element(r, 0), element(r, 1), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, element(r, 2), element(r, 3), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, element(r, 4), element(r, 5), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, element(r, 6), element(r, 7), scale, 3);
  const bool finite = top < 0x7f800000u;  // else an infinity or a NaN
  *exponent = finite ? e : kNanExponent;
  return finite ? w : 0u;
}

// 8 values of a code word into a row.
template <typename T>
__device__ __forceinline__ void store_row(T* p, uint32_t w, uint32_t e) {
  const float scale = __builtin_bit_cast(float, e << 23);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  if constexpr (sizeof(T) == 4) {
    ((f32x4*)p)[0] = f32x4{a[0], a[1], b[0], b[1]};
    ((f32x4*)p)[1] = f32x4{c[0], c[1], d[0], d[1]};
  } else {
    typedef __attribute__((__vector_size__(16))) T vec;
    // neighbouring lanes write whole lines, which go past the caches (a prompt of
    // 262144 tokens written and read: 243 us, 270 through them)
    const vec y = vec{T(a[0]), T(a[1]), T(b[0]), T(b[1]), T(c[0]), T(c[1]), T(d[0]), T(d[1])};
    __builtin_nontemporal_store(y, (vec*)p);
  }
}

// Byte j of word i becomes byte i of word j.
__device__ __forceinline__ void transpose4(uint32_t* w) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);  // 0.0 1.0 0.1 1.1
  const uint32_t b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);  // 0.2 1.2 0.3 1.3
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

constexpr int kGroupElems = 256;  // elements of the heads of a work group, at most
__host__ __device__ constexpr int heads_of_group(int d) { return kGroupElems / d; }

}  // namespace

// Work groups: head group fastest, then the part of the sequence's tiles, then
// the sequence.
template <typename T, int DB, bool WRITE>
__global__ void __launch_bounds__(256) cache_move_kernel(const CacheMoveArgs a, int head_groups, int per_seq) {
  const CacheArgs& c = a.c;
  constexpr int D = 32 * DB, HW = heads_of_group(D);
  constexpr int bytes = 34 * D;  // of a tile
  const int tid = threadIdx.x;
  __shared__ __attribute__((aligned(16))) char image[34 * kGroupElems];
  const int hg = blockIdx.x % head_groups, part = blockIdx.x / head_groups % per_seq;
  const int b = blockIdx.x / (head_groups * per_seq);
  const Seq s = sequence(c, b);
  if (s.n == 0) return;
  const int first = s.len - s.n;  // position of row 0, negative where the first rows have none
  const int h0 = hg * HW, heads = c.H - h0 < HW ? c.H - h0 : HW;
  constexpr int chunks = HW * D / 8;  // 8-element pieces of a token's heads
  const int quad = tid / chunks, chunk = tid % chunks;
  const int h = chunk * 8 / D, e = chunk * 8 % D, blk = e / 32, sub = e / 8 % 4;
  const bool active = quad < 8 && h < heads;
  const int64_t tb = c.q_start ? 0 : b;
  char* const at = image + h * bytes;
  const int kcode = blk * 512 + 4 * quad * 16 + 4 * sub;
  const int vcode = 16 * D + blk * 512 + 4 * sub * 32 + v_token_at(4 * quad);

  for (int t = (first >> 5) + part; 32 * t < s.len; t += per_seq) {
    if (WRITE && t < 0) continue;
    const int64_t page = t < 0 ? -1 : page_of(c, b, t);
    const int p0 = 32 * t + 4 * quad;  // the thread's first token
    const int row = p0 - first;        // and its row
    T* kp = (T*)a.k.p + tb * a.k.b + int64_t(s.row0 + row) * a.k.l + (h0 + h) * a.k.h + e;
    T* vp = (T*)a.v.p + tb * a.v.b + int64_t(s.row0 + row) * a.v.l + (h0 + h) * a.v.h + e;
    char* cache = c.data + (page < 0 ? 0 : tile_at(c, page, h0, t));
    const int64_t next_head = int64_t(bytes) << (c.page_log2 - 5);
    const bool whole = 32 * t >= first && 32 * t + 32 <= s.len;
    if (WRITE) {
      Row8<T> k[4], v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (active && row + j >= 0 && row + j < s.n) {
          k[j] = load_row(kp + j * a.k.l);
          v[j] = load_row(vp + j * a.v.l);
        } else {
          k[j] = v[j] = Row8<T>{};
        }
      if (page < 0) continue;  // here: the rows do not wait for the page
      uint32_t kw[4], ke[4], vw[4], ve[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kw[j] = quantise8(k[j], &ke[j]);
        vw[j] = quantise8(v[j], &ve[j]);
      }
      if (whole) {
        transpose4(vw);
        if (active) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            *(uint32_t*)(at + kcode + 16 * j) = kw[j];
            *(uint32_t*)(at + vcode + 32 * j) = vw[j];
          }
          if (sub == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) at[k_exp_at(D, 4 * quad + j, blk)] = char(ke[j]);
            *(uint32_t*)(at + v_exp_at(D, 4 * quad, blk)) = ve[0] | ve[1] << 8 | ve[2] << 16 | ve[3] << 24;
          }
        }
        __syncthreads();
        const int vecs = bytes / 16;
        for (int i = tid; i < heads * vecs; i += 256) {
          const int g = i / vecs, o = i % vecs * 16;
          *(u32x4*)(cache + g * next_head + o) = *(const u32x4*)(image + g * bytes + o);
        }
        __syncthreads();
      } else if (active) {
        // the other tokens of the tile keep their bytes
        char* dst = cache + h * next_head;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (row + j >= 0 && row + j < s.n) {
            *(uint32_t*)(dst + kcode + 16 * j) = kw[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[vcode + 32 * i + j] = char(vw[j] >> (8 * i));
            if (sub == 0) {
              dst[k_exp_at(D, 4 * quad + j, blk)] = char(ke[j]);
              dst[v_exp_at(D, 4 * quad, blk) + j] = char(ve[j]);
            }
          }
      }
    } else {
      const int vecs = bytes / 16;
      for (int i = tid; i < heads * vecs; i += 256) {
        const int g = i / vecs, o = i % vecs * 16;
        // no page: zeros
        *(u32x4*)(image + g * bytes + o) =
            page < 0 ? u32x4{0u, 0u, 0u, 0u} : *(const u32x4*)(cache + g * next_head + o);
      }
      __syncthreads();
      if (active) {
        uint32_t vw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) vw[j] = *(const uint32_t*)(at + vcode + 32 * j);
        transpose4(vw);
        const uint32_t ve = *(const uint32_t*)(at + v_exp_at(D, 4 * quad, blk));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (row + j >= 0 && row + j < s.n) {
            store_row(kp + j * a.k.l, *(const uint32_t*)(at + kcode + 16 * j),
                      uint8_t(at[k_exp_at(D, 4 * quad + j, blk)]));
            store_row(vp + j * a.v.l, vw[j], (ve >> (8 * j)) & 255u);
          }
      }
      __syncthreads();
    }
  }
}

namespace {

template <typename T, bool WRITE>
void launch_rows(const CacheMoveArgs& a, const dim3& grid, int groups, int per, hipStream_t s) {
  switch (a.c.d / 32) {
#define CQSA_MOVE(DB)                                                                                  \
  case DB:                                                                                             \
    hipLaunchKernelGGL((cache_move_kernel<T, DB, WRITE>), grid, dim3(256), 0, s, a, groups, per);      \
    break;
    CQSA_MOVE(1)
    CQSA_MOVE(2)
    CQSA_MOVE(3)
    CQSA_MOVE(4)
    CQSA_MOVE(5)
    CQSA_MOVE(6)
    CQSA_MOVE(7)
    CQSA_MOVE(8)
#undef CQSA_MOVE
  }
}

template <bool WRITE>
hipError_t launch_move(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  // tiles that a sequence's rows may touch
  const int64_t n = a.c.q_start ? a.c.max_q : a.c.rows;
  const int hw = heads_of_group(a.c.d), groups = (a.c.H + hw - 1) / hw;
  int64_t per = n == 1 ? 1 : (n + 30) / 32 + 1;
  // a work group for each (a prompt of 262144 tokens: 270 us; 16 times fewer groups, 287)
  const int64_t most = (int64_t(1) << 23) / (int64_t(a.c.B) * groups);
  if (per > most) per = most;  // B and the heads are at most 2^23 together
  const dim3 grid(unsigned(per * a.c.B * groups));
  if (dt == CQSA_BF16)
    launch_rows<__bf16, WRITE>(a, grid, groups, int(per), s);
  else if (dt == CQSA_F16)
    launch_rows<_Float16, WRITE>(a, grid, groups, int(per), s);
  else
    launch_rows<float, WRITE>(a, grid, groups, int(per), s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  return launch_move<true>(dt, a, s);
}
hipError_t launch_cache_read(cqsa_dtype dt, const CacheMoveArgs& a, hipStream_t s) {
  return launch_move<false>(dt, a, s);
}

}  // namespace cqsa
