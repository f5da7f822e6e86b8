// sd_q4.hip -- writing rows into a 4-bit cache and reading them back.
//
// Both are bound by memory: 256 bytes (bfloat16) on one side of a row, 68 on
// the other, and some 10 operations per channel pair.  250K positions of 8 KV
// heads take 239 us to append and 266 to load: 5.5 and 5.0 TB/s of reads and
// writes, where a copy reaches 4.8.  Sixteen lanes take a
// row, eight channels each, so that a wave's loads and stores of four rows are
// whole runs of 1 KB and 256 bytes.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

constexpr int kQ4Rows = kBlock / 16;  // rows of a workgroup at once
// Rows of a 16-lane group.  A group with more rows has more bytes under way,
// but scatters its workgroup's writes in time: 250K positions of 8 heads take
// 261, 246, 242 and 253 us to append with 1, 2, 4 and 8 rows (contiguous
// caches 233, 235, 242, 242), and 250, 289, 290 and 293 us to load.
constexpr int kAppendRows = 2, kLoadRows = 1;

// Where packed row t lives: its sequence and position, or b < 0 for a row of
// no sequence.  (T * Hkv rows fit in 31 bits.)
struct TokenPlace {
  int b;
  int j;
};

// The packed rows [first, next) of a sequence, whose first one is at position
// j0 (below 0: before the sequence).
struct TokenRun {
  int b, first, next, j0;
  __device__ __forceinline__ bool holds(int t) const { return t >= first && t < next; }
};

// The run that row t is in; b < 0 and empty if it is in none.
__device__ __forceinline__ TokenRun token_run(const Q4Params &p, int t) {
  TokenRun r{t, t, t + 1, 0};
  if (p.starts) {  // the last sequence that starts at or before t
    int lo = 0, hi = p.batch;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (p.starts[mid] <= t) lo = mid + 1;
      else hi = mid;
    }
    r.b = lo - 1;
    if (r.b < 0) return TokenRun{-1, 0, 0, 0};
    r.first = (int)clamp_start(p.starts, r.b, p.n_rows);
    r.next = (int)clamp_start(p.starts, r.b + 1, p.n_rows);
    if (!r.holds(t)) return TokenRun{-1, 0, 0, 0};
  }
  r.j0 = clamp_len(p.seq_lens, r.b, p.ncap) - (r.next - r.first);
  return r;
}

// Row t's place; run: of the workgroup's first row, which most rows share.
__device__ __forceinline__ TokenPlace token_place(const Q4Params &p, const TokenRun &run, int t) {
  if (run.holds(t)) return TokenPlace{run.b, run.j0 + (t - run.first)};
  const TokenRun r = token_run(p, t);
  return TokenPlace{r.b, r.j0 + (t - r.first)};
}

// Row index in the cache of position j of sequence b, or -1.
template <bool PAGED>
__device__ __forceinline__ int64_t q4_row(const Q4Params &p, const TokenPlace &at, int g) {
  if (at.b < 0 || at.j < 0) return -1;
  if (!PAGED) return ((int64_t)at.b * p.hkv + g) * p.ncap + at.j;
  const int page = p.block_table[(int64_t)at.b * p.max_pages + (at.j >> 4)];
  if (page < 0 || page >= p.n_pages) return -1;
  return ((int64_t)page * p.hkv + g) * kTile + (at.j & 15);
}

// Eight channels of one row, by one lane of sixteen: their codes, and the
// scale byte of the lane's group (the same on its four lanes).
__device__ __forceinline__ void q4_encode(const float x[8], uint32_t &codes, uint32_t &scale) {
  // Largest magnitude as an integer: NaN above infinity above all numbers.
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  // With top = 1.f 2^k: 2^(k - 2), or twice that from 1.75 on, where adding
  // a quarter carries into the exponent.
  const int s = (int)((top + 0x200000u) >> 23) - 2;
  scale = top >= 0x7F800000u ? (uint32_t)kQ4NanScale : (uint32_t)max(s, kQ4MinScale);
  const float f = __uint_as_float(scale << 23);
  codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], f, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], f, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], f, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], f, 3);
  if (scale == (uint32_t)kQ4NanScale) codes = 0;
}

// Eight channels of a row as they lie in memory, and as floats.
template <bool BF16>
struct Channels {
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void *base, int64_t row, int c) {
    const u32x4 *src = BF16 ? (const u32x4 *)((const uint16_t *)base + row * kHeadDim + 8 * c)
                            : (const u32x4 *)((const float *)base + row * kHeadDim + 8 * c);
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = __builtin_nontemporal_load(src + i);
  }
  __device__ __forceinline__ void floats(float x[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const uint32_t y = w[0][i];
        x[2 * i] = bf16_to_f32(y & 0xFFFFu);
        x[2 * i + 1] = __uint_as_float(y & 0xFFFF0000u);
      } else {
        const uint32_t y = w[0][i], z = w[1][i];
        x[i] = __uint_as_float(y);
        x[4 + i] = __uint_as_float(z);
      }
    }
  }
};

// Rows of this workgroup: U per 16-lane group, kQ4Rows apart, so that the
// workgroup's are one run.  Sixteen runs that follow each other are those of one
// XCD: a head's codes and scales of neighbouring positions lie in one cache line,
// which XCDs would otherwise fetch and write each for itself (250K positions
// appended 253 -> 243 us, contiguous 242 -> 235, 64 x 1000 read back 54 -> 50;
// the longest read back from pages 252 -> 266, contiguous 273 -> 259: what is
// appended and read back once is 21 us faster contiguous and 4 us slower on pages).
constexpr uint32_t kXcdRuns = 16;
template <int U>
__device__ __forceinline__ int first_row(const Q4Params &p) {
  constexpr uint32_t n = 8 * kXcdRuns;
  uint32_t i = blockIdx.x;
  if (i < gridDim.x / n * n) i = i / n * n + i % 8 * kXcdRuns + i / 8 % kXcdRuns;
  return ((int)i + p.first) * U * kQ4Rows;
}

template <int U, bool PAGED>
__device__ __forceinline__ int64_t group_row(const Q4Params &p, const TokenRun &run, int u, int &r,
                                             TokenPlace &tp) {
  r = first_row<U>(p) + u * kQ4Rows + (int)(threadIdx.x >> 4);
  if (r >= (int)(p.n_rows * p.hkv)) {
    r = -1;
    return -1;
  }
  tp = token_place(p, run, (int)((uint32_t)r / (uint32_t)p.hkv));
  return q4_row<PAGED>(p, tp, (int)((uint32_t)r % (uint32_t)p.hkv));
}

// The rows' loads are under way before their places are looked up.
template <bool BF16, bool PAGED>
__global__ __launch_bounds__(kBlock) void k_q4_append(Q4Params p) {
  const int rows = (int)(p.n_rows * p.hkv);
  const int c = threadIdx.x & 15;
  Channels<BF16> x[kAppendRows][2];
#pragma unroll
  for (int u = 0; u < kAppendRows; ++u) {
    const int r = first_row<kAppendRows>(p) + u * kQ4Rows + (int)(threadIdx.x >> 4);
    x[u][0].load(p.xk, min(r, rows - 1), c);
    x[u][1].load(p.xv, min(r, rows - 1), c);
  }
  const TokenRun run = token_run(p, (int)((uint32_t)first_row<kAppendRows>(p) / (uint32_t)p.hkv));
#pragma unroll
  for (int u = 0; u < kAppendRows; ++u) {
    int r;
    TokenPlace tp;
    const int64_t at = group_row<kAppendRows, PAGED>(p, run, u, r, tp);
    if (at < 0) continue;  // (a row's sixteen lanes together)
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float y[8];
      x[u][w].floats(y);
      uint32_t codes, scale;
      q4_encode(y, codes, scale);
      // The row's four scale bytes in its first lane.
      scale <<= 8 * (c >> 2);
      scale |= (uint32_t)__shfl_xor((int)scale, 4);
      scale |= (uint32_t)__shfl_xor((int)scale, 8);
      *(uint32_t *)((w ? p.v : p.k) + at * kQ4RowBytes + 4 * c) = codes;
      if (c == 0) *(uint32_t *)((w ? p.vs : p.ks) + at * kQ4Scales) = scale;
    }
  }
}

template <bool BF16, bool PAGED>
__global__ __launch_bounds__(kBlock) void k_q4_load(Q4Params p) {
  const int c = threadIdx.x & 15;
  const TokenRun run = token_run(p, (int)((uint32_t)first_row<kLoadRows>(p) / (uint32_t)p.hkv));
  int r[kLoadRows];
  uint32_t codes[kLoadRows][2], scale[kLoadRows][2];
#pragma unroll
  for (int u = 0; u < kLoadRows; ++u) {
    TokenPlace tp;
    const int64_t at = group_row<kLoadRows, PAGED>(p, run, u, r[u], tp);
    if (r[u] >= 0 && tp.b < 0) r[u] = -1;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      codes[u][w] = scale[u][w] = 0u;
      if (at < 0) continue;
      codes[u][w] = *(const uint32_t *)((w ? p.v : p.k) + at * kQ4RowBytes + 4 * c);
      scale[u][w] = (w ? p.vs : p.ks)[at * kQ4Scales + (c >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < kLoadRows; ++u) {
    if (r[u] < 0) continue;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float f = __uint_as_float(scale[u][w] << 23);
      u32x4 y;
      y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[u][w], f, 0));
      y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[u][w], f, 1));
      y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[u][w], f, 2));
      y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[u][w], f, 3));
      const int64_t at = (int64_t)r[u] * kHeadDim + 8 * c;
      if (BF16) {
        __builtin_nontemporal_store(y, (u32x4 *)((uint16_t *)(w ? p.xv : p.xk) + at));
      } else {
        u32x4 *dst = (u32x4 *)((float *)(w ? p.xv : p.xk) + at);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a = y[2 * i], b = y[2 * i + 1];
          __builtin_nontemporal_store(u32x4{a << 16, a & 0xFFFF0000u, b << 16, b & 0xFFFF0000u}, dst + i);
        }
      }
    }
  }
}

template <bool APPEND>
static hipError_t launch_q4(Q4Params p, bool bf16, bool paged, hipStream_t st) {
  const int64_t per = kQ4Rows * (APPEND ? kAppendRows : kLoadRows);
  const int64_t grid = (p.n_rows * p.hkv + per - 1) / per;
  for (int64_t first = 0; first < grid; first += kMostGroups) {
    const unsigned n = (unsigned)std::min(grid - first, kMostGroups);
    p.first = (int32_t)first;
    if (APPEND) {
      if (bf16 && paged) k_q4_append<true, true><<<n, kBlock, 0, st>>>(p);
      else if (bf16) k_q4_append<true, false><<<n, kBlock, 0, st>>>(p);
      else if (paged) k_q4_append<false, true><<<n, kBlock, 0, st>>>(p);
      else k_q4_append<false, false><<<n, kBlock, 0, st>>>(p);
    } else {
      if (bf16 && paged) k_q4_load<true, true><<<n, kBlock, 0, st>>>(p);
      else if (bf16) k_q4_load<true, false><<<n, kBlock, 0, st>>>(p);
      else if (paged) k_q4_load<false, true><<<n, kBlock, 0, st>>>(p);
      else k_q4_load<false, false><<<n, kBlock, 0, st>>>(p);
    }
  }
  return hipGetLastError();
}

hipError_t launch_q4_append(const Q4Params &p, bool bf16, bool paged, hipStream_t st) {
  return launch_q4<true>(p, bf16, paged, st);
}
hipError_t launch_q4_load(const Q4Params &p, bool bf16, bool paged, hipStream_t st) {
  return launch_q4<false>(p, bf16, paged, st);
}

}  // namespace sd
