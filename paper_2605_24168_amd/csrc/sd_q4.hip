// sd_q4.hip -- writing rows into a 4-bit cache and reading them back.
//
// Both are bound by memory: 256 bytes (bfloat16) on one side of a row, 68 on
// the other, and some 10 operations per channel pair.  Sixteen lanes take a
// row, eight channels each, so that a wave's loads and stores of four rows are
// whole runs of 1 KB and 256 bytes.
#include <hip/hip_runtime.h>

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

constexpr int kQ4Rows = kBlock / 16;  // rows of a workgroup at once
constexpr int kQ4Unroll = 4;          // rows of a 16-lane group

// Where packed row t lives: its sequence and position, or b < 0 for a row of
// no sequence.
struct TokenPlace {
  int b;
  int64_t j;
};

__device__ __forceinline__ TokenPlace token_place(const Q4Params &p, int64_t t) {
  TokenPlace r;
  int64_t first = t, n = 1;
  r.b = (int)t;
  r.j = -1;
  if (p.starts) {  // the last sequence that starts at or before t
    int lo = 0, hi = p.batch;  // starts[lo - 1] <= t < starts[hi + 1], if they are ascending
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (p.starts[mid] <= t) lo = mid + 1;
      else hi = mid;
    }
    r.b = lo - 1;
    if (r.b < 0) return r;
    first = clamp_start(p.starts, r.b, p.n_rows);
    n = clamp_start(p.starts, r.b + 1, p.n_rows) - first;
    if (t - first >= n) {
      r.b = -1;
      return r;
    }
  }
  const int L = clamp_len(p.seq_lens, r.b, p.ncap);
  r.j = L - n + (t - first);
  return r;
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

template <bool BF16>
__device__ __forceinline__ void load_channels(const void *base, int64_t row, int c, float x[8]) {
  if (BF16) {
    const u32x4 w = __builtin_nontemporal_load((const u32x4 *)((const uint16_t *)base + row * kHeadDim + 8 * c));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t y = w[i];
      x[2 * i] = bf16_to_f32(y & 0xFFFFu);
      x[2 * i + 1] = __uint_as_float(y & 0xFFFF0000u);
    }
  } else {
    const f32x4 *src = (const f32x4 *)((const float *)base + row * kHeadDim + 8 * c);
    const f32x4 u = __builtin_nontemporal_load(src), v = __builtin_nontemporal_load(src + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = u[i];
      x[4 + i] = v[i];
    }
  }
}

template <bool BF16, bool PAGED>
__global__ __launch_bounds__(kBlock) void k_q4_append(Q4Params p) {
  const int64_t rows = p.n_rows * p.hkv;
  const int c = threadIdx.x & 15;
#pragma unroll 1
  for (int u = 0; u < kQ4Unroll; ++u) {
    const int64_t r = ((int64_t)blockIdx.x * kQ4Unroll + u) * kQ4Rows + (threadIdx.x >> 4);
    if (r >= rows) return;  // (a row's sixteen lanes leave together)
    const int64_t t = r / p.hkv;
    const int64_t at = q4_row<PAGED>(p, token_place(p, t), (int)(r % p.hkv));
    if (at < 0) continue;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float x[8];
      load_channels<BF16>(w ? p.xv : p.xk, r, c, x);
      uint32_t codes, scale;
      q4_encode(x, codes, scale);
      *(uint32_t *)((w ? p.v : p.k) + at * kQ4RowBytes + 4 * c) = codes;
      if ((c & 3) == 0) (w ? p.vs : p.ks)[at * kQ4Scales + (c >> 2)] = (uint8_t)scale;
    }
  }
}

template <bool BF16, bool PAGED>
__global__ __launch_bounds__(kBlock) void k_q4_load(Q4Params p) {
  const int64_t rows = p.n_rows * p.hkv;
  const int c = threadIdx.x & 15;
#pragma unroll 1
  for (int u = 0; u < kQ4Unroll; ++u) {
    const int64_t r = ((int64_t)blockIdx.x * kQ4Unroll + u) * kQ4Rows + (threadIdx.x >> 4);
    if (r >= rows) return;
    const TokenPlace tp = token_place(p, r / p.hkv);
    if (tp.b < 0) continue;
    const int64_t at = q4_row<PAGED>(p, tp, (int)(r % p.hkv));
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      u32x4 y = {0u, 0u, 0u, 0u};
      if (at >= 0) {
        const uint32_t codes = *(const uint32_t *)((w ? p.v : p.k) + at * kQ4RowBytes + 4 * c);
        const uint32_t scale = (w ? p.vs : p.ks)[at * kQ4Scales + (c >> 2)];
        const float f = __uint_as_float(scale << 23);
        y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 0));
        y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 1));
        y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 2));
        y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, f, 3));
      }
      if (BF16) {
        *(u32x4 *)((uint16_t *)(w ? p.xv : p.xk) + r * kHeadDim + 8 * c) = y;
      } else {
        u32x4 *dst = (u32x4 *)((float *)(w ? p.xv : p.xk) + r * kHeadDim + 8 * c);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a = y[2 * i], b = y[2 * i + 1];
          dst[i] = u32x4{a << 16, a & 0xFFFF0000u, b << 16, b & 0xFFFF0000u};
        }
      }
    }
  }
}

template <bool APPEND>
static hipError_t launch_q4(const Q4Params &p, bool bf16, bool paged, hipStream_t st) {
  const int64_t per = kQ4Rows * kQ4Unroll;
  const int64_t grid = (p.n_rows * p.hkv + per - 1) / per;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  if (grid == 0) return hipSuccess;
  const unsigned n = (unsigned)grid;
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
  return hipGetLastError();
}

hipError_t launch_q4_append(const Q4Params &p, bool bf16, bool paged, hipStream_t st) {
  return launch_q4<true>(p, bf16, paged, st);
}
hipError_t launch_q4_load(const Q4Params &p, bool bf16, bool paged, hipStream_t st) {
  return launch_q4<false>(p, bf16, paged, st);
}

}  // namespace sd
