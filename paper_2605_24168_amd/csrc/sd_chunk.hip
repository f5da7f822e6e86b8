// sd_chunk.hip -- attention of several queries per sequence (chunks of a
// prompt, drafted tokens) over the positions that a window and the first
// tokens leave visible, on float32 and bfloat16 caches.
//
// Bound by the matrix unit: 4 * 128 operations per query head and visible
// position.  A workgroup takes 128 rows of one KV head, a row being one query
// head of one token (the G heads of a token follow each other), so that
// grouped heads share every key and value tile, and short chunks still fill
// the tiles.  Each of its four waves owns 32 rows and walks all tiles of 64
// positions, which the workgroup stages in LDS.
//
// S = K q^T by 32x32 matrix instructions with the keys as the first operand
// leaves lane (row = lane & 31, half = lane >> 5) the scores of positions
// 8 i + 4 half + r of each 32, so that maximum and sum of a row need one
// exchange between two lanes, and the weights are the second operand of
// O^T = V^T p^T as they lie in the registers: the contraction takes the
// positions in that order, and V's operand is read in the same one, by
// transposing LDS reads (bfloat16) or plain ones (float32).
#include <hip/hip_runtime.h>

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkRows = 128;      // rows of a workgroup
constexpr int kChunkKeys = 64;       // positions of a tile
constexpr float kChunkFloor = -1e30f;
constexpr float kChunkSlack = 8.f;

// The workgroup's rows: sequence, its first row there, rows of the sequence.
struct ChunkItem {
  int b;
  int64_t row0;    // of the sequence's n * G rows
  int64_t rows;    // n * G
  int64_t start;   // the sequence's first row of q, in tokens
};

// Item i of the row tiles of all sequences in order; false past the last.
// Every wave finds it for itself: 64 sequences at a time by a prefix sum.
__device__ __forceinline__ bool chunk_item(const WindowParams &p, int64_t i, ChunkItem &it) {
  int64_t before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const int b = b0 + lane_id();
    int64_t s = 0, n = 0;
    if (b < p.batch) {
      s = clamp_start(p.q_starts, b, p.n_rows);
      n = clamp_start(p.q_starts, b + 1, p.n_rows) - s;
      n = n < 0 ? 0 : n;
    }
    const int mine = (int)((n * p.G + kChunkRows - 1) / kChunkRows);
    const int upto = wave_incl_scan(mine);
    const int64_t end = before + upto;
    const uint64_t hit = __ballot(i < end);
    if (hit) {
      const int src = __ffsll((unsigned long long)hit) - 1;
      it.b = b0 + src;
      const int first = __shfl(upto - mine, src);
      it.row0 = (i - before - first) * kChunkRows;
      it.start = __shfl((int)s, src);
      it.rows = (int64_t)__shfl((int)n, src) * p.G;
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

template <int KIND>
struct ChunkLds {
  static constexpr int kRowBytes = KIND == kCacheF32 ? 512 : 256;
  u32x4 k[kChunkKeys * kRowBytes / 16];
  u32x4 v[kChunkKeys * kRowBytes / 16];
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return (uint32_t)f32_to_bf16_rne(a) | ((uint32_t)f32_to_bf16_rne(b) << 16);
}
__device__ __forceinline__ bf16x8 frag(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

// Four rows of one column of 16-bit values: lane i of 16 gives the address of
// row i / 4, columns 4 (i % 4) .. + 3, and gets column i of the four rows.
__device__ __forceinline__ u32x2 read_columns(const char *lds) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lds));
}

template <int KIND, bool PAGED>
__global__ __launch_bounds__(kBlock) void k_chunk_attend(WindowParams p) {
  constexpr bool F32 = KIND == kCacheF32;
  constexpr int kRowBytes = ChunkLds<KIND>::kRowBytes;
  constexpr int kChunks = kRowBytes / 16;            // 16-byte chunks per row
  constexpr int kLoads = kChunkKeys * kChunks / kBlock;  // per thread and tile
  constexpr int kRowsPerLoad = kBlock / kChunks;
  extern __shared__ u32x4 lds_raw[];
  ChunkLds<KIND> &lds = *(ChunkLds<KIND> *)lds_raw;

  const int g = (int)(blockIdx.x % p.hkv);
  ChunkItem it;
  if (!chunk_item(p, blockIdx.x / p.hkv, it)) return;
  const int b = it.b;
  const int L = clamp_len(p.seq_lens, b, p.ncap);
  const int n = (int)(it.rows / p.G);
  const int l = lane_id(), w = wave_id(), col = l & 31, half = l >> 5;

  // This lane's row: its token's position and where its query is.
  const int64_t row = it.row0 + 32 * w + col;
  const bool live = row < it.rows;
  const int tok = (int)((live ? row : it.rows - 1) / p.G);
  const int head = g * p.G + (int)((live ? row : it.rows - 1) % p.G);
  const int pos = L - n + tok;
  const int64_t qat = ((it.start + tok) * p.hq + head) * kHeadDim;

  // Positions of the workgroup's first and last token.
  const int64_t rlast = min(it.row0 + kChunkRows, it.rows) - 1;
  const int pmin = L - n + (int)(it.row0 / p.G), pmax = L - n + (int)(rlast / p.G);

  u32x4 q[F32 ? 16 : 8];
#pragma unroll
  for (int i = 0; i < (F32 ? 16 : 8); ++i) {
    if (F32) q[i] = *(const u32x4 *)((const float *)p.q + qat + 8 * i + 4 * half);
    else q[i] = *(const u32x4 *)((const uint16_t *)p.q + qat + 16 * i + 8 * half);
  }

  f32x16 acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;
  float m = kChunkFloor, ls = 0.f;

  // Tiles: those of the first tokens, then those of the windows.
  const int sink = min(p.n_sink, pmax + 1);
  const int lo = pmin + 1 > p.window ? pmin + 1 - p.window : 0;  // first position of a window
  const int na = sink > 0 ? (sink + kChunkKeys - 1) / kChunkKeys : 0;
  int b0 = lo / kChunkKeys;
  b0 = b0 < na ? na : b0;
  const int end = p.window > 0 && pmax >= 0 ? pmax / kChunkKeys + 1 : 0;
  const int nt = na + (end > b0 ? end - b0 : 0);
  const int lrow = threadIdx.x / kChunks, lchunk = threadIdx.x % kChunks;

  for (int t = 0; t < nt; ++t) {
    const int j0 = (t < na ? t : t - na + b0) * kChunkKeys;
    // Stage the tile.  Rows that none of the workgroup's queries sees become
    // zeros: a weight of 0 times whatever they hold must stay 0.
    uint64_t gone = 0;  // positions on pages outside the pool, by 16
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsPerLoad + lrow, j = j0 + r;
      bool ok = j <= pmax && (j < sink || j >= lo);
      int64_t at = 0;
      if (PAGED) {
        int page = -1;
        if (j <= pmax) page = p.block_table[(int64_t)b * p.max_pages + (j >> 4)];
        ok = ok && page >= 0 && page < p.n_pages;
        at = ((int64_t)page * kTile + (j & 15)) * p.hkv + g;
      } else {
        at = ((int64_t)b * p.hkv + g) * p.ncap + j;
      }
      u32x4 kv = {0u, 0u, 0u, 0u}, vv = {0u, 0u, 0u, 0u};
      if (ok) {
        kv = *(const u32x4 *)(p.k + at * kRowBytes + 16 * lchunk);
        vv = *(const u32x4 *)(p.v + at * kRowBytes + 16 * lchunk);
      }
      if (F32) {
        lds.k[r * kChunks + (lchunk ^ (r & 15))] = kv;
        lds.v[r * kChunks + lchunk] = vv;
      } else {
        lds.k[r * kChunks + (lchunk ^ (r & 15))] = kv;
        lds.v[r * kChunks + (lchunk ^ ((r & 3) << 2))] = vv;
      }
    }
    if (PAGED) {  // which of the tile's pages are not in the pool
#pragma unroll
      for (int i = 0; i < kChunkKeys / kTile; ++i) {
        const int j = j0 + kTile * i;
        int page = -1;
        if (j <= pmax) page = p.block_table[(int64_t)b * p.max_pages + (j >> 4)];
        if (page < 0 || page >= p.n_pages) gone |= 1ull << i;
      }
    }
    __syncthreads();

    f32x16 sc[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[x][r] = 0.f;
      const int kr = 32 * x + col;
#pragma unroll
      for (int i = 0; i < (F32 ? 16 : 8); ++i) {
        const u32x4 kf = lds.k[kr * kChunks + ((2 * i + half) ^ (kr & 15))];
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t kw = kf[e], qw = q[i][e];
            sc[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kw), __uint_as_float(qw),
                                                         sc[x], 0, 0, 0);
          }
        } else {
          sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(kf), frag(q[i]), sc[x], 0, 0, 0);
        }
      }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = j0 + 32 * x + 8 * (r >> 2) + 4 * half + (r & 3);
        const bool sees = j <= pos && (j < p.n_sink || pos - j < p.window) &&
                          !(gone >> (2 * x + (r >> 3)) & 1);
        sc[x][r] = sees ? sc[x][r] : -__builtin_inff();
        top = fmaxf(top, sc[x][r]);
      }
    if (__ballot(top * p.scale2 > m + kChunkSlack)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top * p.scale2);
      const float f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      ls *= f;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= f;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[x][r] = __builtin_amdgcn_exp2f(fmaf(sc[x][r], p.scale2, -m));
        ls += sc[x][r];
      }
    // O^T += V^T p^T.
    if constexpr (F32) {
      const float *v = (const float *)lds.v;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int vr = 32 * x + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
          for (int c = 0; c < 4; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[vr * kHeadDim + 32 * c + col], sc[x][r],
                                                          acc[c], 0, 0, 0);
        }
    } else {
      // (weights round to bfloat16, as the values are: half a step, 2^-9)
      const int i16 = l & 15, c16 = (l >> 4) & 1;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const f32x16 &ss = sc[s >> 1];
        const int r0 = 8 * (s & 1);
        const u32x4 pw = {pack2(ss[r0], ss[r0 + 1]), pack2(ss[r0 + 2], ss[r0 + 3]),
                          pack2(ss[r0 + 4], ss[r0 + 5]), pack2(ss[r0 + 6], ss[r0 + 7])};
        const int vr = 16 * s + 4 * half + (i16 >> 2);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int chunk = 4 * c + 2 * c16 + ((i16 & 3) >> 1);
          const char *base = (const char *)lds.v + 16 * (chunk ^ ((vr & 3) << 2)) + 8 * (i16 & 1);
          const u32x2 x = read_columns(base + vr * 256), y = read_columns(base + (vr + 8) * 256);
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(u32x4{x[0], x[1], y[0], y[1]}),
                                                           frag(pw), acc[c], 0, 0, 0);
        }
      }
    }
    __syncthreads();
  }

  ls += __shfl_xor(ls, 32);
  if (!live) return;
  const float inv = ls > 0.f ? 1.f / ls : 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = qat + 32 * c + 8 * i + 4 * half;
      const float x0 = acc[c][4 * i] * inv, x1 = acc[c][4 * i + 1] * inv;
      const float x2 = acc[c][4 * i + 2] * inv, x3 = acc[c][4 * i + 3] * inv;
      if (F32) *(f32x4 *)((float *)p.out + at) = f32x4{x0, x1, x2, x3};
      else *(u32x2 *)((uint16_t *)p.out + at) = u32x2{pack2(x0, x1), pack2(x2, x3)};
    }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
template <int KIND, bool PAGED>
static hipError_t launch_chunk(const WindowParams &p, hipStream_t st) {
  // Row tiles of all sequences: at most one part-filled tile for each.
  const int64_t tiles = p.n_rows * p.G / kChunkRows + p.batch;
  const int64_t grid = tiles * p.hkv;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  k_chunk_attend<KIND, PAGED><<<(unsigned)grid, kBlock, sizeof(ChunkLds<KIND>), st>>>(p);
  return hipGetLastError();
}

hipError_t launch_chunk_attend(const WindowParams &p, int kind, bool paged, hipStream_t st) {
  if (kind == kCacheF32) return paged ? launch_chunk<kCacheF32, true>(p, st) : launch_chunk<kCacheF32, false>(p, st);
  return paged ? launch_chunk<kCacheBf16, true>(p, st) : launch_chunk<kCacheBf16, false>(p, st);
}

}  // namespace sd
