// sd_token.hip -- attention of one query per sequence over the positions that
// a window and the first tokens leave visible, on float32, bfloat16 and 4-bit
// caches.
//
// Every cached row is used by the G query heads of its KV head only, so the
// kernel is bound by reading keys and values once: 512 bytes per position in
// bfloat16, 136 in 4 bits.
//
// A wave takes tiles of 16 positions, two at a time, straight from global
// memory into the operand registers of the matrix unit; no LDS is touched
// until the end.  With K the first operand, S = K q^T leaves lane (head =
// lane & 15, quarter = lane >> 4) the scores of positions 4 quarter + r of its
// tile, r = 0..3.  The weights p = 2^(scale (s - m)) then are, without any
// move between lanes, the second operand of O^T = V^T p^T over the two tiles,
// because the order in which a contraction runs is free: slot i of quarter a
// stands for position 4a + i of the first tile (i < 4) or 4a + i - 4 of the
// second, and V's rows are loaded in that order.
#include <hip/hip_runtime.h>

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

constexpr int kTokenWaves = 4;
constexpr int kTokenThreads = 64 * kTokenWaves;
constexpr int kUnits = 256;          // compute units of the chip
constexpr float kFloor = -1e30f;     // running maximum before the first position
constexpr float kSlack = 8.f;        // a maximum moves once a score passes it by 2^8

// Tiles of 16 positions that hold a visible position: the first `na`, then
// those from `b0` on, `n` in all.
struct TileRange {
  int L, ns, lo;   // visible: j < ns, and lo <= j < L
  int na, b0, n;
  __device__ __forceinline__ int tile(int t) const { return t < na ? t : t - na + b0; }
};

__device__ __forceinline__ TileRange tile_range(int L, int n_sink, int window) {
  TileRange r;
  r.L = L;
  r.ns = n_sink < L ? n_sink : L;
  r.lo = window < L ? L - window : 0;
  const int end = (L + kTile - 1) / kTile;
  r.na = (r.ns + kTile - 1) / kTile;
  r.b0 = r.lo / kTile;
  if (r.b0 < r.na) r.b0 = r.na;
  r.n = r.na + (end > r.b0 && r.lo < L ? end - r.b0 : 0);
  return r;
}

// One tile's keys and values in registers, per kind of cache.
template <int KIND>
struct Tile;

template <>
struct Tile<kCacheBf16> {
  u32x4 k[4], v[4];
};
template <>
struct Tile<kCacheF32> {
  u32x4 k[8], v[4][2];
};
template <>
struct Tile<kCacheQ4> {
  u32x4 k;
  uint32_t ks;
  uint32_t v[4], vs[4];
};

template <int KIND>
struct QRegs {
  u32x4 v[KIND == kCacheF32 ? 8 : 4];
};

// Query operand: lane (head, quarter a) supplies the channels that the key
// operand of the same instruction and quarter holds.
template <int KIND>
__device__ __forceinline__ void load_query(const WindowParams &p, int b, int g, QRegs<KIND> &qr) {
  const int l = lane_id(), h = l & 15, a = l >> 4;
  constexpr int n = KIND == kCacheF32 ? 8 : 4;
#pragma unroll
  for (int i = 0; i < n; ++i) qr.v[i] = u32x4{0u, 0u, 0u, 0u};
  if (h >= p.G) return;
  const int64_t row = ((int64_t)b * p.hq + (int64_t)g * p.G + h) * kHeadDim;
#pragma unroll
  for (int i = 0; i < n; ++i) {
    if (KIND == kCacheF32) qr.v[i] = *(const u32x4 *)((const float *)p.q + row + 16 * i + 4 * a);
    if (KIND == kCacheBf16) qr.v[i] = *(const u32x4 *)((const uint16_t *)p.q + row + 32 * i + 8 * a);
    if (KIND == kCacheQ4) qr.v[i] = *(const u32x4 *)((const uint16_t *)p.q + row + 32 * a + 8 * i);
  }
}

// Where a tile's rows are: the first row's index in units of rows, and the
// distance between rows (page layouts with the heads inside a row).
struct TilePlace {
  int64_t row0;
  int32_t stride;
  int32_t last;   // largest row of the tile that may be read
};

template <int KIND>
__device__ __forceinline__ void load_tile(const WindowParams &p, const TilePlace &at, Tile<KIND> &t) {
  const int l = lane_id(), m = l & 15, a = l >> 4;
  const int kr = m < at.last ? m : at.last;
  const int64_t krow = at.row0 + (int64_t)kr * at.stride;
  int64_t vrow[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int x = 4 * a + r;
    vrow[r] = at.row0 + (int64_t)(x < at.last ? x : at.last) * at.stride;
  }
  if constexpr (KIND == kCacheBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      t.k[i] = __builtin_nontemporal_load((const u32x4 *)(p.k + krow * 256 + 64 * i + 16 * a));
#pragma unroll
    for (int r = 0; r < 4; ++r)
      t.v[r] = __builtin_nontemporal_load((const u32x4 *)(p.v + vrow[r] * 256 + 16 * m));
  } else if constexpr (KIND == kCacheF32) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      t.k[i] = __builtin_nontemporal_load((const u32x4 *)(p.k + krow * 512 + 64 * i + 16 * a));
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        t.v[r][j] = __builtin_nontemporal_load((const u32x4 *)(p.v + vrow[r] * 512 + 256 * j + 16 * m));
  } else {
    t.k = __builtin_nontemporal_load((const u32x4 *)(p.k + krow * kQ4RowBytes + 16 * a));
    t.ks = (uint32_t)p.ks[krow * kQ4Scales + a];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      t.v[r] = __builtin_nontemporal_load((const uint32_t *)(p.v + vrow[r] * kQ4RowBytes + 4 * m));
      t.vs[r] = *(const uint32_t *)(p.vs + vrow[r] * kQ4Scales);
    }
  }
}

__device__ __forceinline__ uint32_t bits(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// Eight 4-bit codes as bf16 pairs, times the power of two of scale (only its
// exponent counts; 255 makes every value a NaN).
__device__ __forceinline__ void q4_values(uint32_t codes, float scale, uint32_t out[4]) {
  out[0] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  out[1] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  out[2] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  out[3] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

template <int KIND>
__device__ __forceinline__ f32x4 tile_scores(const QRegs<KIND> &q, const Tile<KIND> &t) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (KIND == kCacheF32) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t kw = t.k[i][e], qw = q.v[i][e];
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw), __uint_as_float(qw), s, 0, 0, 0);
      }
  } else if constexpr (KIND == kCacheBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(t.k[i]), as_bf16(q.v[i]), s, 0, 0, 0);
  } else {
    const float scale = __uint_as_float(t.ks << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
      q4_values(t.k[i], scale, w);
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(u32x4{w[0], w[1], w[2], w[3]}),
                                                  as_bf16(q.v[i]), s, 0, 0, 0);
    }
  }
  return s;
}

// Values of a row that is not visible become zeros: whatever it holds, NaN
// included, weighs nothing.
template <int KIND>
__device__ __forceinline__ void drop_row(Tile<KIND> &t, int r) {
  if constexpr (KIND == kCacheF32) {
    t.v[r][0] = t.v[r][1] = u32x4{0u, 0u, 0u, 0u};
  } else if constexpr (KIND == kCacheBf16) {
    t.v[r] = u32x4{0u, 0u, 0u, 0u};
  } else {
    t.v[r] = t.vs[r] = 0u;
  }
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return (uint32_t)f32_to_bf16_rne(a) | ((uint32_t)f32_to_bf16_rne(b) << 16);
}

// O^T += V^T p^T over two tiles.  acc[e] holds, in lane (head, quarter a),
// register r: channel 32 a + 8 r + e (bfloat16 and 4 bits; e = 0..7), or
// 64 (e / 4) + 16 a + 4 r + e % 4 (float32).
template <int KIND>
__device__ __forceinline__ void add_values(f32x4 acc[8], const Tile<KIND> &ta, const Tile<KIND> &tb,
                                           const float pa[4], const float pb[4]) {
  if constexpr (KIND == kCacheF32) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t x = ta.v[r][e >> 2][e & 3], y = tb.v[r][e >> 2][e & 3];
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x), pa[r], acc[e], 0, 0, 0);
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(y), pb[r], acc[e], 0, 0, 0);
      }
  } else {
    // The weights are rounded to bfloat16 (half a step, 2^-9 relative), as
    // the values are: the rounding errors of a row's weights are independent
    // and the output's own rounding is as large.
    const bf16x8 w = as_bf16(u32x4{pack_bf16(pa[0], pa[1]), pack_bf16(pa[2], pa[3]),
                                   pack_bf16(pb[0], pb[1]), pack_bf16(pb[2], pb[3])});
    uint32_t x[8][4];  // channel pairs 2d, 2d + 1 of this lane's 8 rows
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (KIND == kCacheBf16) {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          x[r][d] = ta.v[r][d];
          x[4 + r][d] = tb.v[r][d];
        }
      } else {
        const int sh = 8 * ((lane_id() & 15) >> 2);
        q4_values(ta.v[r], __uint_as_float((ta.vs[r] >> sh & 255u) << 23), x[r]);
        q4_values(tb.v[r], __uint_as_float((tb.vs[r] >> sh & 255u) << 23), x[4 + r]);
      }
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      u32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = low_halves(x[2 * i][d], x[2 * i + 1][d]);
        hi[i] = high_halves(x[2 * i][d], x[2 * i + 1][d]);
      }
      acc[2 * d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(lo), w, acc[2 * d], 0, 0, 0);
      acc[2 * d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(hi), w, acc[2 * d + 1], 0, 0, 0);
    }
  }
}

// LDS of the end of a workgroup: each wave's maxima, sums and outputs.
__host__ __device__ constexpr size_t token_lds_bytes(int G) {
  return sizeof(float) * kTokenWaves * (size_t)G * (kHeadDim + 4 + 2);
}

__device__ __forceinline__ void store_out(const WindowParams &p, int kind, int64_t at, float x) {
  if (kind == kCacheF32) ((float *)p.out)[at] = x;
  else ((uint16_t *)p.out)[at] = f32_to_bf16_rne(x);
}

// grid: splits fastest, then KV heads, then sequences.
template <int KIND, bool PAGED>
__global__ __launch_bounds__(kTokenThreads) void k_token_attend(WindowParams p) {
  extern __shared__ float lds[];
  const int s = (int)(blockIdx.x % p.nsplit);
  const int g = (int)(blockIdx.x / p.nsplit % p.hkv);
  const int b = (int)(blockIdx.x / p.nsplit / p.hkv);
  const int L = clamp_len(p.seq_lens, b, p.ncap);
  const TileRange tr = tile_range(L, p.n_sink, p.window);
  const int nsp = (tr.n + p.span - 1) / p.span;  // splits of this sequence
  if (s > 0 && s >= nsp) return;
  const int64_t orow = (int64_t)b * p.hq + (int64_t)g * p.G;
  if (nsp == 0) {
    for (int i = threadIdx.x; i < p.G * kHeadDim; i += kTokenThreads)
      store_out(p, KIND, orow * kHeadDim + i, 0.f);
    return;
  }
  const int t0 = s * p.span, t1 = min(tr.n, t0 + p.span);
  const int l = lane_id(), a = l >> 4, w = wave_id();

  QRegs<KIND> qr;
  load_query<KIND>(p, b, g, qr);

  float m = kFloor, ls = 0.f;  // of this lane's head; ls over its own positions
  f32x4 acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

  // The tile's place, and whether its positions can be seen at all.
  auto place = [&](int t, bool &ok) {
    TilePlace at;
    const int pt = tr.tile(t);
    ok = t < t1;
    if (PAGED) {
      int page = ok ? p.block_table[(int64_t)b * p.max_pages + pt] : 0;
      if (page < 0 || page >= p.n_pages) {
        page = 0;
        ok = false;
      }
      if (KIND == kCacheQ4) {
        at.row0 = ((int64_t)page * p.hkv + g) * kTile;
        at.stride = 1;
      } else {
        at.row0 = (int64_t)page * kTile * p.hkv + g;
        at.stride = p.hkv;
      }
      at.last = kTile - 1;
    } else {
      const int first = ok ? pt * kTile : 0;
      at.row0 = ((int64_t)b * p.hkv + g) * p.ncap + first;
      at.stride = 1;
      at.last = min(kTile - 1, L - 1 - first);
    }
    return at;
  };

  for (int t = t0 + 2 * w; t < t1; t += 2 * kTokenWaves) {
    Tile<KIND> tile[2];
    bool ok[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const TilePlace at = place(t + u, ok[u]);
      load_tile<KIND>(p, at, tile[u]);
    }
    float z[2][4];
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 sc = tile_scores<KIND>(qr, tile[u]);
      const int j0 = tr.tile(t + u) * kTile;
      const bool whole = ok[u] && j0 + kTile <= L && (j0 + kTile <= tr.ns || j0 >= tr.lo);
#pragma unroll
      for (int r = 0; r < 4; ++r) z[u][r] = sc[r];
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = j0 + 4 * a + r;
          const bool sees = ok[u] && j < L && (j < tr.ns || j >= tr.lo);
          if (!sees) {
            z[u][r] = -__builtin_inff();
            drop_row<KIND>(tile[u], r);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, z[u][r]);
    }
    // The maximum that weights refer to moves only when a score of the wave
    // passes it by more than the slack: weights stay below 2^8.
    if (__ballot(top * p.scale2 > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top * p.scale2);
      const float f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      ls *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= f;
    }
    float pw[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        pw[u][r] = __builtin_amdgcn_exp2f(fmaf(z[u][r], p.scale2, -m));
        ls += pw[u][r];
      }
    add_values<KIND>(acc, tile[0], tile[1], pw[0], pw[1]);
  }

  // Join the waves: per head a common maximum, scaled sums and outputs.
  ls += __shfl_xor(ls, 16);
  ls += __shfl_xor(ls, 32);
  const int h = l & 15;
  float *ml = lds, *o = lds + 2 * kTokenWaves * p.G;
  constexpr int kRow = kHeadDim + 4;  // heads start 4 banks apart
  if (h < p.G) {
    if (a == 0) {
      ml[2 * (w * p.G + h)] = m;
      ml[2 * (w * p.G + h) + 1] = ls;
    }
    float *row = o + (w * p.G + h) * kRow;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = KIND == kCacheF32 ? 64 * (e >> 2) + 16 * a + 4 * r + (e & 3) : 32 * a + 8 * r + e;
        row[c] = acc[e][r];
      }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.G * kHeadDim; i += kTokenThreads) {
    const int hh = i / kHeadDim, c = i % kHeadDim;
    float M = kFloor;
#pragma unroll
    for (int x = 0; x < kTokenWaves; ++x) M = fmaxf(M, ml[2 * (x * p.G + hh)]);
    float sum = 0.f, v = 0.f;
#pragma unroll
    for (int x = 0; x < kTokenWaves; ++x) {
      const float f = __builtin_amdgcn_exp2f(ml[2 * (x * p.G + hh)] - M);
      sum += f * ml[2 * (x * p.G + hh) + 1];
      v += f * o[(x * p.G + hh) * kRow + c];
    }
    if (nsp == 1) {
      store_out(p, KIND, (orow + hh) * kHeadDim + c, sum > 0.f ? v / sum : 0.f);
    } else {
      float *pp = p.part + ((orow + hh) * p.nsplit + s) * kPartStride;
      if (c == 0) {
        pp[0] = M;
        pp[1] = sum;
      }
      pp[2 + c] = v;
    }
  }
}

// Joins the splits of each query head: partials (maximum in powers of two,
// sum, 128 unnormalised channels).  One workgroup per query head; sequences of
// one split are done already.
__global__ __launch_bounds__(kHeadDim) void k_token_merge(WindowParams p, int kind) {
  const int64_t row = blockIdx.x;
  const int b = (int)(row / p.hq);
  const TileRange tr = tile_range(clamp_len(p.seq_lens, b, p.ncap), p.n_sink, p.window);
  const int nsp = (tr.n + p.span - 1) / p.span;
  if (nsp <= 1) return;
  const float *pp = p.part + row * p.nsplit * kPartStride;
  const int c = threadIdx.x;
  float M = kFloor;
  for (int i = 0; i < nsp; ++i) M = fmaxf(M, pp[(int64_t)i * kPartStride]);
  float sum = 0.f, v = 0.f;
  for (int i = 0; i < nsp; ++i) {
    const float *x = pp + (int64_t)i * kPartStride;
    const float f = __builtin_amdgcn_exp2f(x[0] - M);
    sum += f * x[1];
    v += f * x[2 + c];
  }
  store_out(p, kind, row * kHeadDim + c, sum > 0.f ? v / sum : 0.f);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
void window_split(WindowParams &p, int kind) {
  (void)kind;
  const int64_t cap = (p.ncap + kTile - 1) / kTile;
  int64_t tiles = ((int64_t)p.n_sink + kTile - 1) / kTile + ((int64_t)p.window + kTile - 1) / kTile + 1;
  if (tiles > cap) tiles = cap;
  if (tiles < 1) tiles = 1;
  const int64_t items = (int64_t)p.batch * p.hkv;
  const int64_t step = 2 * kTokenWaves;
  int64_t split = items > 0 ? (4LL * kUnits + items - 1) / items : 1;
  const int64_t most = (tiles + step - 1) / step;
  split = split < 1 ? 1 : (split > most ? most : split);
  int64_t span = (tiles + split - 1) / split;
  span = (span + step - 1) / step * step;
  p.span = (int32_t)span;
  p.nsplit = (int32_t)((tiles + span - 1) / span);
}

template <int KIND, bool PAGED>
static hipError_t launch_token(const WindowParams &p, hipStream_t st) {
  const int64_t grid = (int64_t)p.batch * p.hkv * p.nsplit;
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  k_token_attend<KIND, PAGED><<<(unsigned)grid, kTokenThreads, token_lds_bytes(p.G), st>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  k_token_merge<<<(unsigned)(p.batch * p.hq), kHeadDim, 0, st>>>(p, KIND);
  return hipGetLastError();
}

hipError_t launch_token_attend(const WindowParams &p, int kind, bool paged, hipStream_t st) {
  switch (kind) {
    case kCacheF32: return paged ? launch_token<kCacheF32, true>(p, st) : launch_token<kCacheF32, false>(p, st);
    case kCacheBf16: return paged ? launch_token<kCacheBf16, true>(p, st) : launch_token<kCacheBf16, false>(p, st);
    default: return paged ? launch_token<kCacheQ4, true>(p, st) : launch_token<kCacheQ4, false>(p, st);
  }
}

}  // namespace sd
