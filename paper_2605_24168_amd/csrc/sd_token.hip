// sd_token.hip -- attention of one query per sequence over the positions that
// a window and the first tokens leave visible, on float32, bfloat16 and 4-bit
// caches.
//
// Every cached row is used by the G query heads of its KV head only, so the
// kernel is bound by reading keys and values once: 512 bytes per position and
// KV head in bfloat16, 136 in 4 bits.  At 8 KV heads, 64 sequences on pages with
// a window of 4096 take 172 us (6.3 TB/s, a plain read 7.3), 16 of 128K in 4
// bits 350-359 us (6.4-6.5 TB/s), 32 with a window of 16K on pages in 4 bits 94 us (6.0);
// one sequence with a window of 1020 takes 9.6 us on the device, which are the
// latencies of lengths, table, rows and the joining of four parts.
//
// A wave takes tiles of 16 positions, two at a time, straight from global
// memory into the operand registers of the matrix unit, by buffer loads whose
// bounds are the tile's; no LDS is touched until the end.  With K the first operand, S = K q^T leaves lane (head =
// lane & 15, quarter = lane >> 4) the scores of positions 4 r + quarter of its
// tile, r = 0..3 (see row_of).  The weights p = 2^(scale (s - m)) then are, without any
// move between lanes, the second operand of O^T = V^T p^T over the two tiles,
// because the order in which a contraction runs is free: slot i of quarter a
// stands for position 4 i + a of the first tile (i < 4) or 4 (i - 4) + a of
// the second, and V's rows are loaded in that order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sd_cache.hpp"
#include "sd_internal.hpp"
#include "sd_plan.hpp"

namespace sd {

constexpr int kUnits = 256;          // compute units of the chip; a workgroup fills one
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
// operand of the same instruction and quarter holds.  TWICE: heads are 0..7, and
// again on the lanes from 8 on.
template <int KIND, bool TWICE>
__device__ __forceinline__ void load_query(const WindowParams &p, int b, int g, QRegs<KIND> &qr) {
  const int l = lane_id(), h = l & (TWICE ? 7 : 15), a = l >> 4;
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

// Lane (m = lane & 15, quarter a) reads key row row_of(m) as row m of the
// first operand, so that its scores are those of rows 4 r + a; the values of
// one instruction are then four rows in a run.
__device__ __forceinline__ int row_of(int m) { return 4 * (m & 3) + (m >> 2); }

// Byte offsets of a lane's reads from the tile's first row, `stride` rows apart.
template <int KIND>
struct Offsets {
  static constexpr int kBytes = KIND == kCacheF32 ? 512 : (KIND == kCacheBf16 ? 256 : kQ4RowBytes);
  uint32_t k, v[4], ks, vs[4];
  __device__ __forceinline__ explicit Offsets(int stride) {
    const int l = lane_id(), m = l & 15, a = l >> 4;
    const uint32_t kr = (uint32_t)(row_of(m) * stride);
    k = kr * kBytes + 16 * a;
    ks = kr * kQ4Scales + a;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t vr = (uint32_t)((4 * r + a) * stride);
      v[r] = vr * kBytes + (KIND == kCacheQ4 ? 4 : 16) * m;
      vs[r] = vr * kQ4Scales;
    }
  }
};

// Memory from `base` on, of which the first `bytes` may be read: what lies
// behind reads as zeros, without an access.
typedef __amdgpu_buffer_rsrc_t Span;
__device__ __forceinline__ Span span_of(const void *base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes, 0x00020000);
}
constexpr int kNonTemporal = 2;
__device__ __forceinline__ u32x4 load16(Span s, uint32_t at) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(s, at, 0, kNonTemporal));
}

// row0: the tile's first row, in units of rows, of which `rows` from there on
// may be read.
template <int KIND>
__device__ __forceinline__ void load_tile(const WindowParams &p, int64_t row0, int rows,
                                          const Offsets<KIND> &o, Tile<KIND> &t) {
  const Span k = span_of(p.k + row0 * o.kBytes, rows * o.kBytes);
  const Span v = span_of(p.v + row0 * o.kBytes, rows * o.kBytes);
  if constexpr (KIND == kCacheBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t.k[i] = load16(k, o.k + 64 * i);
#pragma unroll
    for (int r = 0; r < 4; ++r) t.v[r] = load16(v, o.v[r]);
  } else if constexpr (KIND == kCacheF32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) t.k[i] = load16(k, o.k + 64 * i);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < 2; ++j) t.v[r][j] = load16(v, o.v[r] + 256 * j);
  } else {
    const Span ks = span_of(p.ks + row0 * kQ4Scales, rows * kQ4Scales);
    const Span vs = span_of(p.vs + row0 * kQ4Scales, rows * kQ4Scales);
    t.k = load16(k, o.k);
    t.ks = __builtin_amdgcn_raw_buffer_load_b8(ks, o.ks, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      t.v[r] = __builtin_amdgcn_raw_buffer_load_b32(v, o.v[r], 0, kNonTemporal);
      t.vs[r] = __builtin_amdgcn_raw_buffer_load_b32(vs, o.vs[r], 0, 0);
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

__device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x),
                                                 __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
}

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
      s = mfma16(t.k[i], q.v[i], s);
  } else {
    const float scale = __uint_as_float(t.ks << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
      q4_values(t.k[i], scale, w);
      s = mfma16(u32x4{w[0], w[1], w[2], w[3]}, q.v[i], s);
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
    t.v[r] = 0u;
    t.vs[r] = 0u;
  }
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// O^T += V^T p^T over two tiles.  acc[e] holds, in lane (head, quarter a),
// register r: channel 32 a + 8 r + e (bfloat16 and 4 bits; e = 0..7), or
// 64 (e / 4) + 16 a + 4 r + e % 4 (float32).
template <int KIND, bool TWICE>
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
    // Two bfloat16 numbers hold a weight, its upper half and what that leaves, so
    // that of the output only its own rounding remains: together they are off by
    // 2^-15 of the weight at most.  (One is off by 2^-8, as much as the output's own
    // rounding, and all weights of a row may be off to one side.)  The matrix unit
    // has the time: 64 sequences of bfloat16 171 us with one and with two.  In 4
    // bits, where the vector unit is busy too, lanes from 8 on hold the second number
    // of the heads below (TWICE) instead of an instruction of its own, and both are
    // cut off (2^-14): 16 of 128K take 366 us, with rounding 372, with instructions
    // 375, and 357 with one number.
    // What is left is never zero (an infinite value times it would be a NaN).
    u32x4 w, rest;
    const bool second = !TWICE || (lane_id() & 8);
    const uint32_t mask = second ? 0xFFFF0000u : 0u;
    const float more = second ? 1.f + 0x1p-23f : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y0 = i < 2 ? pa[2 * i] : pb[2 * i - 4], y1 = i < 2 ? pa[2 * i + 1] : pb[2 * i - 3];
      const float r0 = fmaf(y0, more, -__uint_as_float(__float_as_uint(y0) & mask));
      const float r1 = fmaf(y1, more, -__uint_as_float(__float_as_uint(y1) & mask));
      if constexpr (TWICE) {
        w[i] = high_halves(__float_as_uint(r0), __float_as_uint(r1));
      } else {
        w[i] = high_halves(__float_as_uint(y0), __float_as_uint(y1));
        rest[i] = pack2(r0, r1);
      }
    }
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
        // (the group's scale byte rotated to where a float has its exponent;
        // the conversion looks at nothing else)
        const uint32_t sh = (8 * ((lane_id() & 15) >> 2) + 9) & 31;
        const uint32_t sa = ta.vs[r], sb = tb.vs[r];
        q4_values(ta.v[r], __uint_as_float(__builtin_amdgcn_alignbit(sa, sa, sh)), x[r]);
        q4_values(tb.v[r], __uint_as_float(__builtin_amdgcn_alignbit(sb, sb, sh)), x[4 + r]);
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
      acc[2 * d] = mfma16(lo, w, acc[2 * d]);
      acc[2 * d + 1] = mfma16(hi, w, acc[2 * d + 1]);
      if constexpr (!TWICE) {
        acc[2 * d] = mfma16(lo, rest, acc[2 * d]);
        acc[2 * d + 1] = mfma16(hi, rest, acc[2 * d + 1]);
      }
    }
  }
}

// LDS of the end of a workgroup: each wave's maxima, sums and outputs.
__host__ __device__ constexpr size_t token_lds_bytes(int G, int waves) {
  return sizeof(float) * waves * (size_t)G * (kHeadDim + 4 + 2);
}

template <int KIND>
__device__ __forceinline__ void store_out(const WindowParams &p, int64_t at, float x) {
  if (KIND == kCacheF32) ((float *)p.out)[at] = x;
  else ((uint16_t *)p.out)[at] = f32_to_bf16_rne(x);
}

// Parts of a (sequence, group of KV heads) that are done.
constexpr int kSplitItems = 4096;
static __device__ uint64_t splits_done[kBanks][kSplitItems];

// By all threads of a launch.
__device__ __forceinline__ void set_counters(int bank, uint64_t x) {
  const int all = (int)(gridDim.x * blockDim.x);
  for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x); i < kSplitItems; i += all)
    __hip_atomic_store(&splits_done[bank][i], x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__global__ __launch_bounds__(kBlock) void k_token_counters(int bank, uint64_t x) { set_counters(bank, x); }

// What a workgroup costs beside its tiles, in sixteenths of a step of its waves
// (131 KB of rows and 4.8 us, or 35 KB and 1.3 us in 4 bits; 4 us beside it).
static constexpr int part_cost(int kind) { return kind == kCacheQ4 ? 50 : 13; }

// grid: KV heads fastest, so that the rows of a position are read at about the
// same time, then slots.  HEADS: KV heads of a workgroup, each with NW / HEADS
// waves.  The waves of a workgroup take the steps of two tiles in turn, each
// with the loads of its next step under way while it computes.
template <int KIND, bool PAGED, int NW, int HEADS, bool TWICE>
__global__ __launch_bounds__(64 * NW, KIND == kCacheF32 ? 1 : 2) void k_token_attend(WindowParams p) {
  constexpr int NS = NW / HEADS;   // waves of a head
  extern __shared__ float lds[];
  constexpr bool kInside = PAGED && KIND != kCacheQ4;   // the heads lie inside a position
  const int l = lane_id(), a = l >> 4;
  const int w = __builtin_amdgcn_readfirstlane(wave_id()), sub = w / HEADS;
  const uint32_t groups = p.hkv / HEADS;
  const int g0 = HEADS * (int)(blockIdx.x % groups), g = g0 + w % HEADS;
  // (Cut by the table's capacity instead of a plan over all lengths, uneven
  // batches take longer: 24 contiguous sequences of 100-32K 428 instead of 290
  // us, 128 on pages of 100-16K 1073 instead of 870, 60 in 4 bits of 100-32K 314
  // instead of 219, and 3 of 64K, whose 264 parts were eight too many for one
  // round, 186 instead of 136.)
  constexpr int kStep = 2 * NS;   // tiles that the waves of a head take at once
  if (p.bank) set_counters(next_bank(p.bank), 0);
  const int y = p.first + (int)(blockIdx.x / groups);
  Part part{y, 0, 0, 1, y, INT32_MAX / kStep};
  if (p.plans > 0) {
    auto steps = [&](int i, int &items) {
      items = 1;
      const int n = tile_range(clamp_len(p.seq_lens, i, p.ncap), p.n_sink, p.window).n;
      return max(1, (n + kStep - 1) / kStep);
    };
    if (!find_part(p, y, 1, steps, part)) return;
  }
  const int b = part.b;
  const int L = __builtin_amdgcn_readfirstlane(clamp_len(p.seq_lens, b, p.ncap));
  const TileRange tr = tile_range(L, p.n_sink, p.window);
  const int64_t orow = (int64_t)b * p.hq + (int64_t)g0 * p.G;   // of the workgroup's HEADS * G rows
  const int orows = HEADS * p.G;
  if (tr.n == 0) {
    for (int i = threadIdx.x; i < orows * kHeadDim; i += 64 * NW)
      store_out<KIND>(p, orow * kHeadDim + i, 0.f);
    return;
  }
  const int t0 = part.s * part.span * kStep, t1 = min(tr.n, t0 + part.span * kStep);

  QRegs<KIND> qr;
  load_query<KIND, TWICE>(p, b, g, qr);
  const Offsets<KIND> offs(kInside ? p.hkv : 1);

  float m = kFloor, ls = 0.f;  // of this lane's head; ls over its own positions
  f32x4 acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Step i of this wave: tiles tile_of(i, 0) and the one after it.  Pages: 32
  // steps at a time, a tile per lane; outside: a bit for each that is not in
  // the pool.
  auto tile_of = [&](int i, int u) { return t0 + 2 * (i * NS + sub) + u; };
  const int steps = t0 + 2 * sub < t1 ? (t1 - t0 - 2 * sub + 2 * NS - 1) / (2 * NS) : 0;
  int pages = 0;
  uint64_t outside = 0;
  auto hold_pages = [&](int i) {
    if (!PAGED || (i & 31)) return;
    const int t = tile_of(i + (l >> 1), l & 1);
    pages = 0;
    bool ok = true;
    if (t < t1) {
      pages = p.block_table[(int64_t)b * p.max_pages + tr.tile(t)];
      ok = pages >= 0 && pages < p.n_pages;
    }
    pages = ok ? pages : 0;
    outside = __ballot(!ok);
  };
  struct Step {
    Tile<KIND> tile[2];
    bool ok[2];   // the tile is one of this part's and its page in the pool
  };
  auto load = [&](int i, Step &st) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = tile_of(i, u);
      st.ok[u] = t < t1;
      int64_t row0;
      int rows;
      if (PAGED) {
        const int slot = 2 * (i & 31) + u;
        st.ok[u] = st.ok[u] && !(outside >> slot & 1);
        const int64_t page = __builtin_amdgcn_readlane(pages, slot);
        row0 = kInside ? page * kTile * p.hkv + g : (page * p.hkv + g) * kTile;
        rows = kInside ? kTile * p.hkv - g : kTile;
      } else {
        const int first = tr.tile(t) * kTile;
        row0 = ((int64_t)b * p.hkv + g) * p.ncap + first;
        rows = min(kTile, L - first);
      }
      load_tile<KIND>(p, st.ok[u] ? row0 : 0, st.ok[u] ? rows : 0, offs, st.tile[u]);
    }
  };
  auto compute = [&](int i, Step &st) {
    float z[2][4];
    float top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 sc = tile_scores<KIND>(qr, st.tile[u]);
      const int j0 = tr.tile(tile_of(i, u)) * kTile;
      const bool whole = st.ok[u] && j0 + kTile <= L && (j0 + kTile <= tr.ns || j0 >= tr.lo);
#pragma unroll
      for (int r = 0; r < 4; ++r) z[u][r] = sc[r];
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = j0 + 4 * r + a;
          const bool sees = st.ok[u] & (j < L) & ((j < tr.ns) | (j >= tr.lo));
          if (!sees) {
            z[u][r] = -__builtin_inff();
            drop_row<KIND>(st.tile[u], r);
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
    add_values<KIND, TWICE>(acc, st.tile[0], st.tile[1], pw[0], pw[1]);
  };

  Step st[2];
  hold_pages(0);
  load(0, st[0]);
  // (Loads past the last step touch no memory, and being unconditional let the
  // waits count which ones are due.)
  if (steps == 1) compute(0, st[0]);
  for (int i = 0; steps > 1 && i < steps; i += 2) {
    hold_pages(i + 1);
    load(i + 1, st[1]);
    compute(i, st[0]);
    if (i + 1 >= steps) break;
    hold_pages(i + 2);
    load(i + 2, st[0]);
    compute(i + 1, st[1]);
  }

  uint64_t *const done = &splits_done[p.bank][part.n > 1 ? b * groups + g0 / HEADS : 0];
  if (part.n > 1 && threadIdx.x == 0) call_counter(done, p.call);

  // Join the waves: per head a common maximum, scaled sums and outputs.
  ls += __shfl_xor(ls, 16);
  ls += __shfl_xor(ls, 32);
  const int h = l & 15;
  if constexpr (TWICE) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[e][r] += __shfl_xor(acc[e][r], 8);
  }
  float *ml = lds, *o = lds + 2 * NW * p.G;
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
  for (int i = threadIdx.x; i < orows * kHeadDim; i += 64 * NW) {
    const int hh = i / kHeadDim, c = i % kHeadDim;
    // Row hh is head h of the workgroup's KV head q: in waves q, q + HEADS, ...
    const int q = HEADS == 1 ? 0 : hh / p.G, h = HEADS == 1 ? hh : hh % p.G;
    float M = kFloor;
#pragma unroll
    for (int x = 0; x < NS; ++x) M = fmaxf(M, ml[2 * ((x * HEADS + q) * p.G + h)]);
    float sum = 0.f, v = 0.f;
#pragma unroll
    for (int x = 0; x < NS; ++x) {
      const int row = (x * HEADS + q) * p.G + h;
      const float f = __builtin_amdgcn_exp2f(ml[2 * row] - M);
      sum += f * ml[2 * row + 1];
      v += f * o[row * kRow + c];
    }
    if (part.n == 1) {
      store_out<KIND>(p, (orow + hh) * kHeadDim + c, sum == 0.f ? 0.f : v / sum);
    } else {
      float *pp = p.part + ((int64_t)blockIdx.x * orows + hh) * kPartStride;
      if (c == 0) {
        put_shared(pp, M);
        put_shared(pp + 1, sum);
      }
      put_shared(pp + 2 + c, v);
    }
  }
  if (part.n == 1) return;

  // The workgroup that finishes last joins the splits, a wave per query head.
  // Each one counts itself once its partials have arrived where every compute
  // unit sees them (which fences would ensure too, by writing back and
  // emptying the L2 caches: 5 us more).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) *(uint32_t *)lds = counted_last(done, (uint32_t)part.n);
  __syncthreads();
  if (!*(volatile uint32_t *)lds) return;
  const int64_t first = (int64_t)part.first * groups + g0 / HEADS;   // the item's workgroups
  for (int hh = w; hh < orows; hh += NW) {
    const Joined v = join_splits<true>(p.part + (first * orows + hh) * kPartStride,
                                       (int64_t)groups * orows * kPartStride, part.n);
    const int64_t at = (orow + hh) * kHeadDim + 2 * l;
    store_out<KIND>(p, at, v.x);
    store_out<KIND>(p, at + 1, v.y);
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Waves of a workgroup: eight, so that one fills a compute unit; four for
// float32, whose two steps in registers leave room for one wave per SIMD.
static constexpr int token_waves(int kind) { return kind == kCacheF32 ? 4 : 8; }

// Four KV heads to a workgroup pay on bfloat16 pages, whose rows of one head
// are scattered 256-byte pieces, once there is enough to read: 64 sequences
// with a window of 4096 take 182 us instead of 204, 32 of 100-32K 376 instead
// of 468, 8 of 32K 207 instead of 224; below, the longer joins cost more (32 of
// 1K: 36 instead of 32; one of 64K: 85 instead of 59).
constexpr int64_t kQuadItems = 64;      // sequences times KV heads
constexpr int64_t kQuadTiles = 32768;   // the same times tiles

void window_split(WindowParams &p, int kind, bool paged, size_t scratch) {
  const int waves = token_waves(kind);
  const int64_t cap = (p.ncap + kTile - 1) / kTile;
  int64_t tiles = ((int64_t)p.n_sink + kTile - 1) / kTile + ((int64_t)p.window + kTile - 1) / kTile + 1;
  tiles = std::min(tiles, cap);
  const int64_t all = (int64_t)p.batch * p.hkv;
  p.quad = paged && kind == kCacheBf16 && p.hkv % 4 == 0 && all >= kQuadItems &&
           all * tiles >= kQuadTiles;
  const int heads = p.quad ? 4 : 1;
  const int64_t items = all / heads, groups = p.hkv / heads;
  const int64_t units = tiles * heads / (2 * waves);   // whole steps of a sequence, at most
  const int64_t k0 = (items + kUnits - 1) / kUnits;
  p.plans = 0;
  p.grid = items;
  p.nsplit = kPlanSeqs * kUnits;   // (parts of an item: any number has room)
  p.part_cost = part_cost(kind);
  if (units < 1 || items > kSplitItems || p.batch > kPlanSeqs) return;
  // Plans of as many rounds of workgroups as the items need, one more, and twice as
  // many, which balance better where sequences differ: 24 contiguous ones of 100-32K
  // take 401 us with the first plan alone and 341 with three, 128 on pages of 100-4K
  // 269 and 229, 60 in 4 bits of 100-32K 237 and 212 (but 64 of 100-2K 73 and 81).
  // The first alone where all are longer than their windows, as far as the width of
  // the table tells (64 on pages of 200-65K with a window of 4096: 177 us with more
  // plans, 173 without), where a sequence has four slots anyway (3 and 8 of 1-64K:
  // 80 and 275 us either way), and where there is little to do (32 of 100-1K: 25.9
  // and 23.9 us).
  const bool more = (int64_t)p.n_sink + p.window > p.ncap / 4;
  const int64_t row = (int64_t)(kPartStride * sizeof(float)) * p.G * heads;
  for (const int64_t k : {k0, k0 + 1, 2 * k0 + 1}) {
    const int64_t slots = kUnits * k / groups;
    if (slots * groups * row > (int64_t)scratch) break;
    if (k > k0 && (!more || p.batch * 4 <= p.slots[0] || p.batch * units < 8 * p.slots[0])) break;
    p.slots[p.plans] = (int32_t)slots;
    p.rounds[p.plans++] = (int32_t)k;
  }
  if (!p.plans || p.slots[p.plans - 1] <= p.batch) p.plans = 0;
  else p.grid = p.slots[p.plans - 1] * groups;
}

// Bytes of partials (0: none).
size_t token_part_bytes(const WindowParams &p) {
  if (!p.plans) return 0;
  return (size_t)p.grid * p.G * (p.quad ? 4 : 1) * kPartStride * sizeof(float);
}

// (More sequences than a launch holds are not cut: p.first is the launch's first one.)
template <int KIND, bool PAGED, int HEADS, bool TWICE = false>
static hipError_t launch_token(WindowParams p, hipStream_t st) {
  constexpr int NW = token_waves(KIND);
  const int64_t groups = p.hkv / HEADS, slots = p.grid / groups, most = kMostGroups / groups;
  for (int64_t first = 0; first < slots; first += most) {
    p.first = (int32_t)first;
    k_token_attend<KIND, PAGED, NW, HEADS, TWICE>
        <<<(unsigned)(std::min(slots - first, most) * groups), 64 * NW, token_lds_bytes(p.G, NW), st>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_token_attend(WindowParams p, int kind, bool paged, const Counting &c, hipStream_t st) {
  p.call = c.call;
  p.bank = c.bank;
  const auto set = [&](int bank, uint64_t x) {
    k_token_counters<<<kSplitItems / kBlock, kBlock, 0, st>>>(bank, x);
  };
  if (c.spoil && c.bank == 0) set(0, ((c.call - 1) << kCountBits) + 1);
  if (c.spoil && c.first) set(1, 1), set(2, 1);
  if (c.first) set(c.bank, 0);
  if (p.quad) return launch_token<kCacheBf16, true, 4>(p, st);
  switch (kind) {
    case kCacheF32: return paged ? launch_token<kCacheF32, true, 1>(p, st) : launch_token<kCacheF32, false, 1>(p, st);
    case kCacheBf16: return paged ? launch_token<kCacheBf16, true, 1>(p, st) : launch_token<kCacheBf16, false, 1>(p, st);
  }
  if (p.G <= 8)
    return paged ? launch_token<kCacheQ4, true, 1, true>(p, st) : launch_token<kCacheQ4, false, 1, true>(p, st);
  return paged ? launch_token<kCacheQ4, true, 1>(p, st) : launch_token<kCacheQ4, false, 1>(p, st);
}

}  // namespace sd
