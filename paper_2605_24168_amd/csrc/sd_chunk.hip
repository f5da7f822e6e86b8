// sd_chunk.hip -- attention of several queries per sequence (chunks of a
// prompt, drafted tokens) over the positions that a window and the first
// tokens leave visible, on float32 and bfloat16 caches.
//
// Bound by the matrix unit: 4 * 128 operations per query head and visible
// position.  A workgroup takes rows of one KV head, a row being one query head
// of one token (the G heads of a token follow each other), so that grouped
// heads share every key and value tile, and short chunks still fill the tiles.
// In bfloat16 it takes 128: each of its four waves owns 32 and walks all tiles
// of 64 positions, which the workgroup stages in LDS.
//
// S = K q^T by 32x32 matrix instructions with the keys as the first operand
// leaves lane (row = lane & 31, half = lane >> 5) the scores of positions
// 8 i + 4 half + r of each 32, so that maximum and sum of a row need one
// exchange between two lanes, and the weights are the second operand of
// O^T = V^T p^T as they lie in the registers: the contraction takes the
// positions in that order, and V's operand is read in the same one, by
// transposing LDS reads (bfloat16) or rows from memory (float32).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sd_cache.hpp"
#include "sd_internal.hpp"
#include "sd_plan.hpp"

namespace sd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkRows = 128;      // rows of a workgroup
constexpr int kChunkKeys = 64;       // positions of a tile
constexpr float kChunkFloor = -1e30f;
constexpr float kChunkSlack = 8.f;

// The workgroup's rows: sequence, its first row there, rows of the sequence.
// (T * Hq rows of q fit in 31 bits, so all of these do.)
struct ChunkItem {
  int b;
  int row0;    // of the sequence's n * G rows
  int rows;    // n * G
  int start;   // the sequence's first row of q, in tokens
  int s, n;    // part, parts of what the rows see
};

// Item i of the row tiles (ROWS rows) of all sequences in order; false past the
// last.  Every wave finds it for itself: 64 sequences at a time by a prefix sum.
template <int ROWS>
__device__ __forceinline__ bool chunk_item(const WindowParams &p, int i, ChunkItem &it) {
  int before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const int b = b0 + lane_id();
    int s = 0, n = 0;
    if (b < p.batch) {
      s = (int)clamp_start(p.q_starts, b, p.n_rows);
      n = max(0, (int)clamp_start(p.q_starts, b + 1, p.n_rows) - s);
    }
    const int mine = (n * p.G + ROWS - 1) / ROWS;
    const int upto = wave_incl_scan(mine);
    const uint64_t hit = __ballot(i - before < upto);
    if (hit) {
      const int src = __ffsll((unsigned long long)hit) - 1;
      it.b = b0 + src;
      const int first = __builtin_amdgcn_readlane(upto - mine, src);
      it.row0 = (i - before - first) * ROWS;
      it.start = __builtin_amdgcn_readlane(s, src);
      it.rows = __builtin_amdgcn_readlane(n, src) * p.G;
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

__device__ __forceinline__ bf16x8 frag(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

// Four rows of one column of 16-bit values: lane i of 16 gives the address of
// row i / 4, columns 4 (i % 4) .. + 3, and gets column i of the four rows.
__device__ __forceinline__ u32x2 read_columns(const char *lds) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)lds));
}

// What rows at the positions pmin .. pmax see, as tiles of KEYS positions: those
// of the first tokens, then those of the windows.
template <int KEYS>
struct SeenTiles {
  int sink, lo;      // some row sees j < sink or j >= lo
  int na, b0, n;     // tiles of the first tokens, first one of the windows, all
  __device__ __forceinline__ SeenTiles(const WindowParams &p, int pmin, int pmax) {
    sink = min(p.n_sink, pmax + 1);
    lo = pmin + 1 > p.window ? pmin + 1 - p.window : 0;
    if (p.window == 0) lo = max(pmax + 1, 0);   // no window at all
    na = sink > 0 ? (sink + KEYS - 1) / KEYS : 0;
    b0 = lo / KEYS;
    b0 = b0 < na ? na : b0;
    const int end = p.window > 0 && pmax >= 0 ? pmax / KEYS + 1 : 0;
    n = na + (end > b0 ? end - b0 : 0);
  }
};

// What the rows [row0, row0 + ROWS) of a sequence see, and of its tiles those
// of one part, [t0, t1).
template <int ROWS, int KEYS>
struct ChunkRange {
  int L, n;          // positions, queries of the sequence
  int pmin, pmax;    // positions of the first and last row
  int sink, lo;
  int na, b0, t0, t1;
  __device__ __forceinline__ ChunkRange(const WindowParams &p, const ChunkItem &it) {
    L = __builtin_amdgcn_readfirstlane(clamp_len(p.seq_lens, it.b, p.ncap));
    n = it.rows / p.G;
    pmin = position(p, it, it.row0);
    pmax = position(p, it, it.row0 + ROWS - 1);
    const SeenTiles<KEYS> seen(p, pmin, pmax);
    sink = seen.sink;
    lo = seen.lo;
    na = seen.na;
    b0 = seen.b0;
    t0 = (int)((int64_t)seen.n * it.s / it.n);
    t1 = (int)((int64_t)seen.n * (it.s + 1) / it.n);
  }
  __device__ __forceinline__ int position(const WindowParams &p, const ChunkItem &it, int row) const {
    return L - n + (int)((uint32_t)min(row, it.rows - 1) / (uint32_t)p.G);
  }
  __device__ __forceinline__ int first_of(int t) const { return (t < na ? t : t - na + b0) * KEYS; }
};

// A row's query: where it is in q (and out), and its position.
struct ChunkRow {
  bool live;
  int pos, first;    // first: its visible first tokens
  int64_t at;        // elements
  __device__ __forceinline__ ChunkRow(const WindowParams &p, const ChunkItem &it, int row, int g, int L,
                                      int n) {
    live = row < it.rows;
    const uint32_t r = min(row, it.rows - 1);
    const int tok = (int)(r / (uint32_t)p.G), head = g * p.G + (int)(r % (uint32_t)p.G);
    pos = L - n + tok;
    first = min(p.n_sink, pos + 1);
    at = ((int64_t)(it.start + tok) * p.hq + head) * kHeadDim;
  }
};

// KV head, row tile and part of a workgroup; false: no such rows.  UNIT: tiles of
// KEYS positions in a unit of the plan, of which a part has LEAST.
template <int ROWS, int KEYS, int UNIT, int LEAST>
__device__ __forceinline__ bool chunk_place(const WindowParams &p, int &g, ChunkItem &it) {
  g = (int)(blockIdx.x % (uint32_t)p.hkv);
  const int y = p.first + (int)(blockIdx.x / (uint32_t)p.hkv);
  it.s = 0;
  it.n = 1;
  // (The last row tiles first: without a window they see the most, and what ends
  // a launch should be short: 8192 tokens over themselves 575 -> 535 us, 4096
  // 169 -> 154, float32 2048 316 -> 289.)
  if (p.plans == 0) return chunk_item<ROWS>(p, p.last - y, it);
  auto queries = [&](int b, int &start) {
    start = (int)clamp_start(p.q_starts, b, p.n_rows);
    return max(0, (int)clamp_start(p.q_starts, b + 1, p.n_rows) - start);
  };
  // (Units of the last row tile; those before see as much, or less.)
  auto units = [&](int b, int &items) {
    int start;
    const int n = queries(b, start);
    items = (n * p.G + ROWS - 1) / ROWS;
    const int L = clamp_len(p.seq_lens, b, p.ncap);
    const SeenTiles<KEYS> seen(p, L - n + max(0, items - 1) * ROWS / p.G, L - 1);
    return max(1, (seen.n + UNIT - 1) / UNIT);
  };
  Part part;
  if (!find_part(p, y, LEAST, units, part)) return false;
  it.b = part.b;
  it.row0 = part.item * ROWS;
  it.rows = queries(part.b, it.start) * p.G;
  it.rows = __builtin_amdgcn_readfirstlane(it.rows);
  it.start = __builtin_amdgcn_readfirstlane(it.start);
  it.s = part.s;
  it.n = part.n;
  return true;
}

// Where a row's partial of this part goes.  The first part leaves their number.
__device__ __forceinline__ float *chunk_part(const WindowParams &p, const ChunkItem &it, int64_t row) {
  if (it.s == 0) p.part_n[row] = it.n;
  return p.part + (row * p.nsplit + it.s) * kPartStride;
}

// ---------------------------------------------------------------------------
// float32: bound by the matrix unit, at a sixteenth of its bfloat16 rate, so
// operands come straight from global memory.  The four waves of a workgroup
// share 32 rows and take every fourth tile of 32 positions each; they join at
// the end.  Keys and values pass through the same registers: each group of
// four matrix instructions is followed by the load that refills its operand,
// values behind keys and the next tile's keys behind values, so that sixteen
// loads are always under way and each has half a tile's time to arrive.
// 1024 tokens of 32 heads over 4096 positions: 459-470 us, 128-131 TFLOP/s of the
// 154 that a large product reaches (loads left to the compiler, two under way: 561).
// ---------------------------------------------------------------------------
constexpr int kF32Rows = 32;
constexpr int kF32Keys = 32;

template <bool PAGED>
__global__ __launch_bounds__(kBlock, 2) void k_chunk_f32(WindowParams p) {
  __shared__ float lds_q[kF32Rows * kHeadDim];          // [channel / 4][row][4]
  __shared__ float lds_o[2][kF32Rows * (kHeadDim + 4)];
  __shared__ float lds_ml[kWaves][kF32Rows][2];
  int g;
  ChunkItem it;
  if (!chunk_place<kF32Rows, kF32Keys, kWaves, 1>(p, g, it)) return;
  const ChunkRange<kF32Rows, kF32Keys> cr(p, it);
  const int l = lane_id(), col = l & 31, half = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(wave_id());
  const ChunkRow row(p, it, it.row0 + col, g, cr.L, cr.n);
  for (int i = threadIdx.x >> 5; i < 32; i += kBlock / 32)   // thread: row, 16-byte chunk i
    *(f32x4 *)&lds_q[(i * 32 + col) * 4] = *(const f32x4 *)((const float *)p.q + row.at + 4 * i);
  __syncthreads();

  f32x16 acc[4];   // acc[c], register r: channel 4 (8 (r / 4) + 4 half + r % 4) + c
  float m = kChunkFloor, ls = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;

  // A tile's 32 positions lie on two pages; bad: bits of positions whose page
  // is not in the pool.
  const int step = (PAGED ? p.hkv : 1) * 512;   // bytes from row to row
  struct Where {
    int64_t at[2];    // bytes, of the first and second 16 rows
    uint32_t bad;
  };
  auto locate = [&](int j0) {
    Where x;
    x.bad = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = j0 + kTile * i;
      if (!PAGED) {
        x.at[i] = (((int64_t)it.b * p.hkv + g) * p.ncap + j) * 512;
        continue;
      }
      int page = j <= cr.pmax ? p.block_table[(int64_t)it.b * p.max_pages + (j >> 4)] : 0;
      page = __builtin_amdgcn_readfirstlane(page);
      if (page < 0 || page >= p.n_pages) {
        page = 0;
        x.bad |= 0xFFFFu << (16 * i);
      }
      x.at[i] = ((int64_t)page * kTile * p.hkv + g) * 512;
    }
    return x;
  };
  // Sixteen loads bring a wave's tile of keys, piece i (channels 8 i + 4 half ..)
  // of row col each, and sixteen its values, row 8 (i / 4) + 4 half + i % 4 at
  // channels 4 col ..  (A page has all its rows; of a contiguous cache, only
  // those up to the last position may be read.)
  auto key_row = [&](const Where &wh, int j0) {
    const int y = PAGED ? col & 15 : min(col, cr.pmax - j0);
    return p.k + (PAGED && col >= kTile ? wh.at[1] : wh.at[0]) + (int64_t)(y * step) + 16 * half;
  };
  auto value = [&](const Where &wh, int j0, int i) {
    int y = 8 * (i >> 2) + (i & 3), z = 4 * half;
    if (PAGED) {
      y &= 15;
    } else {
      const int last = cr.pmax - j0;
      y = min(y, last);
      z = min(z, last - y);
    }
    return *(const f32x4 *)(p.v + wh.at[PAGED ? i >> 3 : 0] + (int64_t)y * step +
                            (uint32_t)(z * step + 16 * col));
  };
  f32x4 x[16];   // keys, then the values, then the next tile's keys
  Where next{};
  if (cr.t0 + w < cr.t1) {
    next = locate(cr.first_of(cr.t0 + w));
    const char *src = key_row(next, cr.first_of(cr.t0 + w));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = *(const f32x4 *)(src + 32 * i);
  }
  for (int t = cr.t0 + w; t < cr.t1; t += kWaves) {
    const int j0 = cr.first_of(t), jn = cr.first_of(t + kWaves < cr.t1 ? t + kWaves : t);
    const Where now = next;
    next = locate(jn);
    f32x16 sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
    f32x4 qf = *(const f32x4 *)&lds_q[(half * 32 + col) * 4];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const f32x4 q0 = qf;
      if (i < 15) qf = *(const f32x4 *)&lds_q[((2 * i + 2 + half) * 32 + col) * 4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i][e], q0[e], sc, 0, 0, 0);
      x[i] = value(now, j0, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    // Every row sees all of the tile, or some see part of it.
    const bool whole = !now.bad && j0 + kF32Keys <= cr.pmin + 1 &&
                       (j0 + kF32Keys <= p.n_sink || cr.pmax - j0 < p.window);
    if (!whole) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int y = 8 * (r >> 2) + 4 * half + (r & 3), j = j0 + y;
        const bool sees = (j < row.first) | ((uint32_t)(row.pos - j) < (uint32_t)p.window);
        const bool there = !(now.bad >> y & 1);
        sc[r] = (sees & there) ? sc[r] : -__builtin_inff();
        // A position that no row sees weighs 0, whatever its values hold.
        if (!there || j > cr.pmax || (j >= cr.sink && j < cr.lo)) x[r] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
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
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], p.scale2, -m));
      ls += sc[r];
    }
    const char *src = key_row(next, jn);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[r][c], sc[r], acc[c], 0, 0, 0);
      x[r] = *(const f32x4 *)(src + 32 * r);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Join the waves: to the common maximum, then pairwise sums of outputs.
  ls += __shfl_xor(ls, 32);
  if (half == 0) {
    lds_ml[w][col][0] = m;
    lds_ml[w][col][1] = ls;
  }
  __syncthreads();
  float M = kChunkFloor, sum = 0.f;
#pragma unroll
  for (int x = 0; x < kWaves; ++x) M = fmaxf(M, lds_ml[x][col][0]);
#pragma unroll
  for (int x = 0; x < kWaves; ++x)
    sum += __builtin_amdgcn_exp2f(lds_ml[x][col][0] - M) * lds_ml[x][col][1];
  const float f = __builtin_amdgcn_exp2f(m - M);
  auto each = [&](auto op) {   // op(float4 at channels .., values of this wave)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int c = 4 * (8 * (r >> 2) + 4 * half + (r & 3));
      op(c, f32x4{acc[0][r], acc[1][r], acc[2][r], acc[3][r]});
    }
  };
#pragma unroll
  for (int c = 0; c < 4; ++c) acc[c] *= f;
  float *mine = &lds_o[w & 1][col * (kHeadDim + 4)];
  if (w >= 2) each([&](int c, f32x4 x) { *(f32x4 *)(mine + c) = x; });
  __syncthreads();
  if (w < 2) each([&](int c, f32x4 x) { *(f32x4 *)(mine + c) = x + *(f32x4 *)(mine + c); });
  __syncthreads();
  // Whole rows, 32 lanes each.  (Lane `col` has that row's maximum and sum.)
  const float inv = it.n > 1 ? 1.f : (sum == 0.f ? 0.f : 1.f / sum);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 2 * w + 8 * i + half;   // lanes r and r + 32 hold row r
    const float scale = __shfl(inv, r), rm = __shfl(M, r), rs = __shfl(sum, r);
    const ChunkRow to(p, it, it.row0 + r, g, cr.L, cr.n);
    if (!to.live) continue;
    const int at = r * (kHeadDim + 4) + 4 * col;
    const f32x4 y = (*(f32x4 *)&lds_o[0][at] + *(f32x4 *)&lds_o[1][at]) * scale;
    if (p.plans > 0 && it.n == 1 && col == 0) p.part_n[to.at / kHeadDim] = 1;
    if (it.n == 1) {
      *(f32x4 *)((float *)p.out + to.at + 4 * col) = y;
    } else {
      float *pp = chunk_part(p, it, to.at / kHeadDim);
      if (col == 0) {
        pp[0] = rm;
        pp[1] = rs;
      }
      *(f32x2 *)(pp + 2 + 4 * col) = f32x2{y[0], y[1]};
      *(f32x2 *)(pp + 4 + 4 * col) = f32x2{y[2], y[3]};
    }
  }
}

// ---------------------------------------------------------------------------
// bfloat16: the tiles go from memory straight into LDS, and a wave computes
// the scores of one tile while it turns those of the tile before into weights,
// so that the matrix unit and the vector unit have work at the same time.
// 6618 tokens of 32 heads over windows of 4096: 471-514 us by card and clock,
// 890-972 TFLOP/s of the 1430 that a large product reaches, with the last round of
// workgroups a quarter full (8192 tokens over windows of 16384: 1083).  The matrix
// unit is busy for 51% of the time that a compute unit has work, vector
// instructions for as long, at 1.9 GHz: the clock falls under both (float32 runs at
// 2.4).
// ---------------------------------------------------------------------------
struct ChunkStage {
  u32x4 k[2][kChunkKeys * 16];   // tiles of keys and values, by parity
  u32x4 v[2][kChunkKeys * 16];
};

// Rows that are not to be read come from here.
__device__ const u32x4 chunk_zeros[16] = {};

template <bool PAGED>
__global__ __launch_bounds__(kBlock, 2) void k_chunk_bf16(WindowParams p) {
  extern __shared__ u32x4 lds_raw[];
  ChunkStage &lds = *(ChunkStage *)lds_raw;
  int g;
  ChunkItem it;
  if (!chunk_place<kChunkRows, kChunkKeys, 1, 4>(p, g, it)) return;
  const ChunkRange<kChunkRows, kChunkKeys> cr(p, it);
  const int b = it.b;
  const int l = lane_id(), col = l & 31, half = l >> 5;
  const int w = __builtin_amdgcn_readfirstlane(wave_id());
  const ChunkRow row(p, it, it.row0 + 32 * w + col, g, cr.L, cr.n);
  u32x4 q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = *(const u32x4 *)((const uint16_t *)p.q + row.at + 16 * i + 8 * half);

  const int wmin = cr.position(p, it, it.row0 + 32 * w);
  const int wmax = cr.position(p, it, it.row0 + 32 * w + 31);

  // Pages of 16 tiles at a time, one per lane, from tile `held` on; outside: a
  // bit for each that is not in the pool.
  int pages = 0, held = -16;
  uint64_t outside = 0;
  auto hold_pages = [&](int t) {
    if (!PAGED || t < held + 16) return;
    held = t;
    const int j = cr.first_of(t + (l >> 2)) + kTile * (l & 3);
    pages = 0;
    bool ok = true;
    if (t + (l >> 2) < cr.t1 && j <= cr.pmax) {
      pages = p.block_table[(int64_t)b * p.max_pages + (j >> 4)];
      ok = pages >= 0 && pages < p.n_pages;
    }
    outside = __ballot(!ok);
  };

  f32x16 acc[4];
  float m = kChunkFloor, ls = 0.f;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[c][r] = 0.f;

  // Wave w brings rows 16 w .. 16 w + 15 of a tile (one page), four rows with
  // each instruction, whose lanes fill 1 KB of LDS in order.  Lane (row a of
  // the four, slot s) fetches the chunk of 16 bytes that belongs into slot s
  // of its row: keys are swizzled by the row, values by its last two bits, so
  // that the reads below touch every LDS bank once.
  const int a = l >> 4, s = l & 15;
  const uint32_t step = (uint32_t)(PAGED ? p.hkv : 1) * 256;   // bytes from row to row
  const uint32_t kbase = a * step + 16 * (s ^ a), vbase = a * step + 16 * (s ^ (a << 2));
  typedef __attribute__((address_space(1))) const void gvoid;
  typedef __attribute__((address_space(3))) void lvoid;
  // Where the wave's rows of tile t start, and how many of them (from the
  // first on) are in the cache.
  auto rows_at = [&](int t, int &have) -> int64_t {
    const int j = cr.first_of(t) + kTile * w;
    have = cr.pmax + 1 - j;
    if (have <= 0) return 0;
    if (!PAGED) return (((int64_t)b * p.hkv + g) * p.ncap + j) * 256;
    const int i = 4 * (t - held) + w;
    if (outside >> i & 1) {
      have = 0;
      return 0;
    }
    return ((int64_t)__builtin_amdgcn_readlane(pages, i) * kTile * p.hkv + g) * 256;
  };
  // Keys that no query of the workgroup sees are masked whatever they are, so
  // only what lies outside the cache is replaced; values are replaced
  // wherever none sees them: a weight of 0 times NaN would not be 0.
  auto bring = [&](const char *src, int have, int off, int flip, u32x4 *to, int hide0, int hide1) {
    char *dst = (char *)(to + 256 * w);
    if (have >= kTile && hide0 >= hide1) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_global_load_lds((gvoid *)(src + 4 * i * step + (off ^ (flip * i))),
                                         (lvoid *)(dst + 1024 * i), 16, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *at = src + 4 * i * step + (off ^ (flip * i));
        const int r = 4 * i + a;
        if (r >= have || (r >= hide0 && r < hide1)) at = (const char *)&chunk_zeros[s];
        __builtin_amdgcn_global_load_lds((gvoid *)at, (lvoid *)(dst + 1024 * i), 16, 0, 0);
      }
    }
  };
  auto bring_keys = [&](int t, u32x4 *to) {
    int have;
    const int64_t at = rows_at(t, have);
    bring(p.k + at, have, kbase, 64, to, 0, 0);
  };
  auto bring_values = [&](int t, u32x4 *to) {
    int have;
    const int64_t at = rows_at(t, have);
    const int j = cr.first_of(t) + kTile * w;
    bring(p.v + at, have, vbase, 0, to, max(0, cr.sink - j), min(kTile, cr.lo - j));
  };

  auto scores = [&](const u32x4 *tile, f32x16 sc[2]) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[y][r] = 0.f;
      const int krow = 32 * y + col;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        sc[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            frag(tile[krow * 16 + ((2 * i + half) ^ (krow & 15))]), frag(q[i]), sc[y], 0, 0, 0);
    }
  };
  // Masks the scores of tile t and moves the maximum if it has to.
  auto settle = [&](f32x16 sc[2], int t) {
    const int j0 = cr.first_of(t);
    const uint32_t gone = PAGED ? (uint32_t)(outside >> (4 * (t - held))) & 15u : 0u;
    const bool whole = !gone && j0 + kChunkKeys <= wmin + 1 &&
                       (j0 + kChunkKeys <= p.n_sink || wmax - j0 < p.window);
    if (!whole) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = j0 + 32 * y + 8 * (r >> 2) + 4 * half + (r & 3);
          const bool sees = (j < row.first) | ((uint32_t)(row.pos - j) < (uint32_t)p.window);
          const bool there = !(gone >> (2 * y + (r >> 3)) & 1);
          sc[y][r] = (sees & there) ? sc[y][r] : -__builtin_inff();
        }
    }
    float top = sc[0][0];
#pragma unroll
    for (int r = 1; r < 32; ++r) top = fmaxf(top, sc[r >> 4][r & 15]);
    if (__ballot(top * p.scale2 > m + kChunkSlack)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(m, top * p.scale2);
      const float f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      ls *= f;
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] *= f;
    }
  };
  // The weights round to bfloat16, as the values are: half a step, 2^-8
  // relative at most, independent from position to position.  (The products of a
  // second number for what that leaves, as the decode form has it, would take the
  // matrix unit half as long again: 487 -> 681 us for 6618 tokens of 32 heads over a
  // window of 4096.)  The sum takes the rounded weights, so that what they add to is
  // a mean of the values whatever they are off by (463 -> 473 us).
  auto add = [&](const u32x4 *tile, f32x16 sc[2]) {
    typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
    const b16x2 ones = __builtin_bit_cast(b16x2, 0x3F803F80u);
    const int i16 = l & 15, c16 = (l >> 4) & 1;
#pragma unroll
    for (int x = 0; x < 4; ++x) {   // 16 positions at a time
      uint32_t pw[4];
#pragma unroll
      for (int r = 0; r < 8; ++r)
        sc[x >> 1][8 * (x & 1) + r] =
            __builtin_amdgcn_exp2f(fmaf(sc[x >> 1][8 * (x & 1) + r], p.scale2, -m));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        pw[r] = pack2(sc[x >> 1][8 * (x & 1) + 2 * r], sc[x >> 1][8 * (x & 1) + 2 * r + 1]);
        ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b16x2, pw[r]), ones, ls, false);
      }
      const int vrow = 16 * x + 4 * half + (i16 >> 2);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int chunk = 4 * c + 2 * c16 + ((i16 & 3) >> 1);
        const char *base = (const char *)tile + 16 * (chunk ^ ((vrow & 3) << 2)) + 8 * (i16 & 1);
        const u32x2 lo4 = read_columns(base + vrow * 256), hi4 = read_columns(base + (vrow + 8) * 256);
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            frag(u32x4{lo4[0], lo4[1], hi4[0], hi4[1]}), frag(u32x4{pw[0], pw[1], pw[2], pw[3]}),
            acc[c], 0, 0, 0);
      }
    }
    // One matrix instruction, then what the vector unit can do meanwhile
    // (509 -> 499 us for 6618 tokens of 32 heads over a window of 4096).
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // matrix
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x402, 4, 0);   // vector, transcendental
    }
  };

  if (cr.t0 < cr.t1) {
    f32x16 sa[2], sb[2];
    hold_pages(cr.t0);
    bring_keys(cr.t0, lds.k[0]);
    bring_values(cr.t0, lds.v[0]);
    if (cr.t0 + 1 < cr.t1) bring_keys(cr.t0 + 1, lds.k[1]);
    __syncthreads();
    // A wave without rows only brings its share of the tiles (8 drafted tokens
    // of each of 32 sequences over 4096 positions: 118 -> 103 us).
    const bool idle = it.row0 + 32 * w >= it.rows;
    if (!idle) {
      scores(lds.k[0], sa);
      settle(sa, cr.t0);
    }
    __syncthreads();
    // Tile t's scores are in `now`: bring the tiles after it, score the next
    // one, and add this one's values.
    auto round = [&](int t, int par, f32x16 *now, f32x16 *next) {
      if (t + 1 < cr.t1) bring_values(t + 1, lds.v[par ^ 1]);
      const bool ends = PAGED && t + 2 >= held + 16;   // the held pages end before tile t + 2
      if (t + 2 < cr.t1 && !ends) bring_keys(t + 2, lds.k[par]);
      if (!idle) {
        scores(lds.k[par ^ 1], next);   // (past the last tile: of an old one, unused)
        add(lds.v[par], now);
        if (t + 1 < cr.t1) settle(next, t + 1);
      }
      if (t + 2 < cr.t1 && ends) {
        hold_pages(t + 2);
        bring_keys(t + 2, lds.k[par]);
      }
      __syncthreads();
    };
    for (int t = cr.t0; t < cr.t1; t += 2) {
      round(t, 0, sa, sb);
      if (t + 1 < cr.t1) round(t + 1, 1, sb, sa);
    }
  }

  ls += __shfl_xor(ls, 32);
  if (!row.live) return;
  if (p.plans > 0 && it.n == 1) p.part_n[row.at / kHeadDim] = 1;
  if (it.n > 1) {
    float *pp = chunk_part(p, it, row.at / kHeadDim);
    if (half == 0) {
      pp[0] = m;
      pp[1] = ls;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) pp[2 + 32 * c + 8 * (r >> 2) + 4 * half + (r & 3)] = acc[c][r];
    return;
  }
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(u32x2 *)((uint16_t *)p.out + row.at + 32 * c + 8 * i + 4 * half) =
          u32x2{pack2(acc[c][4 * i] * inv, acc[c][4 * i + 1] * inv),
                pack2(acc[c][4 * i + 2] * inv, acc[c][4 * i + 3] * inv)};
}

// Joins the parts of one row for each wave.
template <bool F32>
__global__ __launch_bounds__(kBlock) void k_chunk_merge(WindowParams p) {
  ChunkItem it;
  const int g = (int)(blockIdx.x % (uint32_t)p.hkv);
  if (!chunk_item<kWaves>(p, (int)(blockIdx.x / (uint32_t)p.hkv), it)) return;
  const int l = lane_id();
  const ChunkRow row(p, it, it.row0 + __builtin_amdgcn_readfirstlane(wave_id()), g, 0, 0);
  if (!row.live) return;
  const int64_t at = row.at / kHeadDim;
  const int n = min(__builtin_amdgcn_readfirstlane(p.part_n[at]), p.nsplit);
  if (n <= 1) return;
  const Joined v = join_splits<false>(p.part + at * p.nsplit * kPartStride, kPartStride, n);
  if (F32) *(float2 *)((float *)p.out + row.at + 2 * l) = float2{v.x, v.y};
  else *(uint32_t *)((uint16_t *)p.out + row.at + 2 * l) = pack2(v.x, v.y);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Row tiles of all sequences: at most one part-filled tile for each that has
// queries.
static int64_t chunk_tiles(const WindowParams &p, int rows) {
  return p.n_rows * p.G / rows + std::min<int64_t>(p.batch, p.n_rows);
}

// Calls with few rows cut what they see over workgroups.  In one round two
// bfloat16 workgroups run on each of the 256 compute units, or one float32
// workgroup, whose waves keep the matrix unit busy alone.  (With as many parts
// for every row tile, uneven batches take longer: 4 drafted tokens of each of 16
// sequences of 500-32K 240 instead of 176 us, 200 of each of 6 of 1-16K 222
// instead of 185, float32 16 of each of 5 of 500-8K 106 instead of 89; even ones
// are 1-5% shorter, 8 of each of 32 sequences of 4K 103 instead of 107.)
void chunk_split(WindowParams &p, int kind, size_t scratch) {
  const bool f32 = kind == kCacheF32;
  const int64_t rows = f32 ? kF32Rows : kChunkRows, round = f32 ? 256 : 512;
  const int64_t least = f32 ? kF32Keys * kWaves : 4 * kChunkKeys;   // positions of a part
  const int64_t bound = chunk_tiles(p, (int)rows);
  p.plans = 0;
  p.nsplit = 1;
  p.grid = bound * p.hkv;
  // (about as many row tiles: where sequences have less than one each, one)
  const int64_t seqs = std::min<int64_t>(p.batch, p.n_rows);
  const int64_t tiles = std::max(p.n_rows * p.G / rows + seqs / 2, seqs);
  const int64_t k0 = (tiles * p.hkv + round - 1) / round;
  const int64_t row = (int64_t)(kPartStride * sizeof(float)) * p.hq * p.n_rows;
  int64_t parts = std::min<int64_t>(p.ncap, (int64_t)p.n_sink + p.window) / least;
  parts = std::min(parts, (int64_t)scratch / (row + 4 * p.hq * p.n_rows));
  if (k0 > 2 || parts < 2 || p.batch > kPlanSeqs) return;
  // A workgroup costs 4 us beside its tiles, and its partials.
  const int64_t fill = std::min<int64_t>(rows, p.n_rows * p.G / tiles);
  p.part_cost = (int32_t)(f32 ? 16 : 32 + 112 * fill / rows);
  // A second plan of one round more than the row tiles need, to choose from where
  // sequences differ (not where all are longer than their windows, as far as the
  // width of the table tells) and have few parts in one.  (It is within 1% of the
  // first alone for 4 to 500 rows of each of 3 to 16 sequences of 1-64K; but 4 of
  // each of 16 of 500-32K, which have more than four slots a row tile, would take
  // 185 us with it instead of 177.)
  const bool more = p.batch > 1 && (int64_t)p.n_sink + p.window > p.ncap / 4;
  for (const int64_t k : {k0, k0 + 1}) {
    const int64_t slots = std::max(round * k / p.hkv, bound);
    if (k > k0 && (!more || tiles * 4 <= p.slots[0] || tiles * parts < 4 * p.slots[0])) break;
    p.slots[p.plans] = (int32_t)slots;
    p.rounds[p.plans++] = (int32_t)k;
  }
  // No cuts with fewer than two slots for a row tile (three float32 sequences of
  // 300-2049, 701 rows at most, of 8 heads over a window of 511: 60 us, cut 65).  With
  // a bound of four slots, 200 rows of each of 6 sequences of 1-16K would take 399 us
  // instead of 187, 500 of each of 2 of 8K 164 instead of 144, and 1000 of one of 32K
  // over a window of 4096 87 instead of 95.
  p.nsplit = (int32_t)parts;
  p.grid = p.slots[p.plans - 1] * (int64_t)p.hkv;
  if (p.plans > 1 || p.slots[0] >= 2 * tiles) return;
  p.plans = 0;
  p.nsplit = 1;
  p.grid = bound * p.hkv;
}

size_t chunk_part_bytes(const WindowParams &p) {
  return p.plans ? (size_t)p.n_rows * p.hq * (p.nsplit * kPartStride * sizeof(float) + sizeof(int32_t)) : 0;
}

hipError_t launch_chunk_attend(WindowParams p, int kind, bool paged, hipStream_t st) {
  const bool f32 = kind == kCacheF32;
  const int64_t slots = p.grid / p.hkv, most = kMostGroups / p.hkv;
  p.last = (int32_t)(slots - 1);
  for (int64_t first = 0; first < slots; first += most) {
    const unsigned n = (unsigned)(std::min(slots - first, most) * p.hkv);
    p.first = (int32_t)first;
    if (f32 && paged) k_chunk_f32<true><<<n, kBlock, 0, st>>>(p);
    else if (f32) k_chunk_f32<false><<<n, kBlock, 0, st>>>(p);
    else if (paged) k_chunk_bf16<true><<<n, kBlock, sizeof(ChunkStage), st>>>(p);
    else k_chunk_bf16<false><<<n, kBlock, sizeof(ChunkStage), st>>>(p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.plans == 0) return e;
  const unsigned merge = (unsigned)(chunk_tiles(p, kWaves) * p.hkv);
  if (f32) k_chunk_merge<true><<<merge, kBlock, 0, st>>>(p);
  else k_chunk_merge<false><<<merge, kBlock, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace sd
