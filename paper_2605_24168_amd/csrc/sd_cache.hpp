// sd_cache.hpp -- what the kernels of window attention, of the 4-bit cache and
// of the pages share: their parameters and host launchers.
#pragma once

#include <hip/hip_runtime.h>

#include "sd_internal.hpp"

namespace sd {

// A launch has less than 2^32 threads: work for more workgroups than this is done in
// several launches, or by several rounds of one's workgroups.
constexpr int64_t kMostGroups = 1 << 22;

// How a cache holds its rows.
enum CacheKind { kCacheF32 = 0, kCacheBf16 = 1, kCacheQ4 = 2 };

constexpr int kQ4RowBytes = kHeadDim / 2;  // codes of a row
constexpr int kQ4Group = 32;               // channels that share a scale
constexpr int kQ4Scales = kHeadDim / kQ4Group;
constexpr int kQ4MinScale = 32;            // smallest scale byte written: 2^-95
constexpr int kQ4NanScale = 255;

// Attention over the positions that windows and first tokens leave visible.
struct WindowParams {
  const void *q;               // [T, Hq, 128]
  void *out;                   // [T, Hq, 128]
  const char *k, *v;           // rows, or codes
  const uint8_t *ks, *vs;      // 4-bit caches: scale bytes
  const int32_t *block_table;  // paged: [batch, max_pages]
  const int32_t *seq_lens;     // [batch]
  const int32_t *q_starts;     // [batch + 1]; null: one query per sequence
  float *part;                 // rows of kPartStride: maximum in powers of two, sum, 128
                               // unnormalised channels of a part; packed queries: [T * Hq]
                               // [nsplit] rows, else those of one workgroup after the other
  int32_t *part_n;             // packed queries: [T * Hq] parts of a row
  int64_t ncap;                // positions addressable per sequence
  int64_t n_rows;              // T
  int32_t n_pages;             // pages of the pool
  int32_t max_pages;
  int32_t batch, hq, hkv, G;
  int32_t n_sink, window;
  float scale2;                // softmax scale times log2(e)
  int64_t grid;                // workgroups
  int32_t first, last;         // groups of KV heads' workgroups: this launch's first one, and the
                               // call's last (a call may have more than a launch holds)
  int32_t quad;                // a workgroup takes four KV heads (one query per sequence)
  int32_t nsplit;              // parts of an item that there is room for
  int32_t plans;               // ways to cut sequences to choose from (0: none is cut)
  int32_t rounds[3];           // of workgroups on all compute units, for each of them
  int32_t slots[3];            // their workgroups for each group of KV heads
  int32_t part_cost;           // of a workgroup beside its units, in sixteenths of one
  uint64_t call;               // see Counting
  int32_t bank;
};

// How the workgroups of a launch find out which of them is the last.  A counter's
// upper bits name the call that counts in it, and calls have ascending numbers, so
// that whatever another call left there counts for nothing, calls that overlapped
// against the rules included.  A captured call comes with its number again and
// again: it has the number 0 and counters of its own, one of two banks, which start
// at 0.  The calls of a graph take the banks in turn, and each of them empties the
// next one's; only the first one's takes a launch (with a launch for each call, a
// sequence with a window of 1020 takes 10.6 instead of 9.6 us).
struct Counting {
  uint64_t call;
  int bank;      // 0: not captured
  bool first;    // of its graph
  bool spoil;    // (for tests) finds what a call before it left unfinished
};
constexpr int kCountBits = 20;   // more than the workgroups that share a counter
constexpr int kBanks = 3;
__host__ __device__ constexpr int next_bank(int bank) { return 3 - bank; }   // of a captured call

// Workgroups of a call, from what the host knows: fills p.grid and what follows.
// Partials take at most `scratch` bytes; *_part_bytes: those that they take (0: no
// sequence is cut).
void window_split(WindowParams &p, int kind, bool paged, size_t scratch);
void chunk_split(WindowParams &p, int kind, size_t scratch);
size_t token_part_bytes(const WindowParams &p);
size_t chunk_part_bytes(const WindowParams &p);
hipError_t launch_token_attend(WindowParams p, int kind, bool paged, const Counting &c, hipStream_t st);
hipError_t launch_chunk_attend(WindowParams p, int kind, bool paged, hipStream_t st);

// Writing and reading a 4-bit cache.
struct Q4Params {
  uint8_t *k, *v, *ks, *vs;    // codes and scale bytes
  void *xk, *xv;               // rows [T, Hkv, 128], float32 or bfloat16
  const int32_t *block_table;
  const int32_t *seq_lens;
  const int32_t *starts;
  int64_t ncap, n_rows;
  int32_t n_pages, max_pages, batch, hkv;
  int32_t first;               // workgroup of the call that this launch begins with
};
hipError_t launch_q4_append(const Q4Params &p, bool bf16, bool paged, hipStream_t st);
hipError_t launch_q4_load(const Q4Params &p, bool bf16, bool paged, hipStream_t st);

// Pages.
constexpr int kMaxPools = 8;
struct Pools {
  char *base[kMaxPools];
  int64_t page_bytes[kMaxPools];
  int32_t n;
  int32_t align;               // largest power of two up to 16 that divides every address and size
};
struct PagesParams {
  int32_t *table, *seq_lens, *refs;
  int32_t n_pages, batch, max_pages;
};
size_t pages_work_bytes(int64_t n_pages, int64_t batch);
hipError_t launch_pages_extend(const PagesParams &p, const int32_t *grow, int32_t *status,
                               char *work, const Counting &c, hipStream_t st);
hipError_t launch_pages_fork(const PagesParams &from, const PagesParams &to,
                             const int32_t *parents, bool keep, const Pools &pools,
                             int32_t *status, char *work, const Counting &c, hipStream_t st);
hipError_t launch_pages_free(const PagesParams &p, const int32_t *rows, int64_t n, hipStream_t st);
hipError_t launch_pages_copy(const Pools &pools, int64_t n_pages, const int32_t *src,
                             const int32_t *dst, int64_t n, hipStream_t st);
hipError_t launch_pages_compact(const PagesParams &p, const Pools &pools, int32_t *remap,
                                int32_t *n_live, char *work, const Counting &c, hipStream_t st);

// Two floats rounded to bfloat16 (to nearest even), the first in the low half.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, b16x2));
}

// A row's partials joined by one wave: lane l gets channels 2l and 2l + 1 of
// the n splits at pp, `step` floats apart, divided by their sum.  Each lane takes a split's maximum
// and sum, so that their loads are under way together.
struct Joined {
  float x, y;
};
// Partials that one workgroup writes and another of the same launch reads:
// past the caches that are not common to both.
__device__ __forceinline__ void put_shared(float *at, float x) {
  __hip_atomic_store(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// One thread of each of the n workgroups that share a counter: call_counter, then
// (with what it is to hand on stored and waited for) counted_last.
__device__ __forceinline__ void call_counter(uint64_t *at, uint64_t call) {
  __hip_atomic_fetch_max(at, call << kCountBits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool counted_last(uint64_t *at, uint32_t n) {
  const uint64_t before = __hip_atomic_fetch_add(at, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return ((uint32_t)before & ((1u << kCountBits) - 1)) == n - 1;
}
template <bool SHARED>
__device__ __forceinline__ float get_partial(const float *at) {
  if (SHARED) return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return *at;
}
template <bool SHARED>
__device__ __forceinline__ Joined join_splits(const float *pp, int64_t step, int n) {
  const int l = lane_id();
  float m = -3e38f;
  for (int s = l; s < n; s += 64) m = fmaxf(m, get_partial<SHARED>(pp + s * step));
  const float M = wave_max(m);
  float sum = 0.f, x = 0.f, y = 0.f;
  for (int s0 = 0; s0 < n; s0 += 64) {
    const int s = s0 + l;
    float f = 0.f;
    if (s < n) {
      f = __builtin_amdgcn_exp2f(get_partial<SHARED>(pp + s * step) - M);
      sum += f * get_partial<SHARED>(pp + s * step + 1);
    }
    const int k = n - s0 < 64 ? n - s0 : 64;
    const float *o = pp + s0 * step + 2 + 2 * l;
    for (int i0 = 0; i0 < k; i0 += 8) {  // eight loads under way together
      float2 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t j = i0 + i < k ? i0 + i : k - 1;
        v[i] = float2{get_partial<SHARED>(o + j * step), get_partial<SHARED>(o + j * step + 1)};
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i0 + i >= k) break;   // (not a factor of zero: a split may hold an infinity)
        const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i0 + i));
        x = fmaf(fi, v[i].x, x);
        y = fmaf(fi, v[i].y, y);
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (NaN stays NaN)
  return Joined{x * inv, y * inv};
}

// Sequence length, clamped to the capacity.
__device__ __forceinline__ int clamp_len(const int32_t *seq_lens, int b, int64_t ncap) {
  int64_t L = seq_lens[b];
  L = L < 0 ? 0 : L;
  return (int)(L > ncap ? ncap : L);
}

// starts[i] of [0, batch], clamped to [0, n_rows] (null: one row each).
__device__ __forceinline__ int64_t clamp_start(const int32_t *starts, int i, int64_t n_rows) {
  if (!starts) return i;
  const int64_t s = starts[i];
  return s < 0 ? 0 : (s > n_rows ? n_rows : s);
}

}  // namespace sd
