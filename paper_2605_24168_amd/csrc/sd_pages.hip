// sd_pages.hip -- the pages of a paged cache: extending and freeing rows of a
// block table, forking rows, copying pages, and moving live pages together.
//
// The tables and counts are small, so these are bound by launches and by the
// latency of a few dependent reads (256 rows of 262144 pages: 4 us to free 64 of
// them, 12 us to extend them; a step of beam search over 32 x 4 rows: 21 us on
// the device); only the copies move bytes that matter (4096 pages of twice 32 KB:
// 106 us, 5.0 TB/s read and written; 16384 moved together: 455 us, 4.7 TB/s).
// Free pages are taken lowest first, which makes results independent of the
// order of workgroups: a first kernel counts the free pages of every stretch
// of the pool, and the workgroup that finishes last turns counts and requests
// into ranks; the next one hands the free pages out by rank.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

constexpr int kPlan = 1024;                       // threads that count and plan
// Consecutive pages of a thread: fewer make more workgroups, of which each finds
// fewer rows, but which count themselves one after the other (256 rows of 262144
// pages extended: 14.7, 11.8 and 12.8 us with 4, 2 and 1).
constexpr int kPerThread = 2;
constexpr int kStretch = kPlan * kPerThread;      // pages counted by one workgroup
// Pools of at most this many pages are handed out (or listed) by the workgroup
// that plans, stretch after stretch; larger ones by the stretches' workgroups of
// a second launch.  (2000 pages moved together in 26 us a call instead of 30,
// 8192 in 27 instead of 30, but 16384 in 41 instead of 34; rows of 8032 pages
// freed and extended in 15.5 instead of 18.)
constexpr int kOneLaunch = 4 * kStretch;
constexpr int64_t kPiece = 16 * 1024;             // bytes a workgroup copies at once
constexpr int kMany = 1 << 29;                    // more than any number of pages

// Scratch of one call (all int32).
struct PageWork {
  int32_t *base;      // [stretches]: counts, then the free (or live) pages before each
  int32_t *scalar;    // [8]: see kLimit ...
  int32_t *first;     // [batch]: extend: rank of the row's first page
  int32_t *have;      // [batch]: extend: pages it held; fork: children of a parent
  int32_t *eldest;    // [batch]: fork: a parent's first child
  int32_t *list;      // [pages / 2]: compact: movers; fork: a child's own last page
  int32_t *hole;      // [pages / 2]: compact: holes; fork: [0, batch) a child's rank among those
                      // that get a page, [batch, ..) the page that it copies
  uint64_t call;      // see Counting
  int32_t bank;
};
enum { kLimit = 0, kMoves = 1, kLive = 2 };

static inline int64_t stretches(int64_t n_pages) { return (n_pages + kStretch - 1) / kStretch; }

static inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

static size_t carve_pages(int64_t n_pages, int64_t batch, char *base, PageWork *w) {
  size_t at = 0;
  auto take = [&](int64_t n) {
    char *ptr = base ? base + at : nullptr;
    at += up256(4 * (size_t)n);
    return (int32_t *)ptr;
  };
  PageWork x;
  x.base = take(stretches(n_pages) + 1);
  x.scalar = take(8);
  x.first = take(batch);
  x.have = take(batch);
  x.eldest = take(batch);
  x.list = take(std::max(n_pages / 2, batch));
  x.hole = take(std::max(n_pages / 2, 2 * batch));
  if (w) *w = x;
  return at;
}

size_t pages_work_bytes(int64_t n_pages, int64_t batch) {
  return carve_pages(n_pages, batch, nullptr, nullptr);
}

__device__ __forceinline__ int row_len(const PagesParams &p, int b) {
  return clamp_len(p.seq_lens, b, (int64_t)p.max_pages * kTile);
}
__device__ __forceinline__ bool in_pool(const PagesParams &p, int page) {
  return page >= 0 && page < p.n_pages;
}

// This thread's pages of stretch `s`: a bit for each that is free (or live).
template <bool LIVE>
__device__ __forceinline__ uint32_t stretch_bits(const PagesParams &p, int s) {
  const int64_t i0 = (int64_t)s * kStretch + threadIdx.x * kPerThread;
  int x[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) x[i] = i0 + i < p.n_pages ? p.refs[i0 + i] : (LIVE ? 0 : 1);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) m |= (LIVE ? x[i] > 0 : x[i] == 0) ? 1u << i : 0u;
  return m;
}

// Workgroups of the counting launch that are done.
static __device__ uint64_t stretches_done[kBanks];

__device__ __forceinline__ void set_counter(int bank, uint64_t x) {
  __hip_atomic_store(&stretches_done[bank], x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__global__ void k_pages_counter(int bank, uint64_t x) { set_counter(bank, x); }

// Counts this workgroup's stretch; true for the workgroup that counts last,
// which finds all counts in w.base.  (They are stored past the caches that
// workgroups do not share, and have arrived before a workgroup counts itself.)
template <bool LIVE>
__device__ __forceinline__ bool count_stretch(const PagesParams &p, const PageWork &w, int *tmp) {
  __shared__ bool last;
  int total;
  uint64_t *const done = &stretches_done[w.bank];
  if (threadIdx.x == 0) {
    call_counter(done, w.call);
    if (w.bank && blockIdx.x == 0) set_counter(next_bank(w.bank), 0);
  }
  block_excl_scan<kPlan>(__popc(stretch_bits<LIVE>(p, blockIdx.x)), tmp, &total);
  if (threadIdx.x == 0) {
    __hip_atomic_store(&w.base[blockIdx.x], total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = counted_last(done, gridDim.x);
  }
  __syncthreads();
  return last;
}

// Counts of the launch's stretches to the pages before each; returns all of
// them.
__device__ __forceinline__ int plan_bases(const PageWork &w, int *tmp) {
  const int n = (int)gridDim.x;
  int before = 0;
  for (int i0 = 0; i0 < n; i0 += kPlan) {
    const int i = i0 + threadIdx.x;
    const int c = i < n ? __hip_atomic_load(&w.base[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    int total;
    const int x = block_excl_scan<kPlan>(c, tmp, &total);
    if (i < n) w.base[i] = before + x;
    before += total;
  }
  return before;
}

// ---------------------------------------------------------------------------
// extend
// ---------------------------------------------------------------------------
// Rows that get pages are those whose ranks end at or below the limit; their
// ranks ascend, so a free page finds its row by bisection, in LDS where the
// rows' first ranks fit (256 rows, 262144 pages: 7.7 instead of 10.6 us, with
// four pages a thread).
constexpr int kRowsLds = 4096;

// Hands out the free pages of stretch s, the first of which has rank `base`.
__device__ __forceinline__ void take_stretch(const PagesParams &p, const PageWork &w, int s, int base,
                                             int limit, int *tmp, const int *first_lds) {
  const bool local = p.batch <= kRowsLds;
  const uint32_t mine = stretch_bits<false>(p, s);
  int total;
  int rank = base + block_excl_scan<kPlan>(__popc(mine), tmp, &total);  // (also a barrier)
  for (uint32_t m = mine; m && rank < limit; m &= m - 1, ++rank) {
    const int page = s * kStretch + threadIdx.x * kPerThread + __ffs(m) - 1;
    int lo = 0, hi = p.batch;  // first row whose ranks start past this one
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if ((local ? first_lds[mid] : w.first[mid]) <= rank) lo = mid + 1;
      else hi = mid;
    }
    const int b = lo - 1;
    p.table[(int64_t)b * p.max_pages + w.have[b] + rank - (local ? first_lds[b] : w.first[b])] = page;
    p.refs[page] = 1;
  }
}

__global__ __launch_bounds__(kPlan) void k_extend_plan(PagesParams p, PageWork w,
                                                       const int32_t *grow, int32_t *status) {
  __shared__ int tmp[kPlan / 64];
  __shared__ int limit;
  __shared__ int first_lds[kRowsLds];
  if (!count_stretch<false>(p, w, tmp)) return;
  const int nfree = plan_bases(w, tmp);
  if (threadIdx.x == 0) limit = 0;
  __syncthreads();
  int before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kPlan) {
    const int b = b0 + threadIdx.x;
    int need = 0, have = 0;
    int64_t L = 0;
    bool fits = true;
    if (b < p.batch) {
      L = row_len(p, b);
      have = (int)((L + kTile - 1) / kTile);
      const int64_t g = grow[b];
      L += g > 0 ? g : 0;
      const int64_t want = (L + kTile - 1) / kTile;
      fits = want <= p.max_pages;
      need = fits ? (int)want - have : 0;
    }
    int total;
    const int first = before + block_excl_scan<kPlan>(need, tmp, &total);
    if (b < p.batch) {
      const bool ok = fits && (need == 0 || first + need <= nfree);
      status[b] = !fits ? 2 : (ok ? 0 : 1);
      if (ok) p.seq_lens[b] = (int32_t)L;
      w.first[b] = first;
      w.have[b] = have;
      if (b < kRowsLds) first_lds[b] = first;
      if (ok && need > 0) atomicMax(&limit, first + need);
    }
    before = min(before + total, kMany);
  }
  __syncthreads();
  if (p.n_pages <= kOneLaunch) {
    for (int s = 0; s < (int)gridDim.x && w.base[s] < limit; ++s)
      take_stretch(p, w, s, w.base[s], limit, tmp, first_lds);
  } else if (threadIdx.x == 0) {
    w.scalar[kLimit] = limit;
  }
}

__global__ __launch_bounds__(kPlan) void k_extend_take(PagesParams p, PageWork w) {
  __shared__ int tmp[kPlan / 64];
  __shared__ int first_lds[kRowsLds];
  const int limit = w.scalar[kLimit];
  const int base = w.base[blockIdx.x];
  if (base >= limit) return;
  if (p.batch <= kRowsLds)
    for (int i = threadIdx.x; i < p.batch; i += kPlan) first_lds[i] = w.first[i];
  take_stretch(p, w, blockIdx.x, base, limit, tmp, first_lds);
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kPlan) void k_fork_plan(PagesParams from, PagesParams to, PageWork w,
                                                     const int32_t *parents, int keep,
                                                     int32_t *status) {
  __shared__ int tmp[kPlan / 64];
  __shared__ int32_t have_lds[kRowsLds], eldest_lds[kRowsLds];
  if (!count_stretch<false>(from, w, tmp)) return;
  const int nfree = plan_bases(w, tmp);
  // Children of each parent and the first of them: in LDS where they fit.
  const bool local = from.batch <= kRowsLds;
  int32_t *have = local ? have_lds : w.have, *eldest = local ? eldest_lds : w.eldest;
  for (int r = threadIdx.x; r < from.batch; r += kPlan) {
    have[r] = 0;
    eldest[r] = INT32_MAX;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < to.batch; i += kPlan) {
    const int r = parents[i];
    if (r >= 0 && r < from.batch) atomicMin(&eldest[r], i);
  }
  __syncthreads();
  int32_t *rank_of = w.hole, *old = w.hole + to.batch;
  int before = 0;
  for (int i0 = 0; i0 < to.batch; i0 += kPlan) {
    const int i = i0 + threadIdx.x;
    int r = -1, L = 0;
    bool need = false;
    if (i < to.batch) {
      r = parents[i];
      if (r < 0 || r >= from.batch) r = -1;
      if (r >= 0) {
        L = row_len(from, r);
        need = L % kTile != 0 &&
               (keep || __hip_atomic_load(&eldest[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != i);
      }
    }
    int total;
    const int rank = before + block_excl_scan<kPlan>(need ? 1 : 0, tmp, &total);
    if (i < to.batch) {
      const bool ok = !need || rank < nfree;
      status[i] = ok ? 0 : 1;
      to.seq_lens[i] = ok ? L : 0;
      rank_of[i] = need && ok ? rank : -1;
      old[i] = need ? from.table[(int64_t)r * from.max_pages + L / kTile] : -1;
      if (ok && r >= 0) atomicAdd(&have[r], 1);
      // (what k_fork_rows makes of the row: its parent, or none)
      w.first[i] = ok ? r : -1;
    }
    before += total;
  }
  if (local) {
    __syncthreads();
    for (int r = threadIdx.x; r < from.batch; r += kPlan) w.have[r] = have[r];
  }
}

// The free page of the given rank: its stretch by bisection over the counts,
// its place there by a prefix sum (nothing writes refs meanwhile).  Called by
// a whole workgroup of kBlock threads; sh: LDS.
__device__ __forceinline__ int page_of_rank(const PagesParams &p, const PageWork &w, int rank, int *tmp,
                                            int *sh) {
  const int n = (int)(((int64_t)p.n_pages + kStretch - 1) / kStretch);
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (w.base[mid] <= rank) lo = mid + 1;
    else hi = mid;
  }
  const int s = lo - 1;
  int left = rank - w.base[s];
  constexpr int kMine = kStretch / kBlock;
  const int64_t i0 = (int64_t)s * kStretch + threadIdx.x * kMine;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i)
    if (i0 + i < p.n_pages && p.refs[i0 + i] == 0) m |= 1u << i;
  int total;
  left -= block_excl_scan(__popc(m), tmp, &total);
  if (left >= 0 && left < __popc(m)) {
    for (; left > 0; --left) m &= m - 1;
    *sh = (int)i0 + __ffs(m) - 1;
  }
  __syncthreads();
  return *sh;
}

// Row i of `to`: its parent's pages, the last one replaced by a page of its
// own where it has to be.
__global__ __launch_bounds__(kBlock) void k_fork_rows(PagesParams from, PagesParams to, PageWork w) {
  __shared__ int tmp[kWaves], page_sh;
  const int i = blockIdx.x;
  const int r = w.first[i], rank = w.hole[i];
  const int L = r >= 0 ? row_len(from, r) : 0;
  const int full = L / kTile, n = (L + kTile - 1) / kTile;
  const int fresh = rank >= 0 ? page_of_rank(from, w, rank, tmp, &page_sh) : -1;
  int32_t *dst = to.table + (int64_t)i * to.max_pages;
  const int32_t *src = from.table + (int64_t)(r < 0 ? 0 : r) * from.max_pages;
  for (int c = threadIdx.x; c < to.max_pages; c += kBlock) {
    int page = -1;
    if (c < n) page = c == full && fresh >= 0 ? fresh : src[c];
    dst[c] = page;
  }
  if (threadIdx.x == 0) w.list[i] = fresh;
}

// Pieces of a page over all pools.
__host__ __device__ static inline int pieces_of(const Pools &pools) {
  int n = 0;
  for (int i = 0; i < pools.n; ++i) n += (int)((pools.page_bytes[i] + kPiece - 1) / kPiece);
  return n;
}

template <class T>
__device__ __forceinline__ void copy_run(const char *src, char *dst, int64_t bytes) {
  constexpr int U = 4;
  const int64_t n = bytes / (int64_t)sizeof(T);
  for (int64_t i0 = 0; i0 < n; i0 += kBlock * U) {
    T x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * kBlock + threadIdx.x;
      if (i < n) x[u] = __builtin_nontemporal_load((const T *)src + i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * kBlock + threadIdx.x;
      if (i < n) __builtin_nontemporal_store(x[u], (T *)dst + i);
    }
  }
}

// Piece `k` of page src to page dst.
__device__ __forceinline__ void copy_piece(const Pools &pools, int64_t src, int64_t dst, int k) {
  for (int i = 0; i < pools.n; ++i) {
    const int64_t bytes = pools.page_bytes[i];
    const int n = (int)((bytes + kPiece - 1) / kPiece);
    if (k < n) {
      const int64_t at = k * kPiece, len = bytes - at < kPiece ? bytes - at : kPiece;
      const char *s = pools.base[i] + src * bytes + at;
      char *d = pools.base[i] + dst * bytes + at;
      if (pools.align == 16) copy_run<u32x4>(s, d, len);
      else if (pools.align >= 4) copy_run<uint32_t>(s, d, len);
      else copy_run<uint8_t>(s, d, len);
      return;
    }
    k -= n;
  }
}

// Workgroups [0, from.batch) count the pages of the parents' rows, and empty
// those that the call ends; the others copy the part-filled pages, a piece of a
// child's page each.
__global__ __launch_bounds__(kBlock) void k_fork_pages(PagesParams from, PagesParams to, PageWork w,
                                                       Pools pools, int pieces, int keep) {
  int64_t i = blockIdx.x;
  if (i < from.batch) {
    const int r = (int)i;
    const int L = row_len(from, r), children = w.have[r];
    int32_t *row = from.table + (int64_t)r * from.max_pages;
    const int delta = keep ? children : children - 1;
    // (the page that the first child takes over keeps its count)
    const int counted = L / kTile + (!keep && children == 0 && L % kTile ? 1 : 0);
    if (delta != 0)
      for (int c = threadIdx.x; c < counted; c += kBlock)
        if (in_pool(from, row[c])) atomicAdd(&from.refs[row[c]], delta);
    if (!keep) {
      for (int c = threadIdx.x; c < from.max_pages; c += kBlock) row[c] = -1;
      __syncthreads();  // (every thread has read the length)
      if (threadIdx.x == 0) from.seq_lens[r] = 0;
    }
    return;
  }
  const int64_t groups = (int64_t)gridDim.x - from.batch;
  for (i -= from.batch; i < (int64_t)to.batch * (pieces + 1); i += groups) {
    const int child = (int)(i / (pieces + 1)), piece = (int)(i % (pieces + 1));
    const int fresh = w.list[child], old = w.hole[to.batch + child];
    if (fresh < 0) continue;
    if (piece == pieces) {
      if (threadIdx.x == 0) from.refs[fresh] = 1;
    } else if (in_pool(from, old)) {
      copy_piece(pools, old, fresh, piece);
    }
  }
}

// ---------------------------------------------------------------------------
// free, copy
// ---------------------------------------------------------------------------
// An entry is exchanged for -1, so that a row listed twice gives its pages
// back once.
__global__ __launch_bounds__(kBlock) void k_pages_free(PagesParams p, const int32_t *rows, int64_t n) {
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int b = rows[i];
    if (b < 0 || b >= p.batch) continue;
    int32_t *row = p.table + (int64_t)b * p.max_pages;
    for (int c = threadIdx.x; c < p.max_pages; c += kBlock) {
      const int page = atomicExch(&row[c], -1);
      if (in_pool(p, page)) atomicAdd(&p.refs[page], -1);
    }
    if (threadIdx.x == 0) p.seq_lens[b] = 0;
  }
}

__global__ __launch_bounds__(kBlock) void k_pages_copy(Pools pools, int64_t n_pages,
                                                       const int32_t *src, const int32_t *dst,
                                                       int64_t n, int pieces) {
  for (int64_t i = blockIdx.x; i < n * pieces; i += gridDim.x) {
    const int64_t s = src[i / pieces], d = dst[i / pieces];
    if (s < 0 || s >= n_pages || d < 0 || d >= n_pages || s == d) continue;
    copy_piece(pools, s, d, (int)(i % pieces));
  }
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------
// Movers and holes of stretch s in ascending order, `before` live pages before
// it; a mover's entry of remap holds its rank i as -2 - i until k_compact_move has
// put the page there.
__device__ __forceinline__ void list_stretch(const PagesParams &p, const PageWork &w, int s, int before,
                                             int n, int below, int32_t *remap, int *tmp) {
  const uint32_t mine = stretch_bits<true>(p, s);
  int total;
  int live = before + block_excl_scan<kPlan>(__popc(mine), tmp, &total);
  const int64_t p0 = (int64_t)s * kStretch + threadIdx.x * kPerThread;
  for (int i = 0; i < kPerThread; ++i) {
    const int64_t page = p0 + i;
    if (page >= p.n_pages) return;
    if (mine >> i & 1) {
      if (page < n) {
        remap[page] = (int)page;
      } else {
        w.list[live - below] = (int)page;
        remap[page] = -2 - (live - below);
      }
      ++live;
    } else {
      remap[page] = -1;
      if (page < n) w.hole[page - live] = (int)page;
    }
  }
}

__global__ __launch_bounds__(kPlan) void k_compact_plan(PagesParams p, PageWork w, int32_t *remap,
                                                        int32_t *n_live) {
  __shared__ int tmp[kPlan / 64];
  if (!count_stretch<true>(p, w, tmp)) return;
  const int n = plan_bases(w, tmp);
  // Live pages below n: those of the stretches before n's, and of its own.
  __syncthreads();
  const int s = n / kStretch;
  int c = 0;
  for (int64_t i = (int64_t)s * kStretch + threadIdx.x; i < n; i += kPlan) c += p.refs[i] > 0;
  int total;
  block_excl_scan<kPlan>(c, tmp, &total);
  const int64_t last = (p.n_pages + kStretch - 1) / kStretch;
  const int below = (s < last ? w.base[s] : n) + total;
  if (threadIdx.x == 0) {
    w.scalar[kLive] = n;
    w.scalar[kMoves] = n - below;
    *n_live = n;
  }
  if (p.n_pages <= kOneLaunch)
    for (int i = 0; i < (int)gridDim.x; ++i) list_stretch(p, w, i, w.base[i], n, below, remap, tmp);
}

__global__ __launch_bounds__(kPlan) void k_compact_lists(PagesParams p, PageWork w, int32_t *remap) {
  __shared__ int tmp[kPlan / 64];
  const int n = w.scalar[kLive];
  list_stretch(p, w, blockIdx.x, w.base[blockIdx.x], n, n - w.scalar[kMoves], remap, tmp);
}

// The table first (workgroups [0, batch)): an entry reads its page's rank or,
// once that is written, its new place.  Then counts and remap by rank, then
// the pages themselves.
__global__ __launch_bounds__(kBlock) void k_compact_move(PagesParams p, PageWork w, Pools pools,
                                                         int32_t *remap, int pieces, int counters) {
  const int moves = w.scalar[kMoves];
  int64_t i = blockIdx.x;
  if (i < p.batch) {
    int32_t *row = p.table + i * p.max_pages;
    for (int c = threadIdx.x; c < p.max_pages; c += kBlock) {
      const int page = row[c];
      if (!in_pool(p, page)) continue;
      const int to = __hip_atomic_load(&remap[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (to != page) row[c] = to <= -2 ? w.hole[-2 - to] : to;
    }
    return;
  }
  i -= p.batch;
  if (i < counters) {
    for (int64_t k = i * kBlock + threadIdx.x; k < moves; k += (int64_t)counters * kBlock) {
      const int from = w.list[k], to = w.hole[k];
      p.refs[to] = p.refs[from];
      p.refs[from] = 0;
      __hip_atomic_store(&remap[from], to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    return;
  }
  i -= counters;
  const int64_t movers = (int64_t)gridDim.x - p.batch - counters;
  for (int64_t k = i; k < (int64_t)moves * pieces; k += movers)
    copy_piece(pools, w.list[k / pieces], w.hole[k / pieces], (int)(k % pieces));
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
static void start_count(PageWork &w, const Counting &c, hipStream_t st) {
  w.call = c.call;
  w.bank = c.bank;
  const auto set = [&](int bank, uint64_t x) { k_pages_counter<<<1, 1, 0, st>>>(bank, x); };
  if (c.spoil && c.bank == 0) set(0, ((c.call - 1) << kCountBits) + 1);
  if (c.spoil && c.first) set(1, 1), set(2, 1);
  if (c.first) set(c.bank, 0);
}

// Workgroups of a counting launch (one at least: it also plans).
static unsigned counters(int64_t n_pages) { return (unsigned)std::max<int64_t>(stretches(n_pages), 1); }

hipError_t launch_pages_extend(const PagesParams &p, const int32_t *grow, int32_t *status,
                               char *work, const Counting &c, hipStream_t st) {
  PageWork w;
  carve_pages(p.n_pages, p.batch, work, &w);
  start_count(w, c, st);
  k_extend_plan<<<counters(p.n_pages), kPlan, 0, st>>>(p, w, grow, status);
  if (p.n_pages > kOneLaunch) k_extend_take<<<counters(p.n_pages), kPlan, 0, st>>>(p, w);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesParams &from, const PagesParams &to,
                             const int32_t *parents, bool keep, const Pools &pools,
                             int32_t *status, char *work, const Counting &c, hipStream_t st) {
  PageWork w;
  carve_pages(from.n_pages, from.batch > to.batch ? from.batch : to.batch, work, &w);
  const int pieces = pieces_of(pools);
  const int64_t last = from.batch + std::min((int64_t)to.batch * (pieces + 1), kMostGroups);
  start_count(w, c, st);
  k_fork_plan<<<counters(from.n_pages), kPlan, 0, st>>>(from, to, w, parents, keep ? 1 : 0, status);
  if (to.batch) k_fork_rows<<<(unsigned)to.batch, kBlock, 0, st>>>(from, to, w);
  k_fork_pages<<<(unsigned)last, kBlock, 0, st>>>(from, to, w, pools, pieces, keep ? 1 : 0);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesParams &p, const int32_t *rows, int64_t n, hipStream_t st) {
  if (n > 0) k_pages_free<<<(unsigned)std::min(n, kMostGroups), kBlock, 0, st>>>(p, rows, n);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const Pools &pools, int64_t n_pages, const int32_t *src,
                             const int32_t *dst, int64_t n, hipStream_t st) {
  const int pieces = pieces_of(pools);
  const int64_t grid = std::min(n * pieces, kMostGroups);
  if (grid > 0) k_pages_copy<<<(unsigned)grid, kBlock, 0, st>>>(pools, n_pages, src, dst, n, pieces);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesParams &p, const Pools &pools, int32_t *remap,
                                int32_t *n_live, char *work, const Counting &c, hipStream_t st) {
  PageWork w;
  carve_pages(p.n_pages, p.batch, work, &w);
  start_count(w, c, st);
  const unsigned n = counters(p.n_pages);
  const int pieces = pieces_of(pools);
  k_compact_plan<<<n, kPlan, 0, st>>>(p, w, remap, n_live);
  if (p.n_pages > kOneLaunch) k_compact_lists<<<n, kPlan, 0, st>>>(p, w, remap);
  const int writers = (int)(n < 64 ? n : 64);
  const int64_t movers = std::min<int64_t>((int64_t)p.n_pages / 2 * pieces, 2048);
  k_compact_move<<<(unsigned)(p.batch + writers + movers), kBlock, 0, st>>>(p, w, pools, remap,
                                                                            pieces, writers);
  return hipGetLastError();
}

}  // namespace sd
