// sd_plan.hpp -- how sequences of different lengths are cut into parts, so that
// every compute unit gets about the same.
//
// A sequence has `items` that read the same positions (its row tiles; one for a
// single query), in `units` steps.  With so many slots (workgroups for each
// group of KV heads), parts of one length are taken, the shortest that the slots
// suffice for.  The host knows no lengths, so the workgroups work this out, each
// of its waves for itself, in 1 to 2 us.
#pragma once

#include "sd_cache.hpp"
#include "sd_internal.hpp"

namespace sd {

constexpr int kPlanChunks = 4;                 // of 64 sequences
constexpr int kPlanSeqs = 64 * kPlanChunks;

struct Part {
  int b, item;    // sequence, and which of its items
  int s, n;       // part, parts of the item
  int first;      // the item's first slot
  int span;       // units of a part
};

// x / d rounded up, for 0 < x, d <= 2^18, with inv = 1 / d but for 2^-23 of it:
// the half keeps the product further from every integer than its rounding moves it.
__device__ __forceinline__ int parts_of(int x, int d, float inv) {
  return (int)(((float)(x + d - 1) + 0.5f) * inv);
}
__device__ __forceinline__ float inverse(int d) { return __builtin_amdgcn_rcpf((float)d); }

// What slot y computes; false: nothing.  sequence(b, items) gives the units of
// sequence b (at least one) and sets its items; `least`: units of a part.
template <class F>
__device__ __forceinline__ bool find_part(const WindowParams &p, int y, int least, F sequence, Part &t) {
  const int l = lane_id();
  int units[kPlanChunks], items[kPlanChunks];   // of this lane's sequences
  int total = 0, n_items = 0, top = 1;
  if (p.batch == 1) {
    int n;
    top = __builtin_amdgcn_readfirstlane(sequence(0, n));
    n_items = __builtin_amdgcn_readfirstlane(n);
    total = top * n_items;
  } else {
#pragma unroll
    for (int c = 0; c < kPlanChunks; ++c) {
      units[c] = items[c] = 0;
      if (64 * c >= p.batch) continue;
      if (64 * c + l < p.batch) units[c] = sequence(64 * c + l, items[c]);
      if (items[c] == 0) units[c] = 0;
      total += __builtin_amdgcn_readlane(wave_incl_scan(items[c] * units[c]), 63);
      n_items += __builtin_amdgcn_readlane(wave_incl_scan(items[c]), 63);
      top = max(top, (int)wave_max_u32((uint32_t)units[c]));
    }
  }
  if (n_items == 0) return false;
  // The least that keeps an item's partials within their room.
  least = max(least, parts_of(top, p.nsplit, inverse(p.nsplit)));
  int span = max(top, least), best = INT32_MAX;
#pragma unroll 1
  for (int i = 0; i < p.plans; ++i) {
    const int slots = p.slots[i];
    if (slots < n_items) continue;
    int lo;
    if (total == top * n_items) {   // sequences of one length
      const int n = (int)(((float)slots + 0.5f) * inverse(n_items));
      lo = parts_of(top, n, inverse(n));
    } else {
      // Between what would do without rounding up each item's parts and what
      // does with a part more for each, four steps of a bisection.
      lo = max(1, (int)((float)total * inverse(slots) - 0.125f));
      int hi = top;
      if (slots > n_items) hi = min(hi, (int)((float)total * inverse(slots - n_items) + 0.125f) + 1);
#pragma unroll 1
      for (int j = 0; j < 4 && lo < hi; ++j) {
        const int mid = (lo + hi) >> 1;
        const float inv = inverse(mid);
        int n = 0;
#pragma unroll
        for (int c = 0; c < kPlanChunks; ++c)
          if (64 * c < p.batch)
            n += __builtin_amdgcn_readlane(wave_incl_scan(items[c] * parts_of(units[c], mid, inv)), 63);
        if (n <= slots) hi = mid;
        else lo = mid + 1;
      }
      lo = hi;
    }
    lo = max(lo, least);
    const int cost = p.rounds[i] * (16 * lo + p.part_cost);
    if (cost < best) {
      best = cost;
      span = lo;
    }
  }
  const float inv = inverse(span);
  t.span = span;
  t.b = t.first = 0;
  t.n = parts_of(top, span, inv);
  if (p.batch == 1) {
    if (y >= t.n * n_items) return false;
  } else {
    int before = 0;
    bool found = false;
#pragma unroll
    for (int c = 0; c < kPlanChunks; ++c) {
      if (64 * c >= p.batch || found) continue;
      const int n = parts_of(units[c], span, inv), upto = wave_incl_scan(items[c] * n);
      const uint64_t hit = __ballot(y - before < upto);
      if (hit) {
        const int src = __ffsll((unsigned long long)hit) - 1;
        t.b = 64 * c + src;
        t.n = __builtin_amdgcn_readlane(n, src);
        t.first = before + __builtin_amdgcn_readlane(upto - items[c] * n, src);
        found = true;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (!found) return false;
  }
  const int at = y - t.first;
  t.item = (int)((uint32_t)at / (uint32_t)t.n);
  t.s = at - t.item * t.n;
  t.first += t.item * t.n;
  return true;
}

}  // namespace sd
