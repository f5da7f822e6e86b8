"""Plain 64-bit implementations of window attention, of the 4-bit format and
of the page operations, with bounds on how far a kernel may be from them.

Bounds on attention, for one output channel sum_j w_j v_j (w the weights, sum
1; all sums below over the visible positions; u = 2^-24):
  * a score q.k of 128 products accumulated in float32 is off by at most
    gamma sum_i |q_i k_i|, gamma = 128 u / (1 - 128 u), twice that allowing for
    the order inside the matrix unit; with the scale, log2(e) and the maximum
    the exponent gets two more roundings of relative size u, and the
    exponential itself 2 u: dz = scale (2 gamma sum |q_i k_i|) + 4 u |z| + 2 u;
  * each weight is thus off by at most a factor e^dz, in the numerator and in
    the sum, and the accumulations of n weights and products add n u each;
  * bfloat16 outputs: every weight of the numerator is rounded once (half a
    step, eps / 2 = 2^-8 relative), and the output once (2^-8);
  so |error| <= (2 (e^dz - 1) + 2 (n + 16) u + r) sum_j w_j |v_j| + r |out|,
  with dz the largest of the visible positions and r = 2^-8 or u.
"""
import math

import numpy as np
import torch

U32 = 2.0**-24
LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def attention(q, k, v, sees, scale, half_step):
    """q [n, Hq, d], k/v [Hkv, L, d], sees [n, L] -> (out, allowance), float64."""
    q, k, v = q.double(), k.double(), v.double()
    n, Hq, d = q.shape
    G = Hq // k.shape[0]
    if sees.numel() == 0:
        return torch.zeros_like(q), torch.full_like(q, 1e-37)
    # (positions that nothing sees count as zeros, whatever they hold)
    used = sees.any(0)
    k = torch.where(used[None, :, None], k, 0.0).repeat_interleave(G, 0)
    v = torch.where(used[None, :, None], v, 0.0).repeat_interleave(G, 0)
    qh = q.transpose(0, 1)
    z = scale * (qh @ k.transpose(1, 2))
    g = d * U32 / (1 - d * U32)
    dz = scale * 2 * g * (qh.abs() @ k.abs().transpose(1, 2)) + 4 * U32 * z.abs() + 2 * U32
    z = torch.where(sees, z, -math.inf)
    dz = torch.where(sees, dz, 0.0).amax(-1, keepdim=True)
    top = torch.clamp(z.amax(-1, keepdim=True), min=-1e300)
    w = torch.exp(z - top)
    w = w / torch.clamp(w.sum(-1, keepdim=True), min=1e-300)
    out, mass = w @ v, w @ v.abs()
    count = sees.sum(-1)[None, :, None].double()
    allow = (2 * torch.expm1(dz) + 2 * (count + 16) * U32 + half_step) * mass + \
        half_step * out.abs() + 1e-37
    return out.transpose(0, 1), allow.transpose(0, 1)


def visible(L, count, n_sink, window):
    """sees [count, L]: query i sits at position L - count + i."""
    p = torch.arange(L - count, L)[:, None]
    j = torch.arange(L)[None]
    return (j <= p) & ((j < n_sink) | (p - j < window))


def q4_round(x):
    """Rows [..., 128] (any float type) -> (values float64, scale bytes)."""
    g = x.double().reshape(x.shape[:-1] + (4, 32))
    top = g.abs().amax(-1)
    bad = ~torch.isfinite(g).all(-1)
    top = torch.where(bad, 1.0, top)
    e = np.full(top.shape, -95, dtype=np.int64)
    t = top.numpy()
    for i in np.ndindex(t.shape):  # the smallest e >= -95 with top < 7 * 2^e
        while t[i] >= 7.0 * 2.0**int(e[i]):
            e[i] += 1
    e = torch.from_numpy(e)
    y = torch.where(bad[..., None], 0.0, g).abs() * torch.pow(2.0, -e.double())[..., None]
    dist = (y[..., None] - LEVELS).abs()
    near = dist.amin(-1, keepdim=True)
    # ties: the level of even index comes first in the order 0, 2, 4, 6, 1, ..
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    index = order[(dist[..., order] == near).int().argmax(-1)]
    val = torch.copysign(LEVELS[index], g) * torch.pow(2.0, e.double())[..., None]
    val = torch.where(bad[..., None], math.nan, val).reshape(x.shape)
    return val, torch.where(bad, 255, e + 127).to(torch.uint8)


def q4_decode(codes, scales):
    """Codes [..., 64] and scale bytes [..., 4] -> values [..., 128], float64."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = torch.where(c >= 8, -LEVELS[c & 7], LEVELS[c & 7])
    s = torch.where(scales == 255, math.nan, torch.pow(2.0, scales.double() - 127))
    return x * s.repeat_interleave(32, -1)


class PagesModel:
    """The page operations, row by row and page by page."""

    def __init__(self, table, lens, refs, pools=()):
        self.table, self.lens, self.refs = np.array(table), np.array(lens), np.array(refs)
        self.pools = [np.array(p) for p in pools]

    def _free(self):
        return [p for p in range(len(self.refs)) if self.refs[p] == 0]

    def extend(self, grow):
        free, at, width = self._free(), 0, self.table.shape[1]
        status = np.zeros(len(self.lens), np.int32)
        for b in range(len(self.lens)):
            L = int(np.clip(self.lens[b], 0, 16 * width))
            new = L + max(0, int(grow[b]))
            have, want = -(-L // 16), -(-new // 16)
            if want > width:
                status[b] = 2
                continue
            need = want - have
            if need and at + need > len(free):
                status[b] = 1
                at += need
                continue
            for c in range(need):
                self.table[b, have + c] = free[at + c]
                self.refs[free[at + c]] = 1
            at += need
            self.lens[b] = new
        return status

    def fork(self, to_rows, parents, keep):
        """-> (table, lens, status) of the children."""
        B, width = self.table.shape
        free, at = self._free(), 0
        table = np.full((to_rows, width), -1, np.int32)
        lens, status = np.zeros(to_rows, np.int32), np.zeros(to_rows, np.int32)
        eldest, children, fresh = {}, [0] * B, []
        for i, r in enumerate(parents):
            if 0 <= r < B:
                eldest.setdefault(int(r), i)
        for i, r in enumerate(parents):
            if not 0 <= r < B:
                continue
            L = int(np.clip(self.lens[r], 0, 16 * width))
            n, own = -(-L // 16), L % 16 != 0 and (keep or eldest[int(r)] != i)
            if own:
                at += 1
                if at > len(free):
                    status[i] = 1
                    continue
            table[i, :n] = self.table[r, :n]
            lens[i] = L
            children[r] += 1
            if own:
                page, old = free[at - 1], self.table[r, n - 1]
                table[i, n - 1] = page
                fresh.append(page)
                if 0 <= old < len(self.refs):
                    for p in self.pools:
                        p[page] = p[old]
        for r in range(B):
            L = int(np.clip(self.lens[r], 0, 16 * width))
            for c in range(L // 16):
                if 0 <= self.table[r, c] < len(self.refs):
                    self.refs[self.table[r, c]] += children[r] - (0 if keep else 1)
            if not keep and not children[r] and L % 16 and 0 <= self.table[r, L // 16] < len(self.refs):
                self.refs[self.table[r, L // 16]] -= 1
        for p in fresh:
            self.refs[p] = 1
        if not keep:
            self.table[:] = -1
            self.lens[:] = 0
        return table, lens, status

    def free(self, rows):
        for b in rows:
            if not 0 <= b < len(self.lens):
                continue
            for page in self.table[b]:
                if 0 <= page < len(self.refs):
                    self.refs[page] -= 1
            self.table[b] = -1
            self.lens[b] = 0

    def copy(self, src, dst):
        n = len(self.refs)
        for s, d in zip(src, dst):
            if 0 <= s < n and 0 <= d < n:
                for p in self.pools:
                    p[d] = p[s]

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] <= 0]
        movers = [p for p in live if p >= n]
        remap = np.full(len(self.refs), -1, np.int32)
        remap[live] = live
        for h, m in zip(holes, movers):
            remap[m] = h
            self.refs[h], self.refs[m] = self.refs[m], 0
            for p in self.pools:
                p[h] = p[m]
        inside = (self.table >= 0) & (self.table < len(self.refs))
        self.table[inside] = remap[self.table[inside]]
        return remap, n
