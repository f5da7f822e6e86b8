"""Operators around the key/value cache, as a serving loop calls them:
attention with a sliding window and visible first tokens (one query per
sequence, or a chunk of them), the cache held in 4 bits (append, load,
attention), and the pages of a paged cache (copy, fork, extend and free,
compact).

Where ``own`` is false, ``run`` computes them in elementary torch operations;
where it is true, through ``paper_2605_24168_amd.sparse_decode``.

The 4-bit cache: a row of 128 channels is 64 bytes of codes (channel 2i in the
low half of byte i) and 4 scale bytes, one per 32 channels.  A code is a sign
bit over an index into 0, 0.5, 1, 1.5, 2, 3, 4, 6; scale byte s stands for
2^(s - 127).  Writing a group whose largest magnitude is a takes the smallest
power of two with a < 7 * 2^e, and rounds to the nearest level, halfway cases
to the even index.
"""
import math
import random

import torch

own = False

D = 128
PAGE = 16
GROUP = 32
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIN_SCALE = 32  # smallest scale byte written
EVERYTHING = 2**31 - 1


# ---------------------------------------------------------------------------
# Cases.
# ---------------------------------------------------------------------------
def _attend(op, batch, q_heads, kv_heads, n, **kw):
    """n: longest sequence, n_min: shortest; tokens: queries of the longest
    chunk (0: one query per sequence, unpacked)."""
    c = {"op": op, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "n": n, "n_min": n,
         "layout": "bhnd", "dtype": "bf16", "sink": 0, "window": EVERYTHING, "tokens": 0}
    c.update(kw)
    return c


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # One user's decode step in a local layer: nothing but latency.
        named("window_token_8k", _attend("window", 1, 32, 8, 8191, layout="paged", sink=4,
                                         window=1020)),
        # Continuous batching in a local layer: 64 sequences of very different
        # lengths on one page pool.
        named("window_ragged64", _attend("window", 64, 32, 8, 65521, layout="paged", n_min=200,
                                         sink=128, window=4096)),
        # Chunks of long prompts: 8K tokens a pass, ragged.
        named("window_chunks_8k", _attend("window", 4, 32, 8, 32768, n_min=9000, sink=128,
                                          window=4096, tokens=2048)),
        # The same in float32, odd sizes (debugging and reference runs).
        named("window_chunks_f32", _attend("window", 3, 8, 2, 2049, n_min=301, dtype="f32", sink=3,
                                           window=511, tokens=701, layout="paged")),
        # One user's decode step on the 4-bit cache: the new token is written,
        # the step attends over everything.
        named("q4_step_8k", _attend("q4_step", 1, 32, 8, 8191, layout="paged")),
        # A large batch over long contexts held in 4 bits: the largest.
        named("q4_dense_128k", _attend("q4", 16, 64, 8, 131072)),
        # Ragged sequences on a 4-bit page pool, window and sinks.
        named("q4_window_ragged32", _attend("q4", 32, 32, 8, 131072, layout="paged", n_min=8192,
                                            sink=128, window=16384)),
        # Prompts written into the 4-bit cache and read back in bfloat16.
        named("q4_fill_256k", _attend("q4_fill", 8, 32, 8, 32749, layout="paged", n_min=30011)),
        # A cached prefix copied page by page (keys and values).
        {"op": "copy", "pages": 16384, "moves": 4096, "kv_heads": 8, "name": "pages_copy_4k"},
        # A step of beam search: 32 prompts of up to 32K tokens, 4 beams each.
        {"op": "beam", "prompts": 32, "beams": 4, "n": 32768, "n_min": 1000, "grown": 500,
         "kv_heads": 8, "keep": False, "name": "pages_beam_32x4"},
        # Half of a 4 GB pool is live, in no order: squeeze it together.
        {"op": "compact", "pages": 65536, "rows": 128, "live": 0.5, "kv_heads": 8,
         "name": "pages_compact_64k"},
        # Continuous batching: 64 of 256 sequences leave and as many prompts of
        # other lengths take their rows.
        {"op": "admit", "pages": 262144, "rows": 256, "leave": 64, "n": 16384, "n_min": 16,
         "name": "pages_admit_256"},
    ]


_HEADS = [(32, 8), (32, 8), (64, 8), (40, 8), (16, 4), (32, 32), (8, 8), (8, 1), (12, 6), (64, 4)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, its sizes log-uniform over the ranges."""
    op = rng.choice(["window", "window", "chunks", "chunks", "q4", "q4", "q4_step", "q4_fill",
                     "copy", "beam", "compact", "admit"])
    if op in ("window", "chunks", "q4", "q4_step", "q4_fill"):
        hq, hkv = rng.choice(_HEADS)
        kw = {"layout": rng.choice(["bhnd", "paged"])}
        n, batch, rows = _log(rng, 64, 131072), _log(rng, 1, 64), 1 << 22
        if op in ("window", "chunks"):
            kw["sink"] = rng.choice([0, 1, 4, 64, 128])
            kw["window"] = _log(rng, 1, 8192)
            kw["dtype"] = "f32" if rng.random() < 0.25 else "bf16"
        if op == "q4":
            rows = 1 << 23
            if rng.random() < 0.5:
                kw["sink"], kw["window"] = rng.choice([0, 4, 128]), _log(rng, 64, 32768)
        if op == "q4_fill":
            n, rows = _log(rng, 64, 32768), 1 << 21
        if op == "chunks":
            op, batch = "window", _log(rng, 1, 8)
            n = min(n, 32768)
            kw["tokens"] = min(n, _log(rng, 2, 2048 if kw["dtype"] == "bf16" else 512))
            kw["window"] = min(kw["window"], 4096)
            while batch > 1 and batch * hq * kw["tokens"] > 1 << 18:
                batch -= 1
        if kw.get("dtype") == "f32":
            rows = 1 << 20
        while batch > 1 and batch * hkv * n > rows:
            batch -= 1
        n = max(2, min(n, rows // (batch * hkv)))
        if kw.get("tokens"):
            kw["tokens"] = min(kw["tokens"], n)
        ragged = batch > 1 and rng.random() < 0.6
        kw["n_min"] = max(1, n // 16) if ragged else n
        return _attend(op, batch, hq, hkv, n, **kw)
    hkv = rng.choice([1, 2, 4, 8, 8])
    if op == "copy":
        pages = _log(rng, 64, 16384)
        return {"op": op, "pages": pages, "moves": _log(rng, 1, pages // 2), "kv_heads": hkv}
    if op == "beam":
        prompts, beams, n = _log(rng, 1, 32), rng.choice([2, 3, 4, 8]), _log(rng, 20, 16384)
        return {"op": op, "prompts": prompts, "beams": beams, "n": n, "n_min": max(1, n // 20),
                "grown": _log(rng, 1, 500), "kv_heads": hkv, "keep": rng.random() < 0.5}
    if op == "compact":
        return {"op": op, "pages": _log(rng, 100, 65536), "rows": _log(rng, 2, 128),
                "live": round(rng.uniform(0.05, 0.98), 2), "kv_heads": hkv}
    rows, n = _log(rng, 4, 256), _log(rng, 20, 16384)
    return {"op": "admit", "pages": rows * (n // PAGE + 1), "rows": rows,
            "leave": _log(rng, 1, rows), "n": n, "n_min": max(1, n // 50)}


# ---------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------
def _dice(case):
    return random.Random(case.get("batch", 1) * 1000003 + case.get("n", case.get("pages", 0)))


def _lens(case):
    """Sequence lengths: the longest first (a property of the case)."""
    r = _dice(case)
    return [case["n"]] + [r.randint(case["n_min"], case["n"]) for _ in range(case["batch"] - 1)]


def _counts(case, lens):
    """Tokens of each sequence that this call brings (queries, or rows to
    write): the longest first; all of a sequence where a cache is filled."""
    if case["op"] == "q4_fill":
        return list(lens)
    if not case["tokens"]:
        return [1] * len(lens)
    r = _dice(case)
    return [min(L, case["tokens"] if b == 0 else r.randint(max(1, case["tokens"] // 3),
                                                          case["tokens"]))
            for b, L in enumerate(lens)]


def _table(lens, gen):
    """Block table of sequences on a pool in random order, and its pages."""
    per = [-(-L // PAGE) for L in lens]
    perm = torch.randperm(sum(per), generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(per)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = perm[at:at + m]
        at += m
    return table, sum(per)


def _prepare_attend(case, gen):
    B, Hq, Hkv, op = case["batch"], case["q_heads"], case["kv_heads"], case["op"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    lens = _lens(case)
    counts = _counts(case, lens)
    paged = case["layout"] == "paged"
    table, pages = _table(lens, gen) if paged else (None, 0)
    dev = {"device": "cuda", "generator": gen}
    s = {"op": op, "paged": paged, "table": table, "lens": torch.tensor(lens, dtype=torch.int32,
                                                                        device="cuda"),
         "sink": case["sink"], "window": case["window"], "most": max(counts), "n": case["n"]}
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    packed = bool(case["tokens"]) or op == "q4_fill"
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda") if packed else None
    T = starts[-1]
    if op != "q4_fill":
        s["q"] = (torch.randn((T, Hq, D), **dev) * 1.5).to(dt)
    # Keys and values with a scale of their own per head.
    head = torch.rand((Hkv, 1), **dev) * 1.5 + 0.5
    if op in ("q4_step", "q4_fill"):  # the tokens that are written
        s["k_new"] = (torch.randn((T, Hkv, D), **dev) * head).to(torch.bfloat16)
        s["v_new"] = (torch.randn((T, Hkv, D), **dev) * head).to(torch.bfloat16)
    if op == "window":
        shape = (pages, PAGE, Hkv, D) if paged else (B, Hkv, case["n"], D)
        by_head = head.view((1, 1, Hkv, 1) if paged else (1, Hkv, 1, 1)).to(dt)
        s["k"] = torch.randn(shape, dtype=dt, **dev).mul_(by_head)
        s["v"] = torch.randn(shape, dtype=dt, **dev).mul_(by_head)
        if own:
            from paper_2605_24168_amd import sparse_decode as sd
            s["cache"] = sd.KVCache(k=s["k"], v=s["v"], layout=case["layout"], block_table=table)
    else:
        rows = (pages, Hkv, PAGE) if paged else (B, Hkv, case["n"])
        by_head = torch.randint(0, 2, (Hkv, 1, 1), dtype=torch.uint8, **dev)
        for name in ("k", "v"):
            if op == "q4_fill":
                s[name] = torch.zeros(rows + (D // 2,), dtype=torch.uint8, device="cuda")
                s[name + "_scales"] = torch.full(rows + (D // GROUP,), MIN_SCALE, dtype=torch.uint8,
                                                 device="cuda")
                continue
            # Rows as writing normal values leaves them, from a bank of such rows.
            codes, scales = _plain_codes(torch.randn((1 << 14, D), **dev) * 0.7)
            pick = torch.randint(0, 1 << 14, rows, **dev)
            s[name], s[name + "_scales"] = codes[pick], scales[pick] + by_head
        if own:
            from paper_2605_24168_amd import sparse_decode as sd
            s["cache"] = sd.Q4Cache(k=s["k"], k_scales=s["k_scales"], v=s["v"],
                                    v_scales=s["v_scales"], layout=case["layout"],
                                    block_table=table)
    return s


def _pools(case, pages, gen):
    shape = (pages, PAGE, case["kv_heads"], D)
    return [torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=gen)
            for _ in range(2)]


def _prepare_pages(case, gen, seed):
    r, sizes = random.Random(seed), _dice(case)
    op = case["op"]
    if op == "copy":
        perm = torch.randperm(case["pages"], generator=gen, device="cuda").to(torch.int32)
        m = case["moves"]
        return {"op": op, "pools": _pools(case, case["pages"], gen), "src": perm[:m].clone(),
                "dst": perm[m:2 * m].clone()}
    rows, lens, pages = [], [], 0  # a row: its pages' numbers before they are shuffled
    if op == "beam":
        for p in range(case["prompts"]):
            prompt = case["n"] if p == 0 else sizes.randint(case["n_min"], case["n"])
            whole = prompt // PAGE  # shared by the prompt's beams
            L = prompt + sizes.randint(1, case["grown"])
            mine = -(-L // PAGE) - whole
            for b in range(case["beams"]):
                rows.append(list(range(pages, pages + whole)) +
                            list(range(pages + whole + b * mine, pages + whole + (b + 1) * mine)))
                lens.append(L)
            pages += whole + case["beams"] * mine
        pages += 2 * len(rows)  # some stay free
    elif op == "compact":
        left = max(case["rows"], int(case["pages"] * case["live"]))
        for b in range(case["rows"]):
            m = left // (case["rows"] - b)
            m = max(1, min(left - (case["rows"] - b - 1), sizes.randint(max(1, m // 2), m + m // 2)))
            rows.append(list(range(pages, pages + m)))
            lens.append(m * PAGE - sizes.randint(0, PAGE - 1))
            pages, left = pages + m, left - m
        pages = max(pages, case["pages"])
    else:
        lens = [case["n"]] + [sizes.randint(case["n_min"], case["n"]) for _ in range(case["rows"] - 1)]
        for L in lens:
            m = -(-L // PAGE)
            rows.append(list(range(pages, pages + m)))
            pages += m
        pages = max(pages, case["pages"])
    most = max(len(x) for x in rows)
    if op == "admit":
        most = -(-case["n"] // PAGE)
    perm = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    flat = torch.tensor([x + [-1] * (most - len(x)) for x in rows], device="cuda")
    table = torch.where(flat >= 0, perm[flat.clamp(min=0)], -1).to(torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs += torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
    s = {"op": op, "table": table, "refs": refs,
         "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    if op == "beam":
        s["pools"], s["keep"] = _pools(case, pages, gen), case["keep"]
        s["parents"] = torch.tensor([i // case["beams"] * case["beams"] +
                                     r.randrange(case["beams"]) for i in range(len(rows))],
                                    dtype=torch.int32, device="cuda")
        s["to_table"] = torch.full_like(table, -1)
        s["to_lens"] = torch.zeros_like(s["lens"])
    elif op == "compact":
        s["pools"] = _pools(case, pages, gen)
    else:
        leave = r.sample(range(case["rows"]), case["leave"])
        grow = [0] * case["rows"]
        for b in leave:
            grow[b] = r.randint(case["n_min"], case["n"])
        s["leave"] = torch.tensor(leave, dtype=torch.int32, device="cuda")
        s["grow"] = torch.tensor(grow, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 2654435761 % (1 << 62) + 29)
    if case["op"] in ("copy", "beam", "compact", "admit"):
        return _prepare_pages(case, gen, seed)
    return _prepare_attend(case, gen)


# ---------------------------------------------------------------------------
# Plain forms.
# ---------------------------------------------------------------------------
def _rows_of(s, cache, pos, head_major):
    """Rows [B, Hkv, C, ...] of a cache at positions pos [B, C]."""
    b = torch.arange(pos.shape[0], device="cuda")[:, None]
    if not s["paged"]:
        return cache[b, :, pos].transpose(1, 2)
    page = s["table"][b, pos // PAGE].long()
    if head_major:
        return cache[page, :, pos % PAGE].transpose(1, 2)
    return cache[page, pos % PAGE].transpose(1, 2)


def _values(codes, scales):
    """What 4-bit rows [..., 64] with scale bytes [..., 4] stand for, float32."""
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device="cuda")
    both = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    x = level[both.int()].unflatten(-1, (D // GROUP, GROUP))
    return (x * torch.exp2(scales.float() - 127.0)[..., None]).flatten(-2)


def _plain_attention(s, keys, values):
    """keys/values: functions from positions [B, C] to float32 rows."""
    lens, most = s["lens"].long(), s["most"]
    B = lens.shape[0]
    starts = s["starts"].long() if s["starts"] is not None else torch.arange(B + 1, device="cuda")
    q = s["q"]
    T, Hq = q.shape[:2]
    counts = starts[1:] - starts[:-1]
    # Positions that some query of the call may see: first tokens, then the
    # stretch from the earliest query's window to the end.
    sink = min(s["sink"], s["n"])
    stretch = min(s["n"], s["window"] + most - 1)
    first = torch.clamp(lens - counts - s["window"] + 1, min=sink)
    pos = torch.cat((torch.arange(sink, device="cuda").expand(B, sink),
                     first[:, None] + torch.arange(stretch, device="cuda")), dim=1)
    there = pos < lens[:, None]
    at = torch.where(there, pos, 0)
    k, v = keys(at), values(at)
    Hkv, C = k.shape[1:3]
    # The packed queries as [B, most]: query i sits at position L - count + i.
    i = torch.arange(most, device="cuda")
    row = torch.clamp(starts[:-1, None] + i, max=T - 1)
    p = (lens - counts)[:, None] + i
    qp = q.float()[row].unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4)
    z = qp.flatten(2, 3) @ k.transpose(2, 3) / math.sqrt(D)
    gap = p[:, :, None] - pos[:, None, :]
    sees = there[:, None, :] & (gap >= 0) & ((pos[:, None, :] < s["sink"]) | (gap < s["window"]))
    z = z.unflatten(2, (Hq // Hkv, most)).masked_fill(~sees[:, None, None], -math.inf)
    z = torch.exp(z - torch.clamp(z.amax(-1, keepdim=True), min=-1e30))
    o = z.flatten(2, 3) @ v
    o = o.unflatten(2, (Hq // Hkv, most)) / torch.clamp(z.sum(-1, keepdim=True), min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)  # [B, most, Hq, D]
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), counts, output_size=T)
    return o[b, torch.arange(T, device="cuda") - starts[b]].to(q.dtype)


def _plain_codes(x):
    """Rows [..., 128] as codes [..., 64] and scale bytes [..., 4]."""
    x = x.float().unflatten(-1, (D // GROUP, GROUP))
    a = x.abs()
    m, e = torch.frexp(a.amax(-1))  # a = m 2^e, 1/2 <= m < 1; 7 2^(e-3) = 0.875 2^e
    scale = torch.clamp(e - 3 + (m >= 0.875).int() + 127, min=MIN_SCALE)
    scale = torch.where(a.amax(-1) > 0, scale, MIN_SCALE)
    a = torch.ldexp(a, (127 - scale)[..., None])
    code = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() \
        + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()
    code = (code + 8 * (x < 0).int()).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.to(torch.uint8)


def _token_places(s):
    """(sequence, position) of each packed token."""
    lens = s["lens"].long()
    B = lens.shape[0]
    starts = s["starts"].long() if s["starts"] is not None else torch.arange(B + 1, device="cuda")
    T = s["k_new"].shape[0]
    counts = starts[1:] - starts[:-1]
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), counts, output_size=T)
    return b, lens[b] - counts[b] + torch.arange(T, device="cuda") - starts[b]


def _plain_append_and_load(s):
    b, pos = _token_places(s)
    if s["paged"]:
        b, pos = s["table"][b, pos // PAGE].long(), pos % PAGE
    out = []
    for name in ("k", "v"):
        codes, scales = _plain_codes(s[name + "_new"])
        s[name][b, :, pos] = codes
        s[name + "_scales"][b, :, pos] = scales
        out.append(_values(s[name][b, :, pos], s[name + "_scales"][b, :, pos]).to(torch.bfloat16))
    return out


def _plain_beam(s, table, lens, refs):
    parents, keep = s["parents"].long(), s["keep"]
    n, width = parents.shape[0], table.shape[1]
    dev = {"device": "cuda"}
    L = lens.long()[parents]
    whole, part = L // PAGE, L % PAGE != 0
    child = torch.arange(n, **dev)
    eldest = torch.full((lens.shape[0],), n, **dev).scatter_reduce(0, parents, child, "amin")
    takes_over = (eldest[parents] == child) & (not keep)
    need = part & ~takes_over
    rank = torch.cumsum(need, 0) - need.long()
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    ok = ~need | (rank < (refs == 0).sum())
    fresh, gets = free[rank.clamp(max=free.shape[0] - 1)], need & ok
    col = torch.arange(width, **dev)
    has = ok[:, None] & (col < (whole + part.long())[:, None])
    new = torch.where(has, table[parents], -1)
    at = whole.clamp(max=width - 1)
    old = table[parents, at].long()
    new = torch.where(gets[:, None] & (col == whole[:, None]), fresh[:, None].to(torch.int32), new)
    s["to_table"].copy_(new)
    s["to_lens"].copy_(torch.where(ok, L, 0))
    children = torch.zeros(lens.shape[0], dtype=torch.int64, **dev).index_add(0, parents, ok.long())
    have = lens.long()
    holds = col < (have // PAGE)[:, None]
    delta = torch.where(holds, (children if keep else children - 1)[:, None], 0)
    if not keep:
        last = (col == (have // PAGE)[:, None]) & (have % PAGE != 0)[:, None]
        delta = torch.where(last & (children == 0)[:, None], -1, delta)
    inside = table >= 0
    refs.index_add_(0, table[inside].long(), delta[inside].to(torch.int32))
    refs[fresh[gets]] = 1
    for pool in s["pools"]:
        pool[fresh[gets]] = pool[old[gets]]
    if not keep:
        table.fill_(-1)
        lens.fill_(0)
    return (~ok).to(torch.int32)


def _plain_compact(s, table, refs):
    live = refs > 0
    n = live.sum()
    page = torch.arange(refs.shape[0], device="cuda")
    holes = torch.nonzero(~live & (page < n)).flatten()
    movers = torch.nonzero(live & (page >= n)).flatten()
    for pool in s["pools"]:
        pool[holes] = pool[movers]
    remap = torch.where(live, page, -1).to(torch.int32)
    remap[movers] = holes.to(torch.int32)
    refs[holes] = refs[movers]
    refs[movers] = 0
    table.copy_(torch.where(table >= 0, remap[table.clamp(min=0).long()], -1))
    return remap, n.to(torch.int32).reshape(1)


def _plain_admit(s):
    table, lens, refs = s["table"], s["lens"], s["refs"]
    goes = torch.zeros(lens.shape[0], dtype=torch.bool, device="cuda")
    goes[s["leave"].long()] = True
    given = table[goes[:, None] & (table >= 0)].long()
    refs.index_add_(0, given, torch.full_like(given, -1, dtype=torch.int32))
    table.masked_fill_(goes[:, None], -1)
    lens.masked_fill_(goes, 0)
    width = table.shape[1]
    L = lens.long()
    want = -(-(L + s["grow"]) // PAGE)
    have = -(-L // PAGE)
    fits = want <= width
    need = torch.where(fits, want - have, 0)
    end = torch.cumsum(need, 0)
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    ok = fits & ((need == 0) | (end <= (refs == 0).sum()))
    col = torch.arange(width, device="cuda")
    takes = ok[:, None] & (col >= have[:, None]) & (col < want[:, None])
    rank = ((end - need - have)[:, None] + col).clamp(0, free.shape[0] - 1)
    page = free[rank]
    table.copy_(torch.where(takes, page.to(torch.int32), table))
    refs[page[takes]] = 1
    lens.copy_(torch.where(ok, L + s["grow"], L))
    return torch.where(fits, (~ok).int(), 2).to(torch.int32)


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    op = s["op"]
    if op == "window":
        return _plain_attention(s, lambda at: _rows_of(s, s["k"], at, False).float(),
                                lambda at: _rows_of(s, s["v"], at, False).float())
    got = {}
    if op in ("q4_step", "q4_fill"):
        got["k"], got["v"] = _plain_append_and_load(s)
    if op in ("q4", "q4_step"):
        def rows(name):
            return lambda at: _values(_rows_of(s, s[name], at, True),
                                      _rows_of(s, s[name + "_scales"], at, True))
        got["out"] = _plain_attention(s, rows("k"), rows("v"))
    elif op == "copy":
        for pool in s["pools"]:
            pool[s["dst"].long()] = pool[s["src"].long()]
        got["pools"] = s["pools"]
    elif op == "admit":
        status = _plain_admit(s)
        got = {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}
    elif op == "beam":  # the state is kept for the next pass: copies of its small arrays change
        table, lens, refs = s["table"].clone(), s["lens"].clone(), s["refs"].clone()
        status = _plain_beam(s, table, lens, refs)
        got = {"old_table": table, "old_lens": lens, "refs": refs, "status": status,
               "table": s["to_table"], "lens": s["to_lens"], "pools": s["pools"]}
    elif op == "compact":
        table, refs = s["table"].clone(), s["refs"].clone()
        remap, live = _plain_compact(s, table, refs)
        got = {"table": table, "refs": refs, "remap": remap, "live": live, "pools": s["pools"]}
    return got


def _run_own(s):
    from paper_2605_24168_amd import sparse_decode as sd
    op = s["op"]
    if op == "window":
        return sd.sparse_decode_window_attention(
            s["q"], s["cache"], s["lens"], sd.Window(n_sink=s["sink"], window=s["window"]),
            q_starts=s["starts"])
    got = {}
    if op in ("q4_step", "q4_fill"):
        sd.sparse_decode_q4_append(s["k_new"], s["v_new"], s["cache"], s["lens"],
                                   starts=s["starts"])
        got["k"], got["v"] = sd.sparse_decode_q4_load(s["cache"], s["lens"], starts=s["starts"],
                                                      tokens=s["k_new"].shape[0])
    if op in ("q4", "q4_step"):
        got["out"] = sd.sparse_decode_q4_attention(
            s["q"], s["cache"], s["lens"], sd.Window(n_sink=s["sink"], window=s["window"]))
    elif op == "copy":
        sd.sparse_decode_pages_copy(s["pools"], s["src"], s["dst"])
        got["pools"] = s["pools"]
    elif op == "admit":
        pages = sd.Pages(block_table=s["table"], seq_lens=s["lens"], refs=s["refs"])
        sd.sparse_decode_pages_free(pages, s["leave"])
        status = sd.sparse_decode_pages_extend(pages, s["grow"])
        got = {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}
    elif op == "beam":
        table, lens, refs = s["table"].clone(), s["lens"].clone(), s["refs"].clone()
        pages = sd.Pages(block_table=table, seq_lens=lens, refs=refs)
        to = sd.Pages(block_table=s["to_table"], seq_lens=s["to_lens"], refs=refs)
        status = sd.sparse_decode_pages_fork(pages, to, s["parents"], pools=s["pools"],
                                             keep=s["keep"])
        got = {"old_table": table, "old_lens": lens, "refs": refs, "status": status,
               "table": s["to_table"], "lens": s["to_lens"], "pools": s["pools"]}
    elif op == "compact":
        table, refs = s["table"].clone(), s["refs"].clone()
        pages = sd.Pages(block_table=table, seq_lens=s["lens"], refs=refs)
        remap, live = sd.sparse_decode_pages_compact(pages, pools=s["pools"])
        got = {"table": table, "refs": refs, "remap": remap, "live": live, "pools": s["pools"]}
    return got


# ---------------------------------------------------------------------------
# Work of a pass.
# ---------------------------------------------------------------------------
def _seen(case, L, c):
    """(positions that some of a sequence's c queries see, pairs of a query
    and a position that it sees)."""
    sink, w = case["sink"], case["window"]
    pairs = 0
    for p in range(L - c, L):
        lo = max(0, p - w + 1)
        pairs += p + 1 - lo + min(sink, lo)
    lo = max(0, L - c - w + 1)
    return L - lo + min(sink, lo), pairs


def work(case):
    op = case["op"]
    if op in ("copy", "beam", "compact", "admit"):
        page = PAGE * case.get("kv_heads", 0) * D * 2 * 2  # key and value
        if op == "copy":
            return {"bytes": 2 * case["moves"] * page + 8 * case["moves"], "flops": 0}
        if op == "beam":
            rows = case["prompts"] * case["beams"]
            entries = rows * ((case["n"] + case["n_min"]) // 2 // PAGE)
            # the tables (read, written), the reference counts, and a part-filled
            # page for most of the children
            fresh = rows if case["keep"] else rows * (case["beams"] - 1) // case["beams"] * 0.6
            return {"bytes": 16 * entries + 2 * fresh * page, "flops": 0}
        if op == "compact":
            moved = case["pages"] * case["live"] * (1 - case["live"])
            return {"bytes": 2 * moved * page + 16 * case["pages"], "flops": 0}
        each = (case["n"] + case["n_min"]) // 2 // PAGE
        return {"bytes": 4 * case["pages"] + 12 * case["leave"] * each, "flops": 0}
    lens = _lens(case)
    counts = _counts(case, lens)
    Hq, Hkv, T = case["q_heads"], case["kv_heads"], sum(counts)
    size = 4 if case["dtype"] == "f32" else 2
    row = D // 2 + D // GROUP if op.startswith("q4") else D * size
    total, flops = 0, 0
    if op in ("q4_step", "q4_fill"):  # read, write; read back, write
        total += 2 * T * Hkv * 2 * (2 * D + row)
    if op != "q4_fill":
        seen = [_seen(case, L, c) for L, c in zip(lens, counts)]
        total += 2 * T * Hq * D * size + 2 * row * Hkv * sum(x for x, _ in seen)
        flops = 4 * D * Hq * sum(x for _, x in seen)
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits.
# ---------------------------------------------------------------------------
def _exact_round(x):
    """What rows [T, H, 128] stand for once written in 4 bits, float64."""
    g = x.double().reshape(x.shape[0], x.shape[1], D // GROUP, GROUP)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, float(MIN_SCALE - 127))
    for t in range(MIN_SCALE - 127, 127):  # the smallest power of two that is large enough
        e = torch.where(top >= 7.0 * 2.0**t, float(t + 1), e)
    y = g.abs() / 2.0**e
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    lower = torch.clamp(torch.searchsorted(level, y.contiguous(), right=True) - 1, 0, 6)
    down, up = y - level[lower], level[lower + 1] - y
    pick = torch.where((down < up) | ((down == up) & (lower % 2 == 0)), lower, lower + 1)
    return (torch.sign(g) * level[pick] * 2.0**e).reshape(x.shape)


def _exact_row_values(s, name, b, L):
    """Keys or values [Hkv, L, 128] of sequence b, float64."""
    t = s[name]
    pages = s["table"][b, :-(-L // PAGE)].long() if s["paged"] else None
    if s["op"] == "window":
        if pages is None:
            return t[b, :, :L].double()
        return t[pages].double().flatten(0, 1)[:L].transpose(0, 1)

    def take(x):
        if pages is None:
            return x[b, :, :L]
        return x[pages].transpose(0, 1).flatten(1, 2)[:, :L]
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    codes, power = take(t).int(), 2.0 ** (take(s[name + "_scales"]).double() - 127.0)
    x = torch.empty(codes.shape[:2] + (D,), dtype=torch.float64, device="cuda")
    for odd in (0, 1):
        c = (codes >> (4 * odd)) & 15
        x[..., odd::2] = torch.where(c >= 8, -level[c & 7], level[c & 7])
    return x * power.repeat_interleave(GROUP, dim=-1)


def exact(case, seed):
    if case["op"] in ("copy", "beam", "compact", "admit"):
        return None
    s = prepare(case, seed)
    lens = _lens(case)
    counts = _counts(case, lens)
    got = {}
    if s["op"] in ("q4_step", "q4_fill"):
        got["k"], got["v"] = _exact_round(s["k_new"]), _exact_round(s["v_new"])
        if s["op"] == "q4_fill":
            return got
    Hkv = case["kv_heads"]
    G = case["q_heads"] // Hkv
    out, at = [], 0
    for b, (L, c) in enumerate(zip(lens, counts)):
        k, v = _exact_row_values(s, "k", b, L), _exact_row_values(s, "v", b, L)
        if s["op"] == "q4_step":  # the tokens of this step are written first
            k[:, L - c:] = got["k"][at:at + c].transpose(0, 1)
            v[:, L - c:] = got["v"][at:at + c].transpose(0, 1)
        q = s["q"][at:at + c].double().reshape(c, Hkv, G, D)
        p = torch.arange(L - c, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        sees = (j <= p) & ((j < case["sink"]) | (p - j < case["window"]))
        o = torch.empty((c, Hkv, G, D), dtype=torch.float64, device="cuda")
        for g in range(Hkv):
            for h in range(G):
                z = torch.where(sees, q[:, g, h] @ k[g].T / math.sqrt(D), -math.inf)
                o[:, g, h] = torch.softmax(z, dim=-1) @ v[g]
        out.append(o.reshape(c, Hkv * G, D))
        at += c
    got["out"] = torch.cat(out)
    return got if s["op"] != "window" else got["out"]
