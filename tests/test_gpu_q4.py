"""The 4-bit cache (sparse_decode_q4_append, _load, _attention) against the
plain 64-bit form: every stored value and scale byte exactly, attention within
its derived bound."""
import math

import numpy as np
import pytest
import torch

from tests import plain64 as R

pytestmark = pytest.mark.gpu
SCALE = 128**-0.5
ALL = 2**31 - 1


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


def new_cache(sd, lens, hkv, layout, seed=0, fill=None):
    """A cache for sequences of these lengths; fill: what its bytes hold."""
    g = torch.Generator().manual_seed(seed)
    cap = max(1, max(lens))
    if layout == "bhnd":
        c = sd.Q4Cache.empty(len(lens), hkv, cap)
    else:
        per = [-(-L // 16) for L in lens]
        perm = torch.randperm(sum(per) + 2, generator=g).int()
        table = torch.full((len(lens), -(-cap // 16)), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(per):
            table[b, :m] = perm[at:at + m]
            at += m
        c = sd.Q4Cache.empty_paged(len(perm), hkv, table.cuda())
    if fill is not None:
        for t in c.pools:
            t.fill_(fill)
    return c


def rows_of(c, codes, scales, b, L):
    """Stored rows [Hkv, L, ...] of sequence b on the host."""
    if c.layout == "bhnd":
        return codes[b, :, :L].cpu(), scales[b, :, :L].cpu()
    pages = c.block_table[b, :-(-L // 16)].long()
    join = lambda t: t[pages].transpose(0, 1).flatten(1, 2)[:, :L].cpu()
    return join(codes), join(scales)


def starts_of(counts):
    return torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device="cuda")


def hard_rows(n, hkv, seed=0):
    """Rows with every kind of group: normal, tiny, huge, zero, ties, at the
    border between two scales, one large value among small ones."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, hkv, 4, 32), generator=g)
    x *= torch.pow(2.0, torch.randint(-20, 20, (n, hkv, 4, 1), generator=g).float())
    kind = torch.randint(0, 8, (n, hkv, 4), generator=g)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    pick = ties[torch.randint(0, 8, (n, hkv, 4, 32), generator=g)]
    x = torch.where((kind == 1)[..., None], pick * x[..., :1].sign(), x)
    x = torch.where((kind == 2)[..., None], 0.0, x)
    edge = torch.tensor([7.0, 6.9375, 7.0625, 3.5, 1.75])[torch.randint(0, 5, (n, hkv, 4, 1), generator=g)]
    x[..., :1] = torch.where((kind == 3)[..., None], edge, x[..., :1])
    x = torch.where((kind == 3)[..., None], x.clamp(-edge, edge), x)
    x = torch.where((kind == 4)[..., None], x * 2.0**-90, x)
    x = torch.where((kind == 5)[..., None], x * 2.0**80, x)
    return x.reshape(n, hkv, 128)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["bhnd", "paged"])
def test_append_stores_the_nearest_levels_and_load_returns_them(sd, dtype, layout):
    lens, counts, hkv = [40, 0, 1, 100, 33], [40, 0, 1, 55, 40], 3
    c = new_cache(sd, lens, hkv, layout, fill=170)
    before = [t.clone() for t in c.pools]
    T = sum(counts)
    k, v = hard_rows(T, hkv, 1).to(dtype), hard_rows(T, hkv, 2).to(dtype)
    dl, st = torch.tensor(lens, dtype=torch.int32, device="cuda"), starts_of(counts)
    sd.sparse_decode_q4_append(k.cuda(), v.cuda(), c, dl, starts=st)
    for got_dtype in (torch.bfloat16, torch.float32):
        lk, lv = sd.sparse_decode_q4_load(c, dl, starts=st, tokens=T, dtype=got_dtype)
        at = 0
        for b, (L, n) in enumerate(zip(lens, counts)):
            real = min(n, L)
            for x, codes, scales, loaded in ((k, c.k, c.k_scales, lk), (v, c.v, c.v_scales, lv)):
                want, wscale = R.q4_round(x[at + n - real:at + n])
                cc, ss = rows_of(c, codes, scales, b, L)
                assert torch.equal(ss[:, L - real:].transpose(0, 1), wscale)
                val = R.q4_decode(cc, ss)[:, L - real:].transpose(0, 1)
                assert torch.equal(val, want)
                assert torch.equal(loaded[at + n - real:at + n].double().cpu(), want)
                assert (loaded[at:at + n - real] == 0).all()    # before the first position
                assert (cc[:, :L - real] == 170).all()          # older rows stay
            at += n
    if layout == "paged":  # pages of no sequence stay
        used = c.block_table[c.block_table >= 0].long()
        free = torch.ones(c.k.shape[0], dtype=torch.bool, device="cuda")
        free[used] = False
        for t, old in zip(c.pools, before):
            assert torch.equal(t[free], old[free])


def test_every_bfloat16_number(sd):
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x)]
    x = x[:x.numel() // 32 * 32].reshape(-1, 32)
    small = torch.randperm(x.numel(), generator=torch.Generator().manual_seed(0)).reshape(x.shape)
    rows = torch.cat((x, x.flatten()[small]))       # groups of neighbours, and mixed ones
    rows = rows[:rows.shape[0] // 4 * 4].reshape(-1, 1, 128)
    n = rows.shape[0]
    c = sd.Q4Cache.empty(1, 1, n)
    dl = torch.tensor([n], dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(rows.cuda(), rows.cuda(), c, dl, starts=starts_of([n]))
    k, v = sd.sparse_decode_q4_load(c, dl, starts=starts_of([n]), tokens=n, dtype=torch.float32)
    want, scale = R.q4_round(rows)
    assert torch.equal(c.k_scales[0, 0].cpu(), scale[:, 0])
    assert torch.equal(R.q4_decode(c.k[0, 0].cpu(), c.k_scales[0, 0].cpu()), want[:, 0])
    fits = want.abs() < 3.4e38          # 6 * 2^126 is above every float32
    assert torch.equal(k.double().cpu()[fits], want[fits]) and torch.equal(k, v)


def test_groups_that_are_not_numbers(sd):
    x = torch.randn(6, 2, 128)
    x[0, 0, 5], x[1, 1, 40], x[2, 0, 127] = math.nan, math.inf, -math.inf
    c = sd.Q4Cache.empty(6, 2, 3)
    dl = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(x.cuda(), x.cuda(), c, dl)
    k, _ = sd.sparse_decode_q4_load(c, dl)
    want, _ = R.q4_round(x)
    assert torch.equal(torch.isnan(k.cpu()), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(k.double().cpu()[ok], want[ok]) and int((~ok).sum()) == 96


def test_append_skips_bad_pages_and_rows_of_no_sequence(sd):
    c = new_cache(sd, [48, 48], 2, "paged", fill=3)
    c.block_table[0, 1], c.block_table[1, 0] = -1, 10**6
    before = [t.clone() for t in c.pools]
    x = torch.randn(100, 2, 128)
    dl = torch.tensor([48, 48], dtype=torch.int32, device="cuda")
    st = torch.tensor([2, 50, 98], dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(x.cuda(), x.cuda(), c, dl, starts=st)
    out = torch.full((100, 2, 128), 7.0, device="cuda")
    out2 = out.clone()
    sd.sparse_decode_q4_load(c, dl, starts=st, k=out, v=out2)
    want, _ = R.q4_round(x)
    assert (out[:2] == 7).all() and (out[98:] == 7).all()
    assert (out[18:34] == 0).all() and (out[50:66] == 0).all()   # the two bad pages
    for a, b in ((2, 18), (34, 50), (66, 98)):
        assert torch.equal(out[a:b].double().cpu(), want[a:b])
    bt = c.block_table
    used = bt[(bt >= 0) & (bt < c.k.shape[0])].long()
    rest = torch.ones(c.k.shape[0], dtype=torch.bool, device="cuda")
    rest[used] = False
    assert all(torch.equal(t[rest], o[rest]) for t, o in zip(c.pools, before))


def random_cache(sd, lens, hkv, layout, seed=0):
    """Random codes and scales in the sequences' rows; scale 255 (NaN) and
    wild codes everywhere else.  Returns the cache and rows [Hkv, L, 128]."""
    g = torch.Generator().manual_seed(seed)
    c = new_cache(sd, lens, hkv, layout, seed, fill=255)
    rows = []
    for b, L in enumerate(lens):
        pair = []
        for codes, scales in ((c.k, c.k_scales), (c.v, c.v_scales)):
            x = torch.randint(0, 256, (hkv, L, 64), generator=g, dtype=torch.uint8)
            s = torch.randint(122, 128, (hkv, L, 4), generator=g, dtype=torch.uint8)
            for t, r in ((codes, x), (scales, s)):
                if layout == "bhnd":
                    t[b, :, :L] = r.cuda()
                else:
                    for j in range(0, L, 16):
                        n = min(16, L - j)
                        t[int(c.block_table[b, j // 16]), :, :n] = r[:, j:j + n].cuda()
            pair.append(R.q4_decode(x, s))
        rows.append(pair)
    return c, rows


def check_attention(sd, lens, hq, hkv, layout, n_sink=0, window=ALL, seed=0, scale=SCALE, null=False,
                    hide=None, change=None):
    c, rows = random_cache(sd, lens, hkv, layout, seed)
    if change is not None:
        change(c)
    q = torch.randn((len(lens), hq, 128), generator=torch.Generator().manual_seed(seed + 9)).bfloat16()
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    w = None if null else sd.Window(n_sink, window, 0.0 if scale == SCALE else scale)
    out = sd.sparse_decode_q4_attention(q.cuda(), c, dl, w)
    got = out.double().cpu()
    for b, L in enumerate(lens):
        sees = R.visible(L, min(1, L), n_sink, window)
        if hide is not None:
            hide(b, sees)
        ref, allow = R.attention(q[b:b + min(1, L)], rows[b][0], rows[b][1], sees, scale, 2.0**-8)
        if L == 0:
            assert (got[b] == 0).all()
            continue
        err = (got[b:b + 1] - ref).abs()
        assert (err <= allow).all(), f"sequence {b} (L {L}): {(err / allow).max():.3g} x the bound"
    return out


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("n_sink,window", [(0, ALL), (0, 1), (0, 0), (4, 0), (1, 16), (17, 33), (128, 64)])
def test_attention(sd, layout, n_sink, window):
    check_attention(sd, [0, 1, 15, 16, 17, 31, 33, 64, 100, 257, 700], 8, 2, layout, n_sink, window)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (12, 6), (7, 1), (16, 1), (32, 2), (64, 8)])
def test_attention_head_groups(sd, hq, hkv):
    check_attention(sd, [50, 333], hq, hkv, "paged", 3, 100, seed=1)
    check_attention(sd, [50, 333], hq, hkv, "bhnd", seed=2, null=True)


def test_attention_long_and_other_scales(sd):
    check_attention(sd, [20011, 6, 4097], 8, 2, "paged", seed=3)
    check_attention(sd, [20011, 6, 4097], 8, 2, "bhnd", 100, 9000, seed=4)
    check_attention(sd, [300], 8, 2, "bhnd", seed=5, scale=1.0)


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("n,most,hq,hkv", [(2, 9000, 4, 1), (9, 5000, 8, 8), (65, 1500, 3, 1),
                                           (200, 700, 2, 2)])
def test_attention_over_very_different_lengths(sd, layout, n, most, hq, hkv):
    lens = np.floor(np.exp(np.random.default_rng(n).uniform(0, np.log(most + 1), n))).astype(int) - 1
    lens = [int(x) for x in lens] + [most]
    check_attention(sd, lens, hq, hkv, layout, seed=n)
    check_attention(sd, lens, hq, hkv, layout, 30, 500, seed=n)


def test_attention_skips_pages_outside_the_pool(sd):
    def change(c):
        c.block_table[0, 0], c.block_table[1, 5] = c.k.shape[0], -3

    def hide(b, sees):
        page = (0, 5)[b]
        sees[:, 16 * page:16 * page + 16] = False
    check_attention(sd, [40, 400], 4, 2, "paged", 32, 350, seed=6, hide=hide, change=change)


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
def test_groups_that_are_not_numbers_reach_the_output(sd, layout):
    lens = [3000, 40]
    c, _ = random_cache(sd, lens, 2, layout, seed=8)
    q = torch.randn((2, 4, 128), device="cuda").bfloat16()
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    at = (0, 0, 2990) if layout == "bhnd" else (int(c.block_table[0, 2990 // 16]), 0, 2990 % 16)
    for scales, channels in ((c.v_scales, range(32, 64)), (c.k_scales, range(128))):
        scales[(*at, 1)] = 255
        nan = torch.isnan(sd.sparse_decode_q4_attention(q, c, dl)).cpu()
        assert nan[0, :2, list(channels)].all()
        assert nan.sum() == 2 * len(channels)


def test_replayed_step(sd):
    """Append, then attend, captured once and replayed with new tokens."""
    B, hq, hkv, cap = 3, 8, 2, 500
    c, rows = random_cache(sd, [cap] * B, hkv, "bhnd", seed=7)
    k, v = torch.randn((2, B, hkv, 128), device="cuda").bfloat16()
    q = torch.randn((B, hq, 128), device="cuda").bfloat16()
    dl = torch.tensor([17, 300, 499], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    sd.sparse_decode_q4_append(k, v, c, dl)
    sd.sparse_decode_q4_attention(q, c, dl, out=out)   # workspace before the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sparse_decode_q4_append(k, v, c, dl)
        sd.sparse_decode_q4_attention(q, c, dl, out=out)
    for step in range(4):
        for t in (k, v, q):
            t.normal_()
        dl += 1 if step else 0
        if step == 3:
            dl[2] = cap
        graph.replay()
        torch.cuda.synchronize()
        got, stored = out.clone(), [t.clone() for t in c.pools]
        sd.sparse_decode_q4_append(k, v, c, dl)
        ref = sd.sparse_decode_q4_attention(q, c, dl)
        assert torch.equal(got, ref)
        assert all(torch.equal(a, b) for a, b in zip(stored, c.pools))
        back, _ = sd.sparse_decode_q4_load(c, dl)
        assert torch.equal(back.double().cpu(), R.q4_round(k.cpu())[0])


def test_offsets_past_32_bits(sd):
    # 4.4 GB of codes, the sequences' rows behind them
    c = sd.Q4Cache.empty(2, 8, 1 << 22)
    q = torch.randn((2, 8, 128)).bfloat16()
    k, v = torch.randn((2, 600, 8, 128)).bfloat16()
    lens, counts = [300, (1 << 22)], [300, 300]
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(k.cuda(), v.cuda(), c, dl, starts=starts_of(counts))
    kk, _ = sd.sparse_decode_q4_load(c, dl, starts=starts_of(counts), tokens=600)
    assert torch.equal(kk.double().cpu(), R.q4_round(k)[0])
    out = sd.sparse_decode_q4_attention(q.cuda(), c, dl, sd.Window(0, 300)).double().cpu()
    for b in range(2):
        kb, vb = (R.q4_round(t[300 * b:300 * b + 300])[0].transpose(0, 1) for t in (k, v))
        ref, allow = R.attention(q[b:b + 1], kb, vb, R.visible(300, 1, 0, 300), SCALE, 2.0**-8)
        assert ((out[b:b + 1] - ref).abs() <= allow).all()
