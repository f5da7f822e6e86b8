"""Window attention (sparse_decode_window_attention) against the plain 64-bit
form, through the binding: one query per sequence and chunks of queries, on
both layouts and types, at lengths around tiles, pages and windows."""
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


DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": R.U32, "bf16": 2.0**-8}


class Problem:
    """Sequences of the given lengths; everything that no sequence reaches
    (rows past a length, pages of no table) holds NaN."""

    def __init__(self, sd, lens, hq, hkv, layout, dtype, counts=None, cap=None, seed=0, gap=0):
        g = torch.Generator().manual_seed(seed)
        self.sd, self.lens, self.hq, self.hkv, self.dtype = sd, lens, hq, hkv, dtype
        self.counts = counts if counts is not None else [1] * len(lens)
        dt = DT[dtype]
        B, cap = len(lens), max(1, cap if cap is not None else max(lens))
        draw = lambda *s: torch.randn(s, generator=g).to(dt)
        self.k = [draw(hkv, L, 128) for L in lens]
        self.v = [draw(hkv, L, 128) for L in lens]
        T = sum(self.counts) + gap
        self.q = draw(T, hq, 128) * 2
        self.starts = torch.tensor(np.concatenate(([0], np.cumsum(self.counts))), dtype=torch.int32)
        nan = float("nan")
        if layout == "bhnd":
            k, v = torch.full((2, B, hkv, cap, 128), nan, dtype=dt)
            for b, L in enumerate(lens):
                k[b, :, :L], v[b, :, :L] = self.k[b], self.v[b]
            self.table = None
        else:
            per = [-(-L // 16) for L in lens]
            width, pages = -(-cap // 16), sum(per) + 3
            perm = torch.randperm(pages, generator=g).int()
            k, v = torch.full((2, pages, 16, hkv, 128), nan, dtype=dt)
            self.table = torch.full((B, width), -1, dtype=torch.int32)
            at = 0
            for b, L in enumerate(lens):
                self.table[b, :per[b]] = perm[at:at + per[b]]
                at += per[b]
                for j in range(0, L, 16):
                    page, n = int(self.table[b, j // 16]), min(16, L - j)
                    k[page, :n] = self.k[b][:, j:j + n].transpose(0, 1)
                    v[page, :n] = self.v[b][:, j:j + n].transpose(0, 1)
        self.cache = sd.KVCache(k=k.cuda(), v=v.cuda(), layout=layout,
                                block_table=self.table.cuda() if self.table is not None else None)
        self.dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def run(self, window, packed, **kw):
        starts = self.starts.cuda() if packed else None
        return self.sd.sparse_decode_window_attention(self.q.cuda(), self.cache, self.dev_lens,
                                                      window, q_starts=starts, **kw)

    def check(self, out, n_sink, window, scale=SCALE, hide=None):
        """hide(b, sees): positions of sequence b that no query sees."""
        out = out.double().cpu()
        at, worst = 0, 0.0
        for b, (L, n) in enumerate(zip(self.lens, self.counts)):
            got = out[at:at + n]
            real = min(n, L)
            assert (got[:n - real] == 0).all(), f"sequence {b}: rows before its first position"
            sees = R.visible(L, real, n_sink, window)
            if hide is not None:
                hide(b, sees)
            ref, allow = R.attention(self.q[at + n - real:at + n], self.k[b], self.v[b], sees,
                                     scale, HALF[self.dtype])
            err = (got[n - real:] - ref).abs()
            assert (err <= allow).all(), f"sequence {b}: {(err / allow).max():.3g} x the bound"
            if err.numel():
                worst = max(worst, float((err / allow).max()))
            at += n
        return worst


LENS = [0, 1, 15, 16, 17, 31, 33, 64, 100, 257, 700]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("n_sink,window", [(0, 2**31 - 1), (0, 1), (0, 0), (4, 0), (1, 16), (17, 33),
                                           (128, 64), (2**31 - 1, 1), (40, 2**31 - 1)])
def test_one_query_per_sequence(sd, dtype, layout, n_sink, window):
    pr = Problem(sd, LENS, 8, 2, layout, dtype)
    out = pr.run(sd.Window(n_sink, window), False)
    pr.check(out, n_sink, window)
    assert (out[0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (12, 6), (7, 1), (16, 1), (32, 2), (5, 5), (64, 8)])
def test_head_groups(sd, dtype, hq, hkv):
    pr = Problem(sd, [50, 333], hq, hkv, "paged", dtype, seed=1)
    pr.check(pr.run(sd.Window(3, 100), False), 3, 100)
    pr = Problem(sd, [50, 333], hq, hkv, "bhnd", dtype, counts=[9, 41], seed=2)
    pr.check(pr.run(sd.Window(3, 100), True), 3, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("n_sink,window", [(0, 2**31 - 1), (0, 1), (0, 0), (5, 0), (1, 16), (70, 33),
                                           (130, 200), (2**31 - 1, 1)])
def test_chunks(sd, dtype, layout, n_sink, window):
    lens = [0, 1, 16, 63, 65, 300, 501, 40, 640]
    counts = [2, 1, 5, 63, 0, 100, 129, 41, 33]   # more queries than positions, and none
    pr = Problem(sd, lens, 6, 2, layout, dtype, counts=counts, seed=3)
    pr.check(pr.run(sd.Window(n_sink, window), True), n_sink, window)


def test_long_sequences_split_over_workgroups(sd):
    for dtype, layout in (("bf16", "paged"), ("bf16", "bhnd"), ("f32", "paged")):
        pr = Problem(sd, [20011, 5], 4, 1, layout, dtype, seed=4)
        pr.check(pr.run(sd.Window(), False), 0, 2**31 - 1)
        pr.check(pr.run(sd.Window(100, 9000), False), 100, 9000)


@pytest.mark.parametrize("hq,hkv", [(32, 8), (16, 16), (8, 4)])
def test_many_sequences_on_pages(sd, hq, hkv):
    # Enough sequences and positions for workgroups of four KV heads, whole
    # and split.
    B = 128 // hkv * 2
    lens = [2100 + 61 * b % 900 for b in range(B)]
    lens[1], lens[2], lens[3] = 0, 1, 33
    pr = Problem(sd, lens, hq, hkv, "paged", "bf16", seed=16)
    pr.check(pr.run(sd.Window(), False), 0, 2**31 - 1)
    pr.check(pr.run(sd.Window(20, 2050), False), 20, 2050)


def test_softmax_scale_and_large_scores(sd):
    for scale in (1.0, 0.01, 3.0):
        pr = Problem(sd, [129, 700], 8, 2, "paged", "f32", seed=5)
        pr.check(pr.run(sd.Window(2, 300, scale), False), 2, 300, scale)
        pr = Problem(sd, [129, 700], 8, 2, "paged", "f32", counts=[100, 3], seed=5)
        pr.check(pr.run(sd.Window(2, 300, scale), True), 2, 300, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rising_scores_move_the_maximum_again_and_again(sd, dtype):
    # Keys grow with the position, so that the running maximum rises by far
    # more than the slack at almost every tile.
    for counts in (None, [70]):
        pr = Problem(sd, [900], 2, 1, "bhnd", dtype, counts=counts, seed=6)
        grow = (torch.arange(900) / 30.0)[None, :, None]
        u = torch.nn.functional.normalize(pr.q[0, 0].float(), dim=0)
        pr.k[0] = (pr.k[0].float() * 0.1 + grow * u).to(DT[dtype])
        pr.cache.k[0, :, :900] = pr.k[0].cuda()
        pr.check(pr.run(sd.Window(4, 800), counts is not None), 4, 800)


def test_equals_the_list_path_with_forced_positions_only(sd):
    # n_sink first and n_local last positions without a budget in between.
    pr = Problem(sd, [1000, 17, 444], 8, 2, "paged", "bf16", seed=7)
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    sp = sd.Sparsity(ratio=1.0, k_override=none, n_sink=20, n_local=200)
    ref, _ = sd.sparse_decode_attention(pr.q.cuda(), pr.cache, pr.dev_lens, sp, k_max=220)
    got = pr.run(sd.Window(20, 200), False)
    assert (ref.float() - got.float()).abs().max() < 2e-2
    pr.check(got, 20, 200)


def test_pages_outside_the_pool_are_seen_by_no_query(sd):
    for packed, counts in ((False, None), (True, [3, 90])):
        for dtype in ("bf16", "f32"):
            pr = Problem(sd, [40, 400], 4, 2, "paged", dtype, counts=counts, seed=8)
            bt = pr.cache.block_table
            bt[1, 3], bt[1, 24], bt[0, 0] = -1, bt.new_tensor(10**9), pr.cache.k.shape[0]

            def hide(b, sees):
                for page in ([0] if b == 0 else [3, 24]):
                    sees[:, 16 * page:16 * page + 16] = False
            pr.check(pr.run(sd.Window(64, 200), packed), 64, 200, hide=hide)
            bt.fill_(-7)
            assert (pr.run(sd.Window(64, 200), packed) == 0).all()


def test_rows_of_no_sequence_are_left(sd):
    pr = Problem(sd, [30, 70], 4, 2, "bhnd", "bf16", counts=[5, 20], gap=7, seed=9)
    pr.starts += 3                      # rows 0..2 before the first, 28..31 behind the last
    pr.q = torch.roll(pr.q, 3, 0)
    out = torch.full_like(pr.q, 9.0).cuda()
    pr.run(sd.Window(2, 10), True, out=out)
    assert (out[:3] == 9).all() and (out[28:] == 9).all()
    pr.q = pr.q[3:28]
    pr.check(out[3:28], 2, 10)


def test_lengths_outside_the_capacity_are_clamped(sd):
    pr = Problem(sd, [64, 64], 4, 2, "paged", "bf16", seed=10)
    pr.dev_lens = torch.tensor([10**6, -5], dtype=torch.int32, device="cuda")
    out = pr.run(sd.Window(2, 10), False)
    assert (out[1] == 0).all()
    pr.lens, pr.counts = [64], [1]
    pr.check(out[:1], 2, 10)


def test_positions_between_sinks_and_window_may_hold_anything(sd):
    for counts in (None, [40]):
        for dtype in ("bf16", "f32"):
            pr = Problem(sd, [300], 4, 2, "bhnd", dtype, counts=counts, seed=11)
            n = 1 if counts is None else 40
            for bad in (float("nan"), float("inf"), -float("inf")):
                pr.cache.k[0, :, 10:300 - n - 100 + 1] = bad
                pr.cache.v[0, :, 10:300 - n - 100 + 1] = bad
                pr.check(pr.run(sd.Window(10, 100), counts is not None), 10, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_a_window_only_the_first_tokens_are_read(sd, dtype):
    for counts in (None, [40], [300]):
        pr = Problem(sd, [300], 4, 2, "bhnd", dtype, counts=counts, seed=17)
        for bad in (float("nan"), float("inf")):
            pr.cache.k[0, :, 5:300] = bad
            pr.cache.v[0, :, 5:300] = bad
            pr.check(pr.run(sd.Window(5, 0), counts is not None), 5, 0)


def uneven(n, most, seed):
    """n lengths from 0 to most, log-uniform."""
    x = np.random.default_rng(seed).uniform(0, np.log(most + 1), n)
    lens = np.floor(np.exp(x)).astype(int) - 1
    lens[n // 2] = most
    return [int(v) for v in lens]


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,most,hq,hkv", [(2, 9000, 4, 1), (9, 5000, 8, 8), (17, 3000, 4, 4),
                                           (65, 1500, 3, 1), (130, 700, 2, 2), (256, 400, 1, 1),
                                           (257, 400, 1, 1)])
def test_sequences_of_very_different_lengths(sd, layout, dtype, n, most, hq, hkv):
    # (cut into parts by a plan over all lengths, 64 sequences at a time)
    pr = Problem(sd, uneven(n, most, n), hq, hkv, layout, dtype, seed=n, cap=2 * most)
    for sink, window in ((0, ALL), (40, 600)):
        pr.check(pr.run(sd.Window(sink, window), False), sink, window)
    same = Problem(sd, [most // 4] * n, hq, hkv, layout, dtype, seed=n + 1)
    same.check(same.run(sd.Window(), False), 0, ALL)


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,most,few,hq,hkv", [(2, 6000, 5, 4, 1), (5, 4000, 40, 8, 2), (1, 5000, 3, 6, 2),
                                               (1, 4000, 130, 8, 2), (70, 1200, 3, 2, 1),
                                               (200, 600, 2, 1, 1), (9, 3000, 70, 16, 1)])
def test_chunks_of_sequences_of_very_different_lengths(sd, layout, dtype, n, most, few, hq, hkv):
    # (few rows over long contexts, cut into parts by a plan over all lengths)
    lens = uneven(n, most, 100 + n)
    counts = [int(c) for c in np.random.default_rng(n).integers(0, few + 1, n)]
    counts[n // 2] = few
    pr = Problem(sd, lens, hq, hkv, layout, dtype, counts=counts, seed=n, cap=2 * most)
    for sink, window in ((0, ALL), (40, most // 2)):
        pr.check(pr.run(sd.Window(sink, window), True), sink, window)
    same = Problem(sd, [most] * min(n, 20), hq, hkv, layout, dtype, counts=[few] * min(n, 20), seed=n + 1)
    same.check(same.run(sd.Window(), True), 0, ALL)


def test_pages_of_four_heads_to_a_workgroup(sd):
    # (enough heads, sequences and tiles for the variant: 64 x 4 x 150)
    pr = Problem(sd, uneven(64, 2399, 3), 8, 4, "paged", "bf16", seed=19)
    pr.check(pr.run(sd.Window(), False), 0, ALL)
    pr = Problem(sd, [2390 - i for i in range(64)], 4, 4, "paged", "bf16", seed=20)
    pr.check(pr.run(sd.Window(33, 2300), False), 33, 2300)


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [None, [33, 1], [2, 7]])
def test_a_nan_that_a_query_sees_reaches_its_output(sd, dtype, layout, counts):
    # Sequence 0's last query sees the position; sequence 1 and the other KV
    # head do not.  (3000 positions: over several workgroups.)
    pr = Problem(sd, [3000, 40], 4, 2, layout, dtype, counts=counts, seed=18)
    at = (0, 0, 2990) if layout == "bhnd" else (int(pr.table[0, 2990 // 16]), 2990 % 16, 0)
    last, w = (0 if counts is None else counts[0] - 1), sd.Window(0, 2500)
    for t, channels in ((pr.cache.v, [5]), (pr.cache.k, list(range(128)))):
        t[(*at, 5)] = float("nan")
        out = pr.run(w, counts is not None)
        nan = torch.isnan(out).cpu()
        assert nan[last, :2, channels].all()
        assert nan[last, :2].sum() == 2 * len(channels)
        assert not nan[:, 2:].any() and not nan[last + 1:].any()


def test_replayed_graphs_and_other_streams(sd):
    for counts in (None, [33, 1]):
        pr = Problem(sd, [3000, 600], 8, 2, "paged", "bf16", counts=counts, seed=12)
        q, starts = pr.q.cuda(), pr.starts.cuda() if counts else None
        w = sd.Window(16, 2000)
        eager = sd.sparse_decode_window_attention(q, pr.cache, pr.dev_lens, w, q_starts=starts)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        other = sd.sparse_decode_window_attention(q, pr.cache, pr.dev_lens, w, q_starts=starts,
                                                  stream=s)
        s.synchronize()
        assert torch.equal(eager, other)
        out = torch.zeros_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sd.sparse_decode_window_attention(q, pr.cache, pr.dev_lens, w, q_starts=starts, out=out)
        for step in range(4):
            pr.dev_lens.fill_(3000 - 7 * step)
            pr.dev_lens[1] = 600 - step
            graph.replay()
            torch.cuda.synchronize()
            ref = sd.sparse_decode_window_attention(q, pr.cache, pr.dev_lens, w, q_starts=starts)
            assert torch.equal(out, ref)
            (out * 2).sum().item()


def test_no_workspace_is_used(sd):
    # Split calls with a caller's workspace too small for any partial.
    for counts in (None, [3]):
        pr = Problem(sd, [20000], 4, 1, "bhnd", "bf16", counts=counts, seed=13)
        eager = pr.run(sd.Window(), counts is not None)
        try:
            sd.set_workspace(torch.empty(256, dtype=torch.uint8, device="cuda"))
            assert torch.equal(pr.run(sd.Window(), counts is not None), eager)
        finally:
            sd.set_workspace(None)
        pr.check(eager, 0, 2**31 - 1)


def test_offsets_past_32_bits(sd):
    # 2.2e9 elements of keys; the sequence's pages are the last ones.
    pages = 135000
    k = torch.empty((pages, 16, 8, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Problem(sd, [500], 16, 8, "paged", "bf16", seed=14)
    n = small.cache.k.shape[0]
    k[-n:], v[-n:] = small.cache.k, small.cache.v
    bt = torch.where(small.cache.block_table >= 0, small.cache.block_table + (pages - n), -1).int()
    small.cache = sd.KVCache(k=k, v=v, layout="paged", block_table=bt)
    small.check(small.run(sd.Window(9, 300), False), 9, 300)
    small.check(small.run(sd.Window(9, 300), True), 9, 300)
    # a contiguous cache whose second sequence starts past 2^32 bytes
    kc = torch.empty((2, 8, 1 << 20, 128), dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    pr = Problem(sd, [400, 333], 8, 8, "bhnd", "bf16", seed=15)
    kc[:, :, :400], vc[:, :, :400] = pr.cache.k, pr.cache.v
    pr.cache = sd.KVCache(k=kc, v=vc)
    pr.check(pr.run(sd.Window(9, 300), False), 9, 300)
    pr.check(pr.run(sd.Window(9, 300), True), 9, 300)


def test_empty_calls(sd):
    pr = Problem(sd, [5], 4, 2, "bhnd", "bf16")
    q = pr.q.cuda()[:0]
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = sd.sparse_decode_window_attention(q, pr.cache, pr.dev_lens, sd.Window(), q_starts=none)
    assert out.shape == (0, 4, 128)


def test_two_graphs_replayed_in_turn(sd):
    # (both keep partials in the library's memory; one stream orders them)
    a = Problem(sd, [5000, 40, 1200], 8, 2, "paged", "bf16", seed=31)
    b = Problem(sd, [4000, 700], 8, 2, "bhnd", "bf16", counts=[6, 2], seed=32)
    calls = []
    for pr, packed in ((a, False), (b, True)):
        q, starts = pr.q.cuda(), pr.starts.cuda() if packed else None
        out = torch.zeros_like(q)
        run = lambda pr=pr, q=q, starts=starts, out=None: sd.sparse_decode_window_attention(
            q, pr.cache, pr.dev_lens, sd.Window(8, 4500), q_starts=starts, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(out=out)
        calls.append((run, graph, out))
    for step in range(4):
        for _, graph, out in calls:
            out.zero_()
            graph.replay()
        calls[step % 2][0]()          # an eager call between the replays
        for run, graph, out in calls:
            graph.replay()
        torch.cuda.synchronize()
        for run, _, out in calls:
            assert torch.equal(out, run())
        a.dev_lens -= 3
        b.dev_lens -= 1
