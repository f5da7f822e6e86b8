"""Calls whose workgroups count each other do not depend on what an earlier call
left in the counters: calls that overlapped against the rules, or lengths that
changed under a call, may spoil their own results only.  The debug switch leaves
in every counter what a call before would have, had it stopped half way."""
import numpy as np
import pytest
import torch

from tests import plain64 as R

pytestmark = pytest.mark.gpu
LEFTOVERS = 128


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


@pytest.fixture
def leftovers(sd):
    yield lambda on: sd.set_debug(LEFTOVERS if on else 0)
    sd.set_debug(0)


def i32(a):
    return torch.tensor(np.array(a), dtype=torch.int32, device="cuda")


def captured(call):
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    return graph


@pytest.mark.parametrize("lens,hq,hkv", [([20011], 4, 1), ([5000, 17, 9000], 8, 2)])
def test_attention_in_parts(sd, leftovers, lens, hq, hkv):
    g = torch.Generator().manual_seed(len(lens))
    B, cap = len(lens), max(lens)
    k, v = torch.randn((2, B, hkv, cap, 128), generator=g).bfloat16().cuda()
    q = torch.randn((B, hq, 128), generator=g).bfloat16().cuda()
    cache, dl = sd.KVCache(k=k, v=v), i32(lens)
    c4 = sd.Q4Cache.empty(B, hkv, cap)
    starts = i32(np.concatenate(([0], np.cumsum(lens))))
    rows = lambda t: torch.cat([t[b, :, :L].transpose(0, 1) for b, L in enumerate(lens)]).contiguous()
    sd.sparse_decode_q4_append(rows(k), rows(v), c4, dl, starts=starts)
    calls = [lambda out=None: sd.sparse_decode_window_attention(q, cache, dl, sd.Window(), out=out),
             lambda out=None: sd.sparse_decode_q4_attention(q, c4, dl, out=out)]
    def others():   # (parts of other results in the library's memory)
        sd.sparse_decode_window_attention(-2 * q, cache, dl, sd.Window())
        sd.sparse_decode_q4_attention(-2 * q, c4, dl)

    for call in calls:
        want = call().clone()
        for on in (True, False, True):
            others()
            leftovers(on)
            assert torch.equal(call(), want)
        out = torch.zeros_like(want)
        for on in (True, False):
            leftovers(on)
            graph = captured(lambda: call(out=out))
            leftovers(True)
            for step in range(3):
                out.zero_()
                others()
                graph.replay()
                others()
                assert torch.equal(call(), want) and torch.equal(out, want)


@pytest.mark.parametrize("first", [False, True])
def test_many_calls_in_a_graph(sd, leftovers, first):
    # Calls of different sizes, in parts and whole, that take their counters in turn;
    # first: the graph begins with a call that needs none.
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn((2, 6, 2, 7000, 128), generator=g).bfloat16().cuda()
    q = torch.randn((6, 8, 128), generator=g).bfloat16().cuda()
    calls = []
    for n, L in ([(2, 30)] if first else []) + [(1, 7000), (6, 5000), (2, 20), (3, 6000), (6, 7000), (1, 900)]:
        cache = sd.KVCache(k=k[:n], v=v[:n])
        lens = i32([L - 7 * b for b in range(n)])
        window = sd.Window(3, 12 if L < 100 else 2**31 - 1)
        out = torch.zeros((n, 8, 128), dtype=torch.bfloat16, device="cuda")
        calls.append((lambda o, n=n, c=cache, l=lens, w=window:
                      sd.sparse_decode_window_attention(q[:n], c, l, w, out=o), out))
    want = [f(torch.zeros_like(out)) for f, out in calls]
    for on in (False, True):
        leftovers(on)
        graphs = [captured(lambda part=part: [f(out) for f, out in part])
                  for part in (calls, calls[::-1], calls[1:2], calls)]
        for step in range(3):
            for graph in graphs:
                for _, out in calls:
                    out.zero_()
                graph.replay()
                leftovers(on and step != 1)
                for i in (step, -1 - step):
                    assert torch.equal(calls[i][0](torch.zeros_like(want[i])), want[i])
                if graph is not graphs[2]:
                    assert all(torch.equal(out, w) for (_, out), w in zip(calls, want))
                else:
                    assert torch.equal(calls[1][1], want[1])


@pytest.mark.parametrize("rows,width,pages", [(3, 40, 100), (20, 300, 5000), (20, 900, 20000)])
def test_page_calls(sd, leftovers, rows, width, pages):
    rng = np.random.default_rng(pages)
    m = R.PagesModel(np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32), np.zeros(pages, np.int32))
    refs = i32(m.refs)
    a = sd.Pages(i32(m.table), i32(m.lens), refs)
    b = sd.Pages(torch.full_like(a.block_table, -1), torch.zeros_like(a.seq_lens), refs)
    grow, parents = i32([0] * rows), i32(range(rows))

    def step():
        sd.sparse_decode_pages_extend(a, grow)
        sd.sparse_decode_pages_fork(a, b, parents, keep=False)
        sd.sparse_decode_pages_extend(b, grow)
        sd.sparse_decode_pages_fork(b, a, parents, keep=False)
        sd.sparse_decode_pages_compact(a)

    def model(g, par):
        for half in range(2):
            m.extend(g)
            m.table, m.lens, _ = m.fork(rows, par, False)
        m.compact()

    leftovers(True)
    graph = captured(step)
    model([0] * rows, range(rows))
    for i in range(6):
        leftovers(i % 2 == 0)
        g, par = rng.integers(0, 16 * width // 6, rows), rng.integers(0, rows, rows)
        grow.copy_(i32(g))
        parents.copy_(i32(par))
        graph.replay() if i % 3 else step()
        model(g, par)
        assert np.array_equal(a.block_table.cpu().numpy(), m.table)
        assert np.array_equal(a.seq_lens.cpu().numpy(), m.lens)
        assert np.array_equal(refs.cpu().numpy(), m.refs)
