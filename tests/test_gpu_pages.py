"""The page operations against a plain model of them, entry by entry."""
import numpy as np
import pytest
import torch

from tests import plain64 as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


def cuda(a):
    return torch.from_numpy(np.array(a)).to("cuda", torch.int32)


def random_state(rng, rows, width, pages, share=0.3, full=0.5):
    """Tables whose rows share their first pages now and then."""
    table = np.full((rows, width), -1, np.int32)
    lens, refs = np.zeros(rows, np.int32), np.zeros(pages, np.int32)
    free = list(rng.permutation(pages))
    for b in range(rows):
        if rng.random() < 0.15:
            continue
        shared = 0
        if b and rng.random() < share:
            r = rng.integers(b)
            shared = int(rng.integers(0, lens[r] // 16 + 1))
            table[b, :shared] = table[r, :shared]
        own = int(min(len(free), rng.integers(0, width - shared + 1), max(1, pages * full / rows)))
        table[b, shared:shared + own] = [free.pop() for _ in range(own)]
        n = shared + own
        lens[b] = 16 * n - (int(rng.integers(0, 16)) if own else 0)
        np.add.at(refs, table[b, :n], 1)
    return table, lens, refs


def pools_for(pages, seed=0, heads=2):
    """Pools of every kind: keys, values, 4-bit codes and scales, labels, and
    one whose pages are an odd number of bytes."""
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn((pages,) + s, generator=g)
    u = lambda *s: torch.randint(0, 256, (pages,) + s, generator=g, dtype=torch.uint8)
    return [f(16, heads, 128).bfloat16(), f(16, heads, 128), u(heads, 16, 64), u(heads, 16, 4),
            torch.arange(pages, dtype=torch.int32).reshape(pages, 1)]


def model_and_pages(sd, state, pools):
    table, lens, refs = state
    m = R.PagesModel(table, lens, refs, [p.float().numpy() for p in pools])
    return m, sd.Pages(cuda(table), cuda(lens), cuda(refs)), [p.cuda() for p in pools]


def same(m, pages, pools=()):
    assert np.array_equal(pages.block_table.cpu().numpy(), m.table)
    assert np.array_equal(pages.seq_lens.cpu().numpy(), m.lens)
    assert np.array_equal(pages.refs.cpu().numpy(), m.refs)
    for got, want in zip(pools, m.pools):
        assert np.array_equal(got.float().cpu().numpy(), want)


SIZES = [(1, 1, 1), (3, 4, 10), (17, 9, 100), (40, 60, 1500), (300, 20, 5000), (5, 3000, 9000)]


@pytest.mark.parametrize("rows,width,pages", SIZES)
def test_extend(sd, rows, width, pages):
    for seed in range(4):
        rng = np.random.default_rng(seed)
        m, p, _ = model_and_pages(sd, random_state(rng, rows, width, pages), [])
        for step in range(4):
            grow = rng.integers(-3, 16 * width // (2 + step) + 2, rows)
            if step == 1:
                grow[:] = 1
            status = sd.sparse_decode_pages_extend(p, cuda(grow))
            assert np.array_equal(status.cpu().numpy(), m.extend(grow))
            same(m, p)


@pytest.mark.parametrize("rows,width,pages", SIZES)
@pytest.mark.parametrize("keep", [True, False])
def test_fork(sd, rows, width, pages, keep):
    for seed in range(3):
        rng = np.random.default_rng(10 + seed)
        small = pages <= 1500
        m, p, pools = model_and_pages(sd, random_state(rng, rows, width, pages, full=0.9 if seed == 2 else 0.5),
                                      pools_for(pages, seed) if small else [])
        n = int(rng.integers(1, 2 * rows + 2))
        parents = rng.integers(-1, rows + 1, n)
        to = sd.Pages(torch.full((n, width), 77, dtype=torch.int32, device="cuda"),
                      torch.full((n,), 77, dtype=torch.int32, device="cuda"), p.refs)
        status = sd.sparse_decode_pages_fork(p, to, cuda(parents), pools=pools, keep=keep)
        table, lens, want = m.fork(n, parents, keep)
        assert np.array_equal(status.cpu().numpy(), want)
        assert np.array_equal(to.block_table.cpu().numpy(), table)
        assert np.array_equal(to.seq_lens.cpu().numpy(), lens)
        same(m, p, pools)


@pytest.mark.parametrize("rows,width,pages", SIZES)
def test_free(sd, rows, width, pages):
    rng = np.random.default_rng(20)
    m, p, _ = model_and_pages(sd, random_state(rng, rows, width, pages), [])
    gone = rng.integers(-2, rows + 2, rows // 2 + 3)
    gone = np.concatenate((gone, gone[:2]))     # rows listed twice
    sd.sparse_decode_pages_free(p, cuda(gone))
    m.free(gone)
    same(m, p)


@pytest.mark.parametrize("rows,width,pages", SIZES)
def test_compact(sd, rows, width, pages):
    for seed in range(3):
        rng = np.random.default_rng(30 + seed)
        pools = pools_for(pages, seed) if pages <= 1500 else pools_for(pages, seed, 1)[2:]
        m, p, pools = model_and_pages(sd, random_state(rng, rows, width, pages, full=(0.2, 0.5, 1.0)[seed]),
                                      pools)
        remap, live = sd.sparse_decode_pages_compact(p, pools=pools)
        want, n = m.compact()
        assert int(live) == n and np.array_equal(remap.cpu().numpy(), want)
        same(m, p, pools)
        remap, live = sd.sparse_decode_pages_compact(p, pools=pools)   # nothing left to do
        want, n = m.compact()
        assert int(live) == n and np.array_equal(remap.cpu().numpy(), want)
        same(m, p, pools)


@pytest.mark.parametrize("pages,n", [(2, 1), (50, 20), (3000, 1500)])
def test_copy(sd, pages, n):
    rng = np.random.default_rng(40)
    pools = pools_for(pages) if pages < 100 else pools_for(pages, heads=1)
    if pages < 100:  # pages of 35 bytes, and a base that is not aligned
        raw = torch.randint(0, 256, (pages * 35 + 1,), dtype=torch.uint8)
        pools.append(raw[1:].reshape(pages, 5, 7))
    m = R.PagesModel([[0]], [0], np.zeros(pages, np.int32), [p.float().numpy() for p in pools])
    dev = [p.cuda() for p in pools]
    if pages < 100:
        dev[-1] = raw.cuda()[1:].reshape(pages, 5, 7)
    perm = rng.permutation(pages)
    src, dst = perm[:n].copy(), perm[n:2 * n].copy()
    if n > 3:
        src[0], dst[1], dst[2] = -1, pages, -5
    sd.sparse_decode_pages_copy(dev, cuda(src), cuda(dst))
    m.copy(src, dst)
    for got, want in zip(dev, m.pools):
        assert np.array_equal(got.float().cpu().numpy(), want)


def test_copy_of_one_misaligned_pool(sd):
    for off, size in ((1, 35), (4, 20), (8, 40)):
        raw = torch.randint(0, 256, (10 * size + off,), dtype=torch.uint8, device="cuda")
        want = raw.clone()
        sd.sparse_decode_pages_copy([raw[off:].reshape(10, size)], cuda([0, 3, 9]), cuda([1, 7, 2]))
        v = want[off:].reshape(10, size)
        v[[1, 7, 2]] = v[[0, 3, 9]]
        assert torch.equal(raw, want)


def test_no_pools_and_no_rows(sd):
    p = sd.Pages(cuda(np.zeros((0, 4), np.int32)), cuda(np.zeros(0)), cuda([1, 0, 1]))
    assert sd.sparse_decode_pages_extend(p, cuda(np.zeros(0))).shape == (0,)
    sd.sparse_decode_pages_free(p, cuda([0, 1]))
    remap, n = sd.sparse_decode_pages_compact(p)
    assert remap.tolist() == [0, -1, 1] and int(n) == 2 and p.refs.tolist() == [1, 1, 0]
    e = sd.Pages(cuda(np.zeros((2, 0), np.int32)), cuda([0, 0]), cuda(np.zeros(0)))
    assert sd.sparse_decode_pages_extend(e, cuda([0, 1])).tolist() == [0, 2]
    sd.sparse_decode_pages_copy([], cuda([0]), cuda([1]))


def test_a_large_pool(sd):
    pages = 1 << 20
    rng = np.random.default_rng(50)
    refs = (rng.random(pages) < 0.7).astype(np.int32)
    m, p, _ = model_and_pages(sd, (np.full((3, 40000), -1, np.int32), np.zeros(3, np.int32), refs), [])
    grow = np.array([16 * 30000, 5, 16 * 39999])
    status = sd.sparse_decode_pages_extend(p, cuda(grow))
    assert np.array_equal(status.cpu().numpy(), m.extend(grow))
    same(m, p)
    sd.sparse_decode_pages_free(p, cuda([0]))
    m.free([0])
    remap, n = sd.sparse_decode_pages_compact(p)
    want, live = m.compact()
    assert int(n) == live and np.array_equal(remap.cpu().numpy(), want)
    same(m, p)


def test_captured_beam_steps(sd):
    """Fork (ending the parents) from one table into the other and back, as a
    captured pair of beam steps, replayed with new parents."""
    rng = np.random.default_rng(60)
    rows, width, pages = 8, 12, 150
    m, a, pools = model_and_pages(sd, random_state(rng, rows, width, pages), pools_for(pages, 3))
    b = sd.Pages(torch.full_like(a.block_table, -1), torch.zeros_like(a.seq_lens), a.refs)
    par, grow = cuda(np.zeros(rows)), cuda(np.zeros(rows))

    def pair():
        sd.sparse_decode_pages_fork(a, b, par, pools=pools, keep=False)
        sd.sparse_decode_pages_extend(b, grow)
        sd.sparse_decode_pages_fork(b, a, par, pools=pools, keep=False)

    def model_pair(parents, g):
        for step in range(2):
            table, lens, _ = m.fork(rows, parents, keep=False)
            m.table, m.lens = table, lens
            if step == 0:
                m.extend(g)
    pair()
    model_pair([0] * rows, [0] * rows)
    same(m, a, pools)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pair()
    for step in range(5):
        parents, g = rng.integers(0, rows, rows), rng.integers(0, 9, rows)
        par.copy_(cuda(parents))
        grow.copy_(cuda(g))
        graph.replay()
        torch.cuda.synchronize()
        model_pair(parents, g)
        same(m, a, pools)
        assert (b.block_table == -1).all() and (b.seq_lens == 0).all()


@pytest.mark.parametrize("rows,width,pages", [(40, 300, 8191), (40, 300, 8192), (40, 300, 8193),
                                              (40, 200, 2048), (40, 200, 4097), (5000, 3, 6000),
                                              (5000, 3, 9000)])
def test_pools_and_rows_around_what_one_workgroup_holds(sd, rows, width, pages):
    # (pools that the planning workgroup hands out itself, and larger ones; rows
    # that fit its LDS, and more)
    rng = np.random.default_rng(pages + rows)
    m, p, _ = model_and_pages(sd, random_state(rng, rows, width, pages), [])
    for step in range(2):
        grow = rng.integers(-3, 16 * width // 2 + 2, rows)
        status = sd.sparse_decode_pages_extend(p, cuda(grow))
        assert np.array_equal(status.cpu().numpy(), m.extend(grow))
        same(m, p)
        gone = rng.integers(-2, rows + 2, rows // 3)
        sd.sparse_decode_pages_free(p, cuda(gone))
        m.free(gone)
        same(m, p)
    remap, live = sd.sparse_decode_pages_compact(p)
    want, n = m.compact()
    assert int(live) == n and np.array_equal(remap.cpu().numpy(), want)
    same(m, p)
    n = rows + 7
    parents = rng.integers(-1, rows + 1, n)
    to = sd.Pages(torch.full((n, width), -1, dtype=torch.int32, device="cuda"),
                  torch.zeros(n, dtype=torch.int32, device="cuda"), p.refs)
    status = sd.sparse_decode_pages_fork(p, to, cuda(parents), keep=False)
    table, lens, want = m.fork(n, parents, False)
    assert np.array_equal(status.cpu().numpy(), want)
    assert np.array_equal(to.block_table.cpu().numpy(), table)
    assert np.array_equal(to.seq_lens.cpu().numpy(), lens)
    same(m, p)
