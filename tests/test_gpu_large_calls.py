"""Calls that the header allows and that have more to do than one launch holds
(less than 2^32 threads)."""
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


def i32(a):
    return torch.tensor(np.array(a), dtype=torch.int32, device="cuda")


def test_four_million_pages_copied_in_four_pools(sd):
    n = 1 << 22                                       # 2^24 pieces
    pools = [torch.randint(0, 256, (2 * n, size), dtype=torch.uint8, device="cuda") for size in (1, 2, 4, 3)]
    perm = torch.randperm(2 * n, device="cuda").int()
    src, dst = perm[:n].contiguous(), perm[n:].contiguous()
    want = [p.clone() for p in pools]
    for w in want:
        w[dst.long()] = w[src.long()]
    sd.sparse_decode_pages_copy(pools, src, dst)
    assert all(torch.equal(p, w) for p, w in zip(pools, want))


def test_a_list_of_seventeen_million_rows_to_free(sd):
    table = np.array([[0, 2, -1], [3, -1, -1], [0, 1, 5]], np.int32)
    m = R.PagesModel(table, [20, 16, 40], [2, 1, 1, 1, 0, 1])
    p = sd.Pages(i32(m.table), i32(m.lens), i32(m.refs))
    rows = torch.full(((1 << 24) + 5,), -1, dtype=torch.int32, device="cuda")
    rows[7], rows[-1], rows[-2] = 1, 2, 99
    sd.sparse_decode_pages_free(p, rows)
    m.free([1, 2])
    assert np.array_equal(p.block_table.cpu().numpy(), m.table)
    assert np.array_equal(p.seq_lens.cpu().numpy(), m.lens) and np.array_equal(p.refs.cpu().numpy(), m.refs)


@pytest.mark.parametrize("keep", [True, False])
def test_a_fork_of_many_rows_with_large_pages(sd, keep):
    # 65535 children, pages of 4 MB: 16.8 million pieces, all but a few of no page.
    pool = torch.randint(0, 256, (12, 257 * 16384), dtype=torch.uint8, device="cuda")
    m = R.PagesModel([[4, 9, -1], [1, 0, -1]], [20, 32], [1, 1, 0, 0, 1, 0, 0, 0, 0, 1, 0, 0],
                     [pool.cpu().numpy()])
    a = sd.Pages(i32(m.table), i32(m.lens), i32(m.refs))
    n = 65535
    parents = np.full(n, -1)
    parents[[0, 5, n - 2, n - 1]] = 0, 1, 0, 0
    to = sd.Pages(torch.full((n, 3), 7, dtype=torch.int32, device="cuda"), i32(np.full(n, 7)), a.refs)
    status = sd.sparse_decode_pages_fork(a, to, i32(parents), pools=[pool], keep=keep)
    table, lens, want = m.fork(n, parents, keep)
    assert np.array_equal(status.cpu().numpy(), want)
    assert np.array_equal(to.block_table.cpu().numpy(), table)
    assert np.array_equal(to.seq_lens.cpu().numpy(), lens)
    assert np.array_equal(a.refs.cpu().numpy(), m.refs)
    assert np.array_equal(a.block_table.cpu().numpy(), m.table)
    assert np.array_equal(pool.cpu().numpy(), m.pools[0])


def one_position(B, heads):
    """Keys, values and queries of B sequences of one position."""
    k, v = torch.randn((2, B, heads, 1, 128), dtype=torch.bfloat16, device="cuda")
    return k, v, torch.randn((B, heads, 128), dtype=torch.bfloat16, device="cuda"), i32([1] * B)


@pytest.mark.parametrize("B,heads,packed", [(65535, 129, False), (257, 65535, True)])
def test_window_attention_of_many_sequences_and_heads(sd, B, heads, packed):
    # 2^23 workgroups of 512 threads, or 2^24 of 256: one position, so its value
    k, v, q, lens = one_position(B, heads)
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda") if packed else None
    out = torch.zeros_like(q)
    sd.sparse_decode_window_attention(q, sd.KVCache(k=k, v=v), lens, sd.Window(), q_starts=starts, out=out)
    assert torch.equal(out, v[:, :, 0])


def test_four_bit_attention_of_many_sequences_and_heads(sd):
    B, heads = 65535, 129
    k, v, q, lens = one_position(B, heads)
    c = sd.Q4Cache.empty(B, heads, 1)
    sd.sparse_decode_q4_append(k[:, :, 0].contiguous(), v[:, :, 0].contiguous(), c, lens)
    _, want = sd.sparse_decode_q4_load(c, lens)
    out = torch.zeros_like(q)
    sd.sparse_decode_q4_attention(q, c, lens, out=out)
    assert torch.equal(out, want)


def test_many_rows_appended_and_read_back(sd):
    # 2^28 rows read back (2^24 workgroups), most of them from before the sequence.
    heads, T, L = 16, (1 << 24) + 77, 300
    if torch.cuda.mem_get_info()[0] < 160e9:
        torch.cuda.empty_cache()
        if torch.cuda.mem_get_info()[0] < 160e9:
            pytest.skip("128 GB of rows")
    c = sd.Q4Cache.empty(1, heads, L)
    lens = i32([L])
    k, v = (torch.full((T, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[-L:].normal_()
    v[-L:].normal_()
    half = T // 2 + 5     # (2^27 rows: in two launches, too)
    sd.sparse_decode_q4_append(k[-half:], v[-half:], c, lens, starts=i32([0, half]))
    want, _ = R.q4_round(k[-L:].cpu())
    sd.sparse_decode_q4_load(c, lens, starts=i32([0, T]), k=k, v=v)
    assert torch.equal(k[-L:].double().cpu(), want)
    for t in (k, v):
        assert not any(bool(t[i:min(i + (1 << 20), T - L)].any()) for i in range(0, T - L, 1 << 20))
    assert not bool((v[-L:] == 7).any())
    del k, v
    torch.cuda.empty_cache()
