"""Long sequences that one workgroup walks from end to end on pages: page numbers
are held a stretch at a time (16 tiles of 64 positions, or 32 steps) and fetched
again, with pages outside the pool and rows of NaN along the way."""
import numpy as np
import pytest
import torch

from tests import plain64 as R
from tests.test_gpu_q4 import random_cache
from tests.test_gpu_window import ALL, HALF, SCALE, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


def lose(table, row, pages, n_pages):
    """Entries of the row point outside the pool."""
    for i, c in enumerate(pages):
        table[row, c] = (-1, n_pages, 2**31 - 1, -2**31)[i % 4]


# More than 256 sequences are not cut into parts: the long ones are walked by one
# workgroup (or the waves of one), 8192 positions and more, or 2048 with four KV
# heads to a workgroup (bfloat16 and hkv = 4).
LONG, MIDDLE = 20011, 9000
LENS = [LONG if b == 200 else MIDDLE if b == 3 else (37 * b) % 90 for b in range(258)]
LOST = [0, 5, 66, 511, 513, 600, 1024, 1250]


def hide_lost(sees):
    for c in LOST:
        sees[:, 16 * c:16 * c + 16] = False


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 4)])
def test_one_query_of_long_sequences(sd, dtype, hq, hkv):
    pr = Problem(sd, LENS, hq, hkv, "paged", dtype, seed=41)
    lose(pr.cache.block_table, 200, LOST, pr.cache.k.shape[0])
    for sink, window in ((0, ALL), (1000, 17000)):
        pr.check(pr.run(sd.Window(sink, window), False), sink, window,
                 hide=lambda b, sees: hide_lost(sees) if b == 200 else None)


@pytest.mark.parametrize("hq,hkv", [(8, 1), (16, 1)])
def test_one_query_of_long_sequences_in_four_bits(sd, hq, hkv):
    c, rows = random_cache(sd, LENS, hkv, "paged", seed=42)
    lose(c.block_table, 200, LOST, c.k.shape[0])
    g = torch.Generator().manual_seed(43)
    q = torch.randn((len(LENS), hq, 128), generator=g).bfloat16()
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    for sink, window in ((0, ALL), (1000, 17000)):
        out = sd.sparse_decode_q4_attention(q.cuda(), c, lens, sd.Window(sink, window)).double().cpu()
        for b, L in enumerate(LENS):
            if L == 0:
                assert (out[b] == 0).all()
                continue
            sees = R.visible(L, 1, sink, window)
            if b == 200:
                hide_lost(sees)
            ref, allow = R.attention(q[b:b + 1], *rows[b], sees, SCALE, 2.0**-8)
            assert ((out[b:b + 1] - ref).abs() <= allow).all(), f"sequence {b}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_few_queries_of_long_sequences(sd, dtype):
    counts = [(b % 4) if b not in (3, 200) else 5 for b in range(len(LENS))]
    pr = Problem(sd, LENS, 6, 2, "paged", dtype, counts=counts, seed=44)
    lose(pr.cache.block_table, 200, LOST, pr.cache.k.shape[0])
    for sink, window in ((0, ALL), (1000, 17000)):
        pr.check(pr.run(sd.Window(sink, window), True), sink, window,
                 hide=lambda b, sees: hide_lost(sees) if b == 200 else None)


@pytest.mark.parametrize("dtype,sink,window", [("bf16", 0, ALL), ("bf16", 70, 1500), ("f32", 70, 1500)])
def test_a_long_chunk(sd, dtype, sink, window):
    # 94 row tiles (375 in float32) of 8 KV heads are more than parts would pay
    # for; a row tile sees up to 41 tiles of 64 positions.
    L, n, hq, hkv = 2611, 1500, 64, 8
    pr = Problem(sd, [L], hq, hkv, "paged", dtype, counts=[n], seed=45)
    lost = [0, 64, 66, 130, 163]
    lose(pr.cache.block_table, 0, lost, pr.cache.k.shape[0])
    out = pr.run(sd.Window(sink, window), True).double().cpu()
    sees = R.visible(L, n, sink, window)
    for c in lost:
        sees[:, 16 * c:16 * c + 16] = False
    for h in (0, 13, 40, 63):        # (a head at a time: its scores alone are 31 MB)
        g = h * hkv // hq
        ref, allow = R.attention(pr.q[:, h:h + 1], pr.k[0][g:g + 1], pr.v[0][g:g + 1], sees, SCALE, HALF[dtype])
        err = (out[:, h:h + 1] - ref).abs()
        assert (err <= allow).all(), f"head {h}: {(err / allow).max():.3g} x the bound"
