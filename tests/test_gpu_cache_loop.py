"""The cache operators together, as a serving loop uses them: prompts are
admitted, written in 4 bits, decoded token by token as beams that fork and
drop, and the pool is squeezed together in between.  Beside the 4-bit pools a
bfloat16 pair of pools holds the same values; every step is checked against
plain rows that the test keeps per beam."""
import numpy as np
import pytest
import torch

from tests import plain64 as R

pytestmark = pytest.mark.gpu
SCALE = 128**-0.5


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


def i32(a):
    return torch.tensor(np.array(a), dtype=torch.int32, device="cuda")


def test_beams_on_a_four_bit_pool(sd):
    rng = np.random.default_rng(0)
    g = torch.Generator().manual_seed(0)
    hq, hkv, width, pages, rows = 8, 2, 16, 120, 6
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    mk = lambda: sd.Pages(torch.full((rows, width), -1, dtype=torch.int32, device="cuda"),
                          torch.zeros(rows, dtype=torch.int32, device="cuda"), refs)
    a, b = mk(), mk()
    q4 = sd.Q4Cache.empty_paged(pages, hkv, a.block_table)
    kb, vb = torch.full((2, pages, 16, hkv, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    pools = list(q4.pools) + [kb, vb]
    kept = [[torch.zeros(0, hkv, 128, dtype=torch.float64) for _ in range(2)] for _ in range(rows)]

    def write(pg, counts):
        """New tokens at the end of each row: in 4 bits, and as their values
        in the bfloat16 pools."""
        T = int(sum(counts))
        k, v = torch.randn((2, T, hkv, 128), generator=g).bfloat16()
        starts = i32(np.concatenate(([0], np.cumsum(counts))))
        cache = sd.Q4Cache(*q4.pools, layout="paged", block_table=pg.block_table)
        sd.sparse_decode_q4_append(k.cuda(), v.cuda(), cache, pg.seq_lens, starts=starts)
        lk, lv = sd.sparse_decode_q4_load(cache, pg.seq_lens, starts=starts, tokens=T)
        at = 0
        for r, n in enumerate(counts):
            for i, (x, loaded) in enumerate(((k, lk), (v, lv))):
                val = R.q4_round(x[at:at + n])[0]
                assert torch.equal(loaded[at:at + n].double().cpu(), val)
                kept[r][i] = torch.cat((kept[r][i], val))
            L = int(pg.seq_lens[r])
            for j in range(L - n, L):
                page = int(pg.block_table[r, j // 16])
                kb[page, j % 16], vb[page, j % 16] = lk[at + j - L + n], lv[at + j - L + n]
            at += n

    def attend(pg):
        q = torch.randn((rows, hq, 128), generator=g).bfloat16()
        cache4 = sd.Q4Cache(*q4.pools, layout="paged", block_table=pg.block_table)
        cache = sd.KVCache(k=kb, v=vb, layout="paged", block_table=pg.block_table)
        for w in (sd.Window(), sd.Window(3, 21)):
            out4 = sd.sparse_decode_q4_attention(q.cuda(), cache4, pg.seq_lens, w).double().cpu()
            out = sd.sparse_decode_window_attention(q.cuda(), cache, pg.seq_lens, w).double().cpu()
            for r in range(rows):
                k, v = (x.transpose(0, 1) for x in kept[r])
                L = k.shape[1]
                if L == 0:
                    assert (out4[r] == 0).all() and (out[r] == 0).all()
                    continue
                ref, allow = R.attention(q[r:r + 1], k, v, R.visible(L, 1, w.n_sink, w.window),
                                         SCALE, 2.0**-8)
                assert ((out4[r:r + 1] - ref).abs() <= allow).all()
                assert ((out[r:r + 1] - ref).abs() <= allow).all()

    # Two prompts, three beams of each (the first ends their rows of one).
    prompts = [37, 64, 0, 0, 0, 0]
    assert (sd.sparse_decode_pages_extend(a, i32(prompts)) == 0).all()
    write(a, prompts)
    now, then = a, b
    parents = [0, 0, 0, 1, 1, 1]
    for step in range(12):
        assert (sd.sparse_decode_pages_fork(now, then, i32(parents), pools=pools, keep=False) == 0).all()
        kept = [[x.clone() for x in kept[p]] for p in parents]
        now, then = then, now
        assert (sd.sparse_decode_pages_extend(now, i32([1] * rows)) == 0).all()
        write(now, [1] * rows)
        attend(now)
        if step % 4 == 3:
            remap, live = sd.sparse_decode_pages_compact(now, pools=pools)
            assert int(live) == int((refs > 0).sum()) and (refs[int(live):] == 0).all()
            attend(now)
        # what refs counts is what the table holds
        held = now.block_table[now.block_table >= 0].long()
        assert torch.equal(torch.bincount(held, minlength=pages).int(), refs)
        parents = [3 * (i // 3) + int(rng.integers(3)) for i in range(rows)]
    # The second prompt's beams end, a new prompt takes one of their rows.
    sd.sparse_decode_pages_free(now, i32([3, 4, 5]))
    kept[3:] = [[torch.zeros(0, hkv, 128, dtype=torch.float64) for _ in range(2)] for _ in range(3)]
    grow = [0, 0, 0, 0, 100, 0]
    assert (sd.sparse_decode_pages_extend(now, i32(grow)) == 0).all()
    write(now, grow)
    attend(now)
    # A chunk of the new prompt's last 30 positions in one call.
    q = torch.randn((30, hq, 128), generator=g).bfloat16()
    starts = i32([0, 0, 0, 0, 0, 30, 30])
    cache = sd.KVCache(k=kb, v=vb, layout="paged", block_table=now.block_table)
    out = sd.sparse_decode_window_attention(q.cuda(), cache, now.seq_lens, sd.Window(2, 40),
                                            q_starts=starts).double().cpu()
    k, v = (x.transpose(0, 1) for x in kept[4])
    ref, allow = R.attention(q, k, v, R.visible(100, 30, 2, 40), SCALE, 2.0**-8)
    assert ((out - ref).abs() <= allow).all()
