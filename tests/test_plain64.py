"""The 64-bit plain implementations against torch's own attention and against
values worked out by hand."""
import math

import numpy as np
import torch

from tests import plain64 as R


def test_attention_equals_torch_in_float64():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in
               ((5, 4, 128), (2, 9, 128), (2, 9, 128)))
    sees = R.visible(9, 5, 2, 3)
    out, allow = R.attention(q, k, v, sees, 128**-0.5, 2.0**-8)
    ref = torch.nn.functional.scaled_dot_product_attention(
        q.transpose(0, 1), k.repeat_interleave(2, 0), v.repeat_interleave(2, 0), attn_mask=sees)
    assert torch.allclose(out, ref.transpose(0, 1), atol=1e-12)
    assert (allow > 0).all() and (allow < 0.1).all()


def test_visible_positions_by_hand():
    assert R.visible(6, 2, 1, 2).int().tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert R.visible(3, 1, 0, 0).int().tolist() == [[0, 0, 0]]
    assert R.visible(2, 4, 0, 9).int().tolist() == [[0, 0], [0, 0], [1, 0], [1, 1]]


def test_q4_levels_ties_and_scales_by_hand():
    x = torch.zeros(1, 128)
    x[0, :9] = torch.tensor([6.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.1])  # scale 1
    x[0, 32] = 7.0          # scale 2: 3.5 goes to the even index, 4
    x[0, 64] = -0.875       # scale 1/4: -3.5, to -4
    x[0, 96] = math.inf
    val, scale = R.q4_round(x)
    assert val[0, :9].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -6]
    assert scale[0].tolist() == [127, 128, 125, 255]
    assert val[0, 32] == 8.0 and val[0, 64] == -1.0
    assert val[0, 96:].isnan().all()
    codes = torch.zeros(1, 64, dtype=torch.uint8)
    codes[0, 0] = 0x97  # channel 0: index 7, channel 1: minus index 1
    assert R.q4_decode(codes, torch.full((1, 4), 128, dtype=torch.uint8))[0, :3].tolist() == [12, -1, 0]


def test_pages_model_by_hand():
    m = R.PagesModel([[0, 2, -1], [0, 3, -1], [-1] * 3], [20, 32, 0], [2, 0, 1, 1, 0, 0],
                     [np.arange(6)])
    table, lens, status = m.fork(3, [0, 0, 1], keep=False)
    assert table.tolist() == [[0, 2, -1], [0, 1, -1], [0, 3, -1]] and lens.tolist() == [20, 20, 32]
    assert m.refs.tolist() == [3, 1, 1, 1, 0, 0] and m.pools[0].tolist() == [0, 2, 2, 3, 4, 5]
    m.table, m.lens = table, lens
    m.free([1, 1])
    assert m.refs.tolist() == [2, 0, 1, 1, 0, 0]
    assert m.extend([13, 0, 40]).tolist() == [0, 0, 2] and m.table[0].tolist() == [0, 2, 1]
    m.free([0])
    remap, n = m.compact()
    assert n == 2 and remap.tolist() == [0, -1, -1, 1, -1, -1] and m.table[2].tolist() == [0, 1, -1]
