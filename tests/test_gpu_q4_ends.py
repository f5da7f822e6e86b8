"""The ends of what a 4-bit cache holds: every code with every scale byte, and
the largest magnitudes that can be written."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_code_with_every_scale_byte(sd, dtype):
    # Values that neither type holds (2^128 and more) read back as infinities.
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).reshape(4, 64)
    c = sd.Q4Cache.empty(1, 1, 1024)
    scales = torch.arange(256, dtype=torch.uint8).repeat_interleave(4)[:, None].expand(1024, 4)
    c.k[0, 0], c.v[0, 0] = codes.repeat(256, 1).cuda(), codes.flip(1).repeat(256, 1).cuda()
    c.k_scales[0, 0], c.v_scales[0, 0] = scales.cuda(), scales.cuda()
    lens = torch.tensor([1024], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 1024], dtype=torch.int32, device="cuda")
    k, v = sd.sparse_decode_q4_load(c, lens, starts=starts, tokens=1024, dtype=dtype)
    for got, stored in ((k, c.k), (v, c.v)):
        want = R.q4_decode(stored[0, 0].cpu(), scales).to(dtype)
        got = got[:, 0].cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_magnitudes(sd, dtype):
    # Below 3.5 * 2^126 the nearest level is at most 3, from there on it is 4:
    # 2^128, an infinity in both types.
    edge = 3.5 * 2.0**126
    below = edge * (1 - (2.0**-8 if dtype is torch.bfloat16 else 2.0**-24))
    x = torch.zeros((1, 4, 128), dtype=dtype)
    x[0, 0, 0], x[0, 1, 0], x[0, 2, 0], x[0, 3, 0] = below, edge, -edge, torch.finfo(dtype).max
    x[0, :, 40] = 1.0
    c = sd.Q4Cache.empty(1, 4, 1)
    lens = torch.ones(1, dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(x.cuda(), x.cuda(), c, lens)
    k, v = sd.sparse_decode_q4_load(c, lens, dtype=dtype)
    inf = float("inf")
    assert k[0, :, 0].tolist() == [3 * 2.0**126, inf, -inf, inf] and torch.equal(k, v)
    assert (k[0, :, 40] == 1).all()
    assert torch.equal(R.q4_round(x)[0].to(dtype), k.cpu())
