"""How exactly softmax weights reach an output of sixteen bits: a mean of equal
values is that value, and one query's weights cost nothing beside the output's
own rounding."""
import math

import pytest
import torch

from tests import plain64 as R

pytestmark = pytest.mark.gpu
LN2 = math.log(2.0)   # as softmax scale: scores are exponents of two


@pytest.fixture(scope="module")
def sd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2605_24168_amd import sparse_decode
    return sparse_decode


def paged(x):
    """[B, Hkv, L, 128] -> pages [B * P, 16, Hkv, 128] and their table."""
    B, H, L, _ = x.shape
    P = -(-L // 16)
    x = torch.nn.functional.pad(x, (0, 0, 0, 16 * P - L))
    table = torch.arange(B * P, dtype=torch.int32, device=x.device).reshape(B, P)
    return x.reshape(B, H, P, 16, 128).permute(0, 2, 3, 1, 4).reshape(B * P, 16, H, 128).contiguous(), table


# Position 0 scores 0, every other one -d, with 2^-d halfway between two bfloat16
# numbers: 0.5 + 2^-9.  A weight that is rounded alone, but not in the sum, is off
# by 2^-8 relative there, all of them to the same side: 31 of 32 positions hold 94%
# of the sum, so that a mean of equal values comes out 0.94 * 2^-8 too large or too
# small, more than half a step of values with a mantissa of 1.07 and more.
# Without that, sums of 32 bits leave (n + 16) 2^-23 at most: half a step is never reached.
FAR = -math.log2(0.5 + 2.0**-9)


def equal_values(B, H, L, seed):
    """Keys as above, and values that are the same at every position."""
    coarse = torch.tensor(FAR).bfloat16()
    fine = torch.tensor(FAR - float(coarse)).bfloat16()
    k = torch.zeros((B, H, L, 128), dtype=torch.bfloat16)
    k[:, :, 1:, 0], k[:, :, 1:, 1] = -coarse, -fine
    g = torch.Generator().manual_seed(seed)
    v = (1 + torch.rand((B, H, 1, 128), generator=g)).bfloat16()
    return k.cuda(), v.expand(B, H, L, 128).contiguous().cuda(), v


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("L", [2, 17, 32, 200, 2399])
@pytest.mark.parametrize("B,hq,hkv", [(1, 8, 2), (3, 16, 1), (64, 8, 4)])
def test_a_mean_of_equal_values_is_that_value(sd, layout, L, B, hq, hkv):
    # (64 x 4 x 2399 on pages: workgroups of four KV heads)
    k, v, value = equal_values(B, hkv, L, L)
    table = None
    if layout == "paged":
        (k, table), (v, _) = paged(k), paged(v)
    cache = sd.KVCache(k=k, v=v, layout=layout, block_table=table)
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    q = torch.zeros((B, hq, 128), dtype=torch.bfloat16, device="cuda")
    q[..., :2] = 1
    want = value[:, :, 0].repeat_interleave(hq // hkv, 1).cuda()
    out = sd.sparse_decode_window_attention(q, cache, lens, sd.Window(softmax_scale=LN2))
    assert torch.equal(out, want)


@pytest.mark.parametrize("hq,hkv", [(8, 1), (16, 1), (6, 2)])
@pytest.mark.parametrize("layout", ["bhnd", "paged"])
def test_a_mean_of_equal_values_in_four_bits(sd, layout, hq, hkv):
    # Keys of level 1 (code 2) on two channels, which the query weights.
    for L in (2, 32, 300):
        lead = (1, hkv, L) if layout == "bhnd" else (-(-L // 16), hkv, 16)
        table = None if layout == "bhnd" else torch.arange(lead[0], dtype=torch.int32, device="cuda")[None]
        full = lambda n, x: torch.full(lead + (n,), x, dtype=torch.uint8, device="cuda")
        k, ks, v, vs = full(64, 0), full(4, 127), full(64, 0x75), full(4, 127)   # values 3, 6, 3, 6 ..
        k[..., 0] = 0xAA          # channels 0 and 1: -1
        k[(0, slice(None), 0)] = 0   # position 0
        q = torch.zeros((1, hq, 128), dtype=torch.bfloat16, device="cuda")
        q[..., 0] = FAR
        q[..., 1] = FAR - q[..., 0].float()
        out = sd.sparse_decode_q4_attention(
            q, sd.Q4Cache(k=k, k_scales=ks, v=v, v_scales=vs, layout=layout, block_table=table),
            torch.tensor([L], dtype=torch.int32, device="cuda"), sd.Window(softmax_scale=LN2))
        assert (out[..., 0::2] == 3).all() and (out[..., 1::2] == 6).all()


def one_query_bound(q, k, v, scale):
    """As R.attention's, with weights kept to 2^-14 instead of rounded once."""
    sees = torch.ones((1, k.shape[1]), dtype=torch.bool)
    ref, rest = R.attention(q, k, v, sees, scale, 0.0)
    both = R.attention(q, k, v, sees, scale, 1.0)[1] - rest   # sum w |v| + |out|
    return ref, rest + 2.0**-14 * both + 2.0**-8 * ref.abs()


@pytest.mark.parametrize("L", [1, 30, 500, 20000])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (16, 1), (2, 1)])
def test_one_query_rounds_its_output_only(sd, L, hq, hkv):
    g = torch.Generator().manual_seed(L)
    q = torch.randn((1, hq, 128), generator=g).bfloat16() * 2
    k, v = torch.randn((2, hkv, L, 128), generator=g).bfloat16()
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    scale = 128**-0.5
    for layout in ("bhnd", "paged"):
        kc, vc, table = k[None].cuda(), v[None].cuda(), None
        if layout == "paged":
            (kc, table), (vc, _) = paged(kc), paged(vc)
        out = sd.sparse_decode_window_attention(
            q.cuda(), sd.KVCache(k=kc, v=vc, layout=layout, block_table=table), lens, sd.Window())
        ref, allow = one_query_bound(q, k, v, scale)
        assert ((out.double().cpu() - ref).abs() <= allow).all()
    c = sd.Q4Cache.empty(1, hkv, L)
    starts = torch.tensor([0, L], dtype=torch.int32, device="cuda")
    sd.sparse_decode_q4_append(k.transpose(0, 1).contiguous().cuda(), v.transpose(0, 1).contiguous().cuda(),
                               c, lens, starts=starts)
    out = sd.sparse_decode_q4_attention(q.cuda(), c, lens)
    ref, allow = one_query_bound(q, R.q4_round(k)[0], R.q4_round(v)[0], scale)
    assert ((out.double().cpu() - ref).abs() <= allow).all()


@pytest.mark.parametrize("layout", ["bhnd", "paged"])
@pytest.mark.parametrize("L,n", [(2, 2), (40, 9), (64, 64), (200, 3), (2399, 130)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (16, 1), (3, 3)])
def test_a_mean_of_equal_values_is_that_value_for_every_query(sd, layout, L, n, hq, hkv):
    k, v, value = equal_values(2, hkv, L, L)
    table = None
    if layout == "paged":
        (k, table), (v, _) = paged(k), paged(v)
    cache = sd.KVCache(k=k, v=v, layout=layout, block_table=table)
    lens = torch.full((2,), L, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, n, n + 1], dtype=torch.int32, device="cuda")
    q = torch.zeros((n + 1, hq, 128), dtype=torch.bfloat16, device="cuda")
    q[..., :2] = 1
    want = value[:, :, 0].repeat_interleave(hq // hkv, 1).cuda()
    out = sd.sparse_decode_window_attention(q, cache, lens, sd.Window(softmax_scale=LN2), q_starts=starts)
    assert torch.equal(out, torch.cat((want[:1].expand(n, -1, -1), want[1:])))


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("L", [1, 31, 700, 9000])
def test_an_infinite_value_is_an_infinite_mean(sd, L, bad):
    # (a weight's second number may be nothing, which an infinity would make a NaN)
    k, v, _ = equal_values(1, 2, L, L)
    for at in (0, L // 2, L - 1):
        v[:, 1, at, 7] = bad
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device="cuda")
    q[..., :2] = 1
    starts = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for packed in (None, starts):
        out = sd.sparse_decode_window_attention(q, sd.KVCache(k=k, v=v), lens, sd.Window(softmax_scale=LN2),
                                                q_starts=packed)
        assert (out[:, 4:, 7] == bad).all()
        out[:, 4:, 7] = 0
        assert torch.isfinite(out).all()
    for hq in (4, 32):      # up to 8 query heads for a KV head, and more
        c = sd.Q4Cache.empty(1, 2, L)
        c.k_scales.fill_(127)
        c.v_scales.fill_(127)
        c.v[0, 1, :, 3] = 0xE2 if bad < 0 else 0x62      # channel 7: +-4, channel 6: 1
        c.v_scales[0, 1, :, 0] = 253                     # 4 * 2^126
        q = torch.ones((1, hq, 128), dtype=torch.bfloat16, device="cuda")
        out = sd.sparse_decode_q4_attention(q, c, lens)
        # (31 times 2^126 is past float32 before it is divided: channel 6 is not looked at)
        assert (out[:, hq // 2:, 7] == bad).all()
        assert torch.isfinite(out[..., 32:]).all() and torch.isfinite(out[:, :hq // 2]).all()
