"""Numbers past their types that window attention and the 4-bit cache refuse on
the host, before any launch."""
import ctypes as C

import pytest

from paper_2605_24168_amd import sparse_decode as sd
from tests.test_cache_refusals import FAKE, INVALID, kv, kv4, q4_call, tensor, window_call


def paged_kv(heads):
    return kv((100, 16, heads, 128), table=FAKE, max_pages=64)


@pytest.mark.parametrize("heads", [0, 65536, 2**32, 2**32 + 8])
def test_heads_of_a_cache_that_pass_16_bits(heads):
    # (2^32 + 8 heads are not 8)
    for cache in (kv((2, heads, 4096, 128)), paged_kv(heads)):
        assert window_call(K=cache, V=cache) == INVALID
    for cache in (kv4(Hkv=heads), kv4(Hkv=heads, paged=True)):
        assert q4_call(K=cache, V=cache) == INVALID
        rows = tensor((9, 8, 128))
        args = [C.byref(rows), C.byref(rows), C.byref(cache), C.byref(cache), FAKE, FAKE, 2, None]
        assert sd.lib.sparse_decode_q4_append(*args) == INVALID


def test_scales_that_are_no_float32_as_exponents_of_two():
    # 2^127 log2(e) is one, the largest float32 times log2(e) is not: zero scores
    # would become NaN.
    for scale in (3.4e38, 2.4e38):
        assert window_call(w=sd.SdWindow(0, 5, scale)) == INVALID
        assert q4_call(w=sd.SdWindow(0, 5, scale)) == INVALID
    nothing = tensor((0, 32, 128), data=None)
    for scale in (2.0**127, -3.4e38):   # (below 0: the default)
        assert window_call(q=nothing, out=nothing, starts=FAKE, w=sd.SdWindow(0, 5, scale)) == 0
