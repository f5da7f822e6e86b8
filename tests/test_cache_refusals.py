"""What window attention, the 4-bit cache and the page operations refuse, on
the host and before any launch: every call here carries exactly one defect
(placeholder addresses stand in for device memory; the checks never read it)."""
import ctypes as C
import math

import pytest
import torch

from paper_2605_24168_amd import sparse_decode as sd

FAKE = 0x100000
INVALID, UNSUPPORTED = sd.SD_ERR_INVALID_ARG, sd.SD_ERR_UNSUPPORTED


def tensor(shape, dtype=sd.SD_BF16, data=FAKE):
    t = sd.SdTensor()
    t.data, t.dtype, t.ndim = data, dtype, len(shape)
    for i, n in enumerate(shape):
        t.shape[i] = n
    return t


def kv(shape=(2, 8, 4096, 128), dtype=sd.SD_BF16, table=None, max_pages=0):
    c = sd.SdKv()
    c.t = tensor(shape, dtype)
    if table is not None:
        c.layout, c.page_size, c.block_table, c.max_pages_per_seq = 1, 16, table, max_pages
    return c


def kv4(B=2, Hkv=8, N=4096, paged=False):
    c = sd.SdKv4()
    lead = (100, Hkv, 16) if paged else (B, Hkv, N)
    c.codes, c.scales = tensor(lead + (64,), sd.SD_U8), tensor(lead + (4,), sd.SD_U8)
    if paged:
        c.layout, c.page_size, c.block_table, c.max_pages_per_seq = 1, 16, FAKE, 64
    return c


def edit(x, **kw):
    """kw: attribute paths with __ for dots, shape indices as shape_i."""
    for path, value in kw.items():
        obj, parts = x, path.split("__")
        for p in parts[:-1]:
            obj = getattr(obj, p)
        if parts[-1].startswith("shape_"):
            obj.shape[int(parts[-1][6:])] = value
        else:
            setattr(obj, parts[-1], value)
    return x


def ref(x):
    return None if x is None else C.byref(x)


def window_call(q=None, K=None, V=None, lens=FAKE, starts=None, batch=2, w=None, out=None):
    q = tensor((2, 32, 128)) if q is None else q
    K, V = kv() if K is None else K, kv() if V is None else V
    w = sd.SdWindow(4, 100, 0.0) if w is None else w
    out = tensor((2, 32, 128)) if out is None else out
    none = lambda x: None if x == "null" else ref(x)
    return sd.lib.sparse_decode_window_attention(none(q), none(K), none(V), lens, starts, batch,
                                                 none(w), none(out), None)


WINDOW = {
    "q null": (dict(q="null"), INVALID),
    "q dims": (dict(q=tensor((2, 32))), INVALID),
    "q dtype": (dict(q=tensor((2, 32, 128), sd.SD_I32)), INVALID),
    "head size": (dict(q=tensor((2, 32, 64))), UNSUPPORTED),
    "q data": (dict(q=tensor((2, 32, 128), data=None)), INVALID),
    "q misaligned": (dict(q=tensor((2, 32, 128), data=FAKE + 8)), INVALID),
    "rows are not sequences": (dict(q=tensor((3, 32, 128)), out=tensor((3, 32, 128))), INVALID),
    "heads do not divide": (dict(q=tensor((2, 30, 128)), out=tensor((2, 30, 128))), INVALID),
    "group of 32": (dict(q=tensor((2, 256, 128)), out=tensor((2, 256, 128))), UNSUPPORTED),
    "too many rows": (dict(q=tensor((2**30, 32, 128)), starts=FAKE, out=tensor((2**30, 32, 128))),
                      UNSUPPORTED),
    "K null": (dict(K="null"), INVALID),
    "V null": (dict(V="null"), INVALID),
    "K dtype": (dict(K=kv(dtype=sd.SD_F32)), INVALID),
    "V dtype": (dict(V=kv(dtype=sd.SD_F32)), INVALID),
    "K misaligned": (dict(K=edit(kv(), t__data=FAKE + 2)), INVALID),
    "V shorter": (dict(V=kv((2, 8, 4095, 128))), INVALID),
    "batch of K": (dict(K=kv((3, 8, 4096, 128)), V=kv((3, 8, 4096, 128))), INVALID),
    "layouts differ": (dict(V=kv((100, 16, 8, 128), table=FAKE, max_pages=256)), INVALID),
    "unknown layout": (dict(K=edit(kv(), layout=7), V=edit(kv(), layout=7)), INVALID),
    "tables differ": (dict(K=kv((100, 16, 8, 128), table=FAKE, max_pages=64),
                           V=kv((100, 16, 8, 128), table=FAKE + 64, max_pages=64)), INVALID),
    "no table": (dict(K=edit(kv((9, 16, 8, 128), table=FAKE, max_pages=4), block_table=None),
                      V=edit(kv((9, 16, 8, 128), table=FAKE, max_pages=4), block_table=None)), INVALID),
    "page size": (dict(K=edit(kv((9, 32, 8, 128), table=FAKE, max_pages=4), page_size=32)), UNSUPPORTED),
    "capacity": (dict(K=kv((2, 8, 2**24 + 1, 128)), V=kv((2, 8, 2**24 + 1, 128))), UNSUPPORTED),
    "lens null": (dict(lens=None), INVALID),
    "negative batch": (dict(batch=-1, starts=FAKE), INVALID),
    "batch too large": (dict(batch=65536, starts=FAKE), UNSUPPORTED),
    "window null": (dict(w="null"), INVALID),
    "negative sinks": (dict(w=sd.SdWindow(-1, 5, 0.0)), INVALID),
    "negative window": (dict(w=sd.SdWindow(0, -5, 0.0)), INVALID),
    "scale nan": (dict(w=sd.SdWindow(0, 5, math.nan)), INVALID),
    "scale inf": (dict(w=sd.SdWindow(0, 5, math.inf)), INVALID),
    "out null": (dict(out="null"), INVALID),
    "out shape": (dict(out=tensor((2, 31, 128))), INVALID),
    "out dtype": (dict(out=tensor((2, 32, 128), sd.SD_F32)), INVALID),
    "out misaligned": (dict(out=tensor((2, 32, 128), data=FAKE + 4)), INVALID),
}


@pytest.mark.parametrize("defect", WINDOW)
def test_window_attention_refuses(defect):
    kw, code = WINDOW[defect]
    assert window_call(**kw) == code


def test_window_attention_of_nothing_is_fine():
    assert window_call(q=tensor((0, 32, 128), data=None), starts=FAKE, out=tensor((0, 32, 128), data=None),
                       lens=None) == 0


def q4_call(q=None, K=None, V=None, lens=FAKE, w=None, out=None):
    q = tensor((2, 32, 128)) if q is None else q
    K, V = kv4() if K is None else K, kv4() if V is None else V
    out = tensor((2, 32, 128)) if out is None else out
    return sd.lib.sparse_decode_q4_attention(ref(q), ref(K), ref(V), lens, ref(w), ref(out), None)


Q4 = {
    "float32": (dict(q=tensor((2, 32, 128), sd.SD_F32)), UNSUPPORTED),
    "q dtype": (dict(q=tensor((2, 32, 128), sd.SD_U8)), INVALID),
    "group of 32": (dict(q=tensor((2, 256, 128)), out=tensor((2, 256, 128))), UNSUPPORTED),
    "heads do not divide": (dict(q=tensor((2, 30, 128)), out=tensor((2, 30, 128))), INVALID),
    "codes dtype": (dict(K=edit(kv4(), codes__dtype=sd.SD_BF16)), INVALID),
    "scales dtype": (dict(V=edit(kv4(), scales__dtype=sd.SD_F32)), INVALID),
    "code bytes": (dict(K=edit(kv4(), codes__shape_3=128)), UNSUPPORTED),
    "scale bytes": (dict(K=edit(kv4(), scales__shape_3=8)), UNSUPPORTED),
    "scales of another length": (dict(K=edit(kv4(), scales__shape_2=4095)), INVALID),
    "codes misaligned": (dict(K=edit(kv4(), codes__data=FAKE + 4)), INVALID),
    "scales misaligned": (dict(V=edit(kv4(), scales__data=FAKE + 4)), INVALID),
    "no scales": (dict(V=edit(kv4(), scales__data=None)), INVALID),
    "layouts differ": (dict(V=kv4(paged=True)), INVALID),
    "tables differ": (dict(K=kv4(paged=True), V=edit(kv4(paged=True), block_table=FAKE + 64)), INVALID),
    "page size": (dict(K=edit(kv4(paged=True), page_size=32)), UNSUPPORTED),
    "batch": (dict(K=kv4(3), V=kv4(3)), INVALID),
    "lens null": (dict(lens=None), INVALID),
    "negative window": (dict(w=sd.SdWindow(0, -1, 0.0)), INVALID),
    "out dtype": (dict(out=tensor((2, 32, 128), sd.SD_F32)), INVALID),
    "out rows": (dict(out=tensor((3, 32, 128))), INVALID),
}


@pytest.mark.parametrize("defect", Q4)
def test_q4_attention_refuses(defect):
    kw, code = Q4[defect]
    assert q4_call(**kw) == code


@pytest.mark.parametrize("defect,kw,code", [
    ("k null", dict(k=None), INVALID),
    ("dtypes differ", dict(v=tensor((9, 8, 128), sd.SD_F32)), INVALID),
    ("dtype", dict(k=tensor((9, 8, 128), sd.SD_U8), v=tensor((9, 8, 128), sd.SD_U8)), INVALID),
    ("rows differ", dict(v=tensor((8, 8, 128))), INVALID),
    ("heads", dict(k=tensor((9, 4, 128)), v=tensor((9, 4, 128))), INVALID),
    ("head size", dict(k=tensor((9, 8, 64)), v=tensor((9, 8, 64))), UNSUPPORTED),
    ("rows are not sequences", dict(starts=None), INVALID),
    ("lens null", dict(lens=None), INVALID),
    ("misaligned", dict(k=tensor((9, 8, 128), data=FAKE + 8)), INVALID),
    ("batch", dict(batch=3), INVALID),
    ("negative batch", dict(batch=-2), INVALID),
    ("layouts differ", dict(K=kv4(paged=True)), INVALID),
])
def test_q4_append_and_load_refuse(defect, kw, code):
    a = dict(k=tensor((9, 8, 128)), v=tensor((9, 8, 128)), K=kv4(), V=kv4(), lens=FAKE, starts=FAKE,
             batch=2)
    a.update(kw)
    assert sd.lib.sparse_decode_q4_append(ref(a["k"]), ref(a["v"]), ref(a["K"]), ref(a["V"]), a["lens"],
                                          a["starts"], a["batch"], None) == code
    assert sd.lib.sparse_decode_q4_load(ref(a["K"]), ref(a["V"]), a["lens"], a["starts"], a["batch"],
                                        ref(a["k"]), ref(a["v"]), None) == code


def pages(table=FAKE, lens=FAKE, refs=FAKE, n=1000, batch=4, width=64):
    return sd.SdPages(table, lens, refs, n, batch, width)


def pool(shape=(1000, 16, 8, 128), dtype=sd.SD_BF16, data=FAKE):
    return tensor(shape, dtype, data)


def pool_array(*ts):
    return (sd.SdTensor * max(1, len(ts)))(*ts), len(ts)


def test_pages_refuse():
    L = sd.lib
    ext = lambda p, grow=FAKE, status=FAKE: L.sparse_decode_pages_extend(ref(p), grow, status, None)
    for bad in (pages(table=None), pages(lens=None), pages(refs=None), pages(n=-1), pages(batch=-1),
                pages(width=-1)):
        assert ext(bad) == INVALID
        assert L.sparse_decode_pages_free(ref(bad), FAKE, 3, None) == INVALID
        assert L.sparse_decode_pages_compact(ref(bad), None, 0, FAKE, FAKE, None) == INVALID
    for bad in (pages(n=2**23 + 1), pages(batch=65536), pages(width=2**20 + 1)):
        assert ext(bad) == UNSUPPORTED
    assert ext(None) == INVALID
    assert ext(pages(), grow=None) == INVALID and ext(pages(), status=None) == INVALID
    assert ext(pages(batch=0)) == 0
    assert L.sparse_decode_pages_free(ref(pages()), None, 3, None) == INVALID
    assert L.sparse_decode_pages_free(ref(pages()), FAKE, -1, None) == INVALID
    assert L.sparse_decode_pages_free(ref(pages()), None, 0, None) == 0


def test_fork_refuses():
    far = 1 << 30

    def fork(a, b, parents=FAKE, keep=1, pools=(), status=FAKE):
        arr, n = pool_array(*pools)
        return sd.lib.sparse_decode_pages_fork(ref(a), ref(b), parents, keep, arr, n, status, None)
    b = lambda **kw: pages(**{**dict(table=far, lens=far), **kw})
    assert fork(pages(), b(refs=FAKE + 16)) == INVALID         # other counts
    assert fork(pages(), b(n=999)) == INVALID
    assert fork(pages(), b(width=63)) == INVALID
    assert fork(pages(), b(table=FAKE + 256)) == INVALID       # tables overlap
    assert fork(pages(), b(lens=FAKE + 12)) == INVALID         # lengths overlap
    assert fork(pages(), b(), keep=2) == INVALID
    assert fork(pages(), b(), parents=None) == INVALID
    assert fork(pages(), b(), status=None) == INVALID
    assert fork(None, b()) == INVALID and fork(pages(), None) == INVALID
    assert fork(pages(), b(), pools=[pool((999, 16, 8, 128))]) == INVALID   # other pages
    assert fork(pages(), b(), pools=[pool(data=None)]) == INVALID
    assert fork(pages(), b(), pools=[pool(dtype=9)]) == INVALID
    assert fork(pages(), b(), pools=[pool()] * 9) == UNSUPPORTED
    assert fork(pages(batch=0), b(batch=0)) == 0


def test_copy_and_compact_refuse():
    L = sd.lib

    def copy(pools, src=FAKE, dst=FAKE, n=3):
        arr, k = pool_array(*pools)
        return L.sparse_decode_pages_copy(arr, k, src, dst, n, None)
    assert copy([pool(), pool((999, 16, 8, 128))]) == INVALID
    assert copy([pool()], src=None) == INVALID and copy([pool()], dst=None) == INVALID
    assert copy([pool()], n=-1) == INVALID
    assert copy([pool()] * 9) == UNSUPPORTED
    assert copy([pool((1000, 2**15, 2**15, 8))]) == UNSUPPORTED      # a page of 16 GB
    assert copy([], src=None, dst=None) == 0 and copy([pool()], n=0) == 0
    assert L.sparse_decode_pages_copy(None, 1, FAKE, FAKE, 1, None) == INVALID
    arr, k = pool_array(pool())
    assert L.sparse_decode_pages_compact(ref(pages()), arr, k, None, FAKE, None) == INVALID
    assert L.sparse_decode_pages_compact(ref(pages()), arr, k, FAKE, None, None) == INVALID
    assert L.sparse_decode_pages_compact(ref(pages(n=5)), arr, k, FAKE, FAKE, None) == INVALID


def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = torch.zeros
    cache = sd.KVCache(k=z(1, 2, 8, 128), v=z(1, 2, 8, 128))
    c4 = sd.Q4Cache.empty(1, 2, 8, device="cpu")
    lens = z(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        sd.sparse_decode_window_attention(z(1, 4, 128), cache, lens, sd.Window())
    with pytest.raises(ValueError):
        sd.sparse_decode_q4_attention(z(1, 4, 128), c4, lens)
    with pytest.raises(ValueError):
        sd.sparse_decode_q4_append(z(1, 2, 128), z(1, 2, 128), c4, lens)
    with pytest.raises(ValueError):
        sd.sparse_decode_q4_load(c4, lens)
    p = sd.Pages(z(1, 4, dtype=torch.int32), lens, z(9, dtype=torch.int32))
    for call in (lambda: sd.sparse_decode_pages_extend(p, lens), lambda: sd.sparse_decode_pages_free(p, lens),
                 lambda: sd.sparse_decode_pages_fork(p, p, lens), lambda: sd.sparse_decode_pages_compact(p),
                 lambda: sd.sparse_decode_pages_copy([], lens, lens)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        sd._window_desc(sd.Window(0, 2**31))


def test_descriptors_match_the_structures():
    w = sd.SdWindow.from_buffer_copy(sd._window_desc(sd.Window(3, 70, 0.5)))
    assert (w.n_sink, w.window, w.softmax_scale) == (3, 70, 0.5)
