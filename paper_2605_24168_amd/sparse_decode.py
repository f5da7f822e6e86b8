"""Python binding of libsparse_decode.so (exact top-k context-sparse decode
attention on MI355X).

Argument marshalling only: every step of the method runs in the library's HIP
kernels.  PyTorch supplies device memory and the current HIP stream.  The
names follow the C ABI in include/sparse_decode.h:

    sparse_decode_score(q, cache, seq_lens, sparsity)        -> scores
    sparse_decode_topk(scores, seq_lens, sparsity, k_max)    -> idx (, vals)
    sparse_decode_attend(q, cache, seq_lens, idx, sparsity)  -> out
    sparse_decode_attention(q, cache, seq_lens, sparsity)    -> (out, idx)
    sparse_decode_attend_weighted(q, cache, seq_lens, idx, weights, sparsity) -> out
    sparse_decode_dense_attention(q, cache, seq_lens)        -> out
    sparse_decode_label_attention(q, cache, labels, seq_lens, sparsity) -> (out, idx)
    sparse_decode_label_score(q, cache, labels, seq_lens, sparsity)     -> scores
    sparse_decode_window_attention(q, cache, seq_lens, window, q_starts) -> out
    sparse_decode_q4_append(k, v, cache4, seq_lens, starts)
    sparse_decode_q4_load(cache4, seq_lens, starts, tokens)  -> (k, v)
    sparse_decode_q4_attention(q, cache4, seq_lens, window)  -> out
    sparse_decode_pages_extend(pages, grow)                  -> status
    sparse_decode_pages_fork(pages, to, parents, pools)      -> status
    sparse_decode_pages_free(pages, rows)
    sparse_decode_pages_copy(pools, src, dst)
    sparse_decode_pages_compact(pages, pools)                -> (remap, n_live)

Calls on one device share the library's memory: they (and replays of graphs that
hold them) have to be ordered, on one stream or by events.

Importing this module raises if the library has not been built; nothing here
falls back to another implementation.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
import struct
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparse_decode.so")
HEADER_PATH = os.path.join(os.path.dirname(_HERE), "include", "sparse_decode.h")

SD_OK, SD_ERR_INVALID_ARG, SD_ERR_UNSUPPORTED, SD_ERR_WORKSPACE, SD_ERR_HIP = 0, -1, -2, -3, -4
SD_F32, SD_BF16, SD_I32, SD_U8 = 0, 1, 2, 3
SD_KV_BHND, SD_KV_PAGED_NHD = 0, 1

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2605_24168_amd.build` "
        "(the HIP path has no fallback)")


class SdTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32), ("ndim", C.c_int32),
                ("shape", C.c_int64 * 4)]


class SdKv(C.Structure):
    _fields_ = [("t", SdTensor), ("layout", C.c_int32), ("page_size", C.c_int32),
                ("block_table", C.c_void_p), ("max_pages_per_seq", C.c_int32)]


class SdSparsity(C.Structure):
    _fields_ = [("ratio", C.c_double), ("k_rounding", C.c_int32), ("group_shared", C.c_int32),
                ("softmax_scale", C.c_float), ("k_override", C.c_void_p),
                ("n_sink", C.c_int32), ("n_local", C.c_int32)]


class SdLabels(C.Structure):
    _fields_ = [("t", SdTensor), ("channels", C.c_void_p)]


class SdWindow(C.Structure):
    _fields_ = [("n_sink", C.c_int32), ("window", C.c_int32), ("softmax_scale", C.c_float)]


class SdKv4(C.Structure):
    _fields_ = [("codes", SdTensor), ("scales", SdTensor), ("layout", C.c_int32),
                ("page_size", C.c_int32), ("block_table", C.c_void_p),
                ("max_pages_per_seq", C.c_int32)]


class SdPages(C.Structure):
    _fields_ = [("block_table", C.c_void_p), ("seq_lens", C.c_void_p), ("refs", C.c_void_p),
                ("n_pages", C.c_int64), ("batch", C.c_int32), ("max_pages", C.c_int32)]


class SdProfile(C.Structure):
    _fields_ = [("pilot_ms", C.c_float), ("score_ms", C.c_float), ("select_ms", C.c_float),
                ("repair_ms", C.c_float), ("attend_ms", C.c_float), ("total_ms", C.c_float),
                ("repaired_rows", C.c_int32), ("valid", C.c_int32)]


_P = C.POINTER
lib = C.CDLL(LIB_PATH)
lib.sparse_decode_score.restype = C.c_int
lib.sparse_decode_score.argtypes = [_P(SdTensor), _P(SdKv), C.c_void_p, _P(SdSparsity),
                                    _P(SdTensor), C.c_void_p]
lib.sparse_decode_topk.restype = C.c_int
lib.sparse_decode_topk.argtypes = [_P(SdTensor), C.c_void_p, _P(SdSparsity), _P(SdTensor),
                                   _P(SdTensor), C.c_void_p]
lib.sparse_decode_attend.restype = C.c_int
lib.sparse_decode_attend.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p, _P(SdTensor),
                                     _P(SdSparsity), _P(SdTensor), C.c_void_p]
lib.sparse_decode_attend_weighted.restype = C.c_int
lib.sparse_decode_attend_weighted.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p,
                                              _P(SdTensor), _P(SdTensor), _P(SdSparsity),
                                              _P(SdTensor), C.c_void_p]
lib.sparse_decode_dense_attention.restype = C.c_int
lib.sparse_decode_dense_attention.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p,
                                              C.c_float, _P(SdTensor), C.c_void_p]
lib.sparse_decode_dense_workspace_size.restype = C.c_int
lib.sparse_decode_dense_workspace_size.argtypes = [_P(SdTensor), _P(SdKv), _P(C.c_size_t)]
lib.sparse_decode_label_attention.restype = C.c_int
lib.sparse_decode_label_attention.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), _P(SdLabels),
                                              C.c_void_p, _P(SdSparsity), _P(SdTensor),
                                              _P(SdTensor), C.c_void_p]
lib.sparse_decode_label_score.restype = C.c_int
lib.sparse_decode_label_score.argtypes = [_P(SdTensor), _P(SdKv), _P(SdLabels), C.c_void_p,
                                          _P(SdSparsity), _P(SdTensor), C.c_void_p]
lib.sparse_decode_attention.restype = C.c_int
lib.sparse_decode_attention.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p,
                                        _P(SdSparsity), _P(SdTensor), _P(SdTensor), C.c_void_p]
lib.sparse_decode_attention_noalloc.restype = C.c_int
lib.sparse_decode_attention_noalloc.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p,
                                                _P(SdSparsity), _P(SdTensor), _P(SdTensor),
                                                C.c_void_p]
lib.sparse_decode_workspace_size.restype = C.c_int
lib.sparse_decode_workspace_size.argtypes = [_P(SdTensor), _P(SdKv), _P(SdSparsity), _P(SdTensor),
                                             _P(C.c_size_t)]
lib.sparse_decode_set_workspace.restype = C.c_int
lib.sparse_decode_set_workspace.argtypes = [C.c_void_p, C.c_size_t]
lib.sparse_decode_budget.restype = C.c_int64
lib.sparse_decode_budget.argtypes = [C.c_int64, _P(SdSparsity)]
lib.sparse_decode_set_profiling.restype = C.c_int
lib.sparse_decode_set_profiling.argtypes = [C.c_int32]
lib.sparse_decode_last_profile.restype = C.c_int
lib.sparse_decode_last_profile.argtypes = [_P(SdProfile)]
lib.sparse_decode_profile_mean.restype = C.c_int
lib.sparse_decode_profile_mean.argtypes = [_P(SdProfile), _P(C.c_int32)]
lib.sparse_decode_set_debug.restype = C.c_int
lib.sparse_decode_set_debug.argtypes = [C.c_int32]
lib.sparse_decode_sampled_attention.restype = C.c_int
lib.sparse_decode_sampled_attention.argtypes = [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p,
                                                _P(SdSparsity), _P(SdTensor), _P(SdTensor),
                                                _P(SdTensor), _P(SdTensor), C.c_void_p]
for _name, _args in {
        "window_attention": [_P(SdTensor), _P(SdKv), _P(SdKv), C.c_void_p, C.c_void_p, C.c_int64,
                             _P(SdWindow), _P(SdTensor), C.c_void_p],
        "q4_append": [_P(SdTensor), _P(SdTensor), _P(SdKv4), _P(SdKv4), C.c_void_p, C.c_void_p,
                      C.c_int64, C.c_void_p],
        "q4_load": [_P(SdKv4), _P(SdKv4), C.c_void_p, C.c_void_p, C.c_int64, _P(SdTensor),
                    _P(SdTensor), C.c_void_p],
        "q4_attention": [_P(SdTensor), _P(SdKv4), _P(SdKv4), C.c_void_p, _P(SdWindow),
                         _P(SdTensor), C.c_void_p],
        "pages_extend": [_P(SdPages), C.c_void_p, C.c_void_p, C.c_void_p],
        "pages_fork": [_P(SdPages), _P(SdPages), C.c_void_p, C.c_int32, _P(SdTensor), C.c_int32,
                       C.c_void_p, C.c_void_p],
        "pages_free": [_P(SdPages), C.c_void_p, C.c_int64, C.c_void_p],
        "pages_copy": [_P(SdTensor), C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p],
        "pages_compact": [_P(SdPages), _P(SdTensor), C.c_int32, C.c_void_p, C.c_void_p,
                          C.c_void_p]}.items():
    getattr(lib, f"sparse_decode_{_name}").restype = C.c_int
    getattr(lib, f"sparse_decode_{_name}").argtypes = _args
lib.sparse_decode_read_probe.restype = C.c_int
lib.sparse_decode_read_probe.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
lib.sparse_decode_status_string.restype = C.c_char_p
lib.sparse_decode_status_string.argtypes = [C.c_int]

# The same entry points for the calls below, which pass descriptors as packed
# bytes (see _desc); `lib` takes the structures and checks their types.
_raw = C.CDLL(LIB_PATH)
for _name in ("score", "topk", "attend", "attend_weighted", "dense_attention",
              "dense_workspace_size", "label_attention", "label_score", "attention",
              "attention_noalloc", "workspace_size", "budget", "sampled_attention",
              "window_attention", "q4_append", "q4_load", "q4_attention", "pages_extend",
              "pages_fork", "pages_free", "pages_copy", "pages_compact"):
    _f, _g = getattr(lib, f"sparse_decode_{_name}"), getattr(_raw, f"sparse_decode_{_name}")
    _g.restype = _f.restype
    _g.argtypes = [C.c_void_p if _t in (_P(SdTensor), _P(SdKv), _P(SdSparsity), _P(SdLabels),
                                        _P(SdWindow), _P(SdKv4), _P(SdPages)) else _t
                   for _t in _f.argtypes]


class SparseDecodeError(RuntimeError):
    def __init__(self, status: int, what: str):
        msg = lib.sparse_decode_status_string(status).decode()
        super().__init__(f"{what}: {msg} ({status})")
        self.status = status


def _check(status: int, what: str) -> None:
    if status != SD_OK:
        raise SparseDecodeError(status, what)


@dataclasses.dataclass
class Sparsity:
    """k = clamp(round(L / ratio), 1, L) per row (rounding 0 = nearest, 1 = ceil)."""
    ratio: float
    rounding: int = 0
    group_shared: bool = False
    softmax_scale: float = 0.0          # <= 0: 1/sqrt(128)
    k_override: Optional[torch.Tensor] = None   # int32 [B] on the device
    n_sink: int = 0                     # first positions always kept
    n_local: int = 0                    # last positions always kept

    def c(self) -> SdSparsity:
        ko = self.k_override
        if ko is not None:
            _need_device(ko, "k_override", torch.int32)
        return SdSparsity(float(self.ratio), int(self.rounding), int(bool(self.group_shared)),
                          float(self.softmax_scale), ko.data_ptr() if ko is not None else None,
                          int(self.n_sink), int(self.n_local))


@dataclasses.dataclass
class KVCache:
    """Key and value caches: "bhnd" [B, Hkv, Ncap, 128] or "paged"
    [pages, 16, Hkv, 128] with an int32 block table [B, max_pages]."""
    k: torch.Tensor
    v: torch.Tensor
    layout: str = "bhnd"
    block_table: Optional[torch.Tensor] = None
    page_size: int = 16

    @property
    def capacity(self) -> int:
        if self.layout == "paged":
            return int(self.block_table.shape[1]) * self.page_size
        return int(self.k.shape[2])

    @property
    def num_kv_heads(self) -> int:
        return int(self.k.shape[2] if self.layout == "paged" else self.k.shape[1])

    def c(self, which: str) -> SdKv:
        t = self.k if which == "k" else self.v
        kv = SdKv()
        kv.t = _tensor(t, which)
        if self.layout == "paged":
            _need_device(self.block_table, "block_table", torch.int32)
            kv.layout = SD_KV_PAGED_NHD
            kv.page_size = self.page_size
            kv.block_table = self.block_table.data_ptr()
            kv.max_pages_per_seq = int(self.block_table.shape[1])
        elif self.layout == "bhnd":
            kv.layout = SD_KV_BHND
            kv.page_size = 0
            kv.block_table = None
            kv.max_pages_per_seq = 0
        else:
            raise ValueError(f"unknown layout {self.layout!r}")
        return kv


_DTYPES = {torch.float32: SD_F32, torch.bfloat16: SD_BF16, torch.int32: SD_I32}


@dataclasses.dataclass
class Labels:
    """Label cache of the low-channel indexer: `t` holds 8 bf16 channels per
    key, [B, Hkv, Ncap, 8] beside a contiguous cache or [pages, Hkv, 16, 8]
    beside a paged one; `channels` (int32 [Hkv, 8], device) names the key
    channel of each column."""
    t: torch.Tensor
    channels: torch.Tensor

    def c(self) -> SdLabels:
        _need_device(self.channels, "channels", torch.int32)
        lab = SdLabels()
        lab.t = _tensor(self.t, "labels")
        lab.channels = self.channels.data_ptr()
        return lab


def _need_device(t: torch.Tensor, name: str, dtype=None) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _tensor(t: torch.Tensor, name: str) -> SdTensor:
    _need_device(t, name)
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if t.dim() > 4:
        raise ValueError(f"{name}: at most 4 dimensions")
    st = SdTensor()
    st.data = t.data_ptr() if t.numel() else None
    st.dtype = _DTYPES[t.dtype]
    st.ndim = t.dim()
    for i, n in enumerate(t.shape):
        st.shape[i] = int(n)
    return st


# The calls below pass descriptors as packed bytes in the structures' native
# layout: filling a ctypes structure field by field took 2-4 us per tensor,
# 17 of the 20 us that a small call spent on the host.
_PACK_TENSOR = struct.Struct("@Pii4q")
_PACK_KV = struct.Struct("@Pii4qiIPi4x")
_PACK_SPARSITY = struct.Struct("@dIIfPII")
_PACK_LABELS = struct.Struct("@Pii4qP")
_PACK_WINDOW = struct.Struct("@iif")
_PACK_KV4 = struct.Struct("@Pii4qPii4qiIPi4x")
_PACK_PAGES = struct.Struct("@PPPqii")
for _s, _t in ((_PACK_TENSOR, SdTensor), (_PACK_KV, SdKv), (_PACK_SPARSITY, SdSparsity),
               (_PACK_LABELS, SdLabels), (_PACK_WINDOW, SdWindow), (_PACK_KV4, SdKv4),
               (_PACK_PAGES, SdPages)):
    if _s.size != C.sizeof(_t):
        raise ImportError(f"descriptor layout of {_t.__name__} does not match")
_U32 = 0xFFFFFFFF  # int32 fields wrap, as a ctypes structure's do
_PAD = ((0, 0, 0, 0), (0, 0, 0), (0, 0), (0,), ())


def _fields(t: torch.Tensor, name: str, dtypes=_DTYPES) -> tuple:
    """The sd_tensor fields of t, in order (the checks of _tensor)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        _need_device(t, name)  # raises
    dtype = dtypes.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    shape = t.shape
    n = len(shape)
    if n > 4:
        raise ValueError(f"{name}: at most 4 dimensions")
    return (0 if 0 in shape else t.data_ptr(), dtype, n, *shape, *_PAD[n])


def _desc(t: torch.Tensor, name: str) -> bytes:
    return _PACK_TENSOR.pack(*_fields(t, name))


def _kv_desc(cache: KVCache, *which: str):
    """KVCache.c(which) as packed bytes (a tuple of them for several)."""
    if cache.layout == "paged":
        bt = cache.block_table
        _need_device(bt, "block_table", torch.int32)
        tail = (SD_KV_PAGED_NHD, cache.page_size & _U32, bt.data_ptr(), bt.shape[1])
    elif cache.layout == "bhnd":
        tail = (SD_KV_BHND, 0, 0, 0)
    else:
        raise ValueError(f"unknown layout {cache.layout!r}")
    got = tuple(_PACK_KV.pack(*_fields(cache.k if w == "k" else cache.v, w), *tail) for w in which)
    return got if len(got) > 1 else got[0]


def _sparsity_desc(sp: Sparsity) -> bytes:
    """Sparsity.c() as packed bytes."""
    ko = sp.k_override
    if ko is not None:
        _need_device(ko, "k_override", torch.int32)
    return _PACK_SPARSITY.pack(float(sp.ratio), int(sp.rounding) & _U32, int(bool(sp.group_shared)),
                               C.c_float(sp.softmax_scale).value,
                               ko.data_ptr() if ko is not None else 0,
                               int(sp.n_sink) & _U32, int(sp.n_local) & _U32)


def _labels_desc(labels: Labels) -> bytes:
    """Labels.c() as packed bytes."""
    _need_device(labels.channels, "channels", torch.int32)
    return _PACK_LABELS.pack(*_fields(labels.t, "labels"), labels.channels.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def budget(L: int, sparsity: Sparsity) -> int:
    """k for a sequence of L positions under the ratio rule."""
    return int(_raw.sparse_decode_budget(int(L), _sparsity_desc(sparsity)))


def rows_of(q: torch.Tensor, cache: KVCache, sparsity: Sparsity) -> int:
    return cache.num_kv_heads if sparsity.group_shared else int(q.shape[1])


def k_max_of(cache: KVCache, sparsity: Sparsity) -> int:
    return budget(cache.capacity, sparsity)


def sparse_decode_score(q, cache: KVCache, seq_lens, sparsity: Sparsity, scores=None, stream=None):
    """float32 scores [B, R, capacity] (-inf beyond each sequence)."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if scores is None:
        scores = torch.empty((q.shape[0], rows_of(q, cache, sparsity), cache.capacity),
                             dtype=torch.float32, device=q.device)
    sp, kq, kk = _sparsity_desc(sparsity), _desc(q, "q"), _kv_desc(cache, "k")
    ks = _desc(scores, "scores")
    _check(_raw.sparse_decode_score(kq, kk, seq_lens.data_ptr(), sp, ks, _stream(stream)),
           "sparse_decode_score")
    return scores


def sparse_decode_topk(scores, seq_lens, sparsity: Sparsity, k_max: Optional[int] = None,
                       idx=None, vals=None, with_vals: bool = False, stream=None):
    """Exact top-k positions (ascending, -1 padded) of each score row."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if k_max is None:
        k_max = budget(scores.shape[2], sparsity)
    if idx is None:
        idx = torch.empty((scores.shape[0], scores.shape[1], k_max), dtype=torch.int32,
                          device=scores.device)
    if with_vals and vals is None:
        vals = torch.empty(idx.shape, dtype=torch.float32, device=scores.device)
    sp, cs, ci = _sparsity_desc(sparsity), _desc(scores, "scores"), _desc(idx, "idx")
    cv = _desc(vals, "vals") if vals is not None else None
    _check(_raw.sparse_decode_topk(cs, seq_lens.data_ptr(), sp, ci, cv, _stream(stream)),
           "sparse_decode_topk")
    return (idx, vals) if vals is not None else idx


def sparse_decode_attend(q, cache: KVCache, seq_lens, idx, sparsity: Sparsity, out=None,
                         stream=None):
    """Softmax attention of each query head over its listed positions."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if out is None:
        out = torch.empty_like(q)
    sp = _sparsity_desc(sparsity)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    ci, co = _desc(idx, "idx"), _desc(out, "out")
    _check(_raw.sparse_decode_attend(cq, kk, kv, seq_lens.data_ptr(), ci, sp, co,
                                     _stream(stream)),
           "sparse_decode_attend")
    return out


def sparse_decode_attend_weighted(q, cache: KVCache, seq_lens, idx, weights, sparsity: Sparsity,
                                  out=None, stream=None):
    """Attention of each query head over its listed positions, entry t of a
    row weighted by weights[b, r, t] (float32, the shape of idx)."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    _need_device(weights, "weights", torch.float32)
    if out is None:
        out = torch.empty_like(q)
    sp = _sparsity_desc(sparsity)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    ci, cw, co = _desc(idx, "idx"), _desc(weights, "weights"), _desc(out, "out")
    _check(_raw.sparse_decode_attend_weighted(cq, kk, kv, seq_lens.data_ptr(), ci, cw, sp, co,
                                              _stream(stream)),
           "sparse_decode_attend_weighted")
    return out


def sparse_decode_dense_attention(q, cache: KVCache, seq_lens, softmax_scale: float = 0.0,
                                  out=None, stream=None):
    """Dense decode attention over every cached position (bfloat16)."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if out is None:
        out = torch.empty_like(q)
    cq, (kk, kv), co = _desc(q, "q"), _kv_desc(cache, "k", "v"), _desc(out, "out")
    _check(_raw.sparse_decode_dense_attention(cq, kk, kv,
                                              seq_lens.data_ptr(), float(softmax_scale),
                                             co, _stream(stream)),
           "sparse_decode_dense_attention")
    return out


def dense_workspace_size(q, cache: KVCache) -> int:
    n = C.c_size_t(0)
    cq, kk = _desc(q, "q"), _kv_desc(cache, "k")
    _check(_raw.sparse_decode_dense_workspace_size(cq, kk, C.byref(n)),
           "sparse_decode_dense_workspace_size")
    return int(n.value)


def sparse_decode_attention(q, cache: KVCache, seq_lens, sparsity: Sparsity, out=None, idx=None,
                            k_max: Optional[int] = None, stream=None):
    """The fused method: returns (out [B, Hq, 128], idx [B, R, k_max])."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if out is None:
        out = torch.empty_like(q)
    if idx is None:
        if k_max is None:
            k_max = k_max_of(cache, sparsity)
        idx = torch.empty((q.shape[0], rows_of(q, cache, sparsity), k_max), dtype=torch.int32,
                          device=q.device)
    sp = _sparsity_desc(sparsity)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    co, ci = _desc(out, "out"), _desc(idx, "idx")
    _check(_raw.sparse_decode_attention(cq, kk, kv, seq_lens.data_ptr(), sp, co, ci,
                                        _stream(stream)),
           "sparse_decode_attention")
    return out, idx


NOALLOC_SCRATCH_BYTES = 64 << 20  # SD_NOALLOC_SCRATCH_BYTES


def sparse_decode_attention_noalloc(q, cache: KVCache, seq_lens, sparsity: Sparsity, out,
                                    idx, stream=None):
    """The fused method with the library's static scratch instead of its
    workspace (no device allocation); out and idx are the caller's."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    sp = _sparsity_desc(sparsity)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    co, ci = _desc(out, "out"), _desc(idx, "idx")
    _check(_raw.sparse_decode_attention_noalloc(cq, kk, kv, seq_lens.data_ptr(), sp, co, ci,
                                                _stream(stream)),
           "sparse_decode_attention_noalloc")
    return out, idx


def sparse_decode_label_attention(q, cache: KVCache, labels: Labels, seq_lens, sparsity: Sparsity,
                                  out=None, idx=None, k_max: Optional[int] = None, stream=None):
    """The method with the low-channel indexer choosing the positions:
    returns (out [B, Hq, 128], idx [B, R, k_max])."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if out is None:
        out = torch.empty_like(q)
    if idx is None:
        if k_max is None:
            k_max = k_max_of(cache, sparsity)
        idx = torch.empty((q.shape[0], rows_of(q, cache, sparsity), k_max), dtype=torch.int32,
                          device=q.device)
    sp, lab = _sparsity_desc(sparsity), _labels_desc(labels)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    co, ci = _desc(out, "out"), _desc(idx, "idx")
    _check(_raw.sparse_decode_label_attention(cq, kk, kv, lab, seq_lens.data_ptr(), sp, co, ci,
                                              _stream(stream)),
           "sparse_decode_label_attention")
    return out, idx


def sparse_decode_label_score(q, cache: KVCache, labels: Labels, seq_lens, sparsity: Sparsity,
                              scores=None, stream=None):
    """float32 approximate label scores [B, R, capacity] (-inf beyond each sequence)."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    if scores is None:
        scores = torch.empty((q.shape[0], rows_of(q, cache, sparsity), cache.capacity),
                             dtype=torch.float32, device=q.device)
    sp, lab = _sparsity_desc(sparsity), _labels_desc(labels)
    cq, kk, ks = _desc(q, "q"), _kv_desc(cache, "k"), _desc(scores, "scores")
    _check(_raw.sparse_decode_label_score(cq, kk, lab, seq_lens.data_ptr(), sp, ks,
                                          _stream(stream)), "sparse_decode_label_score")
    return scores


def workspace_size(q, cache: KVCache, sparsity: Sparsity, idx) -> int:
    n = C.c_size_t(0)
    sp, cq, kk = _sparsity_desc(sparsity), _desc(q, "q"), _kv_desc(cache, "k")
    ci = _desc(idx, "idx")
    _check(_raw.sparse_decode_workspace_size(cq, kk, sp, ci,
                                             C.byref(n)), "sparse_decode_workspace_size")
    return int(n.value)


_workspace_ref = None


def set_workspace(buf: Optional[torch.Tensor]) -> None:
    """Use a caller tensor (device, any dtype) as the library workspace, or
    None to let the library allocate its own."""
    global _workspace_ref
    if buf is None:
        _check(lib.sparse_decode_set_workspace(None, 0), "sparse_decode_set_workspace")
    else:
        _need_device(buf, "workspace")
        _check(lib.sparse_decode_set_workspace(buf.data_ptr(), buf.numel() * buf.element_size()),
               "sparse_decode_set_workspace")
    _workspace_ref = buf


def set_profiling(enable) -> None:
    """True/1: events between every stage; 2: only around the scoring stream."""
    level = 2 if enable == 2 else int(bool(enable))
    _check(lib.sparse_decode_set_profiling(level), "sparse_decode_set_profiling")


def last_profile() -> dict:
    p = SdProfile()
    _check(lib.sparse_decode_last_profile(C.byref(p)), "sparse_decode_last_profile")
    return {f: getattr(p, f) for f, _ in SdProfile._fields_}


def profile_mean() -> dict:
    """Mean stage times (ms) over the profiled calls since set_profiling(True)."""
    p, n = SdProfile(), C.c_int32(0)
    _check(lib.sparse_decode_profile_mean(C.byref(p), C.byref(n)), "sparse_decode_profile_mean")
    d = {f: getattr(p, f) for f, _ in SdProfile._fields_}
    d["calls"] = int(n.value)
    return d


def sparse_decode_sampled_attention(q, cache: KVCache, seq_lens, sparsity: Sparsity, draws,
                                    out=None, idx=None, weights=None, k_max: Optional[int] = None,
                                    stream=None):
    """Exact top-k plus s importance-weighted uniform draws of the rest of
    each row (draws: int32 [B, R, s], read as uint32 bits).  Returns (out,
    idx [B, R, k_max + s], weights, same shape)."""
    _need_device(seq_lens, "seq_lens", torch.int32)
    _need_device(draws, "draws", torch.int32)
    s = int(draws.shape[2])
    if idx is None:
        km = k_max_of(cache, sparsity) if k_max is None else k_max
        idx = torch.empty((q.shape[0], rows_of(q, cache, sparsity), km + s), dtype=torch.int32,
                          device=q.device)
    if weights is None:
        weights = torch.empty(idx.shape, dtype=torch.float32, device=q.device)
    if out is None:
        out = torch.empty_like(q)
    sp = _sparsity_desc(sparsity)
    cq, (kk, kv) = _desc(q, "q"), _kv_desc(cache, "k", "v")
    cd, co, ci, cw = _desc(draws, "draws"), _desc(out, "out"), _desc(idx, "idx"), \
        _desc(weights, "weights")
    _check(_raw.sparse_decode_sampled_attention(cq, kk, kv, seq_lens.data_ptr(), sp, cd, co, ci, cw,
                                                _stream(stream)),
           "sparse_decode_sampled_attention")
    return out, idx, weights


# ---------------------------------------------------------------------------
# Window attention, the 4-bit cache, and the pages of a paged cache.
# ---------------------------------------------------------------------------
@dataclasses.dataclass
class Window:
    """What a query at position p sees: the positions j <= p with j < n_sink
    or p - j < window.  window = EVERYTHING: all of them."""
    n_sink: int = 0
    window: int = 2**31 - 1
    softmax_scale: float = 0.0          # <= 0: 1/sqrt(128)


EVERYTHING = 2**31 - 1


@dataclasses.dataclass
class Q4Cache:
    """Keys and values in 4 bits: codes "bhnd" [B, Hkv, Ncap, 64] with scales
    [B, Hkv, Ncap, 4], or "paged" [pages, Hkv, 16, 64] with [pages, Hkv, 16, 4]
    (uint8 all) and an int32 block table [B, max_pages]."""
    k: torch.Tensor
    k_scales: torch.Tensor
    v: torch.Tensor
    v_scales: torch.Tensor
    layout: str = "bhnd"
    block_table: Optional[torch.Tensor] = None
    page_size: int = 16

    @classmethod
    def empty(cls, batch: int, kv_heads: int, capacity: int, device="cuda") -> "Q4Cache":
        """A contiguous cache of empty rows."""
        return cls(*cls._rows((batch, kv_heads, capacity), device))

    @classmethod
    def empty_paged(cls, pages: int, kv_heads: int, block_table: torch.Tensor,
                    device="cuda") -> "Q4Cache":
        """A pool of empty pages behind a block table."""
        return cls(*cls._rows((pages, kv_heads, 16), device), layout="paged",
                   block_table=block_table)

    @staticmethod
    def _rows(shape, device):
        return [torch.zeros(shape + (n,), dtype=torch.uint8, device=device) for n in (64, 4, 64, 4)]

    @property
    def pools(self) -> tuple:
        """The tensors whose first dimension counts pages (paged layout)."""
        return self.k, self.k_scales, self.v, self.v_scales

    @property
    def num_kv_heads(self) -> int:
        return int(self.k.shape[1])


@dataclasses.dataclass
class Pages:
    """The pages of a paged cache: sequence b holds the pages
    block_table[b, :ceil(seq_lens[b] / 16)] (the other entries are -1), refs[p]
    counts the rows that hold page p (0: free).  int32, changed in place."""
    block_table: torch.Tensor           # [B, max_pages]
    seq_lens: torch.Tensor              # [B]
    refs: torch.Tensor                  # [pages]


_DTYPES_U8 = {**_DTYPES, torch.uint8: SD_U8}


def _window_desc(w: Window) -> bytes:
    return _PACK_WINDOW.pack(_int32(w.n_sink, "n_sink"), _int32(w.window, "window"),
                             C.c_float(w.softmax_scale).value)


def _int32(x, name: str) -> int:
    x = int(x)
    if not -2**31 <= x < 2**31:
        raise ValueError(f"{name} must fit in 32 bits")
    return x


# Descriptors of the calls below, of tensors that have to be on device `index`.
# What is as it should be takes one look at each property (a call's tensors cost
# 0.3 us of host time each); everything else goes on to the checks that raise.
_I32 = torch.int32
_PACK_ROWS = struct.Struct("@Pii3q8x").pack      # an sd_tensor of three dimensions


def _device_of(t: torch.Tensor, name: str) -> int:
    index = t.get_device() if isinstance(t, torch.Tensor) else -1
    if index < 0:
        _need_device(t, name)  # raises
    return index


def _same_device(t: torch.Tensor, name: str, index: int) -> None:
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the call on device {index}")


def _rows_desc(t: torch.Tensor, name: str, index: int) -> bytes:
    """[rows, heads, channels]"""
    try:
        if t.get_device() == index and t.is_contiguous():
            shape = t.shape
            if len(shape) == 3:
                return _PACK_ROWS(t.data_ptr(), _DTYPES[t.dtype], 3, *shape)
    except (AttributeError, KeyError):
        pass
    desc = _desc(t, name)
    _same_device(t, name, index)
    return desc


def _pool_fields(t: torch.Tensor, name: str, index: int, dtypes) -> tuple:
    """_fields of a cache's tensor."""
    try:
        if t.get_device() == index and t.is_contiguous():
            shape = t.shape
            if len(shape) == 4:
                return t.data_ptr(), dtypes[t.dtype], 4, *shape
    except (AttributeError, KeyError):
        pass
    fields = _fields(t, name, dtypes)
    _same_device(t, name, index)
    return fields


def _vector(t: torch.Tensor, name: str, index: int, n: Optional[int] = None) -> int:
    """Address of an int32 vector (of n entries)."""
    try:
        if t.get_device() == index and t.dtype is _I32 and t.is_contiguous() and \
                t.dim() == 1 and (n is None or t.shape[0] == n):
            return t.data_ptr()
    except AttributeError:
        pass
    _need_device(t, name, _I32)
    _same_device(t, name, index)
    raise ValueError(f"{name} must have the shape [{'n' if n is None else n}]")


def _places(cache, batch: int, index: int) -> tuple:
    """What a cache's descriptors hold beside its tensors."""
    if cache.layout == "paged":
        bt = cache.block_table
        try:
            if bt.get_device() == index and bt.dtype is _I32 and bt.is_contiguous():
                shape = bt.shape
                if len(shape) == 2 and shape[0] == batch:
                    return SD_KV_PAGED_NHD, cache.page_size & _U32, bt.data_ptr(), shape[1]
        except AttributeError:
            pass
        _need_device(bt, "block_table", _I32)
        _same_device(bt, "block_table", index)
        raise ValueError(f"block_table must have the shape [{batch}, max_pages]")
    if cache.layout != "bhnd":
        raise ValueError(f"unknown layout {cache.layout!r}")
    return SD_KV_BHND, 0, 0, 0


def _kv_descs(cache: KVCache, batch: int, index: int) -> tuple:
    tail = _places(cache, batch, index)
    return (_PACK_KV.pack(*_pool_fields(cache.k, "k", index, _DTYPES), *tail),
            _PACK_KV.pack(*_pool_fields(cache.v, "v", index, _DTYPES), *tail))


def _q4_descs(cache: Q4Cache, batch: int, index: int) -> tuple:
    tail = _places(cache, batch, index)
    return (_PACK_KV4.pack(*_pool_fields(cache.k, "k", index, _DTYPES_U8),
                           *_pool_fields(cache.k_scales, "k_scales", index, _DTYPES_U8), *tail),
            _PACK_KV4.pack(*_pool_fields(cache.v, "v", index, _DTYPES_U8),
                           *_pool_fields(cache.v_scales, "v_scales", index, _DTYPES_U8), *tail))


def _batch_of(seq_lens: torch.Tensor, index: int) -> tuple:
    """Sequences of a call, and where their lengths are."""
    at = _vector(seq_lens, "seq_lens", index)
    return seq_lens.shape[0], at


def _starts(starts, name: str, batch: int, index: int) -> Optional[int]:
    return None if starts is None else _vector(starts, name, index, batch + 1)


def _call(fn, index: int, stream, *args) -> None:
    """One library call on device `index`, with the stream appended."""
    if index == torch._C._cuda_getDevice():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None
                    else _stream(stream))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _stream(stream))
    if status != SD_OK:
        _check(status, fn.__name__)


def _empty(like: torch.Tensor, shape, dtype, stream) -> torch.Tensor:
    """An output on the device of `like`, from the memory of the stream that the
    call runs on (the device's current stream without one)."""
    if stream is None:
        if like.get_device() == torch._C._cuda_getDevice():
            return like.new_empty(shape, dtype=dtype)
        with torch.cuda.device(like.device):
            return like.new_empty(shape, dtype=dtype)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream), device=like.device)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _empty_like(q: torch.Tensor, stream) -> torch.Tensor:
    if stream is None and q.is_contiguous() and q.get_device() == torch._C._cuda_getDevice():
        return torch.empty_like(q)
    return _empty(q, q.shape, q.dtype, stream)


def sparse_decode_window_attention(q, cache: KVCache, seq_lens, window: Window, q_starts=None,
                                   out=None, stream=None):
    """Attention over the positions that `window` leaves visible: one query
    per sequence (q [B, Hq, 128], at the sequence's last position), or with
    q_starts (int32 [B + 1]) sequence b's last positions as the rows
    q_starts[b] .. q_starts[b + 1] of q [T, Hq, 128].  Rows of no sequence
    are left as they are in `out` (unset without one)."""
    index = _device_of(q, "q")
    batch, lens = _batch_of(seq_lens, index)
    starts = _starts(q_starts, "q_starts", batch, index)
    if out is None:
        out = _empty_like(q, stream)
    cq, co = _rows_desc(q, "q", index), _rows_desc(out, "out", index)
    kk, kv = _kv_descs(cache, batch, index)
    _call(_raw.sparse_decode_window_attention, index, stream, cq, kk, kv, lens, starts, batch,
          _window_desc(window), co)
    return out


def sparse_decode_q4_append(k, v, cache: Q4Cache, seq_lens, starts=None, stream=None) -> None:
    """Write the rows of k and v [T, Hkv, 128] as the last positions of their
    sequences (seq_lens counts them): row b of sequence b, or with starts
    (int32 [B + 1]) the rows starts[b] .. starts[b + 1]."""
    index = _device_of(k, "k")
    batch, lens = _batch_of(seq_lens, index)
    starts = _starts(starts, "starts", batch, index)
    ck, cv = _rows_desc(k, "k", index), _rows_desc(v, "v", index)
    kk, kv = _q4_descs(cache, batch, index)
    _call(_raw.sparse_decode_q4_append, index, stream, ck, cv, kk, kv, lens, starts, batch)


def sparse_decode_q4_load(cache: Q4Cache, seq_lens, starts=None, tokens: Optional[int] = None,
                          k=None, v=None, dtype=torch.bfloat16, stream=None):
    """The last positions of each sequence as what their codes stand for: k
    and v [T, Hkv, 128], rows as in sparse_decode_q4_append (tokens = T, when
    k and v are not given and starts is).  Rows of no sequence are left as
    they are (unset in new tensors)."""
    index = _device_of(cache.k, "cache.k")
    batch, lens = _batch_of(seq_lens, index)
    if (k is None or v is None) and tokens is None:
        if starts is not None:
            raise ValueError("tokens: the rows of k and v must be given beside starts")
        tokens = batch
    starts = _starts(starts, "starts", batch, index)
    kk, kv = _q4_descs(cache, batch, index)
    shape = (tokens, cache.num_kv_heads, 128)
    if k is None and v is None:
        k = _empty(cache.k, shape, dtype, stream)
        v = _empty_like(k, stream)
    elif k is None or v is None:
        new = _empty(cache.k, shape, dtype, stream)
        k, v = (new, v) if k is None else (k, new)
    ck, cv = _rows_desc(k, "k", index), _rows_desc(v, "v", index)
    _call(_raw.sparse_decode_q4_load, index, stream, kk, kv, lens, starts, batch, ck, cv)
    return k, v


def sparse_decode_q4_attention(q, cache: Q4Cache, seq_lens, window: Optional[Window] = None,
                               out=None, stream=None):
    """Decode attention over a 4-bit cache (bfloat16 q [B, Hq, 128]): every
    position, or those that `window` leaves visible."""
    index = _device_of(q, "q")
    batch, lens = _batch_of(seq_lens, index)
    if q.shape[0] != batch:
        raise ValueError("q and seq_lens must have the same number of sequences")
    if out is None:
        out = _empty_like(q, stream)
    cq, co = _rows_desc(q, "q", index), _rows_desc(out, "out", index)
    kk, kv = _q4_descs(cache, batch, index)
    cw = _window_desc(window) if window is not None else None
    _call(_raw.sparse_decode_q4_attention, index, stream, cq, kk, kv, lens, cw, co)
    return out


def _pages_desc(pages: Pages, index: int) -> bytes:
    bt = pages.block_table
    if bt.dtype is not _I32 or not bt.is_contiguous():
        _need_device(bt, "block_table", _I32)  # raises
    shape = bt.shape
    if len(shape) != 2:
        raise ValueError("block_table must have the shape [batch, max_pages]")
    lens = _vector(pages.seq_lens, "seq_lens", index, shape[0])
    refs = _vector(pages.refs, "refs", index)
    return _PACK_PAGES.pack(bt.data_ptr(), lens, refs, pages.refs.shape[0], *shape)


def _pools_desc(pools: Sequence[torch.Tensor], index: int) -> tuple:
    for t in pools:
        _device_of(t, "pools")
        _same_device(t, "pools", index)
    return b"".join(_PACK_TENSOR.pack(*_fields(t, "pools", _DTYPES_U8)) for t in pools), len(pools)


def sparse_decode_pages_extend(pages: Pages, grow, status=None, stream=None):
    """Pages for grow[b] more positions of each row (int32 [B]), the lowest
    free ones first; seq_lens grows.  Returns status int32 [B]: 0 done, 1 no
    free pages left, 2 longer than the table; such rows stay as they are."""
    index = _device_of(pages.block_table, "block_table")
    cp, batch = _pages_desc(pages, index), pages.block_table.shape[0]
    at = _vector(grow, "grow", index, batch)
    if status is None:
        status = _empty(grow, (batch,), _I32, stream)
    _call(_raw.sparse_decode_pages_extend, index, stream, cp, at,
          _vector(status, "status", index, batch))
    return status


def sparse_decode_pages_fork(pages: Pages, to: Pages, parents, pools: Sequence[torch.Tensor] = (),
                             keep: bool = True, status=None, stream=None):
    """Row i of `to` becomes a child of row parents[i] of `pages` (int32;
    outside its rows: an empty row): full pages are shared, a part-filled last
    page is copied in every pool.  keep=False ends the parents' rows (a step
    of beam search).  Returns status int32: 0 done, 1 no free page left."""
    index = _device_of(pages.block_table, "block_table")
    if _device_of(to.block_table, "block_table") != index:
        _same_device(to.block_table, "block_table", index)  # raises
    cp, ct, batch = _pages_desc(pages, index), _pages_desc(to, index), to.block_table.shape[0]
    at = _vector(parents, "parents", index, batch)
    if status is None:
        status = _empty(parents, (batch,), _I32, stream)
    pl, n = _pools_desc(pools, index)
    _call(_raw.sparse_decode_pages_fork, index, stream, cp, ct, at, int(bool(keep)), pl, n,
          _vector(status, "status", index, batch))
    return status


def sparse_decode_pages_free(pages: Pages, rows, stream=None) -> None:
    """The listed rows (int32) give back their pages and are left empty."""
    index = _device_of(pages.block_table, "block_table")
    cp, at = _pages_desc(pages, index), _vector(rows, "rows", index)
    _call(_raw.sparse_decode_pages_free, index, stream, cp, at, rows.shape[0])


def sparse_decode_pages_copy(pools: Sequence[torch.Tensor], src, dst, stream=None) -> None:
    """Page dst[i] = page src[i] in every pool (int32; a page is not both a
    source and a destination, nor a destination twice)."""
    index = _device_of(src, "src")
    at, moves = _vector(src, "src", index), src.shape[0]
    to = _vector(dst, "dst", index, moves)
    pl, n = _pools_desc(pools, index)
    _call(_raw.sparse_decode_pages_copy, index, stream, pl, n, at, to, moves)


def sparse_decode_pages_compact(pages: Pages, pools: Sequence[torch.Tensor] = (), remap=None,
                                n_live=None, stream=None):
    """Move the live pages to the front of the pools; table and refs follow.
    Returns (remap int32 [pages]: where each page is now, -1 if it was free;
    n_live int32 [1])."""
    index = _device_of(pages.block_table, "block_table")
    cp, n = _pages_desc(pages, index), pages.refs.shape[0]
    remap = _empty(pages.refs, (n,), _I32, stream) if remap is None else remap
    n_live = _empty(pages.refs, (1,), _I32, stream) if n_live is None else n_live
    pl, count = _pools_desc(pools, index)
    _call(_raw.sparse_decode_pages_compact, index, stream, cp, pl, count,
          _vector(remap, "remap", index, n), _vector(n_live, "n_live", index, 1))
    return remap, n_live


def read_probe(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """One plain streaming read of buf (device, contiguous, 16-byte aligned):
    the device's reference read rate when timed.  sink: a device int32/uint32
    scalar the kernel may write."""
    _need_device(buf, "buf")
    _need_device(sink, "sink")
    if not buf.is_contiguous():
        raise ValueError("buf must be contiguous")
    nbytes = buf.numel() * buf.element_size()
    _check(lib.sparse_decode_read_probe(buf.data_ptr(), nbytes, sink.data_ptr(), _stream(stream)),
           "sparse_decode_read_probe")


def set_debug(flags: int) -> None:
    _check(lib.sparse_decode_set_debug(int(flags)), "sparse_decode_set_debug")


def cache_from_inputs(inp, device="cuda") -> tuple:
    """Copy a host decode-step description (uint16 bfloat16 bits or float32
    arrays) to the device: returns (q, KVCache, seq_lens)."""
    def dev(a):
        t = torch.from_numpy(a)
        if a.dtype.name == "uint16":
            t = t.view(torch.bfloat16)
        return t.to(device)
    q = dev(inp.q)
    cache = KVCache(k=dev(inp.k), v=dev(inp.v), layout=inp.layout,
                    block_table=(torch.from_numpy(inp.block_table).to(device)
                                 if inp.block_table is not None else None),
                    page_size=inp.page_size)
    seq_lens = torch.from_numpy(inp.seq_lens.astype("int32")).to(device)
    return q, cache, seq_lens


def sparsity_from_inputs(inp, **kw) -> Sparsity:
    kw.setdefault("n_sink", int(getattr(inp, "n_sink", 0) or 0))
    kw.setdefault("n_local", int(getattr(inp, "n_local", 0) or 0))
    return Sparsity(ratio=inp.ratio, rounding=inp.rounding, group_shared=inp.group_shared, **kw)
