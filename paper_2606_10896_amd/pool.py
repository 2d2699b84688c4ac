"""Python binding of the paged cache's page pool (``csrc/kvpool.hip``) and of beam search's selection
(``csrc/beam.hip``).

Argument marshalling only, with the names of the C ABI in ``include/flashgmm.h``.  ``ref`` [pages]
int32 counts the table entries that name a page; tables are ``total`` [rows] and ``pages``
[rows, max_pages], int32.  Beam j of sequence b is row b * beams + j of a table.  A call runs on the
device of its tensors, which have to be on one.
"""
from __future__ import annotations

import ctypes

import torch

import paper_2606_10896_amd as _base

from .kv import _CP, _F64, _I32, _I64, _SZ, _VP, _dtype

_TABLE = [_VP, _VP, _I32, _I32, _I64]                 # total, pages, rows, max_pages, stride

#: argument types of the C entry points
SIGNATURES = {
    "gmm_kv_copy": [_CP, _CP, _VP, _VP, _I64, _VP],
    "gmm_kv_fork": [_CP, _VP, *_TABLE, _VP, _VP, _I32, _I32, _VP, _VP, _I32, _I64, _VP],
    "gmm_kv_pool_workspace_bytes": [_CP, _I32],
    "gmm_kv_grow": [_CP, _VP, _VP, *_TABLE, _VP, _VP, _SZ, _VP],
    "gmm_kv_compact": [_CP, _VP, *_TABLE, _VP, _VP, _VP, _SZ, _VP],
    "gmm_beam_workspace_bytes": [_I32, _I32, _I32],
    "gmm_beam_select": [_VP, _I32, _I64, _I64, _I32, _I32, _I32, _VP, _VP, _VP, _I32, _VP, _I64,
                        _F64, _I32, _VP, _VP, _VP, _VP, _VP, _SZ, _VP],
}


_FN = {}


def bind(lib):
    """Sets the entry points' argument and result types."""
    for name, args in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_size_t if name.endswith("_bytes") else ctypes.c_int
        _FN[name] = fn


# A decoding step's bookkeeping takes a few microseconds on the GPU: the checks look at each tensor
# once, and only a tensor that fails is looked at for what is wrong.

def _call(name, dev, *args):
    """Calls an entry point with device `dev` as the current one."""
    if not _FN:
        _base.load_library()
    if dev == torch._C._cuda_getDevice():
        rc = _FN[name](*args)
    else:
        with torch.cuda.device(dev):
            rc = _FN[name](*args)
    if rc:
        raise _base.GMMError(name, rc)


def _stream(stream, dev):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _wrong(t, dtype, numel, name, dev):
    """The error of a tensor that is not a contiguous `dtype` one on device `dev`."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()):
        return TypeError(f"{name} must be a contiguous {dtype} CUDA tensor")
    if t.get_device() != dev:
        return ValueError(f"{name} is on {t.device}, the call's other tensors on cuda:{dev}")
    return ValueError(f"{name} holds {t.numel()} elements, {numel} needed")


def _flat(t, dtype, numel, name, dev):
    """Address of a contiguous CUDA tensor of `numel` elements or more on device `dev`."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == dev and \
            t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    raise _wrong(t, dtype, numel, name, dev)


def _table(total, pages, dev, names=("total", "pages")):
    """(total, pages, rows, max_pages, stride) of a table."""
    if not (isinstance(pages, torch.Tensor) and pages.dtype is torch.int32 and pages.dim() == 2 and
            pages.is_cuda):
        raise TypeError(f"{names[1]} must be an int32 CUDA tensor [rows, max_pages]")
    (rows, width), (stride, inner) = pages.shape, pages.stride()
    if inner != 1 and width > 1:
        raise TypeError(f"{names[1]} must have contiguous rows")
    if pages.get_device() != dev:
        raise ValueError(f"{names[1]} is on {pages.device}, the call's other tensors on cuda:{dev}")
    at = _flat(total, torch.int32, rows, names[0], dev)
    if total.numel() != rows:
        raise ValueError(f"{names[1]} has {rows} rows for {total.numel()} in {names[0]}")
    return at, pages.data_ptr(), rows, width, stride if rows > 1 else max(stride, width)


def _ws(ws, dev):
    at, size = _base._ws(ws)
    if ws is not None and ws.get_device() != dev:
        raise ValueError(f"ws is on {ws.device}, the call's other tensors on cuda:{dev}")
    return at, size


def kv_pool(cache):
    """Counts of an empty pool for the cache's pages: int32 zeros [pages]."""
    return torch.zeros(cache.pages, dtype=torch.int32, device=cache.k.device)


def kv_pool_workspace_bytes(cache, rows):
    """Workspace size of gmm_kv_grow and gmm_kv_compact for tables of up to `rows` rows."""
    return int(_base.load_library().gmm_kv_pool_workspace_bytes(cache._ref, int(rows)))


def kv_pool_workspace(cache, rows):
    """A workspace tensor (uint8) for tables of up to `rows` rows."""
    nb = kv_pool_workspace_bytes(cache, rows)
    if nb == 0:
        raise _base.GMMError("gmm_kv_pool_workspace_bytes", _base.GMM_ERR_UNSUPPORTED)
    return torch.empty(nb, dtype=torch.uint8, device=cache.k.device)


def gmm_kv_copy(src, dst, src_pages, dst_pages, stream=None):
    """Copies pages src_pages [n] int32 of the cache src to pages dst_pages [n] of the cache dst
    (which may be src): keys, values and boxes."""
    dev, n = src.k.get_device(), src_pages.numel()
    if dst.k.get_device() != dev:
        raise ValueError(f"dst is on {dst.k.device}, src on {src.k.device}")
    if dst_pages.numel() != n:
        raise ValueError(f"{n} source pages, {dst_pages.numel()} destinations")
    _call("gmm_kv_copy", dev, src._ref, dst._ref, _flat(src_pages, torch.int32, n, "src_pages", dev),
          _flat(dst_pages, torch.int32, n, "dst_pages", dev), n, _stream(stream, dev))


def gmm_kv_fork(cache, ref, total, pages, parent, total_out, pages_out, keep=None, release=True,
                stream=None):
    """New rows total_out [rows], pages_out [rows, >= max_pages] with the pages of the rows
    parent [rows] of (total, pages), of their first keep [rows] keys if given.  release: the old
    rows are given up, and pages that nobody names any more are free."""
    dev, rows = cache.k.get_device(), parent.numel()
    new = _table(total_out, pages_out, dev, ("total_out", "pages_out"))
    if new[2] != rows:
        raise ValueError(f"pages_out has {new[2]} rows for {rows} parents")
    _call("gmm_kv_fork", dev, cache._ref, _flat(ref, torch.int32, cache.pages, "ref", dev),
          *_table(total, pages, dev), _flat(parent, torch.int32, rows, "parent", dev),
          None if keep is None else _flat(keep, torch.int32, rows, "keep", dev), rows,
          1 if release else 0, new[0], new[1], new[3], new[4], _stream(stream, dev))


def gmm_kv_grow(cache, ref, held, total, pages, short_by, ws, stream=None):
    """Gives the rows of `pages` [rows, max_pages] pages for growing from held [rows] to total
    [rows] keys, copies of shared pages that they write into among them; short_by [1] int32: how
    many pages are missing (then nothing changes), or 0."""
    dev = cache.k.get_device()
    tb = _table(total, pages, dev)
    _call("gmm_kv_grow", dev, cache._ref, _flat(ref, torch.int32, cache.pages, "ref", dev),
          _flat(held, torch.int32, tb[2], "held", dev), *tb,
          _flat(short_by, torch.int32, 1, "short_by", dev), *_ws(ws, dev), _stream(stream, dev))


def gmm_kv_compact(cache, ref, total, pages, where, used, ws, stream=None):
    """Moves the used pages to the numbers below their count used [1] int32, rewrites the tables,
    and says in where [cache pages] int32 where every page's contents are now (-1: it was free)."""
    dev = cache.k.get_device()
    _call("gmm_kv_compact", dev, cache._ref, _flat(ref, torch.int32, cache.pages, "ref", dev),
          *_table(total, pages, dev), _flat(where, torch.int32, cache.pages, "where", dev),
          _flat(used, torch.int32, 1, "used", dev), *_ws(ws, dev), _stream(stream, dev))


def beam_workspace_bytes(batch, beams, vocab):
    """Workspace size of gmm_beam_select."""
    return int(_base.load_library().gmm_beam_workspace_bytes(int(batch), int(beams), int(vocab)))


def beam_workspace(batch, beams, vocab, device="cuda"):
    """A workspace tensor (uint8) for gmm_beam_select."""
    nb = beam_workspace_bytes(batch, beams, vocab)
    if nb == 0:
        raise _base.GMMError("gmm_beam_workspace_bytes", _base.GMM_ERR_UNSUPPORTED)
    return torch.empty(nb, dtype=torch.uint8, device=device)


def gmm_beam_select(logits, score, out_score, out_parent, out_token, ws, done=None, out_done=None,
                    eos=-1, weight=None, mask=None, scale=1.0, stream=None):
    """The m = out_score.shape[1] best continuations of every sequence's beams.  logits
    [batch, beams, vocab] fp32, bf16 or fp16 (words contiguous), score [batch, beams] fp32;
    out_score [batch, m] fp32, out_parent [batch, m] int32 (rows: b * beams + beam) and out_token
    [batch, m] int32.  done / out_done: bool, finished beams (their one continuation is eos);
    weight [batch, beams] fp32: factors of the scores where they are compared; mask
    [batch, beams, words] int32: bit v % 32 of word v // 32 allows word v."""
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 3):
        raise TypeError("logits must be a CUDA tensor [batch, beams, vocab]")
    batch, beams, vocab = logits.shape
    dev, rows = logits.get_device(), batch * beams
    s0, s1, s2 = logits.stride()
    if s2 != 1 and vocab > 1 and rows:
        raise TypeError("logits must have contiguous rows")
    if out_score.dim() != 2 or out_score.shape[0] != batch:
        raise ValueError(f"out_score must be [{batch}, m]")
    m = out_score.shape[1]
    opt = lambda t, dt, n, name: None if t is None else _flat(t, dt, n, name, dev)
    words = 0
    if mask is not None:
        if mask.dim() != 3 or mask.shape[:2] != (batch, beams):
            raise ValueError(f"mask must be [{batch}, {beams}, words]")
        words = mask.shape[2]
    _call("gmm_beam_select", dev, logits.data_ptr(), _dtype(logits.dtype), s0, s1, batch, beams,
          vocab, _flat(score, torch.float32, rows, "score", dev),
          opt(weight, torch.float32, rows, "weight"), opt(done, torch.bool, rows, "done"), eos,
          opt(mask, torch.int32, rows * words, "mask"), words, scale, m,
          _flat(out_score, torch.float32, batch * m, "out_score", dev),
          _flat(out_parent, torch.int32, batch * m, "out_parent", dev),
          _flat(out_token, torch.int32, batch * m, "out_token", dev),
          opt(out_done, torch.bool, batch * m, "out_done"), *_ws(ws, dev), _stream(stream, dev))
