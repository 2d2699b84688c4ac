"""Python binding of the paged key/value cache: rotary positions, appending, page selection and
attention (``csrc/kvcache.hip``).

Argument marshalling only, with the names of the C ABI in ``include/flashgmm.h``.  A batch is
given by three int32 CUDA tensors: ``cu`` [batch + 1] (first row of every sequence's new tokens),
``total`` [batch] (keys of the sequence with them) and ``pages`` [batch, max_pages] (page table).
Keys are appended before the queries of the same tokens attend.
"""
from __future__ import annotations

import ctypes
import math

import torch

import paper_2606_10896_amd as _base

GMM_F32 = 0
GMM_BF16 = 1
GMM_F16 = 2


class _CCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("box", ctypes.c_void_p),
                ("box_scale", ctypes.c_void_p), ("pages", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("page", ctypes.c_int32), ("d", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class _CBatch(ctypes.Structure):
    _fields_ = [("cu", ctypes.c_void_p), ("total", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("pages_stride", ctypes.c_int64)]


_VP, _I64, _I32, _F32, _F64, _SZ = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                    ctypes.c_float, ctypes.c_double, ctypes.c_size_t)
_CP, _BP = ctypes.POINTER(_CCache), ctypes.POINTER(_CBatch)
_STRIDED = [_VP, _I64, _I64]

#: argument types of the C entry points
SIGNATURES = {
    "gmm_rope_table": [_VP, _I32, _F64, _I32, _VP, _VP],
    "gmm_rope": [*_STRIDED, *_STRIDED, _I64, _I32, _I32, _I32, _VP, _VP, _I32, _I32, _I32, _I32,
                 _VP],
    "gmm_kv_append": [_CP, _BP, _I64, *_STRIDED, *_STRIDED, _VP, _VP, _I32, _I32, _I32, *_STRIDED,
                      *_STRIDED, _I32, _VP],
    "gmm_kv_workspace_bytes": [_CP, _I64, _I32, _I32, _I32],
    "gmm_kv_select": [_CP, _BP, _I64, *_STRIDED, _I32, _I32, _I32, _I32, _VP, _VP, _SZ, _VP],
    "gmm_kv_attend": [_CP, _BP, _I64, *_STRIDED, _I32, _F32, _I32, _VP, _I32, _VP, _VP, _VP, _SZ,
                      _VP],
}


def bind(lib):
    """Sets the entry points' argument and result types."""
    for name, args in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_size_t if name == "gmm_kv_workspace_bytes" else ctypes.c_int


_CODES = {torch.float32: GMM_F32, torch.bfloat16: GMM_BF16, torch.float16: GMM_F16}


def _dtype(t):
    code = _CODES.get(t)
    if code is None:
        raise TypeError(f"{t} is not a type of these calls")
    return code


# A step of a single token is a few microseconds on the GPU: the binding keeps its own share of
# a call small (addresses as plain integers, one look at a tensor's strides, the stream's handle
# without a Stream object).

def _stream(stream, t):
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _flat(t, dtype, numel, name):
    """Address of a contiguous CUDA tensor of at least numel elements."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous {dtype} CUDA tensor")
    if t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, {numel} needed")
    return t.data_ptr()


class KVCache:
    """Pages of keys and values: k [pages, heads, page, d], v [pages, heads, d, page] (a page's
    values transposed), bfloat16 or float16; box [pages, heads, 2, d] int8 and box_scale
    [pages, heads] fp32 for gmm_kv_select, or None for a cache without boxes."""

    def __init__(self, k, v, box=None, box_scale=None):
        dev = _base._dev
        pages, heads, page, d = k.shape
        if k.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("k must be bfloat16 or float16")
        dev(k, k.dtype, "k")
        dev(v, k.dtype, "v")
        if tuple(v.shape) != (pages, heads, d, page):
            raise ValueError(f"v must be [pages, heads, d, page] = {[pages, heads, d, page]}")
        if (box is None) != (box_scale is None):
            raise ValueError("box and box_scale come together")
        if box is not None:
            dev(box, torch.int8, "box", pages * heads * 2 * d)
            dev(box_scale, torch.float32, "box_scale", pages * heads)
        self.k, self.v, self.box, self.box_scale = k, v, box, box_scale
        self.pages, self.heads, self.page, self.d = pages, heads, page, d
        at = lambda t: None if t is None else t.data_ptr()
        self._c = _CCache(at(k), at(v), at(box), at(box_scale), pages, heads, page, d,
                          _dtype(k.dtype))
        self._ref = ctypes.byref(self._c)

    def box_values(self):
        """The boxes as numbers, fp32 [pages, heads, 2, d]: upper, then lower bounds."""
        return self.box * self.box_scale.view(self.pages, self.heads, 1, 1)


def kv_cache(pages, heads, page, d, dtype=None, boxes=True, device="cuda"):
    """An empty KVCache (bfloat16 unless dtype says otherwise)."""
    dtype = torch.bfloat16 if dtype is None else dtype
    k = torch.zeros(pages, heads, page, d, dtype=dtype, device=device)
    v = torch.zeros(pages, heads, d, page, dtype=dtype, device=device)
    box = torch.zeros(pages, heads, 2, d, dtype=torch.int8, device=device) if boxes else None
    scale = torch.zeros(pages, heads, dtype=torch.float32, device=device) if boxes else None
    return KVCache(k, v, box, scale)


def rope_frequencies(rot, base=10000.0, factor=1.0, trained=None, slow=1.0, fast=32.0):
    """Rotation frequencies base^(-2i / rot), i < rot / 2, as a list.  factor > 1 stretches them
    for contexts `factor` times as long: all of them (trained None: positions are interpolated),
    or by parts: a pair that turns fewer than `slow` times in the `trained` positions is divided
    by factor, one that turns more than `fast` times is kept, in between the share is linear in
    its turns."""
    if rot < 2 or rot % 2 or base <= 0 or factor <= 0:
        raise ValueError("rot must be even and positive, base and factor positive")
    if trained is not None and not 0 <= slow < fast:
        raise ValueError("0 <= slow < fast")
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        keep = 0.0
        if trained is not None:
            keep = min(1.0, max(0.0, (trained * f / (2 * math.pi) - slow) / (fast - slow)))
        out.append(f * keep + f / factor * (1.0 - keep))
    return out


def gmm_rope_table(freq, table, scale=1.0, stream=None):
    """Fills table [positions, rot] fp32 (rot/2 cosines, then rot/2 sines of every position,
    times scale) from the frequencies freq [rot/2] (fp64 CUDA tensor)."""
    positions, rot = table.shape
    if rot % 2:
        raise ValueError("table must hold an even number of columns")
    rc = _base.load_library().gmm_rope_table(
        _base._ptr(_base._dev(freq, torch.float64, "freq", rot // 2)), rot // 2, float(scale),
        positions, _base._ptr(_base._dev(table, torch.float32, "table")), _stream(stream, table))
    _base._check("gmm_rope_table", rc)


def _rows(t, dtype, tokens, heads, d, name):
    """(address, token stride, head stride) of a CUDA tensor [tokens, heads, d] whose rows are
    contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype):
        raise TypeError(f"{name} must be a {dtype} CUDA tensor")
    if t.shape != (tokens, heads, d):
        raise ValueError(f"{name} must have the shape {[tokens, heads, d]}, has {list(t.shape)}")
    st = t.stride()
    if st[2] != 1 and t.numel():
        raise TypeError(f"{name} must have contiguous rows")
    return t.data_ptr(), st[0], st[1]


def gmm_rope(x, pos, table, out, interleaved=False, inverse=False, stream=None):
    """Rotates x [tokens, heads, d] by the positions pos [tokens] int32 into out (which may be x):
    the first rot = table.shape[1] dimensions in pairs (i, i + rot/2), or (2i, 2i + 1) if
    interleaved.  inverse applies the transposed rotation: the gradient."""
    tokens, heads, d = x.shape
    dt = x.dtype
    rc = _base.load_library().gmm_rope(
        *_rows(x, dt, tokens, heads, d, "x"), *_rows(out, dt, tokens, heads, d, "out"), tokens,
        heads, d, _dtype(dt), _flat(pos, torch.int32, tokens, "pos"),
        _flat(table, torch.float32, 0, "table"), table.shape[0], table.shape[1],
        1 if interleaved else 0, 1 if inverse else 0, _stream(stream, x))
    if rc:
        raise _base.GMMError("gmm_rope", rc)


def _batch(cu, total, pages):
    batch = total.numel()
    if not (isinstance(pages, torch.Tensor) and pages.is_cuda and pages.dtype is torch.int32 and
            pages.dim() == 2 and (pages.stride(1) == 1 or pages.shape[1] == 1)):
        raise TypeError("pages must be an int32 CUDA tensor [batch, max_pages] with contiguous rows")
    rows, width = pages.shape
    if rows != batch:
        raise ValueError(f"pages has {rows} rows for {batch} sequences")
    stride = max(pages.stride(0), width) if batch == 1 else pages.stride(0)
    return ctypes.byref(_CBatch(_flat(cu, torch.int32, batch + 1, "cu"),
                                _flat(total, torch.int32, batch, "total"), pages.data_ptr(), batch,
                                width, stride))


def gmm_kv_append(cache, k, v, cu, total, pages, pos=None, table=None, q=None, q_out=None,
                  interleaved=False, stream=None):
    """Stores the new tokens' keys (rotated if a table is given) and values [tokens, heads, d] in
    the cache and renews the boxes of their pages; rotates q [tokens, hq, d] into q_out.  pos
    [tokens] int32: rotation positions, a token's slot in its sequence if None."""
    tokens = k.shape[0]
    dt, heads, d = cache.k.dtype, cache.heads, cache.d
    qs = qo = (0, 0, 0)
    hq = 0
    if q is not None:
        hq = q.shape[1]
        qs = _rows(q, dt, tokens, hq, d, "q")
        qo = _rows(q_out, dt, tokens, hq, d, "q_out")
    tb = (0, 0, 0)
    if table is not None:
        tb = _flat(table, torch.float32, 0, "table"), table.shape[0], table.shape[1]
    rc = _base.load_library().gmm_kv_append(
        cache._ref, _batch(cu, total, pages), tokens, *_rows(k, dt, tokens, heads, d, "k"),
        *_rows(v, dt, tokens, heads, d, "v"),
        0 if pos is None else _flat(pos, torch.int32, tokens, "pos"), *tb,
        1 if interleaved else 0, *qs, *qo, hq, _stream(stream, k))
    if rc:
        raise _base.GMMError("gmm_kv_append", rc)


def kv_workspace_bytes(cache, tokens, hq, batch, max_pages):
    """Workspace size of gmm_kv_select and gmm_kv_attend."""
    return int(_base.load_library().gmm_kv_workspace_bytes(
        cache._ref, int(tokens), int(hq), int(batch), int(max_pages)))


def kv_workspace(cache, tokens, hq, batch, max_pages):
    """A workspace tensor (uint8) for calls with up to these sizes."""
    nb = kv_workspace_bytes(cache, tokens, hq, batch, max_pages)
    if nb == 0:
        raise _base.GMMError("gmm_kv_workspace_bytes", _base.GMM_ERR_UNSUPPORTED)
    return torch.empty(nb, dtype=torch.uint8, device=cache.k.device)


def gmm_kv_select(cache, q, cu, total, pages, idx, ws, keep_first=1, keep_last=1, stream=None):
    """The m = idx.shape[2] best pages of every new token and cache head into idx
    [tokens, heads, m] int32 (indexes into the page table, ascending, -1 at the end)."""
    tokens, hq = q.shape[:2]
    if idx.dim() != 3 or idx.shape[0] != tokens or idx.shape[1] != cache.heads:
        raise ValueError(f"idx must be [{tokens}, {cache.heads}, m]")
    rc = _base.load_library().gmm_kv_select(
        cache._ref, _batch(cu, total, pages), tokens, *_rows(q, cache.k.dtype, tokens, hq, cache.d, "q"),
        hq, idx.shape[2], keep_first, keep_last, _flat(idx, torch.int32, 0, "idx"), *_base._ws(ws),
        _stream(stream, q))
    if rc:
        raise _base.GMMError("gmm_kv_select", rc)


def gmm_kv_attend(cache, q, cu, total, pages, out, ws, lse=None, scale=None, window=0, sel=None,
                  stream=None):
    """Attention of the new tokens' queries q [tokens, hq, d] over their sequences' keys (causal;
    the last `window` keys if window > 0; the pages listed in sel [tokens, heads, m] if given)
    into out [tokens, hq, d] and lse [tokens, hq] fp32.  scale is 1/sqrt(d) if None."""
    tokens, hq = q.shape[:2]
    dt, d = cache.k.dtype, cache.d
    sp, m = 0, 0
    if sel is not None:
        sp, m = _flat(sel, torch.int32, 0, "sel"), sel.shape[-1]
        if sel.dim() != 3 or sel.shape[0] != tokens or sel.shape[1] != cache.heads:
            raise ValueError(f"sel must be [{tokens}, {cache.heads}, m]")
    rc = _base.load_library().gmm_kv_attend(
        cache._ref, _batch(cu, total, pages), tokens, *_rows(q, dt, tokens, hq, d, "q"), hq,
        1.0 / math.sqrt(d) if scale is None else scale, window, sp, m,
        _flat(out, dt, tokens * hq * d, "out"),
        0 if lse is None else _flat(lse, torch.float32, tokens * hq, "lse"), *_base._ws(ws),
        _stream(stream, q))
    if rc:
        raise _base.GMMError("gmm_kv_attend", rc)
