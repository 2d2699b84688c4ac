"""The paged cache's calls without a GPU: bad arguments are refused on the host, before anything
is enqueued, by the C entry points and by the binding."""
import ctypes

import pytest
import torch

import paper_2606_10896_amd as gmm
from paper_2606_10896_amd.kv import _CBatch, _CCache

BAD, UNSUP, WS, OK = (gmm.GMM_ERR_INVALID_ARG, gmm.GMM_ERR_UNSUPPORTED, gmm.GMM_ERR_WORKSPACE,
                      gmm.GMM_OK)
P = 0x100000


@pytest.fixture(scope="module")
def lib():
    return gmm.load_library()


def _cache(**kw):
    f = dict(k=P, v=P, box=P, box_scale=P, pages=10, heads=2, page=64, d=128, dtype=1)
    f.update(kw)
    return _CCache(*(f[n] for n, _ in _CCache._fields_))


def _batch(**kw):
    f = dict(cu=P, total=P, pages=P, batch=3, max_pages=4, pages_stride=4)
    f.update(kw)
    return _CBatch(*(f[n] for n, _ in _CBatch._fields_))


CACHES = [(dict(k=None), BAD), (dict(v=None), BAD), (dict(pages=0), BAD), (dict(heads=0), BAD),
          (dict(page=0), BAD), (dict(d=0), BAD), (dict(k=P + 8), BAD), (dict(v=P + 2), BAD),
          (dict(box=None), BAD), (dict(box_scale=None), BAD), (dict(dtype=0), UNSUP),
          (dict(dtype=7), UNSUP), (dict(d=24), UNSUP), (dict(d=272), UNSUP), (dict(page=16), UNSUP),
          (dict(page=48), UNSUP), (dict(page=512), UNSUP), (dict(heads=2000), UNSUP)]
BATCHES = [(dict(cu=None), BAD), (dict(total=None), BAD), (dict(pages=None), BAD),
           (dict(batch=0), BAD), (dict(max_pages=0), BAD), (dict(pages_stride=3), BAD),
           (dict(max_pages=1 << 26, pages_stride=1 << 26), UNSUP), (dict(batch=1 << 21), UNSUP)]


def _append(lib, c, b, tokens=5, k=P, v=P, table=None, positions=0, rot=0, q=None, qo=None, hq=0):
    return lib.gmm_kv_append(ctypes.byref(c) if c else None, ctypes.byref(b) if b else None, tokens,
                             k, 256, 128, v, 256, 128, None, table, positions, rot, 0, q, 512, 128,
                             qo, 512, 128, hq, None)


def _select(lib, c, b, tokens=5, q=P, hq=4, m=4, first=1, last=1, idx=P, ws=P, nb=1 << 40):
    return lib.gmm_kv_select(ctypes.byref(c) if c else None, ctypes.byref(b) if b else None, tokens,
                             q, 512, 128, hq, m, first, last, idx, ws, nb, None)


def _attend(lib, c, b, tokens=5, q=P, hq=4, scale=0.1, window=0, sel=None, m=0, out=P, lse=None,
            ws=P, nb=1 << 40):
    return lib.gmm_kv_attend(ctypes.byref(c) if c else None, ctypes.byref(b) if b else None, tokens,
                             q, 512, 128, hq, scale, window, sel, m, out, lse, ws, nb, None)


@pytest.mark.parametrize("call", [_append, _select, _attend])
def test_caches_and_batches(lib, call):
    for kw, want in CACHES:
        assert call(lib, _cache(**kw), _batch()) == want, kw
    for kw, want in BATCHES:
        assert call(lib, _cache(), _batch(**kw)) == want, kw
    assert call(lib, None, _batch()) == BAD
    assert call(lib, _cache(), None) == BAD
    assert call(lib, _cache(), _batch(), tokens=-1) == BAD
    assert call(lib, _cache(), _batch(), tokens=(1 << 24) + 1) == UNSUP
    assert call(lib, _cache(), _batch(), tokens=0) == OK


def test_append(lib):
    c, b = _cache(), _batch()
    assert _append(lib, c, b, k=None) == BAD
    assert _append(lib, c, b, v=None) == BAD
    for rot in (0, 3, 130, -2):
        assert _append(lib, c, b, table=P, positions=9, rot=rot) == BAD
    assert _append(lib, c, b, table=P, positions=0, rot=64) == BAD
    assert _append(lib, c, b, q=P, qo=P, hq=4) == BAD                      # no table
    assert _append(lib, c, b, table=P, positions=9, rot=64, q=P, hq=4) == BAD
    assert _append(lib, c, b, table=P, positions=9, rot=64, q=P, qo=P, hq=3) == BAD
    assert _append(lib, c, b, table=P, positions=9, rot=64, q=P, qo=P, hq=0) == BAD
    assert _append(lib, c, b, table=P, positions=9, rot=64, q=P, qo=P, hq=130) == UNSUP


def test_select(lib):
    c, b = _cache(), _batch()
    assert _select(lib, _cache(box=None, box_scale=None), b) == BAD
    for kw in (dict(q=None), dict(idx=None), dict(hq=3), dict(hq=0), dict(m=0), dict(first=-1),
               dict(last=0), dict(m=3, first=2, last=2)):
        assert _select(lib, c, b, **kw) == BAD, kw
    assert _select(lib, c, b, m=4097) == UNSUP
    assert _select(lib, c, b, hq=130) == UNSUP
    need = lib.gmm_kv_workspace_bytes(ctypes.byref(c), 5, 4, 3, 4)
    assert need > 0 and need % 256 == 0
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
        assert _select(lib, c, b, **kw) == WS, kw


def test_attend(lib):
    c, b = _cache(), _batch()
    for kw in (dict(q=None), dict(out=None), dict(out=P + 4), dict(hq=3), dict(hq=0), dict(window=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(m=4), dict(sel=P, m=0),
               dict(sel=P, m=4, window=3)):
        assert _attend(lib, c, b, **kw) == BAD, kw
    assert _attend(lib, c, b, sel=P, m=4097) == UNSUP
    assert _attend(lib, c, b, hq=130) == UNSUP
    need = lib.gmm_kv_workspace_bytes(ctypes.byref(c), 5, 4, 3, 4)
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
        assert _attend(lib, c, b, **kw) == WS, kw


def test_workspace(lib):
    size = lambda c, *a: lib.gmm_kv_workspace_bytes(ctypes.byref(c), *a)
    for kw, _ in CACHES:
        assert size(_cache(**kw), 5, 4, 3, 4) == 0
    for a in ((-1, 4, 3, 4), (5, 3, 3, 4), (5, 4, 0, 4), (5, 4, 3, 0), ((1 << 24) + 1, 4, 3, 4),
              (5, 4, 3, 1 << 26)):
        assert size(_cache(), *a) == 0
    # the scores of every (token, head, page) fit
    assert size(_cache(), 100, 4, 3, 1001) >= 100 * 2 * 1001 * 4


def test_rope(lib):
    call = lambda x=P, out=P, tokens=5, heads=2, d=64, dt=1, pos=P, table=P, n=9, rot=64: \
        lib.gmm_rope(x, 128, 64, out, 128, 64, tokens, heads, d, dt, pos, table, n, rot, 0, 0, None)
    for kw in (dict(x=None), dict(out=None), dict(pos=None), dict(table=None), dict(tokens=-1),
               dict(heads=0), dict(d=1), dict(n=0), dict(rot=0), dict(rot=3), dict(rot=66)):
        assert call(**kw) == BAD, kw
    for kw in (dict(dt=3), dict(d=1026), dict(heads=1025), dict(tokens=(1 << 24) + 1)):
        assert call(**kw) == UNSUP, kw
    assert call(tokens=0) == OK
    table = lambda f=P, half=4, scale=1.0, n=9, t=P: lib.gmm_rope_table(f, half, scale, n, t, None)
    for kw in (dict(f=None), dict(t=None), dict(half=0), dict(n=0), dict(scale=float("nan"))):
        assert table(**kw) == BAD, kw
    assert table(half=513) == UNSUP
    assert table(half=512, n=2 ** 31 - 1) == UNSUP


def test_binding_refuses_what_is_no_gpu_tensor():
    k = torch.zeros(2, 1, 32, 16, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        gmm.KVCache(k, k.transpose(2, 3).contiguous())
    with pytest.raises(TypeError):
        gmm.KVCache(k.float(), k.float())
    with pytest.raises(TypeError):
        gmm.gmm_rope(k[0], torch.zeros(1, dtype=torch.int32), torch.zeros(4, 16), k[0])
    for kw in (dict(rot=3), dict(rot=0), dict(rot=8, base=0.0), dict(rot=8, factor=0.0),
               dict(rot=8, trained=100, slow=3.0, fast=2.0)):
        with pytest.raises(ValueError):
            gmm.rope_frequencies(**kw)
