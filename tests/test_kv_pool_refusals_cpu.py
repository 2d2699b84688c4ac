"""The page pool's and the selection's calls without a GPU: bad arguments are refused on the host,
before anything is enqueued, by the C entry points and by the binding."""
import ctypes

import pytest
import torch

import paper_2606_10896_amd as gmm
from test_kv_refusals_cpu import BAD, CACHES, OK, UNSUP, WS, P, _cache

Q = 0x900000                    # another address, far from P
ROWS = 65536                    # rows of a table at most


@pytest.fixture(scope="module")
def lib():
    return gmm.load_library()


def _ref(c):
    return ctypes.byref(c) if c else None


def _copy(lib, c, dst=None, a=P, b=Q, n=5):
    return lib.gmm_kv_copy(_ref(c), _ref(dst if dst else c), a, b, n, None)


def _fork(lib, c, ref=P, total=P, pages=P, batch=3, width=4, stride=4, parent=P, keep=None, rows=3,
          release=1, nt=Q, npg=Q, nwidth=4, nstride=4):
    return lib.gmm_kv_fork(_ref(c), ref, total, pages, batch, width, stride, parent, keep, rows,
                           release, nt, npg, nwidth, nstride, None)


def _grow(lib, c, ref=P, held=P, total=P, pages=P, batch=3, width=4, stride=4, short=P, ws=P,
          nb=1 << 40):
    return lib.gmm_kv_grow(_ref(c), ref, held, total, pages, batch, width, stride, short, ws, nb,
                           None)


def _compact(lib, c, ref=P, total=P, pages=P, batch=3, width=4, stride=4, where=P, used=P, ws=P,
             nb=1 << 40):
    return lib.gmm_kv_compact(_ref(c), ref, total, pages, batch, width, stride, where, used, ws, nb,
                              None)


def _beam(lib, x=P, dt=1, s0=4000, s1=1000, batch=2, beams=4, vocab=1000, score=P, weight=None,
          done=None, eos=-1, mask=None, mstride=0, scale=1.0, m=4, os=P, op=P, ot=P, od=None, ws=P,
          nb=1 << 40):
    return lib.gmm_beam_select(x, dt, s0, s1, batch, beams, vocab, score, weight, done, eos, mask,
                               mstride, scale, m, os, op, ot, od, ws, nb, None)


TABLES = [(dict(batch=0), BAD), (dict(width=0), BAD), (dict(stride=3), BAD),
          (dict(batch=ROWS + 1), UNSUP), (dict(width=1 << 25, stride=1 << 25), UNSUP),
          (dict(ref=None), BAD), (dict(total=None), BAD), (dict(pages=None), BAD)]


@pytest.mark.parametrize("call", [_copy, _fork, _grow, _compact])
def test_caches(lib, call):
    for kw, want in CACHES:
        assert call(lib, _cache(**kw)) == want, kw
    assert call(lib, None) == BAD


@pytest.mark.parametrize("call", [_fork, _grow, _compact])
def test_tables(lib, call):
    for kw, want in TABLES:
        assert call(lib, _cache(), **kw) == want, kw
    assert call(lib, _cache(pages=(1 << 26) + 1)) == UNSUP


def test_copy(lib):
    for kw in (dict(heads=3), dict(page=32), dict(d=64), dict(dtype=2),
               dict(box=None, box_scale=None)):
        assert _copy(lib, _cache(), _cache(**kw)) == BAD, kw
    for kw, want in (((dict(a=None)), BAD), (dict(b=None), BAD), (dict(n=-1), BAD),
                     (dict(n=(1 << 30) + 1), UNSUP), (dict(n=0), OK),
                     (dict(n=0, a=None, b=None), OK)):
        assert _copy(lib, _cache(), **kw) == want, kw


def test_fork(lib):
    c = _cache()
    for kw in (dict(parent=None), dict(nt=None), dict(npg=None), dict(rows=-1), dict(nwidth=3),
               dict(nwidth=6, nstride=5)):
        assert _fork(lib, c, **kw) == BAD, kw
    assert _fork(lib, c, rows=ROWS + 1) == UNSUP
    assert _fork(lib, c, nwidth=1 << 25, nstride=1 << 25) == UNSUP
    # rows 0 and nothing to give up: nothing to do
    assert _fork(lib, c, rows=0, release=0, parent=None, nt=None, npg=None) == OK


def test_fork_refuses_tables_that_overlap(lib):
    c = _cache()
    # the old tables take 3 x 4 entries from P on, the new ones 3 x 4
    for off in (0, 4, 44, -44):
        assert _fork(lib, c, npg=P + off) == BAD, off
    for off in (0, 8, -8):
        assert _fork(lib, c, nt=P + off) == BAD, off
        assert _fork(lib, c, parent=Q + 4096 + off, nt=Q + 4096) == BAD, off
        assert _fork(lib, c, keep=Q + 4096 + off, nt=Q + 4096) == BAD, off
        for name in ("total", "parent", "keep"):
            assert _fork(lib, c, nt=Q + 8192, npg=Q + 4096, **{name: Q + 4096 + off}) == BAD, name
    assert _fork(lib, c, nt=P + 16) == BAD             # into the old table of pages


def test_workspaces(lib):
    c = _cache()
    size = lambda c, n: lib.gmm_kv_pool_workspace_bytes(ctypes.byref(c), n)
    for kw, _ in CACHES:
        assert size(_cache(**kw), 3) == 0
    assert size(c, 0) == 0 and size(c, ROWS + 1) == 0 and size(c, ROWS) > 0
    assert size(_cache(pages=(1 << 26) + 1), 3) == 0
    need = size(c, 3)
    assert need % 256 == 0
    assert size(_cache(pages=100), 3) >= 3 * 4 * 100
    for call in (_grow, _compact):
        for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
            assert call(lib, c, **kw) == WS, kw
    need = lib.gmm_beam_workspace_bytes(2, 4, 1000)
    for kw in (dict(ws=None), dict(ws=P + 16), dict(nb=need - 1)):
        assert _beam(lib, **kw) == WS, kw
    for a in ((0, 4, 1000), (2, 0, 1000), (2, 4, 0), (2, 65, 1000), (2, 4, (1 << 24) + 1),
              (1 << 24, 2, 1000), (1 << 19, 64, 1000), (1 << 15, 64, 1 << 24), (1 << 23, 1, 10)):
        assert lib.gmm_beam_workspace_bytes(*a) == 0, a


def test_grow_and_compact(lib):
    c = _cache()
    for kw in (dict(held=None), dict(short=None)):
        assert _grow(lib, c, **kw) == BAD, kw
    for kw in (dict(where=None), dict(used=None)):
        assert _compact(lib, c, **kw) == BAD, kw


def test_select(lib):
    for kw in (dict(batch=-1), dict(beams=0), dict(vocab=0), dict(m=0), dict(eos=1000),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e7),
               dict(scale=1e-7), dict(done=P, eos=3), dict(done=P, od=P, eos=-1),
               dict(mask=P, mstride=31), dict(x=None), dict(score=None), dict(os=None),
               dict(op=None), dict(ot=None), dict(x=P + 1), dict(x=P + 2, dt=0)):
        assert _beam(lib, **kw) == BAD, kw
    for kw in (dict(dt=3), dict(m=65), dict(beams=65), dict(vocab=(1 << 24) + 1),
               dict(batch=1 << 23)):
        assert _beam(lib, **kw) == UNSUP, kw
    assert _beam(lib, batch=0, x=None, score=None) == OK


def test_select_refuses_results_over_what_it_reads(lib):
    # scores, weights and flags: 2 x 4; the workspace is refused where they are not
    for off in (4, -4, 28, -28):
        assert _beam(lib, os=P + off, ws=None) == BAD, off
        assert _beam(lib, weight=Q, os=Q + off, ws=None) == BAD, off
    for off in (1, -1, 7, -7):
        assert _beam(lib, done=Q, od=Q + off, eos=3, ws=None) == BAD, off
    for off in (32, -32):
        assert _beam(lib, os=P + off, ws=None) == WS, off
    assert _beam(lib, done=Q, od=Q, eos=3, ws=None) == WS
    # in place only with as many results as beams
    assert _beam(lib, m=3, ws=None) == BAD
    assert _beam(lib, m=3, os=Q, done=Q + 64, od=Q + 64, eos=3, ws=None) == BAD
    assert _beam(lib, m=3, os=Q, ws=None) == WS


def test_binding_refuses_what_is_no_gpu_tensor():
    f, i = torch.zeros(1, 2), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(TypeError):
        gmm.gmm_beam_select(torch.zeros(1, 2, 50), f, f, i, i, None)
    with pytest.raises(TypeError):
        gmm.pool._flat(i, torch.int32, 2, "x", 0)
    with pytest.raises(TypeError):
        gmm.pool._table(i, i, 0)


def test_the_binding_checks_every_workspace():
    with open(gmm.pool.__file__) as f:
        text = f.read()
    assert "ws.data_ptr()" not in text and text.count("_base._ws(ws)") == 1
