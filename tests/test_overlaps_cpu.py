"""Results that overlap what is read for them, or each other, are refused before anything is
enqueued: other workgroups would read what one of them has written."""
import itertools

import pytest

import paper_2606_10896_amd as gmm
from test_kv_refusals_cpu import BAD, UNSUP, WS, _cache
from test_kv_pool_refusals_cpu import _beam, _compact, _fork

BATCH, BEAMS, M = 2, 4, 3
AT = {"score": 0x910000, "weight": 0x920000, "done": 0x930000, "os": 0x940000, "op": 0x950000,
      "ot": 0x960000, "od": 0x970000}
SIZE = {"score": 32, "weight": 32, "done": 8, "os": 24, "op": 24, "ot": 24, "od": 6}
RESULTS, READ = ("os", "op", "ot", "od"), ("score", "weight", "done")


@pytest.fixture(scope="module")
def lib():
    return gmm.load_library()


def _select(lib, m=M, **kw):
    return _beam(lib, batch=BATCH, beams=BEAMS, m=m, eos=3, **{**AT, **kw})


def _places(a, b):
    """Addresses of `a` at which it shares a byte with `b`, first and last, and the same one."""
    return AT[b] - SIZE[a] + 1, AT[b], AT[b] + SIZE[b] - 1


@pytest.mark.parametrize("out,read", itertools.product(RESULTS, READ))
def test_results_over_scores_weights_and_flags(lib, out, read):
    for at in _places(out, read):
        assert _select(lib, **{out: at}) == BAD, at


@pytest.mark.parametrize("a,b", itertools.permutations(RESULTS, 2))
def test_results_over_each_other(lib, a, b):
    for at in _places(a, b):
        assert _select(lib, **{a: at}) == BAD, at


def test_in_place_with_as_many_results_as_beams(lib):
    """Only scores and weights by scores, flags by flags; the workspace is refused after these."""
    allowed = {("os", "score"), ("os", "weight"), ("od", "done")}
    for out, read in itertools.product(RESULTS, READ):
        if (out, read) in allowed:
            assert _select(lib, m=BEAMS, ws=None, **{out: AT[read]}) == WS, (out, read)
        else:
            assert _select(lib, m=BEAMS, **{out: AT[read]}) == BAD, (out, read)


def test_a_forks_totals_and_tables(lib):
    """New totals [3] and new tables [3, 4], and the counts [10 pages], at addresses of their own but
    for one."""
    at = dict(ref=0x910000, total=0x920000, pages=0x930000, parent=0x940000, nt=0x950000, npg=0x960000)
    size = dict(ref=40, nt=12, npg=48)
    for a, b in itertools.permutations(size, 2):
        for off in (1 - size[a], 0, size[b] - 1):
            assert _fork(lib, _cache(), **{**at, a: at[b] + off}) == BAD, (a, b, off)


def test_compacting_refuses_tables_past_a_launch(lib):
    rows = 65536
    assert _compact(lib, _cache(), batch=rows, width=1 << 16, stride=1 << 16, ws=None) == WS
    for heads in (2, 1):                               # large and small pages
        cache = _cache(heads=heads, page=32, d=64)
        assert _compact(lib, cache, batch=rows, width=1 << 16, stride=1 << 16) == UNSUP
