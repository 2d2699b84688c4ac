"""Values that are NaN or infinite reach the rows that see their key, in their dimension, and no
other: not the rows of earlier tokens of the same call, not rows whose window has moved on."""
import math

import pytest
import torch

from kvcheck import Batch, attend64
from test_kv_attend_gpu import _attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


# new tokens and keys, query heads, cache heads, width, page
CASES = [
    ([(1, 200), (1, 33)], 4, 2, 64, 32),
    ([(1, 1500)], 8, 2, 128, 64),
    ([(6, 400), (3, 3), (2, 90)], 4, 2, 128, 32),
    ([(9, 1000)], 4, 1, 96, 64),
    ([(14, 500), (4, 40)], 4, 1, 208, 32),
    ([(60, 60), (20, 700)], 3, 3, 48, 32),
    ([(100, 260), (40, 140)], 2, 1, 64, 32),
    ([(90, 1300)], 4, 2, 64, 64),
    ([(140, 900)], 1, 1, 128, 64),
    ([(300, 420), (5, 70), (0, 3)], 2, 2, 112, 128),
    ([(90, 400)], 1, 1, 240, 32),
    ([(150, 150), (70, 70)], 2, 2, 128, 64),
]


def _spoil(bt, window, seed, kinds):
    """Some values of every sequence become NaN or infinite: among the last keys, where the rows of a
    call differ, at its windows' first keys, and anywhere.  Returns {(sequence, head, key, dim): value}."""
    g = torch.Generator().manual_seed(seed)
    pick = lambda n: int(torch.randint(n, (1,), generator=g))
    spots = {}
    for b, (n, t) in enumerate(bt.seqs):
        if t == 0:
            continue
        near = [t - 1, t - 2, t - max(n, 1), t - n // 2 - 1, pick(t), max(0, t - 1 - pick(40))]
        if window:
            near += [t - n - window, t - n - window + 1, t - window - n // 2, t - window]
        for key in near:
            if not 0 <= key < t:
                continue
            h, dim = pick(bt.hk), pick(bt.d)
            x = kinds[pick(len(kinds))]
            bt.v[int(bt.pages[b, key // bt.page]), h, dim, key % bt.page] = x
            bt.vals[b][h, key, dim] = 0.0
            spots[b, h, key, dim] = x              # what was written last
    return spots


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kinds", [[math.nan], [math.inf], [math.nan, math.inf, -math.inf]])
@pytest.mark.parametrize("window", [0, 1, 50, 130])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_only_rows_that_see_the_key(gmm, dtype, kinds, window, case):
    seqs, hq, hk, d, page = CASES[case]
    print(f"not finite {dtype} {kinds} {window} {CASES[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 400)
    spots = _spoil(bt, window, case, kinds)
    out, lse = _attend(gmm, bt, window=window)
    o, l, tol, ltol = attend64(bt, 1.0 / math.sqrt(d), window)       # of the finite values
    hit = torch.zeros(bt.rows, hq, d)
    for (b, h, key, dim), x in spots.items():
        for r in range(bt.rows):
            s = bt.row_slot[r]
            if bt.row_seq[r] == b and key <= s and not (window and key <= s - window):
                hit[r, h * (hq // hk):(h + 1) * (hq // hk), dim] += x
    seen = ~hit.isfinite()
    assert bool((~out.isfinite() == seen).all())
    assert bool(((out - o).abs() <= tol)[~seen].all())
    assert bool((out[seen].isnan() == hit[seen].isnan()).all())
    assert bool((out[hit == math.inf] == math.inf).all())
    assert bool((out[hit == -math.inf] == -math.inf).all())
    assert bool(((lse - l).abs() <= ltol)[l > -math.inf].all())


@pytest.mark.parametrize("seqs,hq,d", [([(1, 700)], 4, 64), ([(3, 2000)], 4, 128), ([(100, 900)], 1, 128)])
def test_a_value_that_every_row_sees(gmm, seqs, hq, d):
    """In a range of keys of its own, also where its weight is too small for fp32."""
    bt = Batch(seqs, hq, 1, d, 32, "bf16", seed=5)
    bt.v[int(bt.pages[0, 2]), 0, 7, 9] = math.inf
    for scale in (0.1, 60.0):
        out, _ = _attend(gmm, bt, scale=scale)
        assert bool((~out[:, :, 7].isfinite()).all())
        assert bool(out[:, :, :7].isfinite().all()) and bool(out[:, :, 8:].isfinite().all())


def test_selected_pages_and_values_after_the_row(gmm):
    """Lists: a token's own page may hold later tokens' values of the same call."""
    bt = Batch([(4, 200)], 4, 2, 64, 32, "bf16", seed=6)
    bt.v[int(bt.pages[0, 6]), 1, 3, 199 % 32] = math.nan       # the last token's own
    bt.vals[0][1, 199, 3] = 0.0
    sel = torch.tensor([[[0, 6, -1], [6, 2, 1]]] * 4, dtype=torch.int32)
    out, _ = _attend(gmm, bt, sel=sel)
    o, _, tol, _ = attend64(bt, 0.125, sel=sel)
    assert bool(((out - o).abs() <= tol)[:3].all())
    assert bool(out[3, 2:, 3].isnan().all())
    out[3, 2:, 3] = o[3, 2:, 3]
    assert bool(((out - o).abs() <= tol)[3].all())


@pytest.mark.parametrize("window", [0, 60])
@pytest.mark.parametrize("x", [math.nan, math.inf])
@pytest.mark.parametrize("case", [2, 4, 5, 7, 9])
def test_every_value_not_finite(gmm, x, window, case):
    seqs, hq, hk, d, page = CASES[case]
    bt = Batch(seqs, hq, hk, d, page, "bf16", seed=case)
    bt.v.fill_(x)
    out, lse = _attend(gmm, bt, window=window)
    seen = torch.tensor(bt.row_slot) >= 0
    assert bool((out[seen].isnan() if x != x else out[seen] == x).all())
    assert bool(lse[seen].isfinite().all())
