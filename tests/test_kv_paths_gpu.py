"""The paged cache's kernels that the sizes of the other tests do not reach: every tile of many
query rows, with windows, missing pages and opposite signs; rankings of many pages; and the
clustered-cache example, whose steps run the operators together with the library's k-means."""
import math
import os
import sys

import pytest
import torch

from kvcheck import Batch, attend64, select_exact
from test_kv_attend_gpu import _attend, _check
from test_kv_select_gpu import _select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


# rows of a head: 65 .. 128 (four waves) and more (eight waves from 65 to 128 dimensions)
TILES = [
    ([(100, 260)], 1, 1, 96, 32),
    ([(70, 500), (129, 129)], 2, 1, 96, 64),
    ([(90, 1000)], 1, 1, 128, 32),
    ([(33, 777)], 8, 2, 112, 128),
    ([(260, 260), (5, 70), (0, 3), (300, 900)], 3, 3, 128, 64),
    ([(120, 400)], 2, 2, 176, 32),
    ([(200, 330)], 1, 1, 256, 256),
    ([(128, 128)], 2, 1, 32, 32),
    ([(66, 3000)], 16, 1, 64, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(TILES)))
def test_tiles(gmm, dtype, case):
    seqs, hq, hk, d, page = TILES[case]
    print(f"attend {dtype} {TILES[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 100)
    _check(bt, _attend(gmm, bt), attend64(bt, 1.0 / math.sqrt(d)))


@pytest.mark.parametrize("window", [1, 40, 64, 333])
@pytest.mark.parametrize("case", [0, 1, 3, 4, 5, 8])
def test_tiles_with_a_window(gmm, window, case):
    seqs, hq, hk, d, page = TILES[case]
    print(f"attend window {window} {TILES[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, "f16", seed=case + 120)
    _check(bt, _attend(gmm, bt, window=window), attend64(bt, 1.0 / math.sqrt(d), window))


@pytest.mark.parametrize("factor", [0.0, -0.2, 5.0])
@pytest.mark.parametrize("case", [2, 4, 7])
def test_tiles_scale(gmm, factor, case):
    seqs, hq, hk, d, page = TILES[case]
    bt = Batch(seqs, hq, hk, d, page, "bf16", seed=case + 140)
    _check(bt, _attend(gmm, bt, scale=factor), attend64(bt, factor))


@pytest.mark.parametrize("case", [2, 4, 5])
def test_tiles_leave_out_pages_out_of_range(gmm, case):
    """A page number out of range: the keys of its slots do not exist for any row."""
    seqs, hq, hk, d, page = TILES[case]
    bt = Batch(seqs, hq, hk, d, page, "bf16", seed=case + 160)
    gone = [1, 4]
    sel = torch.full((bt.rows, hk, bt.width), -1, dtype=torch.int32)
    for r in range(bt.rows):
        for p in range(bt.row_slot[r] // page + 1):
            if bt.row_seq[r] != 0 or p not in gone:
                sel[r, :, p] = p
    ref = attend64(bt, 1.0 / math.sqrt(d), sel=sel)
    for i, p in enumerate(gone):
        if p < bt.width:
            bt.pages[0, p] = -7 if i else bt.npages
    _check(bt, _attend(gmm, bt), ref)


def test_tiles_with_rows_before_the_first_key(gmm):
    bt = Batch([(200, 70), (80, 80)], 1, 1, 128, 32, "bf16")
    assert bt.row_slot[0] == -130
    _check(bt, _attend(gmm, bt), attend64(bt, 1.0 / math.sqrt(128)))


def test_tiles_with_rows_before_the_first_key_of_a_long_context(gmm):
    bt = Batch([(200, 70), (80, 80), (2, 1500)], 2, 1, 128, 32, "bf16")
    _check(bt, _attend(gmm, bt), attend64(bt, 1.0 / math.sqrt(128)))


# prompts that are most of their own context (four waves), and the same with longer contexts
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,hq,hk,d,page", [
    ([(300, 300)], 1, 1, 128, 64),
    ([(500, 640), (0, 0), (411, 411)], 4, 2, 128, 32),
    ([(129, 129), (257, 258)], 3, 3, 96, 128),
    ([(300, 601)], 1, 1, 128, 64),
    ([(500, 640), (0, 0), (411, 1411)], 4, 2, 128, 32),
    ([(2050, 2050)], 1, 1, 80, 256),
])
def test_prompts(gmm, dtype, seqs, hq, hk, d, page):
    print(f"attend {dtype} {seqs} {hq} {hk} {d} {page}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=len(seqs) + d)
    _check(bt, _attend(gmm, bt), attend64(bt, 1.0 / math.sqrt(d)))


def test_tiles_move_their_maximum(gmm):
    """Keys whose scores grow along the sequence: every step moves the running maximum."""
    bt = Batch([(140, 900)], 1, 1, 128, 64, "bf16", seed=9)
    ramp = torch.linspace(0.1, 6.0, 900)[None, :, None]
    base = torch.randn(1, 1, 128, generator=torch.Generator().manual_seed(1))
    bt.keys[0] = (base * ramp).to(bt.dt)
    for s in range(900):
        bt.k[int(bt.pages[0, s // 64]), :, s % 64] = bt.keys[0][:, s]
    q = (base[0] + 0.1 * torch.randn(140, 1, 128, generator=torch.Generator().manual_seed(2)))
    q = q.to(bt.dt)
    _check(bt, _attend(gmm, bt, q=q, scale=0.3), attend64(bt, 0.3, q=q))


def test_one_chunk_equals_single_tokens(gmm):
    """A prompt attended in one call and token by token differ by roundings only."""
    bt = Batch([(90, 90)], 4, 2, 64, 32, "bf16", seed=21)
    ref = attend64(bt, 0.125)
    whole = _attend(gmm, bt)
    _check(bt, whole, ref)
    for t in (0, 31, 32, 89):
        one = Batch([(1, t + 1)], 4, 2, 64, 32, "bf16")
        one.k, one.v, one.pages, one.width = bt.k, bt.v, bt.pages, bt.width
        out, lse = _attend(gmm, one, q=bt.q[t:t + 1])
        assert bool(((out[0] - ref[0][t]).abs() <= ref[2][t]).all())
        assert bool(((lse[0] - ref[1][t]).abs() <= ref[3][t]).all())


class _Boxes(Batch):
    """Random boxes of many pages; the keys themselves are not read by the selection."""

    def __init__(self, pages, new, hq, hk, d, seed):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.hq, self.hk, self.d, self.page = [(new, pages * 32)], hq, hk, d, 32
        self.dt, self.npages, self.width = torch.bfloat16, pages + 2, pages
        self.k = torch.zeros(self.npages, hk, 32, d, dtype=self.dt)
        self.v = torch.zeros(self.npages, hk, d, 32, dtype=self.dt)
        self.pages = torch.randperm(self.npages, generator=g)[:pages].to(torch.int32)[None]
        self.rows = new
        self.cu = torch.tensor([0, new], dtype=torch.int32)
        self.total = torch.tensor([pages * 32], dtype=torch.int32)
        self.q = torch.randn(new, hq, d, generator=g).to(self.dt)
        self.row_seq, self.row_slot = [0] * new, [pages * 32 - new + i for i in range(new)]
        hi = torch.randint(-20, 128, (self.npages, hk, d), generator=g)
        lo = torch.minimum(hi, torch.randint(-127, 40, (self.npages, hk, d), generator=g))
        self.box = torch.stack([hi, lo], 2).to(torch.int8)
        # few different units: many pages with equal scores
        self.unit = torch.randint(1, 4, (self.npages, hk), generator=g).float() / 64


@pytest.mark.parametrize("pages,m", [(500, 33), (513, 1 + 2), (2049, 64), (16384, 500),
                                     (16385, 4096), (40000, 100)])
def test_rankings_of_many_pages(gmm, pages, m):
    print(f"select {pages} {m}", flush=True)
    bt = _Boxes(pages, 3, 2, 1, 16, seed=pages)
    got = _select(gmm, bt, bt.box, bt.unit, m, 2, 1)
    assert torch.equal(got, select_exact(bt, bt.box, bt.unit, m, 2, 1))


def test_rankings_with_few_different_scores(gmm):
    bt = _Boxes(3000, 2, 1, 1, 16, seed=5)
    box = (bt.box > 60).to(torch.int8)
    unit = torch.ones_like(bt.unit)
    q = torch.ones_like(bt.q)
    got = _select(gmm, bt, box, unit, 700, 1, 1, q=q)
    assert torch.equal(got, select_exact(bt, box, unit, 700, 1, 1, q=q))


def test_example(gmm):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                    "examples"))
    try:
        import clustered_cache
    finally:
        sys.path.pop(0)
    res = clustered_cache.run(prompt=8192, steps=4, pages_read=6)
    (mass0, err0), (mass1, err1) = res["prompt order"], res["cluster order"]
    assert 0.0 < mass0 <= 1.0 + 1e-3 and 0.0 < mass1 <= 1.0 + 1e-3
    # pages of alike keys hold more of the mass and leave a smaller error
    assert mass1 > mass0 and err1 < err0
