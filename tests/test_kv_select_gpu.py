"""Page selection on the GPU against its definition in whole numbers: equal, entry by entry."""
import pytest
import torch

from kvcheck import Batch, select_exact, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


def _select(gmm, bt, box, scale, m, keep_first=1, keep_last=1, q=None):
    cache = gmm.KVCache(bt.k.cuda(), bt.v.cuda(), box.cuda(), scale.cuda())
    idx = torch.full((bt.rows, bt.hk, m), 77, dtype=torch.int32, device="cuda")
    ws = gmm.kv_workspace(cache, bt.rows, bt.hq, len(bt.seqs), bt.width)
    ws.fill_(255)
    gmm.gmm_kv_select(cache, strided(bt.q if q is None else q), bt.cu.cuda(), bt.total.cuda(),
                      bt.pages.cuda(), idx, ws, keep_first=keep_first, keep_last=keep_last)
    return idx.cpu()


CASES = [
    ([(1, 1)], 1, 1, 16, 32, 1, 0, 1),
    ([(1, 3000), (1, 100), (1, 2049), (0, 64), (1, 32)], 8, 2, 128, 32, 7, 1, 1),
    ([(3, 2500), (9, 700), (1, 65)], 6, 2, 96, 64, 5, 1, 2),
    ([(5, 1700)], 7, 1, 256, 32, 16, 2, 3),
    ([(2, 3000)], 40, 1, 64, 32, 20, 0, 1),
    ([(40, 2000)], 3, 3, 80, 32, 9, 1, 1),
    ([(1, 9000), (1, 20)], 16, 1, 48, 32, 100, 1, 1),
    ([(1, 300)] * 9, 64, 1, 32, 32, 3, 1, 1),
    ([(4, 40000)], 2, 1, 16, 32, 64, 1, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_selection(gmm, dtype, case):
    seqs, hq, hk, d, page, m, first, last = CASES[case]
    print(f"select {dtype} {CASES[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 20)
    box, scale = bt.boxes()
    got = _select(gmm, bt, box, scale, m, first, last)
    assert torch.equal(got, select_exact(bt, box, scale, m, first, last))


def test_ties_go_to_the_lower_page(gmm):
    bt = Batch([(1, 3200)], 2, 1, 32, 32, "bf16")
    box = torch.ones(bt.npages, 1, 2, 32, dtype=torch.int8)
    scale = torch.ones(bt.npages, 1)
    got = _select(gmm, bt, box, scale, 6)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 99]
    zero = torch.zeros_like(bt.q)                       # a query without a direction: all scores 0
    got = _select(gmm, bt, *bt.boxes(), 4, q=zero)
    assert got[0, 0].tolist() == [0, 1, 2, 99]


def test_scores_below_zero_and_minus_zero(gmm):
    bt = Batch([(1, 320)], 1, 1, 32, 32, "bf16")
    box = torch.zeros(bt.npages, 1, 2, 32, dtype=torch.int8)
    scale = torch.ones(bt.npages, 1)
    q = torch.ones(1, 1, 32, dtype=bt.dt)
    for lp in range(10):
        box[bt.pages[0, lp]] = -lp if lp < 8 else 0     # page 8: dot 0 times a unit of 0 below
    scale[bt.pages[0, 8]] = 0.0
    got = _select(gmm, bt, box, scale, 4, 0, 1, q=q)
    assert torch.equal(got, select_exact(bt, box, scale, 4, 0, 1, q=q))
    assert got[0, 0].tolist() == [0, 1, 8, 9]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_pages_and_queries_without_bounds(gmm, bad):
    bt = Batch([(2, 1600), (1, 700)], 4, 2, 32, 32, "bf16")
    box, scale = bt.boxes()
    for lp in (5, 17):
        scale[bt.pages[0, lp], 1] = float("inf")
        box[bt.pages[0, lp], 1] = 0
    got = _select(gmm, bt, box, scale, 6)
    assert torch.equal(got, select_exact(bt, box, scale, 6))
    assert 5 in got[0, 1].tolist() and 17 in got[0, 1].tolist()
    q = bt.q.clone()
    q[0, 3, 4] = bad
    got = _select(gmm, bt, box, scale, 6, q=q)
    assert torch.equal(got, select_exact(bt, box, scale, 6, q=q))


def test_a_table_narrower_than_the_sequence_and_no_keys(gmm):
    bt = Batch([(3, 1000), (2, 2)], 2, 1, 64, 32, "bf16")
    box, scale = bt.boxes()
    bt.width = 9
    bt.pages = bt.pages[:, :9].contiguous()
    assert torch.equal(_select(gmm, bt, box, scale, 4), select_exact(bt, box, scale, 4))
    # more new tokens than keys: a row before slot 0 sees no page
    bt.total[1] = 1
    bt.row_slot[3], bt.row_slot[4] = -1, 0
    got = _select(gmm, bt, box, scale, 4)
    assert got[3].tolist() == [[-1] * 4] and got[4].tolist() == [[0, -1, -1, -1]]


def test_bound_holds(gmm):
    """Without the rounding of the query, the score of a page bounds every inner product in it."""
    bt = Batch([(1, 640)], 1, 1, 64, 32, "bf16", seed=3)
    box, scale = bt.boxes()
    q = torch.randint(-127, 128, (1, 1, 64)).to(torch.bfloat16)
    q[0, 0, 0] = 127.0                      # unit 1: exact in 8 bits
    for lp in range(20):
        ph = int(bt.pages[0, lp])
        hi, lo = box[ph, 0].double() * float(scale[ph, 0])
        qq = q[0, 0].double()
        bound = (qq.clamp(min=0) * hi + qq.clamp(max=0) * lo).sum()
        top = (bt.keys[0][0, lp * 32:(lp + 1) * 32].double() @ qq).max()
        assert float(bound) >= float(top) - 1e-3
