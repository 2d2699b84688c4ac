"""Page selection over tables with entries out of range: they hold no key and take no place."""
import numpy as np
import pytest
import torch

from kvcheck import Batch
from test_kv_paths_gpu import _Boxes
from test_kv_select_gpu import _select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


def select_held(bt, box, scale, m, keep_first, keep_last):
    """The definition, in whole numbers, over the entries that are pages of the cache."""
    q, grp = bt.q.float().numpy(), bt.hq // bt.hk
    unit = np.abs(q).max(2).astype(np.float32) * (np.float32(1) / np.float32(127))
    q8 = np.rint(q / unit[..., None]).astype(np.int64)
    bx, sc = box.numpy().astype(np.int64), scale.numpy()
    out = np.full((bt.rows, bt.hk, m), -1, np.int32)
    for r in range(bt.rows):
        nv = min(bt.row_slot[r] // bt.page + 1, bt.width)
        ph = bt.pages[bt.row_seq[r], :nv].numpy()
        held = [p for p in range(nv) if 0 <= ph[p] < bt.npages]
        for h in range(bt.hk):
            rank = {}
            for p in held:
                u = []
                for j in range(h * grp, (h + 1) * grp):
                    dot = (np.maximum(q8[r, j], 0) * bx[ph[p], h, 0] +
                           np.minimum(q8[r, j], 0) * bx[ph[p], h, 1]).sum()
                    u.append(np.float32(unit[r, j] * sc[ph[p], h]) * np.float32(dot))
                rank[p] = (p < keep_first or p >= nv - keep_last, max(u))
            best = sorted(held, key=lambda p: (not rank[p][0], -rank[p][1], p))[:m]
            out[r, h, :len(best)] = sorted(best)
    return torch.from_numpy(out)


def _punch(bt, b, entries):
    """Entries of sequence b's table are set to numbers below and above the cache's pages."""
    for i, p in enumerate(entries):
        bt.pages[b, p] = (-1, bt.npages, -2 ** 31, 2 ** 31 - 1, bt.npages + 7)[i % 5]


def _largest(bt, box, scale):
    """Physical page 0, which no sequence need hold, gets the largest box of all."""
    box[0, :, 0], box[0, :, 1] = 127, -127
    scale[0] = 100.0


@pytest.mark.parametrize("m,first,last", [(4, 1, 1), (3, 0, 1), (7, 2, 3), (12, 1, 1), (30, 1, 1),
                                          (100, 0, 1)])
@pytest.mark.parametrize("holes", [[3], [0, 1, 2, 5, 9], [12, 13], [0, 24], list(range(1, 24))])
def test_entries_out_of_range_take_no_place(gmm, m, first, last, holes):
    bt = Batch([(3, 800), (1, 800), (2, 100)], 4, 2, 64, 32, "bf16", seed=m)
    box, scale = bt.boxes()
    _largest(bt, box, scale)
    _punch(bt, 0, holes)
    _punch(bt, 1, [p for p in (0, 7, 24) if p not in holes])
    got = _select(gmm, bt, box, scale, m, first, last)
    assert torch.equal(got, select_held(bt, box, scale, m, first, last))


# every kernel of the ranking, more and fewer pages left than asked for
@pytest.mark.parametrize("pages", [400, 2000, 9000, 20000])
@pytest.mark.parametrize("left", [25, 26, 27, 300])
def test_tables_that_are_mostly_empty(gmm, pages, left):
    print(f"select {pages} {left}", flush=True)
    bt = _Boxes(pages, 2, 2, 1, 16, seed=pages + left)
    _largest(bt, bt.box, bt.unit)
    g = torch.Generator().manual_seed(left)
    _punch(bt, 0, torch.randperm(pages, generator=g)[left:].tolist())
    for m in (26, 60):
        got = _select(gmm, bt, bt.box, bt.unit, m, 1, 1)
        assert torch.equal(got, select_held(bt, bt.box, bt.unit, m, 1, 1))


def test_a_table_without_a_page(gmm):
    bt = Batch([(2, 300), (1, 90)], 2, 1, 64, 32, "bf16")
    box, scale = bt.boxes()
    _punch(bt, 0, range(bt.width))
    got = _select(gmm, bt, box, scale, 5)
    assert bool((got[:2] == -1).all())
    assert got[2, 0].tolist() == [0, 1, 2, -1, -1]
    assert bool((_select(gmm, bt, box, scale, 20)[:2] == -1).all())


@pytest.mark.parametrize("d", [16, 96, 128, 240])
def test_query_rows_of_any_alignment(gmm, d):
    """Rows that allow 16-byte loads and rows that do not: by address, by token and by head stride."""
    bt = Batch([(5, 900), (1, 70)], 6, 2, d, 32, "bf16", seed=d)
    box, scale = bt.boxes()
    cache = gmm.KVCache(bt.k.cuda(), bt.v.cuda(), box.cuda(), scale.cuda())
    ws = gmm.kv_workspace(cache, bt.rows, 6, 2, bt.width)
    args = bt.cu.cuda(), bt.total.cuda(), bt.pages.cuda()
    want = select_held(bt, box, scale, 6, 1, 1)
    q = bt.q.cuda()

    def view(offset, token, head):
        flat = torch.zeros(offset + bt.rows * token, dtype=bt.dt, device="cuda")
        x = flat.as_strided((bt.rows, 6, d), (token, head, 1), offset)
        x.copy_(q)
        return x
    for x in (q, view(0, 6 * d, d), view(8, 6 * d + 8, d), view(1, 6 * d, d), view(0, 6 * d + 3, d),
              view(0, 6 * d + 24, d + 4), view(0, 6 * d + 48, d + 8)):
        idx = torch.full((bt.rows, 2, 6), 77, dtype=torch.int32, device="cuda")
        gmm.gmm_kv_select(cache, x, *args, idx, ws)
        assert torch.equal(idx.cpu(), want)
