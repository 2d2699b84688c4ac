"""Appending to the paged cache on the GPU: what is stored where, the boxes, what is left alone."""
import numpy as np
import pytest
import torch

from kvcheck import TYPES, UNIT, Batch, box_of, rope64, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


def _table(gmm, positions, rot):
    freq = torch.tensor(gmm.rope_frequencies(rot), dtype=torch.float64, device="cuda")
    table = torch.empty(positions, rot, device="cuda")
    gmm.gmm_rope_table(freq, table)
    return table


def _run(gmm, bt, rot, interleaved, pos=None, boxes=True, with_q=True, layout=strided, seed=9):
    """Appends fresh keys and values; returns them with the GPU cache's new state."""
    g = torch.Generator().manual_seed(seed)
    kn = torch.randn(bt.rows, bt.hk, bt.d, generator=g).to(bt.dt)
    vn = torch.randn(bt.rows, bt.hk, bt.d, generator=g).to(bt.dt)
    box = torch.full((bt.npages, bt.hk, 2, bt.d), 55, dtype=torch.int8, device="cuda")
    scale = torch.full((bt.npages, bt.hk), 7.5, device="cuda")
    cache = gmm.KVCache(bt.k.cuda(), bt.v.cuda(), box if boxes else None,
                        scale if boxes else None)
    table = _table(gmm, max([t for _, t in bt.seqs] + [1]), rot) if rot else None
    qo = torch.empty(bt.rows, bt.hq, bt.d, dtype=bt.dt, device="cuda")
    gmm.gmm_kv_append(cache, layout(kn), layout(vn), bt.cu.cuda(), bt.total.cuda(),
                      bt.pages.cuda(), pos=None if pos is None else pos.cuda(), table=table,
                      q=layout(bt.q) if rot and with_q else None,
                      q_out=qo if rot and with_q else None, interleaved=interleaved)
    torch.cuda.synchronize()
    return kn, vn, cache, table, qo


def _check(bt, rot, interleaved, kn, vn, cache, table, qo, pos=None, boxes=True, with_q=True):
    p = torch.tensor(bt.row_slot) if pos is None else pos
    kr = rope64(kn, p, table.cpu(), interleaved) if rot else kn.double()
    # two fp32 products, a sum, one rounding to the type
    mag = 4 * 2.0 ** -24 * float(kn.double().abs().max()) + \
        (2.0 ** -25 if bt.dt == torch.float16 else 0)
    k, v = cache.k.cpu(), cache.v.cpu()
    left_k, left_v = torch.ones(k.shape[0], k.shape[2], dtype=torch.bool), None
    pages = set()
    for r in range(bt.rows):
        s = bt.row_slot[r]
        ph = int(bt.pages[bt.row_seq[r], s // bt.page])
        pages.add((bt.row_seq[r], s // bt.page))
        got = k[ph, :, s % bt.page].double()
        assert bool(((got - kr[r]).abs() <= UNIT[bt.dt] * kr[r].abs() + mag).all()), r
        assert torch.equal(v[ph, :, :, s % bt.page], vn[r])
        left_k[ph, s % bt.page] = False
    # every other slot as it was
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))
    for ph in range(bt.npages):
        keep = left_k[ph]
        assert same(k[ph][:, keep], bt.k[ph][:, keep])
        assert same(v[ph][:, :, keep].contiguous(), bt.v[ph][:, :, keep].contiguous())
    if boxes:
        box, scale = cache.box.cpu(), cache.box_scale.cpu()
        done = torch.zeros(bt.npages, dtype=torch.bool)
        for b, lp in pages:
            ph = int(bt.pages[b, lp])
            filled = min(bt.page, bt.seqs[b][1] - lp * bt.page)
            bx, sc = box_of(k[ph, :, :filled].float().numpy())
            np.testing.assert_array_equal(box[ph].numpy(), bx)
            np.testing.assert_array_equal(scale[ph].numpy(), sc)
            done[ph] = True
        assert bool((box[~done] == 55).all()) and bool((scale[~done] == 7.5).all())
    if rot and with_q:
        qr = rope64(bt.q, p, table.cpu(), interleaved)
        tol = UNIT[bt.dt] * qr.abs() + 4 * 2.0 ** -24 * float(bt.q.double().abs().max()) + \
            (2.0 ** -25 if bt.dt == torch.float16 else 0)
        assert bool(((qo.cpu().double() - qr).abs() <= tol).all())


CASES = [
    ([(1, 1)], 1, 1, 16, 32),
    ([(1, 33), (1, 32), (1, 64), (0, 5), (1, 1)], 4, 2, 128, 32),
    ([(70, 100), (0, 0), (3, 67), (200, 200), (1, 129)], 6, 3, 96, 64),
    ([(5, 300)], 2, 1, 256, 128),
    ([(260, 300)], 2, 2, 64, 256),
    ([(1, 40)] * 70, 2, 1, 48, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append(gmm, dtype, interleaved, case):
    seqs, hq, hk, d, page = CASES[case]
    print(f"append {dtype} {interleaved} {CASES[case][1:]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case)
    for rot in sorted({d, d // 2, 0, 10}):
        res = _run(gmm, bt, rot, interleaved)
        _check(bt, rot, interleaved, *res)


def test_no_boxes_no_queries_and_given_positions(gmm):
    bt = Batch([(40, 90), (1, 7)], 4, 2, 64, 32, "bf16")
    res = _run(gmm, bt, 64, False, boxes=False)
    _check(bt, 64, False, *res, boxes=False)
    res = _run(gmm, bt, 64, False, with_q=False)
    _check(bt, 64, False, *res, with_q=False)
    pos = torch.randperm(41, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    pos[3] = -1
    res = _run(gmm, bt, 64, False, pos=pos)
    _check(bt, 64, False, *res, pos=pos)


def test_rows_that_allow_no_wide_access(gmm):
    def odd(x):
        base = torch.zeros(x.numel() + x.shape[0] * x.shape[1] + 1, dtype=x.dtype, device="cuda")
        view = base[1:].view(x.shape[0], x.shape[1], x.shape[2] + 1)[:, :, :x.shape[2]]
        view.copy_(x)
        return view
    bt = Batch([(40, 90), (1, 7)], 4, 2, 64, 32, "f16")
    res = _run(gmm, bt, 64, True, layout=odd)
    _check(bt, 64, True, *res)


def test_one_token_at_a_time_equals_a_chunk(gmm):
    """The cache and the boxes after 70 single appends are those of one append of 70."""
    d, page = 64, 32
    g = torch.Generator().manual_seed(4)
    kn, vn = (torch.randn(70, 2, d, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    pages = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    table = _table(gmm, 70, d)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    a, b = (gmm.kv_cache(3, 2, page, d) for _ in range(2))
    gmm.gmm_kv_append(a, kn, vn, i32(0, 70), i32(70), pages, table=table)
    for t in range(70):
        gmm.gmm_kv_append(b, kn[t:t + 1], vn[t:t + 1], i32(0, 1), i32(t + 1), pages, table=table)
    for x, y in ((a.k, b.k), (a.v, b.v), (a.box, b.box), (a.box_scale, b.box_scale)):
        assert torch.equal(x, y)


def test_pages_out_of_range_and_slots_beyond_the_table_are_left_out(gmm):
    bt = Batch([(60, 90), (2, 40)], 2, 1, 32, 32, "bf16", spare=2)
    bt.pages[0, 1] = bt.npages            # out of range
    bt.pages[1, 1] = -5
    kn = torch.ones(62, 1, 32, dtype=bt.dt, device="cuda")
    cache = gmm.KVCache(bt.k.cuda(), bt.v.cuda())
    gmm.gmm_kv_append(cache, kn, kn, bt.cu.cuda(), bt.total.cuda(), bt.pages[:, :2].contiguous().cuda())
    k = cache.k.cpu()
    ph = int(bt.pages[0, 0])              # slots 30, 31 are new, the rest as before
    assert bool((k[ph, 0, 30:32] == 1).all())
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert same(k[ph, :, :30], bt.k[ph, :, :30])
    others = [p for p in range(bt.npages) if p != ph]
    assert same(k[others], bt.k[others])
    # fewer keys than new tokens: those before slot 0 are left out
    total = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    gmm.gmm_kv_append(cache, kn, kn, bt.cu.cuda(), total, bt.pages[:, :1].contiguous().cuda())
    assert bool((cache.k.cpu()[ph, 0, 0] == 1).all())
    assert same(cache.k.cpu()[ph, :, 1:30], bt.k[ph, :, 1:30])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_key_that_is_no_number_leaves_a_page_without_bounds(gmm, bad):
    cache = gmm.kv_cache(2, 2, 32, 32)
    kn = torch.randn(40, 2, 32).to(torch.bfloat16)
    kn[3, 1, 7] = bad
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    gmm.gmm_kv_append(cache, kn.cuda(), kn.cuda(), i32(0, 40), i32(40),
                      torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    assert float(cache.box_scale[1, 1]) == float("inf") and bool((cache.box[1, 1] == 0).all())
    assert bool(cache.box_scale[1, 0].isfinite()) and bool(cache.box_scale[0].isfinite().all())


def test_zero_keys(gmm):
    cache = gmm.kv_cache(1, 1, 32, 16)
    z = torch.zeros(3, 1, 16, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache.box.fill_(3)
    gmm.gmm_kv_append(cache, z, z, i32(0, 3), i32(3), torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    assert float(cache.box_scale[0, 0]) == 0.0 and bool((cache.box == 0).all())
