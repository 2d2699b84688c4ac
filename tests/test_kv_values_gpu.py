"""Attention over values and scores at the ends of their types' ranges, against 64 bits."""
import math

import pytest
import torch

from kvcheck import Batch, attend64
from test_kv_attend_gpu import _attend, _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


# up to 64 rows a head, and tiles of 128 and 256 rows, one range of keys and several
HUGE = [
    ([(1, 300)], 4, 2, 32, 32),
    ([(9, 900)], 4, 1, 128, 64),
    ([(100, 260)], 1, 1, 32, 32),
    ([(140, 2100)], 2, 1, 128, 64),
    ([(300, 700), (3, 70)], 2, 2, 96, 64),
    ([(80, 400)], 2, 2, 240, 32),
]


@pytest.mark.parametrize("dtype,size,scale", [("bf16", 1e30, 0.25), ("bf16", 1e9, 1.0),
                                              ("f16", 2000.0, 1e7), ("f16", 2000.0, -3e4)])
@pytest.mark.parametrize("case", range(len(HUGE)))
def test_scores_of_every_size(gmm, dtype, size, scale, case):
    """Where a row's largest score leads by more than fp32's spacing there, it takes all the
    weight: neighbouring numbers at 1e10 lie 1024 apart."""
    seqs, hq, hk, d, page = HUGE[case]
    print(f"huge {dtype} {size} {scale} {HUGE[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 300)
    q = (bt.q.float() * size).to(bt.dt)
    out, lse = _attend(gmm, bt, q=q, scale=scale)
    clear = 0
    for r in range(bt.rows):
        b, slot = bt.row_seq[r], bt.row_slot[r]
        for j in range(hq):
            h = j // (hq // hk)
            k, v = bt.keys[b][h, :slot + 1].double(), bt.vals[b][h, :slot + 1].double()
            s = (k @ q[r, j].double()) * scale
            # a score's error: d fp32 products and additions, and the scaling
            mag = float((k.abs() @ q[r, j].double().abs()).max()) * abs(scale)
            err = (d + 8) * 2.0 ** -24 * mag
            top = s.sort(descending=True).values
            assert abs(float(lse[r, j] - top[0])) <= err + 2.0 ** -21 * abs(float(top[0])) + 8
            if slot > 0 and float(top[0] - top[1]) <= 2 * err + 40:      # e^-40 of weight
                continue
            clear += 1
            assert torch.equal(out[r, j], v[int(s.argmax())]), (r, j)
    assert clear >= 0.9 * bt.rows * hq


def _with_keys(bt, b, keys):
    """bt with sequence b's keys [heads, t, d] replaced."""
    bt.keys[b] = keys.to(bt.dt)
    for s in range(keys.shape[1]):
        bt.k[int(bt.pages[b, s // bt.page]), :, s % bt.page] = bt.keys[b][:, s]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("offset", [3000.0, -3000.0])
@pytest.mark.parametrize("ramp", [False, True])
@pytest.mark.parametrize("seqs,d", [([(3, 500)], 128), ([(140, 900)], 128), ([(100, 300)], 32),
                                    ([(70, 300)], 208)])
def test_large_scores_that_differ_by_little(gmm, dtype, offset, ramp, seqs, d):
    """All of a row's scores are near the offset, or grow to it along the sequence."""
    print(f"offset {dtype} {offset} {ramp} {seqs} {d}", flush=True)
    bt = Batch(seqs, 1, 1, d, 64, dtype, seed=d + 17)
    g = torch.Generator().manual_seed(d)
    n, t = seqs[0]
    keys = 0.25 * torch.randn(1, t, d, generator=g)
    # one dimension carries the offset, its factors powers of two and thus exact
    keys[:, :, 0] = 64.0
    if ramp:
        keys[:, :, 0] = 64.0 * torch.linspace(0.01, 1.0, t)
    q = torch.randn(n, 1, d, generator=g)
    q[:, :, 0] = 2.0 if offset > 0 else -2.0
    _with_keys(bt, 0, keys)
    q = q.to(bt.dt)
    scale = abs(offset) / 128.0
    _check(bt, _attend(gmm, bt, q=q, scale=scale), attend64(bt, scale, q=q))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("seqs,hq,d", [([(1, 60000)], 2, 64), ([(8, 9000)], 1, 64), ([(100, 8300)], 1, 64),
                                       ([(200, 9000)], 1, 128), ([(1, 9000)], 64, 192)])
def test_many_small_weights_under_one_large_one(gmm, dtype, seqs, hq, d):
    """Weights of e^-18.25, each below the smallest number of fp16, that the row's sum keeps and its
    result has to keep as well."""
    print(f"small weights {dtype} {seqs} {hq} {d}", flush=True)
    bt = Batch(seqs, hq, 1, d, 64, dtype, seed=3)
    n, t = seqs[0]
    keys = torch.zeros(1, t, d)
    keys[:, 1:, 0] = -18.25
    _with_keys(bt, 0, keys)
    g = torch.Generator().manual_seed(4)
    bt.vals[0] = (2.0 + torch.randn(1, t, d, generator=g)).to(bt.dt)
    bt.vals[0][:, 0] = 0.0
    for s in range(t):
        bt.v[int(bt.pages[0, s // 64]), :, :, s % 64] = bt.vals[0][:, s]
    q = torch.zeros(n, hq, d, dtype=bt.dt)
    q[:, :, 0] = 8.0
    out, lse = _attend(gmm, bt, q=q, scale=0.125)
    w, v = math.exp(-18.25), bt.vals[0][0].double()
    many = n * hq > 64
    for i in range(n):
        held = t - n + i + 1
        z = 1 + (held - 1) * w
        o = w * v[1:held].sum(0) / z
        u = 2.0 ** -11 if dtype == "f16" else 2.0 ** -8
        # one rounding of the result; of a weight, exact to its square where the rest is added; a
        # fp32 exponential of -26; for fp16 half the spacing of its smallest weights
        tol = u * o.abs() + (u if many else u * u) * w * v[1:held].abs().sum(0) / z + 1e-5 * o.abs()
        if dtype == "f16":
            tol += held * (2.0 ** -32 if many else 2.0 ** -40) * v.abs().max() + 2.0 ** -25
        for j in range(hq):
            assert bool(((out[i, j] - o).abs() <= tol).all()), float(((out[i, j] - o).abs() - tol).max())
            assert abs(float(lse[i, j]) - math.log(z)) <= 2.0 ** -20
