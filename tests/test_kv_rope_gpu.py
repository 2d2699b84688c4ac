"""Rotary positions on the GPU: the table and the rotation against 64 bits, every layout, the
gradient against the formula and against differences."""
import math

import numpy as np
import pytest
import torch

from kvcheck import TYPES, UNIT, rope64, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


def _table(gmm, positions, rot, **kw):
    freq = torch.tensor(gmm.rope_frequencies(rot, **kw), dtype=torch.float64, device="cuda")
    table = torch.empty(positions, rot, device="cuda")
    gmm.gmm_rope_table(freq, table)
    return table


@pytest.mark.parametrize("positions,rot,kw", [(1, 2, {}), (1000, 128, {}),
                                              (70001, 64, {"base": 5e5, "factor": 8.0}),
                                              (40000, 96, {"factor": 4.0, "trained": 8192})])
def test_table(gmm, positions, rot, kw):
    table = _table(gmm, positions, rot, **kw).cpu().numpy()
    f = np.array(gmm.rope_frequencies(rot, **kw))
    a = np.arange(positions)[:, None] * f
    # one rounding to fp32 of numbers up to 1, and fp64's own error in the angle
    np.testing.assert_allclose(table, np.concatenate([np.cos(a), np.sin(a)], 1), rtol=0,
                               atol=2.0 ** -25 + 1e-9)


def test_table_scale(gmm):
    freq = torch.tensor([1.0, 0.25], dtype=torch.float64, device="cuda")
    table = torch.empty(3, 4, device="cuda")
    gmm.gmm_rope_table(freq, table, scale=1.5)
    a = np.arange(3)[:, None] * np.array([1.0, 0.25])
    np.testing.assert_allclose(table.cpu().numpy(), 1.5 * np.concatenate([np.cos(a), np.sin(a)], 1),
                               rtol=2.0 ** -23, atol=1e-9)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("tokens,heads,d,rot", [(1, 1, 16, 16), (5, 3, 128, 128), (3, 2, 80, 32),
                                                (4, 5, 33, 10), (2, 40, 256, 96), (7, 1, 6, 2),
                                                (300, 2, 64, 64), (2, 3, 128, 44)])
def test_rotation(gmm, dtype, interleaved, inverse, tokens, heads, d, rot):
    print(f"rope {dtype} {interleaved} {inverse} {tokens} {heads} {d} {rot}", flush=True)
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(d + rot)
    x = torch.randn(tokens, heads, d, generator=g).to(dt)
    pos = torch.randint(0, 500, (tokens,), generator=g).to(torch.int32)
    if tokens > 2:
        pos[1] = -1
    table = _table(gmm, 500, rot)
    ref = rope64(x, pos, table.cpu(), interleaved, inverse)
    # two products and a sum in fp32 of numbers a, b, and one rounding to the type
    mag = x.double().abs().max()
    tol = UNIT[dt] * ref.abs() + 4 * 2.0 ** -24 * mag + (2.0 ** -25 if dt == torch.float16 else 0)
    for xin in (x.cuda(), strided(x), x.cuda().transpose(0, 1).contiguous().transpose(0, 1)):
        out = torch.empty(tokens, heads, d, dtype=dt, device="cuda")
        gmm.gmm_rope(xin, pos.cuda(), table, out, interleaved=interleaved, inverse=inverse)
        assert bool(((out.cpu().double() - ref).abs() <= tol).all())
        assert torch.equal(out.cpu()[..., rot:], x[..., rot:])
        gmm.gmm_rope(xin, pos.cuda(), table, xin, interleaved=interleaved, inverse=inverse)
        assert torch.equal(xin, out)                       # in place: the same


def test_addresses_and_strides_that_allow_no_wide_access(gmm):
    g = torch.Generator().manual_seed(2)
    base = torch.randn(9 * 4 * 65 + 1, generator=g).to(torch.bfloat16).cuda()
    x = base[1:].view(9, 4, 65)[:, :, :64]
    pos = torch.arange(9, dtype=torch.int32)
    table = _table(gmm, 9, 64)
    out = torch.empty(9, 4, 64, dtype=torch.bfloat16, device="cuda")
    want = torch.empty_like(out)
    gmm.gmm_rope(x, pos.cuda(), table, out)
    gmm.gmm_rope(x.contiguous(), pos.cuda(), table, want)
    assert torch.equal(out, want)


def test_positions_past_the_table_give_nan(gmm):
    x = torch.ones(3, 2, 32, dtype=torch.float32, device="cuda")
    table = _table(gmm, 10, 16)
    pos = torch.tensor([9, 10, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    gmm.gmm_rope(x, pos, table, out)
    assert bool(out[0].isfinite().all()) and bool(out[1:, :, :16].isnan().all())
    assert bool((out[1:, :, 16:] == 1).all())


def test_no_tokens(gmm):
    x = torch.empty(0, 2, 32, dtype=torch.float32, device="cuda")
    gmm.gmm_rope(x, torch.empty(0, dtype=torch.int32, device="cuda"), _table(gmm, 4, 32), x)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (48, 20)])
def test_gradient_against_the_formula_and_differences(gmm, interleaved, d, rot):
    """L = sum w . R(x): its gradient is R^T w.  L is linear in x, so a difference quotient of any
    step is exact up to rounding."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(4, 3, d, generator=g)
    w = torch.randn(4, 3, d, generator=g)
    pos = torch.tensor([0, 1, 77, 499], dtype=torch.int32)
    table = _table(gmm, 500, rot)
    grad = torch.empty(4, 3, d, device="cuda")
    gmm.gmm_rope(w.cuda(), pos.cuda(), table, grad, interleaved=interleaved, inverse=True)
    ref = rope64(w, pos, table.cpu(), interleaved, True)
    assert float((grad.cpu().double() - ref).abs().max()) <= 8 * 2.0 ** -24 * float(w.abs().max())

    def loss(v):
        out = torch.empty(4, 3, d, device="cuda")
        gmm.gmm_rope(v.cuda(), pos.cuda(), table, out, interleaved=interleaved)
        return (out.cpu().double() * w.double()).sum(2)        # per (token, head)
    for e in (0, 1, rot // 2, rot - 1, d - 1):
        up, dn = x.clone(), x.clone()
        up[..., e] += 1.0
        dn[..., e] -= 1.0
        step = (up[..., e].double() - dn[..., e].double())
        num = (loss(up) - loss(dn)) / step
        # fp32 outputs of size |x| + 1 in a sum with two of them per entry
        tol = 16 * 2.0 ** -24 * float(x.abs().max() + 1) * float(w.abs().max()) * 4
        assert float((num - grad.cpu().double()[..., e]).abs().max()) <= tol


def test_frequencies(gmm):
    f = gmm.rope_frequencies(8, base=10000.0)
    np.testing.assert_allclose(f, [1.0, 0.1, 0.01, 0.001])
    np.testing.assert_allclose(gmm.rope_frequencies(8, factor=4.0), np.array(f) / 4)
    # turns in 2 pi 1000 positions: 1000, 100, 10, 1
    g = gmm.rope_frequencies(8, factor=4.0, trained=2 * math.pi * 1000, slow=5.0, fast=15.0)
    np.testing.assert_allclose(g, [1.0, 0.1, 0.01 * 0.5 + 0.0025 * 0.5, 0.00025])
