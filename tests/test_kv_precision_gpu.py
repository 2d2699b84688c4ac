"""Attention of few rows keeps the rest of the weights' rounding: within a bound that one rounding of
the weights would break (test_kv_precision_cpu)."""
import math

import pytest

from kvcheck import Batch
from kvprecise import CASES, attend_precise
from test_kv_attend_gpu import _attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gmm():
    import paper_2606_10896_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_few_rows(gmm, dtype, case):
    seqs, hq, hk, d, page = CASES[case]
    print(f"precise {dtype} {CASES[case]}", flush=True)
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 500)
    assert -(-bt.rows // len(seqs)) * (hq // hk) <= 64
    o, tol = attend_precise(bt, 1.0 / math.sqrt(d))
    out, _ = _attend(gmm, bt)
    assert bool(((out - o).abs() <= tol).all()), float(((out - o).abs() - tol).max())
