"""The bound of the tests for few rows tells a second term for the weights' rounding from none."""
import math

import pytest

from kvcheck import Batch
from kvprecise import CASES, attend_precise, attend_rounded_once


# (of fp16, whose own rounding is finer, where the scores' error leaves it visible)
@pytest.mark.parametrize("dtype,case", [("bf16", 0), ("bf16", 1), ("bf16", 4), ("bf16", 5), ("bf16", 7),
                                        ("bf16", 8), ("f16", 1), ("f16", 7), ("f16", 8)])
def test_one_rounding_breaks_the_bound(dtype, case):
    seqs, hq, hk, d, page = CASES[case]
    bt = Batch(seqs, hq, hk, d, page, dtype, seed=case + 500)
    scale = 1.0 / math.sqrt(d)
    o, tol = attend_precise(bt, scale)
    once = attend_rounded_once(bt, scale)
    assert int(((once - o).abs() > tol).sum()) > 10
