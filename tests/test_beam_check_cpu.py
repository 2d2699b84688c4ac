"""The check of beam search's selection itself: results with a mistake in them are refused, also where
some words of the sequence are far below the others."""
import pytest
import torch

from beamexact import check, scores

M = 4


def _case(low):
    x = torch.randn(1, 3, 500, generator=torch.Generator().manual_seed(4)) * 3
    x[0, 0, 100:] = low
    x[0, 0, 77] = 9.0
    return x, torch.tensor([[-1.0, -1.5, -2.0]])


def _right(x, s):
    l = scores(x, s)[0]
    best = torch.sort(l.reshape(-1), descending=True, stable=True)
    at = best.indices[:M]
    return (best.values[:M].float()[None], (at // 500).int()[None], (at % 500).int()[None], None)


@pytest.mark.parametrize("low", [-50.0, -1e10, -1e30, -3e38])
def test_mistakes_are_found(low):
    x, s = _case(low)
    check(_right(x, s), x, s, M)
    lost = torch.tensor([[-float("inf"), -1.5, -2.0]])            # beam 0 is lost altogether
    with pytest.raises(AssertionError):
        check(_right(x, lost), x, s, M)
    score, parent, token, _ = _right(x, s)
    for i in range(M):
        off = score.clone()
        off[0, i] += 2e-5
        with pytest.raises(AssertionError):
            check((off, parent, token, None), x, s, M)
        other = token.clone()
        other[0, i] = (other[0, i] + 1) % 500
        with pytest.raises(AssertionError):
            check((score, parent, other, None), x, s, M)
    order = [1, 0, 2, 3]
    with pytest.raises(AssertionError):
        check((score[:, order], parent[:, order], token[:, order], None), x, s, M)
    fewer = [t.clone() for t in (score, parent, token)]
    for t, v in zip(fewer, (-float("inf"), -1, -1)):
        t[0, M - 1] = v
    with pytest.raises(AssertionError):
        check((*fewer, None), x, s, M)
