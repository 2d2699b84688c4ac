"""Beam search's selection where a sequence has more runs of 2048 words than are ranked together, or a
beam more than a wave has lanes: 64 results kept from chunk to chunk, ties across chunks, finished
beams and whole chunks without a word."""
import math

import pytest
import torch

from beamexact import check
from test_beam_gpu import TYPES, _select

pytestmark = pytest.mark.gpu
RUN, CHUNK = 2048, 1024


def _inputs(batch, beams, vocab, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(batch, beams, vocab, generator=g) * 3).to(TYPES[dtype])
    return x, -10.0 - 2.0 * torch.rand(batch, beams, generator=g), g


@pytest.mark.parametrize("m", [1, 16, 17, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,beams,vocab", [(1, 32, 131072), (1, 8, 300001), (2, 17, 133121),
                                               (1, 64, 40000)])
def test_more_runs_than_a_chunk(batch, beams, vocab, dtype, m):
    x, s, _ = _inputs(batch, beams, vocab, dtype, seed=vocab + m)
    x, s = x.cuda(), s.cuda()
    check(_select(x, s, m), x, s, m)


@pytest.mark.parametrize("m", [5, 16, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_finished_beams_and_empty_chunks(dtype, m):
    beams, vocab = 12, 250007                      # 123 runs a beam, two chunks
    x, s, g = _inputs(2, beams, vocab, dtype, seed=m)
    eos = vocab - 3                                # in the last run
    done = torch.zeros(2, beams, dtype=torch.bool)
    done[0, 0] = done[0, 9] = done[0, 11] = done[1, 11] = True
    words = (vocab + 31) // 32
    mask = torch.full((2, beams, words), -1, dtype=torch.int32)
    mask[0, 9:] = 0                                # the second chunk: finished beams alone
    mask[1, :8] = 0                                # the first: 8 beams without a word, a part of one
    mask[1, 8, :37 * RUN // 32] = 0
    mask[1, 8, 37 * RUN // 32] = -2 ** 31
    weight = 0.5 + torch.rand(2, beams, generator=g)
    x, s, kw = x.cuda(), s.cuda(), dict(mask=mask.cuda(), done=done.cuda(), eos=eos)
    check(_select(x, s, m, **kw), x, s, m, **kw)
    kw["weight"] = weight.cuda()
    check(_select(x, s, m, **kw), x, s, m, **kw)
    # nothing but finished beams, and nothing at all
    kw = dict(done=torch.ones_like(done).cuda(), eos=eos)
    check(_select(x, s, m, **kw), x, s, m, **kw)
    out = _select(x, torch.full_like(s, -math.inf), m)
    assert (out[1] == -1).all() and (out[2] == -1).all() and (out[0] == -math.inf).all()


@pytest.mark.parametrize("m", [1, 16, 17, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_ties_across_chunks(dtype, m):
    """Equal words in all runs, in each run one, and behind larger ones of a later chunk."""
    beams, vocab = 9, 262145                       # 129 runs a beam, 1161 in all
    s = torch.full((1, beams), -3.0, device="cuda")
    x = torch.ones(1, beams, vocab, dtype=TYPES[dtype], device="cuda")
    out = _select(x, s, m)
    assert out[1][0].tolist() == [0] * m and out[2][0].tolist() == list(range(m))
    x.fill_(-4.0)
    x[..., 77::RUN] = 2.0                          # 128 runs of a beam hold one
    out = _select(x, s, m)
    assert out[1][0].tolist() == [0] * m and out[2][0].tolist() == [77 + RUN * i for i in range(m)]
    # the last beam, in the second chunk, has larger ones as well, in place of two of its words
    x[0, 8, 5 * RUN + 77], x[0, 8, 100 * RUN + 77] = 3.0, 2.5
    x[0, :8, 77] = -4.0                            # and the others one fewer: their sums differ
    out = _select(x, s, m)
    z = [float(torch.logsumexp(x[0, j].double(), 0)) for j in range(beams)]
    cand = [(-(float(x[0, j, v]) - z[j if j == 8 else 0]), j, v) for j in range(beams)
            for v in range(77, vocab, RUN) if float(x[0, j, v]) > 0]
    want = sorted(cand)[:m]
    assert list(zip(out[1][0].tolist(), out[2][0].tolist())) == [c[1:] for c in want]


@pytest.mark.parametrize("m", [3, 64])
def test_runs_beyond_several_chunks(m):
    """A chunk brings nothing, and a later one does: 3 beams of 1100 runs."""
    vocab = 1100 * RUN - 5
    x, s, _ = _inputs(1, 3, vocab, "bf16", seed=2)
    x[0, 0, :] = -20.0
    x[0, 0, 3:3 + m] = 9.0
    x[0, 1, :] = -20.0
    x[0, 2, vocab - 1 - m:] = 20.0
    x, s = x.cuda(), s.cuda()
    check(_select(x, s, m), x, s, m)
