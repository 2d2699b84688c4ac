"""gmm_beam_select's definition in 64 bits for logits of any size, and a check whose bounds are those
of the places that are compared."""
import math

import torch

from poolcheck import INF, allowed


def scores(x, score, done=None, eos=-1, mask=None, scale=1.0):
    """l [batch, beams, vocab] in 64 bits, -inf for no continuation.  From the differences to the
    beam's largest logit: products of large logits would cancel, also in 64 bits."""
    x = allowed(x.cpu().double(), None if mask is None else mask.cpu(), x.shape[2])
    s = score.cpu().double()
    top = x.amax(2, keepdim=True)
    bad = ~torch.isfinite(top) | torch.isnan(x).any(2, keepdim=True)
    d = torch.where(bad, -INF, x - top) * scale
    l = torch.where(bad, -INF, s[..., None] + (d - torch.log(torch.exp(d).sum(2, keepdim=True))))
    if done is not None:
        end = torch.full_like(l, -INF)
        end[..., eos] = s
        l = torch.where(done.cpu()[..., None], end, l)
    return torch.where(torch.isfinite(s)[..., None], l, -INF)


def logz_tolerance(l, vocab):
    """Bound of the error of l before it is rounded to fp32, in units of u = 2^-24 that of log Z: the
    exponentials 4 u, their arguments (difference, constant and product, 3 u of |argument|, twice: a
    term of weight w has |argument| log2(1 / w) at most, their mean is log2(vocab) at most), sums 16
    u, a run's factor 2 u.  Sums and products in 64 bits: four roundings of |l| or less."""
    return 2.0 ** -24 * (22 + 4.2 * math.log2(max(vocab, 2))) + 2.0 ** -51 * abs(l)


def check(out, x, score, m, weight=None, done=None, eos=-1, mask=None, scale=1.0):
    """Checks gmm_beam_select's outputs (score, parent, token, done or None): the i-th place's key
    against the i-th largest, within the bounds of these two; words of one beam in the order of their
    logits; every score within its own bound."""
    got_s, got_p, got_t, got_d = (None if t is None else t.cpu() for t in out)
    l = scores(x, score, done, eos, mask, scale)
    batch, beams, vocab = l.shape
    xs = allowed(x.cpu().double(), None if mask is None else mask.cpu(), vocab)
    w = torch.ones(batch, beams, dtype=torch.float64) if weight is None else weight.cpu().double()
    ok = torch.isfinite(w) & (w > 0)
    key = torch.where(ok[..., None] & (l > -INF), torch.where(ok, w, 0.0)[..., None] * l, -INF)
    for b in range(batch):
        best = torch.sort(key[b].reshape(-1), descending=True, stable=True)
        want = min(m, int((best.values > -INF).sum()))
        assert got_p[b].tolist()[want:] == [-1] * (m - want) == got_t[b].tolist()[want:], b
        assert got_s[b].tolist()[want:] == [-INF] * (m - want), b
        seen = {}
        for i in range(want):
            j, v = int(got_p[b, i]) - b * beams, int(got_t[b, i])
            assert 0 <= j < beams and 0 <= v < vocab, (b, i, j, v)
            exact, there = float(l[b, j, v]), int(best.indices[i])
            # the returned score: half a step of its own besides
            tol = logz_tolerance(exact, vocab) + 2.0 ** -24 * abs(exact)
            assert abs(float(got_s[b, i]) - exact) <= tol, (b, i, j, v, float(got_s[b, i]), exact)
            gap = sum(float(w[b, r]) * logz_tolerance(float(l[b, r, c]), vocab)
                      for r, c in ((j, v), (there // vocab, there % vocab)))
            assert abs(float(key[b, j, v]) - float(best.values[i])) <= gap, \
                (b, i, (j, v), (there // vocab, there % vocab))
            seen.setdefault(j, []).append(v)
            fin = done is not None and bool(done[b, j])
            assert got_d is None or bool(got_d[b, i]) == (fin or v == eos), (b, i)
        for j, vs in seen.items():
            if done is not None and bool(done[b, j]):
                assert vs == [eos], (b, j)
            else:
                order = torch.sort(xs[b, j], descending=True, stable=True).indices[:len(vs)]
                assert vs == order.tolist(), (b, j)
        assert got_d is None or not got_d[b, want:].any(), b
