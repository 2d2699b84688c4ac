"""Plain forms of the page pool's calls and of beam search's selection, for the tests: the
bookkeeping entry by entry on the host, the scores in 64 bits."""
import math

import torch

INF = math.inf


def pages_of(t, page):
    return max(0, -(-t // page))


class Pool:
    """Counts and tables as lists; the cache's pages are stood for by their history: `data[p]` is
    what page p holds."""

    def __init__(self, pages, page):
        self.page, self.ref, self.data = page, [0] * pages, [("new", p) for p in range(pages)]

    def ok(self, p):
        return 0 <= p < len(self.ref)

    def count(self, p, by):
        if self.ok(p):
            self.ref[p] += by

    def fork(self, total, pages, width, parent, out_width, keep=None, release=True):
        nt, npg = [], []
        for i, p in enumerate(parent):
            t, row = 0, []
            if 0 <= p < len(total):
                t = max(total[p], 0)
                if keep is not None:
                    t = min(t, max(keep[i], 0))
                row = list(pages[p][:min(pages_of(t, self.page), width)])
            for q in row:
                self.count(q, 1)
            nt.append(t)
            npg.append(row + [-1] * (out_width - len(row)))
        if release:
            for t, row in zip(total, pages):
                for q in row[:min(pages_of(t, self.page), width)]:
                    self.count(q, -1)
        return nt, npg

    def grow(self, held, total, pages, width):
        """The rows' entries change in place; returns the number of missing pages."""
        page, need, writers = self.page, [], {}
        for r, (h, t) in enumerate(zip(held, total)):
            if h > 0 and t > h and h % page and h // page < width:
                p = pages[r][h // page]
                if self.ok(p) and self.ref[p] > 1:
                    writers.setdefault(p, []).append(r)
        copies = {r: p for p, rows in writers.items()
                  for i, r in enumerate(rows) if i > 0 or self.ref[p] > len(rows)}
        for r, (h, t) in enumerate(zip(held, total)):
            if r in copies:
                need.append((r, h // page, copies[r]))
            need += [(r, e, None) for e in range(pages_of(h, page), min(pages_of(t, page), width))]
        free = [p for p, c in enumerate(self.ref) if c <= 0]
        if len(need) > len(free):
            return len(need) - len(free)
        for (r, e, src), p in zip(need, free):
            if src is not None:
                self.ref[src] -= 1
                self.data[p] = self.data[src]
            pages[r][e] = p
            self.ref[p] = 1
        return 0

    def compact(self, total, pages, width):
        used = sum(c > 0 for c in self.ref)
        high = [p for p in range(used, len(self.ref)) if self.ref[p] > 0]
        low = [p for p in range(used) if self.ref[p] <= 0]
        where = [p if c > 0 else -1 for p, c in enumerate(self.ref)]
        for a, b in zip(high, low):
            where[a], self.ref[b], self.ref[a], self.data[b] = b, self.ref[a], 0, self.data[a]
        for r, t in enumerate(total):
            for e in range(min(pages_of(t, self.page), width)):
                p = pages[r][e]
                if self.ok(p) and where[p] >= 0:
                    pages[r][e] = where[p]
        return used, where


# ------------------------------------------------------------------ selection

def beam_tolerance(l, vocab):
    """Bound of a returned score's error.  The score is rounded once (half a step of |l|); log Z
    carries, in units of u = 2^-24 relative to Z: the exponentials' own error (two results with a
    run's factor, each within 2 u: 4 u), their arguments' (difference, constant and product, 3 u
    each of |argument|, twice; a term of weight w has |argument| log2(1 / w) at most, whose mean
    is at most log2(vocab): 2 * 3 ln 2 log2(vocab) u), and sums of 8 terms, 2 and 6 pairs (16 u);
    a multiply for a run's factor and one rounding to it (2 u)."""
    return 2.0 ** -24 * (abs(l) + 22 + 4.2 * math.log2(max(vocab, 2)))


def allowed(x, mask, vocab):
    """x with -inf where the mask forbids."""
    if mask is None:
        return x
    v = torch.arange(vocab)
    bits = (mask[..., v // 32].to(torch.int64) >> (v % 32)) & 1
    return torch.where(bits == 1, x, torch.full_like(x, -INF))


def beam_keys(x, score, weight=None, done=None, eos=-1, mask=None, scale=1.0):
    """(keys, scores l) of every continuation [batch, beams, vocab] in 64 bits, -inf for none."""
    vocab = x.shape[2]
    x = allowed(x.cpu().double(), None if mask is None else mask.cpu(), vocab)
    s = score.cpu().double()
    w = torch.ones_like(s) if weight is None else weight.cpu().double()
    z = torch.logsumexp(x * scale, 2)
    l = s[..., None] + (x * scale - z[..., None])
    bad = ~torch.isfinite(z) | torch.isnan(x).any(2) | (x == INF).any(2)
    l = torch.where(bad[..., None] | (x == -INF), -INF, l)
    if done is not None:
        end = torch.full_like(l, -INF)
        end[..., eos] = s
        l = torch.where(done.cpu()[..., None], end, l)
    none = ~torch.isfinite(s) | ~(torch.isfinite(w) & (w > 0))
    l = torch.where(none[..., None], -INF, l)
    return torch.where(l > -INF, w[..., None] * l, -INF), l


def check_beam(out, x, score, m, weight=None, done=None, eos=-1, mask=None, scale=1.0):
    """Checks gmm_beam_select's outputs (score, parent, token, done or None).  Words of one beam
    are ordered by their logits, exactly; places of different beams may differ from the 64-bit
    order only where keys are within twice the bound of a score."""
    got_s, got_p, got_t, got_d = (None if t is None else t.cpu() for t in out)
    key, l = beam_keys(x, score, weight, done, eos, mask, scale)
    batch, beams, vocab = key.shape
    xs = allowed(x.cpu().double(), None if mask is None else mask.cpu(), vocab)
    w = torch.ones(batch, beams, dtype=torch.float64) if weight is None else weight.cpu().double()
    w = torch.where(torch.isfinite(w) & (w > 0), w, 0.0)
    for b in range(batch):
        flat = key[b].reshape(-1)
        top = torch.sort(flat, descending=True, stable=True).values[:m]
        want = int((top > -INF).sum())
        assert (got_p[b] >= 0).sum() == want and (got_p[b, want:] == -1).all()
        assert (got_t[b, want:] == -1).all() and (got_s[b, want:] == -INF).all()
        seen = {}
        for i in range(want):
            j, v = int(got_p[b, i]) - b * beams, int(got_t[b, i])
            assert 0 <= j < beams and 0 <= v < vocab, (b, i, j, v)
            exact = float(l[b, j, v])
            tol = beam_tolerance(exact, vocab)
            assert abs(float(got_s[b, i]) - exact) <= tol, (b, i, j, v, float(got_s[b, i]), exact)
            gap = 2 * float(w[b].max()) * beam_tolerance(float(l[b][l[b] > -INF].min()), vocab)
            assert abs(float(key[b, j, v]) - float(top[i])) <= gap, (b, i, j, v)
            seen.setdefault(j, []).append(v)
            fin = done is not None and bool(done[b, j])
            if got_d is not None:
                assert bool(got_d[b, i]) == (fin or v == eos)
        for j, vs in seen.items():
            if done is not None and bool(done[b, j]):
                assert vs == [eos]
                continue
            order = torch.sort(xs[b, j], descending=True, stable=True).indices[:len(vs)]
            assert vs == order.tolist(), (b, j)
        if got_d is not None:
            assert not got_d[b, want:].any()
