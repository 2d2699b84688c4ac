"""Attention of few rows in 64 bits, with the bound of a kernel that adds the rest of the weights'
rounding as a second term: what one rounding of the weights costs is not in it."""
import math

import torch

from kvcheck import UNIT

# up to 64 query rows a cache head in the mean
CASES = [
    ([(1, 300), (1, 33), (0, 50)], 8, 2, 128, 32),
    ([(1, 2500), (1, 5)], 12, 4, 64, 64),
    ([(1, 900)], 40, 1, 96, 32),
    ([(1, 400)], 64, 1, 256, 128),
    ([(5, 400), (2, 2), (7, 129)], 6, 3, 80, 64),
    ([(9, 700)], 4, 1, 128, 64),
    ([(16, 333)], 4, 1, 192, 32),
    # few keys and narrow heads: weights' roundings that do not average out, scores of small error
    ([(1, 6), (1, 9), (1, 17), (1, 40)], 48, 1, 16, 32),
    ([(3, 12), (2, 25)], 8, 2, 32, 32),
]


def rows_of(bt):
    """(row, query head, keys, values, scores' factor q) of every row that sees a key."""
    grp = bt.hq // bt.hk
    for r in range(bt.rows):
        b, slot = bt.row_seq[r], bt.row_slot[r]
        if slot < 0:
            continue
        for j in range(bt.hq):
            k, v = bt.keys[b][j // grp, :slot + 1].double(), bt.vals[b][j // grp, :slot + 1].double()
            yield r, j, k, v, bt.q[r, j].double()


def attend_precise(bt, scale):
    """out [rows, hq, d] in 64 bits and its bound: u u a weight (the rest's own rounding), fp32 scores
    and sums, one rounding of the result."""
    u = UNIT[bt.dt]
    out = torch.zeros(bt.rows, bt.hq, bt.d, dtype=torch.float64)
    tol = torch.zeros_like(out)
    for r, j, k, v, q in rows_of(bt):
        s = (k @ q) * scale
        p = torch.softmax(s, 0)
        o, a = p @ v, p @ v.abs()
        # the same terms as for many rows, but for the weights' rounding
        mag = float((k.abs() @ q.abs()).max()) * abs(scale)
        ds = (bt.d + 8) * 2.0 ** -24 * mag + 2.0 ** -21
        sums = (k.shape[0] / 16 + 64) * 2.0 ** -24
        err = (u * u + 2 * ds + 2 * sums) * a
        if bt.dt == torch.float16:         # weights down to 2^-40 of the largest, small results
            err += 2.0 ** -40 * v.abs().sum(0) + 2.0 ** -25
        out[r, j], tol[r, j] = o, err + u * (o.abs() + err)
    return out, tol


def attend_rounded_once(bt, scale):
    """The same with the weights rounded to the type and nothing added, on the CPU."""
    out = torch.zeros(bt.rows, bt.hq, bt.d, dtype=torch.float64)
    for r, j, k, v, q in rows_of(bt):
        s = (k @ q) * scale
        e = torch.exp(s - s.max())
        out[r, j] = ((e.to(bt.dt).double() @ v) / e.sum()).to(bt.dt).double()
    return out
