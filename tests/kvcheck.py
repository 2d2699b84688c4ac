"""Inputs and plain 64-bit definitions for the tests of the paged key/value cache, on the CPU and
written from the formulas, one sequence, head and row at a time where it matters."""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# unit roundoff: half the distance of neighbours, relative
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


class Batch:
    """Sequences (new tokens, keys with them) over a cache whose pages are handed out in random
    order, with `spare` unused ones; everything on the CPU."""

    def __init__(self, seqs, hq, hk, d, page, dtype, seed=0, spare=3, stale=math.nan, width=None):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.hq, self.hk, self.d, self.page = seqs, hq, hk, d, page
        self.dt = TYPES[dtype]
        need = [(t + page - 1) // page for _, t in seqs]
        self.npages = sum(need) + spare
        perm = torch.randperm(self.npages, generator=g).to(torch.int32)
        self.width = max(need + [1]) if width is None else width
        self.pages = torch.full((len(seqs), self.width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.pages[b, :n] = perm[at:at + n]
            at += n
        rn = lambda *s: torch.randn(*s, generator=g)
        self.k = torch.full((self.npages, hk, page, d), stale).to(self.dt)
        self.v = torch.full((self.npages, hk, d, page), stale).to(self.dt)
        self.keys, self.vals = [], []
        for b, (_, t) in enumerate(seqs):
            kk = (rn(hk, t, d) * 0.8 + rn(hk, 1, d)).to(self.dt)
            vv = rn(hk, t, d).to(self.dt)
            self.keys.append(kk)
            self.vals.append(vv)
            for s in range(t):
                p = int(self.pages[b, s // page])
                self.k[p, :, s % page] = kk[:, s]
                self.v[p, :, :, s % page] = vv[:, s]
        self.rows = sum(n for n, _ in seqs)
        cu = [0]
        for n, _ in seqs:
            cu.append(cu[-1] + n)
        self.cu = torch.tensor(cu, dtype=torch.int32)
        self.total = torch.tensor([t for _, t in seqs], dtype=torch.int32)
        self.q = rn(self.rows, hq, d).to(self.dt)
        self.row_seq = [b for b, (n, _) in enumerate(seqs) for _ in range(n)]
        self.row_slot = [t - n + i for n, t in seqs for i in range(n)]

    def boxes(self):
        """(box int8, scale fp32) of every page from its keys, in numpy."""
        box = np.zeros((self.npages, self.hk, 2, self.d), np.int8)
        scale = np.zeros((self.npages, self.hk), np.float32)
        for b, (_, t) in enumerate(self.seqs):
            for lp in range((t + self.page - 1) // self.page):
                kk = self.keys[b][:, lp * self.page:(lp + 1) * self.page].float().numpy()
                box[self.pages[b, lp]], scale[self.pages[b, lp]] = box_of(kk)
        return torch.from_numpy(box), torch.from_numpy(scale)


def box_of(kk):
    """8-bit bounds of keys kk [heads, n, d] (fp32 values): box [heads, 2, d], scale [heads]."""
    heads, _, d = kk.shape
    box, scale = np.zeros((heads, 2, d), np.int8), np.zeros(heads, np.float32)
    for h in range(heads):
        if not np.isfinite(kk[h]).all():
            scale[h] = np.inf
            continue
        hi, lo = kk[h].max(0), kk[h].min(0)
        u = np.float32(np.abs(kk[h]).max()) * (np.float32(1) / np.float32(127))
        scale[h] = u
        if u > 0:
            box[h, 0] = np.clip(np.ceil(hi / u), -127, 127)
            box[h, 1] = np.clip(np.floor(lo / u), -127, 127)
    return box, scale


def rope64(x, pos, table, interleaved=False, inverse=False):
    """The rotation in 64 bits: x [tokens, heads, d], table [positions, rot]."""
    out = x.double().clone()
    h = table.shape[1] // 2
    for t in range(x.shape[0]):
        p = int(pos[t])
        if p < 0:
            continue
        for i in range(h):
            c, s = float(table[p, i]), float(table[p, h + i])
            if inverse:
                s = -s
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, h + i)
            a, b = x[t, :, ia].double(), x[t, :, ib].double()
            out[t, :, ia] = a * c - b * s
            out[t, :, ib] = b * c + a * s
    return out


def select_exact(bt, box, scale, m, keep_first=1, keep_last=1, q=None):
    """Selected pages [rows, hk, m] from the definition, in whole numbers."""
    q = (bt.q if q is None else q).float().numpy()
    grp = bt.hq // bt.hk
    out = np.full((bt.rows, bt.hk, m), -1, np.int32)
    unit = np.abs(q).max(2).astype(np.float32) * (np.float32(1) / np.float32(127))
    ok = np.isfinite(q).all(2)
    with np.errstate(all="ignore"):
        q8 = np.where((ok & (unit > 0))[..., None], np.rint(q / unit[..., None]), 0.0)
    q8 = q8.astype(np.int64)
    unit = np.where(ok, unit, np.inf).astype(np.float32)
    bx, sc = box.numpy().astype(np.int64), scale.numpy()
    for r in range(bt.rows):
        if bt.row_slot[r] < 0:
            continue
        nv = min(bt.row_slot[r] // bt.page + 1, bt.width)
        ph = bt.pages[bt.row_seq[r], :nv].numpy()
        for h in range(bt.hk):
            best = np.full(nv, -np.inf, np.float32)
            for j in range(h * grp, (h + 1) * grp):
                dot = (np.maximum(q8[r, j], 0) * bx[ph, h, 0] +
                       np.minimum(q8[r, j], 0) * bx[ph, h, 1]).sum(1)
                with np.errstate(all="ignore"):
                    u = (unit[r, j] * sc[ph, h]).astype(np.float32) * dot.astype(np.float32)
                best = np.maximum(best, np.where(np.isnan(u), np.inf, u))
            # kept pages outrank every score
            rank = np.where((np.arange(nv) < keep_first) | (np.arange(nv) >= nv - keep_last), 1, 0)
            order = sorted(range(nv), key=lambda p: (-rank[p], -best[p], p))[:m]
            out[r, h, :len(order)] = sorted(order)
    return torch.from_numpy(out)


def attend64(bt, scale, window=0, sel=None, q=None):
    """out [rows, hq, d], lse [rows, hq] in 64 bits, and a bound of what fp32 sums, weights
    rounded to the type and one rounding of the result may differ from them by."""
    q = (bt.q if q is None else q).double()
    grp, u = bt.hq // bt.hk, UNIT[bt.dt]
    out = torch.zeros(bt.rows, bt.hq, bt.d, dtype=torch.float64)
    lse = torch.full((bt.rows, bt.hq), -math.inf, dtype=torch.float64)
    tol = torch.zeros_like(out)
    ltol = torch.zeros_like(lse)
    for r in range(bt.rows):
        b, slot = bt.row_seq[r], bt.row_slot[r]
        lo = max(0, slot - window + 1) if window else 0
        for h in range(bt.hk):
            if slot < 0:
                continue
            if sel is None:
                keys = torch.arange(lo, slot + 1)
            else:
                keys = [s for p in sel[r, h].tolist() if p >= 0
                        for s in range(p * bt.page, min((p + 1) * bt.page, slot + 1))]
                keys = torch.tensor(keys, dtype=torch.long)
            if keys.numel() == 0:
                continue
            k, v = bt.keys[b][h, keys].double(), bt.vals[b][h, keys].double()
            for j in range(h * grp, (h + 1) * grp):
                s = (k @ q[r, j]) * scale
                z = torch.logsumexp(s, 0)
                p = torch.exp(s - z)
                o = p @ v
                out[r, j], lse[r, j] = o, z
                # error of a score: d fp32 additions of products, the scaling, and the base-2
                # exponential of an argument of that size
                mag = float((k.abs() @ q[r, j].abs()).max()) * abs(scale)
                ds = (bt.d + 8) * 2.0 ** -24 * mag + 2.0 ** -21
                sums = (keys.numel() / 16 + 64) * 2.0 ** -24
                a = p @ v.abs()
                tol[r, j] = (u + 2 * ds + 2 * sums) * a + u * o.abs()
                if bt.dt == torch.float16:      # spacing of its smallest weights and results
                    tol[r, j] += 2.0 ** -25 * (v.abs().sum(0) + 1)
                ltol[r, j] = 2 * ds + sums + 2.0 ** -22 * (1 + abs(float(z)))
    return out, lse, tol, ltol


def strided(x, dt=None):
    """x's values on the GPU as the first heads of rows that hold more of them."""
    big = torch.zeros(x.shape[0], x.shape[1] + 3, x.shape[2], dtype=x.dtype, device="cuda")
    big[:, :x.shape[1]] = x.cuda()
    return big[:, :x.shape[1]]
