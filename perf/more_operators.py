"""Beam search over the paged key/value cache as measurable cases: the selection over beams and
vocabulary, and the bookkeeping of the cache's pages (copying, forking, growing, compacting).

A case is one pass through one operator.  `own` false computes it in elementary torch operations,
`own` true makes the calls of this library.

Layouts (those of the library):
  cache    k [pages, heads, page, d], v [pages, heads, d, page], box [pages, heads, 2, d] int8 in
           units of box_scale [pages, heads] fp32
  tables   row r holds total[r] keys; key t is slot t % page of page pages[r, t // page]
  counts   ref [pages] int32: how many table entries name a page; 0 is a free page
  beams    row b * beams + j is beam j of sequence b
A call that changes counts or tables in place starts from those that `prepare` made: `run` puts
them back first, one copy of a few kilobytes on both sides.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _beam(batch, beams, vocab, m, dtype, mask=False, done=False, weight=False, strided=False,
          first=False, scale=1.0, name=None):
    """done: some beams are finished; first: the first step, one live beam a sequence."""
    c = {"op": "beam", "batch": batch, "beams": beams, "vocab": vocab, "m": m, "dtype": dtype,
         "mask": mask, "done": done, "weight": weight, "strided": strided, "first": first,
         "scale": scale}
    return c if name is None else {**c, "name": name}


def _copy(n, pool, heads, page, d, dtype, boxes=True, two=True, name=None):
    """n pages of `pool`, into a second cache or (two false) free pages of the same one."""
    c = {"op": "copy", "n": n, "pool": pool, "heads": heads, "page": page, "d": d,
         "dtype": dtype, "boxes": boxes, "two": two}
    return c if name is None else {**c, "name": name}


def _book(op, seqs, group, keys, page, heads, d, dtype, fill, lens=1, new=0, fan=1, keep=False,
          release=True, boxes=False, tight=False, name=None):
    """Tables of seqs * group rows: the `group` rows of a sequence share the pages of its
    prompt, of up to `keys` keys (lengths spread, seeded by lens).  fill: the used part of the
    pool; new: tokens a row grows by; fan: new rows an old one is forked into; keep: a few
    tokens are rolled back; tight: the pool is too small."""
    c = {"op": op, "seqs": seqs, "group": group, "keys": keys, "page": page, "heads": heads,
         "d": d, "dtype": dtype, "fill": fill, "lens": lens, "new": new, "fan": fan,
         "keep": keep, "release": release, "boxes": boxes, "tight": tight}
    return c if name is None else {**c, "name": name}


def listed():
    return [
        # the first step of one request: one live beam, latency
        _beam(1, 4, 32768, 4, "f32", first=True, name="beam_first"),
        # a step of 32 requests with 8 beams each
        _beam(32, 8, 131072, 8, "bf16", name="beam_step"),
        # odd vocabulary in padded rows, words that a grammar forbids, finished beams, scores
        # normalised by length, twice as many candidates as beams
        _beam(5, 3, 50001, 6, "f16", mask=True, done=True, weight=True, strided=True, scale=0.7,
              name="beam_grammar"),
        # many requests with wide beams, logits kept in fp32
        _beam(64, 16, 131072, 16, "f32", done=True, name="beam_wide"),
        # requests that give way are moved to a second cache
        _copy(2048, 3000, 8, 64, 128, "bf16", name="copy_swap"),
        # some small pages within a cache: latency
        _copy(9, 300, 4, 32, 96, "f16", boxes=False, two=False, name="copy_few"),
        # the beams of 64 requests of up to 32,768 keys take their parents' tables
        _book("fork", 64, 8, 32768, 64, 1, 16, "bf16", 0.7, name="fork_beams"),
        # drafted tokens of 20 requests are rolled back
        _book("fork", 20, 1, 9000, 32, 1, 16, "f16", 0.5, lens=5, keep=True, name="fork_rollback"),
        # one more token for every beam; beams of one parent share the page that they write
        _book("grow", 64, 8, 3000, 64, 8, 128, "bf16", 0.8, lens=3, new=1, boxes=True,
              name="grow_beams"),
        # pages for the prompts of 9 new requests, many pages
        _book("grow", 9, 1, 1, 32, 1, 32, "f16", 0.01, lens=7, new=20000, name="grow_prompts"),
        # a scattered pool is pushed together
        _book("compact", 48, 1, 8000, 64, 8, 128, "bf16", 0.55, lens=9, boxes=True,
              name="compact_pool"),
        # few small pages
        _book("compact", 6, 2, 900, 32, 4, 64, "f16", 0.3, lens=11, name="compact_small"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the same calls, sizes between and around the listed ones."""
    op = rng.choice(["beam", "beam", "copy", "fork", "grow", "compact"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "beam":
        batch, beams, vocab = _log(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 8, 8, 12, 16, 32]), \
            _log(rng, 100, 200000)
        while batch * beams * vocab > 64 * 16 * 131072:
            batch = (batch + 1) // 2
        return _beam(batch, beams, vocab, min(64, rng.choice([1, beams, beams, 2 * beams])),
                     rng.choice([dtype, "f32"]), mask=rng.random() < 0.3, done=rng.random() < 0.5,
                     weight=rng.random() < 0.5, strided=rng.random() < 0.3,
                     first=rng.random() < 0.2, scale=rng.choice([1.0, 1.0, 0.7, 1.3]))
    heads, page, d = rng.choice([1, 2, 4, 8]), rng.choice([32, 64, 64, 128]), \
        rng.choice([64, 128, 128, rng.randrange(32, 257, 16)])
    boxes = rng.random() < 0.5
    if op == "copy":
        n = _log(rng, 1, 2048)
        while n * heads * page * d > 2048 * 8 * 64 * 128:
            n = (n + 1) // 2
        return _copy(n, n + rng.randint(0, n) if n > 1 else 3, heads, page, d, dtype, boxes=boxes,
                     two=rng.random() < 0.5)
    group = rng.choice([1, 1, 4, 8, rng.randint(2, 12)])
    lens, fill = rng.randrange(1 << 20), rng.uniform(0.2, 0.95)
    if op == "fork":
        fan = rng.choice([1, 1, rng.randint(2, 20)])
        seqs = _log(rng, 1, 512 // (group * fan) + 1)
        return _book("fork", seqs, group, _log(rng, 1, 32768), page, 1, 16, dtype, fill, lens=lens,
                     fan=fan, keep=rng.random() < 0.4, release=fan == 1 or rng.random() < 0.5)
    if op == "grow":
        if rng.random() < 0.5:
            return _book("grow", _log(rng, 1, 64), group, _log(rng, 1, 3000), page, heads,
                         rng.choice([64, 128]), dtype, fill, lens=lens, new=rng.randint(1, 8),
                         boxes=boxes, tight=rng.random() < 0.1)
        return _book("grow", _log(rng, 1, 9), 1, _log(rng, 1, 3000), page, 1, 32, dtype,
                     rng.uniform(0.01, 0.9), lens=lens, new=_log(rng, 10, 20000),
                     tight=rng.random() < 0.1)
    seqs, keys = _log(rng, 1, 48), _log(rng, 32, 8000)
    while seqs * keys * heads * d > 48 * 6000 * 8 * 128:
        keys = (keys + 1) // 2
    return _book("compact", seqs, group if seqs * group < 96 else 1, keys, page, heads, d, dtype,
                 fill, lens=lens, boxes=boxes)


# ------------------------------------------------------------------ tables

def _np(t, page):
    return (t + page - 1) // page


def _layout(case):
    """Keys of every row and logical numbers of its pages (lists), pages in all, before the
    call.  Rows of a sequence share its prompt's full pages; what follows is each row's own."""
    rng = random.Random(case["lens"])
    page, totals, rows, at = case["page"], [], [], 0
    for s in range(case["seqs"]):
        t = case["keys"]
        if s > 0 and t > 1:
            t = min(t, _log(rng, max(1, t // 8), t))
        if case["op"] == "grow" and case["keys"] == 1:
            t = 0
        common = t * 3 // 4 // page
        head = list(range(at, at + common))
        at += common
        for _ in range(case["group"]):
            own_pages = _np(t, page) - common
            rows.append(head + list(range(at, at + own_pages)))
            totals.append(t)
            at += own_pages
    if case["op"] == "grow" and case["group"] > 1:
        # what a fork leaves: rows of a sequence continue the table of one of them
        par = _parents(case, rng)
        rows, totals = [rows[p] for p in par], [totals[p] for p in par]
        seen = {}
        rows = [[seen.setdefault(p, len(seen)) for p in r] for r in rows]
        at = len(seen)
    return totals, rows, at


def _parents(case, rng):
    g = case["group"]
    par = []
    for s in range(case["seqs"]):
        for _ in range(g * case["fan"]):
            par.append(s * g + rng.randrange(g))
    return par


def _new_totals(case, totals):
    rng = random.Random(case["lens"] + 1)
    return [t + (case["new"] if case["new"] <= 8 else _log(rng, 1, case["new"])) for t in totals]


def _pool(case, totals, used):
    """Pages of the pool."""
    page = case["page"]
    size = max(used + 1, int(used / case["fill"]))
    if case["op"] == "grow":
        need = sum(_np(n, page) - _np(t, page) for t, n in zip(totals, _new_totals(case, totals)))
        if case["tight"]:
            return used + max(need - 1, 0) // 2 + 1
        size = max(size, int(need / (1 - case["fill"]))) if used == 0 else size
        return max(size, used + need + case["seqs"] * case["group"])
    return size


def _cache(case, pages, g):
    """Random contents of a cache: what is moved is looked at whole."""
    dt = TYPES[case["dtype"]]
    h, page, d = case["heads"], case["page"], case["d"]
    st = {"k": torch.empty(pages, h, page, d, dtype=dt, device=DEV).normal_(generator=g),
          "v": torch.empty(pages, h, d, page, dtype=dt, device=DEV).normal_(generator=g),
          "box": None, "scale": None}
    if case["boxes"]:
        st["box"] = torch.randint(-127, 128, (pages, h, 2, d), generator=g, device=DEV,
                                  dtype=torch.int8)
        st["scale"] = torch.rand(pages, h, generator=g, device=DEV)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    st = {"case": case}
    if own:
        import paper_2606_10896_amd as gmm
        st["gmm"] = gmm
    if case["op"] == "beam":
        bt, bm, vocab, m = (case[c] for c in ("batch", "beams", "vocab", "m"))
        dt = TYPES[case["dtype"]]
        pad = 24 if case["strided"] else 0
        x = torch.empty(bt, bm, vocab + pad, device=DEV).normal_(generator=g).mul_(3.0).to(dt)
        # the beams' last words differ, their probabilities are close
        s = -12.0 - 3.0 * torch.rand(bt, bm, generator=g, device=DEV)
        if case["first"]:
            s[:, 0] = 0.0
            s[:, 1:] = -math.inf
        elif bm > 2:
            # two beams that came from the same words
            x[0, 2], s[0, 2] = x[0, 1], s[0, 1]
        st.update(x=x[..., :vocab], s=s, done=None, weight=None, mask=None, out_done=None,
                  eos=vocab // 3)
        if case["done"]:
            st["done"] = torch.rand(bt, bm, generator=g, device=DEV) < 0.2
            st["out_done"] = torch.empty(bt, m, dtype=torch.bool, device=DEV)
        if case["weight"]:
            st["weight"] = 0.05 + 0.1 * torch.rand(bt, bm, generator=g, device=DEV)
        if case["mask"]:
            words = (vocab + 31) // 32
            bits = torch.randint(-2 ** 31, 2 ** 31, (3, bt, bm, words), generator=g, device=DEV,
                                 dtype=torch.int64).to(torch.int32)
            st["mask"] = bits[0] | bits[1] | bits[2]
            # a grammar that has come to its end leaves nothing
            st["mask"][bt - 1, bm - 1] = 0
        st["out_s"] = torch.empty(bt, m, device=DEV)
        st["out_p"] = torch.empty(bt, m, dtype=torch.int32, device=DEV)
        st["out_t"] = torch.empty(bt, m, dtype=torch.int32, device=DEV)
        if own:
            st["ws"] = gmm.beam_workspace(bt, bm, vocab)
        return st
    if case["op"] == "copy":
        n, pool = case["n"], case["pool"]
        st["src"] = _cache(case, pool if case["two"] else pool + n, g)
        st["dst"] = _cache(case, pool, g) if case["two"] else st["src"]
        perm = torch.randperm(st["src"]["k"].shape[0], generator=g, device=DEV).to(torch.int32)
        st["from"] = perm[:n].contiguous()
        st["to"] = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)[:n].contiguous() \
            if case["two"] else perm[n:2 * n].contiguous()
        if own:
            for c in ("src", "dst"):
                s = st[c]
                s["cache"] = gmm.KVCache(s["k"], s["v"], s["box"], s["scale"])
        return st

    totals, rows, used = _layout(case)
    pool = _pool(case, totals, used)
    page, nrows = case["page"], len(rows)
    after = _new_totals(case, totals) if case["op"] == "grow" else totals
    width = max(1, max(_np(t, page) for t in after))
    table = torch.full((nrows, width), -1, dtype=torch.int32)
    for r, p in enumerate(rows):
        table[r, :len(p)] = torch.tensor(p, dtype=torch.int32)
    # a used pool is scattered; a young one has given out its first pages
    perm = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    table = table.to(DEV)
    table = torch.where(table >= 0, perm[table.clamp(min=0).long()], table)
    # counts and tables in one piece: one copy puts both back
    book0 = torch.zeros(pool + nrows * width, dtype=torch.int32, device=DEV)
    ref0, tab0 = book0[:pool], book0[pool:].view(nrows, width)
    tab0.copy_(table)
    ref0.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    book = book0.clone()
    st.update(book0=book0, book=book, ref=book[:pool], pages=book[pool:].view(nrows, width),
              total=i32(totals), width=width)
    if case["op"] == "fork":
        case_rng = random.Random(seed + 1)
        par = list(range(nrows)) if case["keep"] and case["fan"] == 1 else _parents(case, case_rng)
        st["parent"] = i32(par)
        st["keep"] = i32([max(0, totals[p] - rng.randint(0, 40)) for p in par]) \
            if case["keep"] else None
        st["new_total"] = torch.empty(len(par), dtype=torch.int32, device=DEV)
        st["new_pages"] = torch.empty(len(par), width, dtype=torch.int32, device=DEV)
        if own:
            # the bookkeeping does not touch the keys: narrow pages stand for any
            st["cache"] = gmm.kv_cache(pool, 1, page, 16, TYPES[case["dtype"]], boxes=False)
        return st
    st.update(_cache(case, pool, g))
    if case["op"] == "grow":
        st["new_total"] = i32(after)
        st["short"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    else:
        st["where"] = torch.empty(pool, dtype=torch.int32, device=DEV)
        st["used"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if own:
        st["cache"] = gmm.KVCache(st["k"], st["v"], st["box"], st["scale"])
        st["ws"] = gmm.kv_pool_workspace(st["cache"], nrows)
    return st


# ------------------------------------------------------------------ one pass

def _plain_beam(st):
    """In 64 bits: scores of different beams are compared next to each other."""
    case, x, s = st["case"], st["x"].double(), st["s"].double()
    bt, bm, vocab = x.shape
    if st["mask"] is not None:
        v = torch.arange(vocab, device=DEV)
        ok = (st["mask"][..., v // 32] >> (v % 32).to(torch.int32)) & 1
        x = x.masked_fill(ok == 0, -math.inf)
    x = x * case["scale"]
    mx = x.amax(2, keepdim=True)
    lse = mx + torch.log(torch.exp(x - mx.clamp(min=-1e300)).sum(2, keepdim=True))
    total = torch.where(x > -math.inf, s[..., None] + (x - lse), -math.inf)
    if st["done"] is not None:
        word = torch.where(torch.arange(vocab, device=DEV) == st["eos"], s[..., None], -math.inf)
        total = torch.where(st["done"][..., None], word, total)
    key = total if st["weight"] is None else st["weight"].double()[..., None] * total
    key, at = torch.sort(key.view(bt, bm * vocab), dim=1, descending=True, stable=True)
    m = min(case["m"], bm * vocab)
    key, at = key[:, :m], at[:, :m]
    ok = key > -math.inf
    row = torch.arange(bt, device=DEV)[:, None] * bm + at // vocab
    score = torch.full((bt, case["m"]), -math.inf, dtype=torch.float64, device=DEV)
    parent = torch.full((bt, case["m"]), -1, dtype=torch.int32, device=DEV)
    word = torch.full((bt, case["m"]), -1, dtype=torch.int32, device=DEV)
    score[:, :m] = torch.where(ok, total.view(bt, -1).gather(1, at), -math.inf)
    parent[:, :m] = torch.where(ok, row, -1).to(torch.int32)
    word[:, :m] = torch.where(ok, at % vocab, -1).to(torch.int32)
    if st["done"] is None:
        return score.float(), parent, word
    done = torch.zeros(bt, case["m"], dtype=torch.bool, device=DEV)
    done[:, :m] = ok & (st["done"].view(-1)[row] | (at % vocab == st["eos"]))
    return score.float(), parent, word, done


def _contents(c):
    """A cache's tensors, boxes as the values that they stand for."""
    if c["box"] is None:
        return c["k"], c["v"]
    return c["k"], c["v"], c["box"] * c["scale"][..., None, None]


def _move(src, dst, a, b):
    for t in ("k", "v", "box", "scale"):
        if src[t] is not None:
            dst[t][b] = src[t][a]


def _plain_copy(st):
    _move(st["src"], st["dst"], st["from"].long(), st["to"].long())
    return _contents(st["dst"])


def _entries(total, page, width):
    return torch.arange(width, device=DEV) < _np(total, page)[:, None]


def _plain_fork(st):
    case, ref = st["case"], st["ref"]
    par = st["parent"].long()
    total = st["total"][par]
    if st["keep"] is not None:
        total = torch.minimum(total, st["keep"])
    used = _entries(total, case["page"], st["width"])
    pages = torch.where(used, st["pages"][par], -1)
    named = pages[used]
    ref.index_add_(0, named.long(), torch.ones_like(named))
    if case["release"]:
        named = st["pages"][_entries(st["total"], case["page"], st["width"])]
        ref.index_add_(0, named.long(), torch.full_like(named, -1))
    return total, pages, ref


def _plain_grow(st):
    case, ref, pages, page = st["case"], st["ref"], st["pages"], st["case"]["page"]
    held, total = st["total"], st["new_total"]
    rows = torch.arange(held.numel(), device=DEV)
    new = (_np(total, page) - _np(held, page)).clamp(min=0)
    # rows that write into a page that others hold too
    last = pages[rows, (held // page).clamp(max=st["width"] - 1).long()]
    part = (held % page > 0) & (total > held) & (last >= 0)
    cnt = ref[last.clamp(min=0).long()]
    part &= cnt > 1
    same = part[:, None] & part[None] & (last[:, None] == last[None])
    first = ~(same & (rows[None] < rows[:, None])).any(1)
    copy = part & ~(first & (cnt <= same.sum(1)))
    need = new + copy
    free = torch.nonzero(ref == 0).view(-1).to(torch.int32)
    want = int(need.sum())
    short = torch.full_like(st["short"], max(0, want - free.numel()))
    if 0 < want <= free.numel():
        at = need.cumsum(0) - need
        b = rows[copy]
        src, dst = last[copy].long(), free[at[copy]].long()
        _move(st, st, src, dst)
        ref.index_add_(0, src, torch.full_like(last[copy], -1))
        pages[b, (held[copy] // page).long()] = dst.to(torch.int32)
        e = torch.arange(st["width"], device=DEV) - _np(held, page)[:, None]
        fresh = (e >= 0) & (e < new[:, None])
        pages[fresh] = free[((at + copy)[:, None] + e)[fresh]]
        ref[free[:want].long()] = 1
    return (short, pages, ref) + _contents(st)


def _plain_compact(st):
    case, ref, pages = st["case"], st["ref"], st["pages"]
    used = ref > 0
    n = used.sum()
    p = torch.arange(ref.numel(), device=DEV, dtype=torch.int32)
    src, dst = torch.nonzero(used & (p >= n)).view(-1), torch.nonzero(~used & (p < n)).view(-1)
    where = torch.where(used, p, -1)
    where[src] = dst.to(torch.int32)
    _move(st, st, src, dst)
    ref[dst] = ref[src]
    ref[src] = 0
    live = _entries(st["total"], case["page"], st["width"])
    pages.copy_(torch.where(live, where[pages.clamp(min=0).long()], pages))
    return (n.to(torch.int32).view(1), where, pages, ref) + _contents(st)


def run(st):
    case, op = st["case"], st["case"]["op"]
    if op in ("grow", "compact"):
        st["book"].copy_(st["book0"])
    elif op == "fork":
        st["ref"].copy_(st["book0"][:st["ref"].numel()])
    if not own:
        return {"beam": _plain_beam, "copy": _plain_copy, "fork": _plain_fork,
                "grow": _plain_grow, "compact": _plain_compact}[op](st)
    gmm = st["gmm"]
    if op == "beam":
        gmm.gmm_beam_select(st["x"], st["s"], st["out_s"], st["out_p"], st["out_t"], st["ws"],
                            done=st["done"], out_done=st["out_done"], eos=st["eos"],
                            weight=st["weight"], mask=st["mask"], scale=case["scale"])
        out = st["out_s"], st["out_p"], st["out_t"]
        return out if st["done"] is None else out + (st["out_done"],)
    if op == "copy":
        gmm.gmm_kv_copy(st["src"]["cache"], st["dst"]["cache"], st["from"], st["to"])
        return _contents(st["dst"])
    if op == "fork":
        gmm.gmm_kv_fork(st["cache"], st["ref"], st["total"], st["pages"], st["parent"],
                        st["new_total"], st["new_pages"], keep=st["keep"],
                        release=case["release"])
        return st["new_total"], st["new_pages"], st["ref"]
    if op == "grow":
        gmm.gmm_kv_grow(st["cache"], st["ref"], st["total"], st["new_total"], st["pages"],
                        st["short"], st["ws"])
        return (st["short"], st["pages"], st["ref"]) + _contents(st)
    gmm.gmm_kv_compact(st["cache"], st["ref"], st["total"], st["pages"], st["where"], st["used"],
                       st["ws"])
    return (st["used"], st["where"], st["pages"], st["ref"]) + _contents(st)


# ------------------------------------------------------------------ what a pass cannot do without

def _page_bytes(case):
    h, d = case["heads"], case["d"]
    return 4 * h * case["page"] * d + (h * (2 * d + 4) if case["boxes"] else 0)


def work(case):
    if case["op"] == "beam":
        rows = case["batch"] * case["beams"]
        n = rows * case["vocab"]
        es = 4 if case["dtype"] == "f32" else 2
        return {"bytes": n * es + (n // 8 if case["mask"] else 0) + rows * 9 +
                case["batch"] * case["m"] * 13, "flops": 4 * n}
    if case["op"] == "copy":
        return {"bytes": case["n"] * (2 * _page_bytes(case) + 8), "flops": 0}
    totals, rows, used = _layout(case)
    page, entries = case["page"], sum(len(r) for r in rows)
    if case["op"] == "fork":
        new = len(rows) * case["fan"]
        width = max(1, max(_np(t, page) for t in totals))
        return {"bytes": 4 * (min(entries * case["fan"], entries if case["release"] else
                                  new * width) + new * width + 3 * new), "flops": 0}
    pool = _pool(case, totals, used)
    if case["op"] == "grow":
        after = _new_totals(case, totals)
        fresh = sum(_np(a, page) - _np(t, page) for t, a in zip(totals, after))
        cnt, writers = {}, {}
        for r in rows:
            for p in r:
                cnt[p] = cnt.get(p, 0) + 1
        for t, r in zip(totals, rows):
            if t % page:
                writers[r[-1]] = writers.get(r[-1], 0) + 1
        copies = sum(w - 1 if cnt[p] <= w else w for p, w in writers.items() if cnt[p] > 1)
        if case["tight"]:
            fresh = copies = 0
        return {"bytes": 4 * pool + 2 * copies * _page_bytes(case) + 8 * (fresh + copies) +
                12 * len(rows), "flops": 0}
    # pages above the used ones, in a pool filled evenly
    moved = used * (pool - used) // pool
    return {"bytes": 8 * pool + 8 * entries + 2 * moved * _page_bytes(case), "flops": 0}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_beam(st, case):
    """Beam by beam: the m best words of each, and the best of those on the host."""
    bt, bm, vocab = st["x"].shape
    m, inf = case["m"], math.inf
    score = torch.full((bt, m), -inf, dtype=torch.float64)
    parent = torch.full((bt, m), -1, dtype=torch.int32)
    word = torch.full((bt, m), -1, dtype=torch.int32)
    flag = torch.zeros(bt, m, dtype=torch.bool)
    for b in range(bt):
        found = []
        for j in range(bm):
            s = float(st["s"][b, j])
            w = 1.0 if st["weight"] is None else float(st["weight"][b, j])
            if s == -inf:
                continue
            if st["done"] is not None and bool(st["done"][b, j]):
                found.append((-w * s, j, st["eos"], s, True))
                continue
            x = st["x"][b, j].double()
            if st["mask"] is not None:
                word_bits = st["mask"][b, j].to(torch.int64) & 0xFFFFFFFF
                bits = (word_bits[:, None] >> torch.arange(32, device=DEV)) & 1
                x = torch.where(bits.view(-1)[:vocab] == 1, x, -inf)
            top, at = torch.sort(x, descending=True, stable=True)
            z = float(torch.logsumexp(x * case["scale"], 0))
            for v, t in zip(at[:m].tolist(), top[:m].tolist()):
                if t > -inf:
                    tot = s + (t * case["scale"] - z)
                    found.append((-w * tot, j, v, tot, v == st["eos"]))
        for i, (_, j, v, tot, f) in enumerate(sorted(found)[:m]):
            score[b, i], parent[b, i], word[b, i], flag[b, i] = tot, b * bm + j, v, f
    out = score.to(DEV), parent.to(DEV), word.to(DEV)
    return out if st["done"] is None else out + (flag.to(DEV),)


def _exact_contents(src, dst, pairs):
    """dst's tensors in 64 bits with the pages `pairs` (from, to) of src in them."""
    out = []
    order = list(range(dst["k"].shape[0]))
    for a, b in pairs:
        order[b] = a if src is dst else -1 - a
    idx = torch.tensor(order, device=DEV)
    take = lambda s, d: torch.where((idx >= 0).view(-1, *[1] * (d.dim() - 1)),
                                    d[idx.clamp(min=0)], s[(-1 - idx).clamp(min=0)])
    for t in ("k", "v"):
        out.append(take(src[t], dst[t]).double())
    if dst["box"] is not None:
        out.append(take(src["box"], dst["box"]).double() *
                   take(src["scale"], dst["scale"]).double()[..., None, None])
    return tuple(out)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "beam":
        return _exact_beam(st, case)
    if case["op"] == "copy":
        return _exact_contents(st["src"], st["dst"],
                               list(zip(st["from"].tolist(), st["to"].tolist())))
    # the bookkeeping, page by page on the host
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    page, ref, pages, totals = case["page"], st["ref"].tolist(), st["pages"].tolist(), \
        st["total"].tolist()
    if case["op"] == "fork":
        keep = st["keep"].tolist() if st["keep"] is not None else None
        nt, npg = [], []
        for i, p in enumerate(st["parent"].tolist()):
            t = totals[p] if keep is None else min(totals[p], keep[i])
            row = pages[p][:_np(t, page)]
            for q in row:
                ref[q] += 1
            nt.append(t)
            npg.append(row + [-1] * (st["width"] - len(row)))
        if case["release"]:
            for t, row in zip(totals, pages):
                for q in row[:_np(t, page)]:
                    ref[q] -= 1
        return i32(nt), i32(npg), i32(ref)
    if case["op"] == "grow":
        free = [p for p, c in enumerate(ref) if c == 0]
        after, writers, need = st["new_total"].tolist(), {}, []
        for r, (t, a) in enumerate(zip(totals, after)):
            if t % page and a > t and ref[pages[r][t // page]] > 1:
                writers.setdefault(pages[r][t // page], []).append(r)
        copies = {r: p for p, rs in writers.items()
                  for i, r in enumerate(rs) if i or ref[p] > len(rs)}
        for r, (t, a) in enumerate(zip(totals, after)):
            if r in copies:
                need.append((r, t // page, copies[r]))
            need.extend((r, e, -1) for e in range(_np(t, page), _np(a, page)))
        pairs, short = [], max(0, len(need) - len(free))
        for (r, e, src), p in zip([] if short else need, free):
            if src >= 0:
                ref[src] -= 1
                pairs.append((src, p))
            pages[r][e] = p
            ref[p] = 1
        return (i32([short]), i32(pages), i32(ref)) + _exact_contents(st, st, pairs)
    n = sum(c > 0 for c in ref)
    high = [p for p in range(n, len(ref)) if ref[p] > 0]
    low = [p for p in range(n) if ref[p] == 0]
    where = [p if c > 0 else -1 for p, c in enumerate(ref)]
    for a, b in zip(high, low):
        where[a], ref[b], ref[a] = b, ref[a], 0
    for r, t in enumerate(totals):
        for e in range(_np(t, page)):
            pages[r][e] = where[pages[r][e]]
    return (i32([n]), i32(where), i32(pages), i32(ref)) + \
        _exact_contents(st, st, list(zip(high, low)))
