"""The page pool's calls (copy, fork, grow, compact) against the bookkeeping on the host, entry by
entry, and the contents of every page."""
import random

import pytest
import torch

import paper_2606_10896_amd as gmm
from poolcheck import Pool, pages_of

pytestmark = pytest.mark.gpu


def _i32(v, dev="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _cache(pages, heads=1, page=32, d=16, dtype=torch.bfloat16, boxes=True, seed=0):
    """A cache of random contents."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = gmm.kv_cache(pages, heads, page, d, dtype, boxes=boxes)
    c.k.normal_(generator=g)
    c.v.normal_(generator=g)
    if boxes:
        c.box.copy_(torch.randint(-127, 128, c.box.shape, generator=g, device="cuda"))
        c.box_scale.uniform_(generator=g)
    return c


def _tensors(c):
    return [t for t in (c.k, c.v, c.box, c.box_scale) if t is not None]


def _snapshot(c):
    return [t.clone() for t in _tensors(c)]


def _check_contents(c, before, data):
    """Page p holds what page data[p] held before."""
    at = torch.tensor(data, device="cuda")
    for t, b in zip(_tensors(c), before):
        assert torch.equal(t, b[at])


class Both:
    """A pool on the GPU and its bookkeeping on the host."""

    def __init__(self, pages, page=32, width=8, seed=0, **kw):
        self.cache = _cache(pages, page=page, seed=seed, **kw)
        self.host, self.page, self.width = Pool(pages, page), page, width
        self.ref = gmm.kv_pool(self.cache)
        self.total, self.pages = [], []
        self.tt = _i32([])
        self.tp = torch.empty(0, width, dtype=torch.int32, device="cuda")

    def check(self):
        assert self.ref.tolist() == self.host.ref
        assert self.tt.tolist() == self.total and self.tp.tolist() == self.pages

    def fork(self, parent, keep=None, release=True, width=None, check=True):
        width = width or self.width
        old_t, old_p = self.tt, self.tp
        if not self.total:                               # rows of an empty table
            old_t, old_p = _i32([0]), torch.full((1, self.width), -1, dtype=torch.int32,
                                                 device="cuda")
        nt = torch.full((len(parent),), 99, dtype=torch.int32, device="cuda")
        npg = torch.full((len(parent), width), 99, dtype=torch.int32, device="cuda")
        gmm.gmm_kv_fork(self.cache, self.ref, old_t, old_p, _i32(parent), nt, npg,
                        keep=None if keep is None else _i32(keep), release=release)
        self.total, self.pages = self.host.fork(self.total, self.pages, self.width, parent, width,
                                                keep, release)
        self.tt, self.tp, self.width = nt, npg, width
        if check:
            self.check()

    def grow(self, total):
        short = _i32([-7])
        before = _snapshot(self.cache)
        self.host.data = list(range(len(self.host.ref)))
        new = _i32(total)
        gmm.gmm_kv_grow(self.cache, self.ref, self.tt, new, self.tp, short,
                        gmm.kv_pool_workspace(self.cache, len(total)).fill_(255))
        missing = self.host.grow(self.total, total, self.pages, self.width)
        assert short.item() == missing
        if missing == 0:
            self.tt, self.total = new, list(total)
        self.check()
        _check_contents(self.cache, before, self.host.data)
        return missing

    def compact(self):
        n = len(self.host.ref)
        where, used = torch.full((n,), 99, dtype=torch.int32, device="cuda"), _i32([-7])
        before = _snapshot(self.cache)
        self.host.data = list(range(n))
        gmm.gmm_kv_compact(self.cache, self.ref, self.tt, self.tp, where, used,
                           gmm.kv_pool_workspace(self.cache, len(self.total)).fill_(255))
        u, w = self.host.compact(self.total, self.pages, self.width)
        assert used.item() == u and where.tolist() == w
        self.check()
        _check_contents(self.cache, before, self.host.data)


# ------------------------------------------------------------------ copy

@pytest.mark.parametrize("heads,page,d,dtype,boxes", [
    (1, 32, 16, torch.bfloat16, True), (3, 32, 48, torch.float16, True),
    (8, 64, 128, torch.bfloat16, True), (2, 128, 256, torch.float16, False),
    (5, 256, 80, torch.bfloat16, True)])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_copy_between_caches(heads, page, d, dtype, boxes, n):
    src = _cache(50, heads, page, d, dtype, boxes, seed=1)
    dst = _cache(45, heads, page, d, dtype, boxes, seed=2)
    g = torch.Generator().manual_seed(n)
    a, b = torch.randperm(50, generator=g)[:n].tolist(), torch.randperm(45, generator=g)[:n].tolist()
    want = _snapshot(dst)
    # numbers out of range: the pair is skipped
    fa, fb = a + [50, -1, 3, 4, 2 ** 31 - 1, -2 ** 31], b + [b[0], b[0], 45, -1, 0, 0]
    for t, s in zip(want, _tensors(src)):
        for p, q in zip(a, b):
            t[q] = s[p]
    kept = _snapshot(src)
    gmm.gmm_kv_copy(src, dst, _i32(fa), _i32(fb))
    for t, w in zip(_tensors(dst), want):
        assert torch.equal(t, w)
    for t, w in zip(_tensors(src), kept):
        assert torch.equal(t, w)


def test_copy_within_a_cache_and_of_nothing():
    c = _cache(20, 2, 64, 64, seed=3)
    before = _snapshot(c)
    gmm.gmm_kv_copy(c, c, _i32([]), _i32([]))
    _check_contents(c, before, list(range(20)))
    gmm.gmm_kv_copy(c, c, _i32([4, 5, 9, 4]), _i32([1, 0, 9, 19]))
    data = list(range(20))
    data[1], data[0], data[19] = 4, 5, 4
    _check_contents(c, before, data)


def test_copy_of_many_pages_past_32_bits_of_bytes():
    """A cache of more than 4 GiB of keys."""
    pages = 17000
    try:
        c = gmm.kv_cache(pages, 8, 64, 256, boxes=True)
    except torch.OutOfMemoryError:
        pytest.skip("no memory")
    src = list(range(100)) + [8500]
    dst = list(range(pages - 100, pages)) + [pages - 101]
    for i, p in enumerate(src):
        c.k[p] = i + 1
        c.v[p] = -i - 1
        c.box_scale[p] = i + 1
    gmm.gmm_kv_copy(c, c, _i32(src), _i32(dst))
    for i, p in enumerate(dst):
        assert (c.k[p] == i + 1).all() and (c.v[p] == -i - 1).all()
        assert (c.box_scale[p] == i + 1).all()
    assert (c.k[200:8400] == 0).all() and (c.k[8501:pages - 101] == 0).all()


# ------------------------------------------------------------------ fork

def test_fork_shares_rolls_back_and_frees():
    b = Both(60, width=8)
    b.fork([-1] * 3)
    assert b.grow([200, 33, 0]) == 0
    b.fork([0, 0, 1, 0, 2, 5, -4, 3])                     # two parents that are no rows
    b.fork([0, 1, 2, 3, 4, 5, 6, 7], keep=[200, 64, 33, 65, 9, 9, 0, -5])
    b.fork([0, 2, 2], keep=[10 ** 9, 1, 32], width=11)
    b.fork([1], release=False)
    assert sum(b.host.ref) > 1
    b.fork([])
    # what the rows left behind still counts
    assert b.ref.sum().item() == sum(b.host.ref)


def test_free_everything():
    b = Both(40, width=20)
    b.fork([-1, -1])
    b.grow([500, 300])
    b.fork([0, 1, 0, 1, 1])
    b.fork([])
    assert (b.ref == 0).all()


def test_fork_leaves_entries_that_are_no_pages_alone():
    """Entries out of range in the used part of a row are passed on and not counted."""
    c = _cache(10)
    ref = gmm.kv_pool(c) + 1
    total, pages = _i32([160, 64]), _i32([[0, -3, 10, 2 ** 31 - 1, 9, 5], [1, 2, 77, 77, 77, 77]])
    nt, npg = _i32([0, 0, 0]), torch.zeros(3, 6, dtype=torch.int32, device="cuda")
    gmm.gmm_kv_fork(c, ref, total, pages, _i32([0, 0, 1]), nt, npg)
    assert nt.tolist() == [160, 160, 64]
    assert npg.tolist() == [[0, -3, 10, 2 ** 31 - 1, 9, -1]] * 2 + [[1, 2, -1, -1, -1, -1]]
    assert ref.tolist() == [2, 1, 1, 1, 1, 1, 1, 1, 1, 2]


def test_fork_of_totals_past_the_table():
    b = Both(30, width=3)
    b.fork([-1])
    b.grow([1000])                                       # three entries of 32 keys
    assert sum(b.host.ref) == 3
    b.fork([0, 0], keep=[90, 999])
    b.fork([])
    assert (b.ref == 0).all()


@pytest.mark.parametrize("rows,width", [(700, 3), (3, 5000), (1, 1025)])
def test_fork_of_many_rows_and_long_rows(rows, width):
    rng = random.Random(rows)
    n = rows * width
    c = _cache(n)
    perm = list(range(n))
    rng.shuffle(perm)
    page, host = 32, Pool(n, 32)
    total = [rng.randint(0, width * page) for _ in range(rows)]
    pages = [perm[r * width:(r + 1) * width] for r in range(rows)]
    for t, p in zip(total, pages):
        for q in p[:pages_of(t, page)]:
            host.ref[q] += 1
    parent = [rng.randint(-1, rows) for _ in range(rows + 5)]
    keep = [rng.randint(-3, width * page + 9) for _ in parent]
    ref, tt, tp = _i32(host.ref), _i32(total), _i32(pages)
    nt = torch.empty(len(parent), dtype=torch.int32, device="cuda")
    # rows of a wider buffer: what lies between them stays
    buf = torch.full((len(parent), width + 9), 55, dtype=torch.int32, device="cuda")
    gmm.gmm_kv_fork(c, ref, tt, tp, _i32(parent), nt, buf[:, 2:width + 4], keep=_i32(keep))
    wt, wp = host.fork(total, pages, width, parent, width + 2, keep)
    assert nt.tolist() == wt and buf[:, 2:width + 4].tolist() == wp and ref.tolist() == host.ref
    assert (buf[:, :2] == 55).all() and (buf[:, width + 4:] == 55).all()


# ------------------------------------------------------------------ grow

def test_grow_copies_what_others_hold():
    b = Both(40, heads=3, d=48)
    b.fork([-1, -1])
    b.grow([70, 64])
    b.fork([0, 0, 0, 1, 1])
    # three writers of one shared page: the first keeps it; a full last page is not written
    assert b.grow([71, 70, 100, 65, 64]) == 0
    b.fork([0, 0, 1, 1], release=True)
    # one writer, the other holder does not write: a copy
    assert b.grow([72, 71, 70, 200]) == 0


def test_grow_keeps_a_page_that_a_table_outside_holds():
    b = Both(40)
    b.fork([-1])
    b.grow([40])
    outside = (b.tt, b.tp)
    total, pages = list(b.total), [list(r) for r in b.pages]
    b.fork([0, 0], release=False)
    assert b.grow([41, 41]) == 0                         # both get copies
    assert outside[0].tolist() == total and outside[1].tolist() == pages
    assert b.ref[pages[0][1]].item() == 1


def test_grow_that_is_short_changes_nothing():
    b = Both(9, width=8)
    b.fork([-1, -1])
    assert b.grow([100, 140]) == 0                       # 4 and 5 pages: all
    assert b.grow([100, 140]) == 0                       # nothing needed
    assert b.grow([129, 140]) == 1
    b.fork([0, 0])
    assert b.grow([101, 101]) == 0                       # the second row's copy, 5 pages are free
    b.fork([0, 1, 0, 1, 1])
    # five copies but two are kept: 3 of the 4 free ones
    assert b.grow([102] * 5) == 0
    assert b.grow([200] * 5) > 0


def test_grow_rows_that_do_not_and_edges():
    b = Both(50, width=4)
    b.fork([-1] * 6)
    assert b.grow([0, 1, 32, 33, 128, 10 ** 6]) == 0      # past the table: its four entries
    assert b.grow([1, 0, 33, 33, 129, 10 ** 6 + 5]) == 0
    assert b.host.ref.count(1) == sum(b.host.ref)


@pytest.mark.parametrize("pages", [1, 63, 64, 65, 1023, 1025, 65535, 65536, 65537, 140001])
def test_grow_finds_the_lowest_free_pages(pages):
    """Pools of many sizes, sparse and dense, with the free pages anywhere."""
    c = _cache(pages, boxes=False)
    rng = random.Random(pages)
    for used in (0.0, 0.5, 0.999, 1.0):
        ref = [1 if rng.random() < used else 0 for _ in range(pages)]
        if used == 1.0:
            ref[-1] = 0                                  # the last page of all
        free = [p for p, r in enumerate(ref) if r == 0]
        for want in {0, 1, min(len(free), 700), len(free), len(free) + 1}:
            rows = 3
            each = [want // 2, 0, want - want // 2]
            width = max(1, *each)
            if width * 32 > 1 << 30:
                continue
            tr, tp = _i32(ref), torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
            short = _i32([-1])
            gmm.gmm_kv_grow(c, tr, _i32([0] * rows), _i32([32 * e for e in each]), tp, short,
                            gmm.kv_pool_workspace(c, rows))
            assert short.item() == max(0, want - len(free))
            wr = torch.tensor(ref, dtype=torch.int32)
            wp = torch.full((rows, width), -1, dtype=torch.int32)
            if want <= len(free):
                wr[free[:want]] = 1
                wp[0, :each[0]] = torch.tensor(free[:each[0]], dtype=torch.int32)
                wp[2, :each[2]] = torch.tensor(free[each[0]:want], dtype=torch.int32)
            assert torch.equal(tr.cpu(), wr) and torch.equal(tp.cpu(), wp)


def test_grow_of_thousands_of_rows():
    rows = 5000
    b = Both(30000, width=3)
    b.fork([-1] * rows)
    rng = random.Random(1)
    assert b.grow([rng.randint(0, 64) for _ in range(rows)]) == 0
    b.fork([rng.randrange(rows // 3) for _ in range(rows)])
    assert b.grow([t + rng.randint(0, 40) for t in b.total]) == 0


def test_need_past_32_bits():
    """The sum of what rows ask for does not wrap."""
    c = _cache(100, boxes=False)
    rows, width = 300, 1 << 25                           # of one table, rows 0 apart: not written
    one = torch.full((1, 64), -1, dtype=torch.int32, device="cuda")
    short = _i32([-1])
    lib = gmm.load_library()
    ws = gmm.kv_pool_workspace(c, rows)
    ref = gmm.kv_pool(c)
    held, total = _i32([0] * rows), _i32([1 << 30] * rows)
    rc = lib.gmm_kv_grow(c._ref, ref.data_ptr(), held.data_ptr(), total.data_ptr(), one.data_ptr(),
                         rows, width, width, short.data_ptr(), ws.data_ptr(), ws.numel(),
                         torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert short.item() == 2 ** 31 - 1                   # 300 x 2^25 - 100, as far as it goes
    assert (ref == 0).all() and (one == -1).all()


# ------------------------------------------------------------------ compact

@pytest.mark.parametrize("pages", [1, 2, 64, 65, 900, 1024, 1025, 5000, 65536, 66000, 131073])
@pytest.mark.parametrize("used", [0.0, 0.03, 0.5, 0.97, 1.0])
def test_compact(pages, used):
    rng = random.Random(pages)
    b = Both(pages, width=5, boxes=pages < 2000)
    live = [p for p in range(pages) if rng.random() < used]
    rng.shuffle(live)
    rows = max(1, min(200, len(live) // 4))
    b.pages, b.total, at = [], [], 0
    for r in range(rows):
        n = min(5, len(live) - at)
        b.pages.append(live[at:at + n] + [-1] * (5 - n))
        b.total.append(n * 32 - rng.randint(0, 31) if n else 0)
        at += n
    # pages that other tables hold move, too
    for p in live:
        b.host.ref[p] = rng.randint(1, 3)
    b.ref, b.tt, b.tp = _i32(b.host.ref), _i32(b.total), _i32(b.pages)
    b.compact()
    b.compact()                                          # nothing moves


def test_compact_leaves_the_rest_of_a_row():
    b = Both(12, width=6)
    b.host.ref = [0, 0, 0, 0, 0, 0, 0, 0, 1, 2, 0, 1]
    b.total, b.pages = [70, 0, 1000], [[9, 8, 11, 9, 55, -1], [9, 9, 9, 9, 9, 9],
                                       [9, -5, 12, 8, 0, 11]]
    b.ref, b.tt, b.tp = _i32(b.host.ref), _i32(b.total), _i32(b.pages)
    b.compact()
    assert b.pages == [[1, 0, 2, 9, 55, -1], [9] * 6, [1, -5, 12, 0, 0, 2]]


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("seed", [0, 1, 2])
def test_random_programs(seed):
    """Forks, growth, roll-back and compaction in any order keep counts, tables and contents."""
    rng = random.Random(seed)
    b = Both(rng.choice([90, 300]), page=rng.choice([32, 64]), width=7, heads=2, d=32, seed=seed)
    b.fork([-1] * 4)
    for step in range(40):
        n = len(b.total)
        what = rng.choice(["fork", "grow", "grow", "roll", "compact"])
        if what == "fork":
            b.fork([rng.randint(-1, n - 1) for _ in range(rng.randint(1, 9))])
        elif what == "roll":
            b.fork(list(range(n)), keep=[max(0, t - rng.randint(0, 40)) for t in b.total])
        elif what == "compact":
            b.compact()
        else:
            b.grow([t + rng.choice([0, 1, 1, 5, 70]) for t in b.total])
        counts = [0] * len(b.host.ref)
        for t, row in zip(b.total, b.pages):
            for p in row[:min(pages_of(t, b.page), 7)]:
                counts[p] += 1
        assert counts == b.host.ref


def test_captured_step():
    """Fork, growth and copies in a graph: two tables in turn, replayed with eager work between."""
    c = _cache(64, heads=2, d=32, seed=4)
    ref, ws = gmm.kv_pool(c), gmm.kv_pool_workspace(c, 4)
    tot = [_i32([0] * 4), _i32([0] * 4)]
    pg = [torch.full((4, 6), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    grown, parent, short = _i32([0] * 4), _i32([0, 0, 1, 1]), _i32([0])

    def step():
        for i in (0, 1):
            gmm.gmm_kv_fork(c, ref, tot[i], pg[i], parent, tot[1 - i], pg[1 - i])
            torch.add(tot[1 - i], 5, out=grown)
            gmm.gmm_kv_grow(c, ref, tot[1 - i], grown, pg[1 - i], short, ws)
            tot[1 - i].copy_(grown)

    start = [t.clone() for t in (ref, *tot, *pg, c.k, c.v, c.box, c.box_scale)]
    state = (ref, *tot, *pg, c.k, c.v, c.box, c.box_scale)
    eager = []
    for _ in range(4):
        step()
        eager.append([t.clone() for t in state])
    for t, s in zip(state, start):
        t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, s in zip(state, start):
        t.copy_(s)
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(state, want):
            assert torch.equal(t, w)
        (c.k.float().sum() + 1).item()
        assert short.item() == 0


@pytest.mark.parametrize("rows", [3000, 65536])
def test_fork_of_the_most_rows(rows):
    """Every row forked twice, dropped or kept: counts of 3000 and 65,536 rows."""
    c = _cache(2 * rows, boxes=False)
    g = torch.Generator().manual_seed(rows)
    pages = torch.randperm(2 * rows, generator=g).to(torch.int32).view(rows, 2).cuda()
    total = torch.randint(0, 65, (rows,), generator=g).to(torch.int32).cuda()
    parent = torch.randint(-2, rows, (rows,), generator=g).to(torch.int32).cuda()
    named = lambda t: (t[:, None] + 31 >= torch.tensor([32, 64], device="cuda"))
    ref = gmm.kv_pool(c)
    ref[pages[named(total)].long()] = 1
    nt, npg = torch.empty_like(total), torch.empty_like(pages)
    gmm.gmm_kv_fork(c, ref, total, pages, parent, nt, npg)
    ok = parent >= 0
    wt = torch.where(ok, total[parent.clamp(min=0).long()], 0)
    wp = torch.where(named(wt), pages[parent.clamp(min=0).long()], -1)
    want = torch.bincount(wp[wp >= 0].long(), minlength=2 * rows).to(torch.int32)
    assert torch.equal(nt, wt) and torch.equal(npg, wp) and torch.equal(ref, want)


def test_binding_checks_sizes_and_types():
    c, small = _cache(10), _cache(10, heads=2)
    ref, ws = gmm.kv_pool(c), gmm.kv_pool_workspace(c, 2)
    t, p, s = _i32([0, 0]), _i32([[0, 1, 2]] * 2), _i32([0])
    nt, npg = _i32([0, 0]), _i32([[0, 1, 2]] * 2)
    good = dict(ref=ref, total=t, pages=p, parent=_i32([0, 1]), total_out=nt, pages_out=npg)
    for kw, err in ((dict(ref=ref[:9]), ValueError), (dict(ref=ref.float()), TypeError),
                    (dict(total=_i32([0])), ValueError), (dict(total=_i32([0, 0, 0])), ValueError),
                    (dict(pages=p.long()), TypeError), (dict(pages=p.t()), TypeError),
                    (dict(parent=_i32([0])), ValueError), (dict(parent=[0, 1]), AttributeError),
                    (dict(keep=_i32([1])), ValueError), (dict(pages_out=npg[:, :2]), gmm.GMMError),
                    (dict(pages_out=p), gmm.GMMError), (dict(total_out=t), gmm.GMMError)):
        with pytest.raises(err):
            gmm.gmm_kv_fork(c, **{**good, **kw})
    for args in ((_i32([0]), t, p, s), (t, t, p, s.long()), (t, t, p, s[:0])):
        with pytest.raises((TypeError, ValueError)):
            gmm.gmm_kv_grow(c, ref, *args, ws)
    with pytest.raises(gmm.GMMError):
        gmm.gmm_kv_grow(c, ref, t, t, p, s, ws[:256])
    with pytest.raises(gmm.GMMError):
        gmm.gmm_kv_copy(c, small, s, s)
    with pytest.raises(ValueError):
        gmm.gmm_kv_copy(c, c, s, _i32([0, 1]))
    with pytest.raises(ValueError):
        gmm.gmm_kv_compact(c, ref, t, p, ref[:5].clone(), s, ws)
    assert (ref == 0).all()
