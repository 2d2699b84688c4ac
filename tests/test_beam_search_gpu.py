"""A beam search as a user runs it: selection, fork, growth, append, attention, logits, step after
step, against every beam's own words.  The keys and values that a beam attends to are those of its
words, whichever pages hold them."""
import math
from types import SimpleNamespace

import pytest
import torch

import paper_2606_10896_amd as gmm
from kvcheck import attend64, rope64
from poolcheck import INF, check_beam

pytestmark = pytest.mark.gpu

VOCAB, D, HQ, HK, PAGE, WIDTH = 211, 32, 4, 2, 32, 5


class Model:
    """Tables in place of a network: a word's query, key and value, and a projection to words."""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g)
        self.q, self.k, self.v = (rn(VOCAB, h, D).bfloat16() for h in (HQ, HK, HK))
        self.head = (rn(HQ * D, VOCAB) * 0.7).cuda()
        self.freq = torch.tensor(gmm.rope_frequencies(D), dtype=torch.float64, device="cuda")
        self.table = torch.empty(PAGE * WIDTH, D, device="cuda")
        gmm.gmm_rope_table(self.freq, self.table)

    def expected(self, words):
        """attend64 of the last word of every row, from the rows' words alone."""
        keys, vals, q = [], [], []
        for w in words:
            t = torch.tensor(w)
            pos, tb = torch.arange(len(w)), self.table.cpu()
            keys.append(rope64(self.k[t], pos, tb).bfloat16().transpose(0, 1))
            vals.append(self.v[t].transpose(0, 1))
            q.append(rope64(self.q[t[-1:]], pos[-1:], tb).bfloat16())
        bt = SimpleNamespace(hq=HQ, hk=HK, d=D, dt=torch.bfloat16, rows=len(words), page=PAGE,
                             q=torch.cat(q), row_seq=list(range(len(words))),
                             row_slot=[len(w) - 1 for w in words], keys=keys, vals=vals)
        return attend64(bt, 1 / math.sqrt(D))


def test_beam_search():
    batch, beams, steps, eos = 3, 4, 40, 7
    rows = batch * beams
    m = Model(1)
    cache = gmm.kv_cache(60, HK, PAGE, D)
    cache.k.fill_(math.nan)
    cache.v.fill_(math.nan)
    ref = gmm.kv_pool(cache)
    pool_ws = gmm.kv_pool_workspace(cache, rows)
    ws = gmm.kv_workspace(cache, 100, HQ, rows, WIDTH)
    beam_ws = gmm.beam_workspace(batch, beams, VOCAB)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    tables = [(i32(rows), i32(rows, WIDTH) - 1) for _ in range(2)]
    short = i32(1)
    word_of = lambda t: t.clamp(min=0).cpu().long()

    def attend(tokens, cu, total, pages):
        """Appends the words and attends; rows of logits."""
        n = len(tokens)
        q, k, v = (t[tokens].cuda() for t in (m.q, m.k, m.v))
        q_rot, out = torch.empty_like(q), torch.empty_like(q)
        gmm.gmm_kv_append(cache, k, v, cu, total, pages, table=m.table, q=q, q_out=q_rot)
        gmm.gmm_kv_attend(cache, q_rot, cu, total, pages, out, ws)
        return out, out.float().view(n, -1) @ m.head

    # prompts, one row each, grown and appended at once
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(VOCAB, (n,), generator=g).tolist() for n in (33, 1, 64)]
    lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
    first_pages = i32(batch, WIDTH) - 1
    gmm.gmm_kv_grow(cache, ref, i32(batch), lens, first_pages, short, pool_ws)
    cu = torch.cat([i32(1), lens.cumsum(0).to(torch.int32)])
    out, logits = attend(torch.tensor(sum(prompts, [])), cu, lens, first_pages)
    last = cu[1:].long() - 1
    # the rows of a prompt's beams share its pages; one of them is live
    gmm.gmm_kv_fork(cache, ref, lens, first_pages,
                    torch.arange(batch, dtype=torch.int32, device="cuda").repeat_interleave(beams),
                    *tables[0])
    words = [list(p) for p in prompts for _ in range(beams)]
    score = torch.full((batch, beams), -INF, device="cuda")
    score[:, 0] = 0.0
    done = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    logits = logits[last].repeat_interleave(beams, 0).view(batch, beams, VOCAB)
    cur, cu = 0, torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    for step in range(steps):
        if step > 8:
            logits[:, :, eos] += 2.0
        new_score = torch.empty(batch, beams, device="cuda")
        parent, token = i32(batch, beams), i32(batch, beams)
        new_done = torch.empty_like(done)
        weight = torch.where(done, 1.0 / (step + 1), 1.0 / (step + 2))
        gmm.gmm_beam_select(logits, score, new_score, parent, token, beam_ws, done=done,
                            out_done=new_done, eos=eos, weight=weight)
        check_beam((new_score, parent, token, new_done), logits, score, beams, weight=weight,
                   done=done, eos=eos)
        score, done = new_score, new_done
        (old_t, old_p), (held, pages) = tables[cur], tables[1 - cur]
        cur = 1 - cur
        gmm.gmm_kv_fork(cache, ref, old_t, old_p, parent.view(-1), held, pages)
        total = held + 1
        gmm.gmm_kv_grow(cache, ref, held, total, pages, short, pool_ws)
        assert short.item() == 0
        words = [words[p] + [t] for p, t in zip(parent.view(-1).tolist(), token.view(-1).tolist())]
        out, logits = attend(word_of(token.view(-1)), cu, total, pages)
        logits = logits.view(batch, beams, VOCAB)
        tables[cur] = (total, pages)
        want, _, tol, _ = m.expected(words)
        assert bool(((out.cpu().double() - want).abs() <= tol).all()), step
        assert bool((ref >= 0).all()) and int(ref.sum()) == sum(-(-len(w) // PAGE) for w in words)
        if step % 13 == 12:
            # the pool is pushed together under way
            where, used = i32(cache.pages), i32(1)
            gmm.gmm_kv_compact(cache, ref, total, pages, where, used, pool_ws)
            assert bool((ref[:used.item()] > 0).all()) and not ref[used.item():].any()
    assert bool(done.any()), "no beam has met the end word"
    gmm.gmm_kv_fork(cache, ref, *tables[cur], i32(0), i32(0), i32(0, WIDTH))
    assert not ref.any()


def test_requests_moved_to_another_cache_and_back():
    """The pages of a row are copied out, given up, and brought back to other places."""
    g = torch.Generator(device="cuda").manual_seed(0)
    cache, store = gmm.kv_cache(20, HK, PAGE, D), gmm.kv_cache(9, HK, PAGE, D)
    ref, ws, short = gmm.kv_pool(cache), gmm.kv_pool_workspace(cache, 2), None
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    short, total, pages = i32([0]), i32([100, 70]), i32([[-1] * WIDTH] * 2)
    gmm.gmm_kv_grow(cache, ref, i32([0, 0]), total, pages, short, ws)
    k, v = (torch.randn(170, HK, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    gmm.gmm_kv_append(cache, k, v, i32([0, 100, 170]), total, pages)
    q = torch.randn(2, HQ, D, generator=g, device="cuda").bfloat16()
    attn_ws = gmm.kv_workspace(cache, 2, HQ, 2, WIDTH)

    def look(t, p):
        out = torch.empty_like(q)
        gmm.gmm_kv_attend(cache, q[:t.numel()], i32(list(range(t.numel() + 1))), t, p,
                          out[:t.numel()], attn_ws)
        return out[:t.numel()]

    want = look(total, pages)
    slots = torch.arange(4, dtype=torch.int32, device="cuda") + 3
    gmm.gmm_kv_copy(cache, store, pages[0, :4].contiguous(), slots)
    left_t, left_p = i32([0]), i32([[0] * WIDTH])
    gmm.gmm_kv_fork(cache, ref, total, pages, i32([1]), left_t, left_p)
    assert ref.sum().item() == 3
    # another request takes the pages that became free
    other = i32([[-1] * WIDTH])
    gmm.gmm_kv_grow(cache, ref, i32([0]), i32([60]), other, short, ws)
    cache.k[other[0, :2].long()] = 5.0
    back = i32([[-1] * WIDTH])
    gmm.gmm_kv_grow(cache, ref, i32([0]), i32([100]), back, short, ws)
    gmm.gmm_kv_copy(store, cache, slots, back[0, :4].contiguous())
    got = look(i32([100, 70]), torch.cat([back, left_p]))
    assert short.item() == 0 and torch.equal(got, want)
