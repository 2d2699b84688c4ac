"""Long-context decoding over a paged key/value cache whose pages hold clusters of keys.

A prompt's keys are clustered with the library's k-means (k-means++ seeding, then Lloyd
iterations), and appended to the cache in cluster order: softmax attention does
not depend on the order of the keys, and every later token sees the whole prompt.  A page then
holds keys that are alike, its box of per-dimension bounds is tight, and a token's query needs
few pages.  Each decoding step is three calls: append (with the rotation of queries and keys),
select, attend.  The same steps over the prompt in its own order, and over every key, say what
the clusters are worth.

    python examples/clustered_cache.py [--prompt 32768] [--steps 16] [--pages-read 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_10896_amd as gmm  # noqa: E402

PAGE, HQ, HK, D, ROT = 64, 32, 8, 128, 32
DEV = "cuda"


def synthetic_prompt(n, topics, seed):
    """Keys around `topics` centres that follow each other in short passages, values, and the
    centres (which queries of later tokens look for)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    centres = torch.randn(topics, HK, D, device=DEV, generator=g)
    passages = torch.randint(topics, ((n + 15) // 16,), device=DEV, generator=g)
    topic = passages.repeat_interleave(16)[:n]
    keys = centres[topic] + 0.5 * torch.randn(n, HK, D, device=DEV, generator=g)
    values = torch.randn(n, HK, D, device=DEV, generator=g)
    return keys.bfloat16(), values.bfloat16(), centres, g


def cluster_order(keys, k, iters=4):
    """Order of the keys by k-means cluster (all heads of a token together), in place of theirs."""
    n = keys.shape[0]
    x = keys.float().reshape(n, -1)
    x = x / x.norm(dim=1, keepdim=True)
    d = x.shape[1]
    seeds = torch.empty(k, dtype=torch.int64, device=DEV)
    centres, var = (torch.empty(k, d, device=DEV) for _ in range(2))
    gmm.gmm_kmeanspp(x, torch.rand(k, dtype=torch.float64, device=DEV), seeds, centres)
    weights = torch.empty(k, device=DEV)
    assign = torch.empty(n, dtype=torch.int32, device=DEV)
    gmm.gmm_kmeans(x, weights, centres, var, iters, assign, gmm.workspace(n, d, k, 1))
    return torch.argsort(assign, stable=True)


class Decoder:
    """One sequence: its cache, page table and rotation table."""

    def __init__(self, max_keys, pages_read):
        pages = (max_keys + PAGE - 1) // PAGE
        self.cache = gmm.kv_cache(pages, HK, PAGE, D)
        self.pages = torch.randperm(pages, device=DEV).to(torch.int32)[None]
        self.table = torch.empty(max_keys, ROT, device=DEV)
        freq = torch.tensor(gmm.rope_frequencies(ROT), dtype=torch.float64, device=DEV)
        gmm.gmm_rope_table(freq, self.table)
        self.total = 0
        self.one = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
        self.sel = torch.empty(1, HK, pages_read, dtype=torch.int32, device=DEV)
        self.ws = gmm.kv_workspace(self.cache, 1, HQ, 1, pages)
        self.q = torch.empty(1, HQ, D, dtype=torch.bfloat16, device=DEV)

    def prompt(self, keys, values, order):
        n = keys.shape[0]
        self.total = n
        cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        total = torch.tensor([n], dtype=torch.int32, device=DEV)
        gmm.gmm_kv_append(self.cache, keys[order].contiguous(), values[order].contiguous(), cu,
                          total, self.pages, pos=order.to(torch.int32), table=self.table)

    def step(self, q, k, v, every_key=False):
        """One new token: its output, after its key and value went into the cache."""
        self.total += 1
        total = torch.tensor([self.total], dtype=torch.int32, device=DEV)
        batch = (self.one, total, self.pages)
        gmm.gmm_kv_append(self.cache, k, v, *batch, table=self.table, q=q, q_out=self.q)
        out = torch.empty_like(self.q)
        lse = torch.empty(1, HQ, device=DEV)
        sel = None
        if not every_key:
            gmm.gmm_kv_select(self.cache, self.q, *batch, self.sel, self.ws)
            sel = self.sel
        gmm.gmm_kv_attend(self.cache, self.q, *batch, out, self.ws, lse=lse, sel=sel)
        return out, lse


def run(prompt=32768, steps=16, pages_read=8, seed=0, say=print):
    """Mean share of the softmax mass that the selected pages hold, and relative error of the
    outputs, for pages in prompt order and in cluster order."""
    topics = max(8, prompt // 128)
    keys, values, centres, g = synthetic_prompt(prompt, topics, seed)
    k = max(8, prompt // 128)
    orders = {"prompt order": torch.arange(prompt, device=DEV),
              "cluster order": cluster_order(keys, k)}
    tokens = []
    for _ in range(steps):
        t = torch.randint(topics, (1,), device=DEV, generator=g)
        q = centres[t].repeat_interleave(HQ // HK, 1) + \
            0.5 * torch.randn(1, HQ, D, device=DEV, generator=g)
        kn = centres[t] + 0.5 * torch.randn(1, HK, D, device=DEV, generator=g)
        vn = torch.randn(1, HK, D, device=DEV, generator=g)
        tokens.append([x.bfloat16() for x in (q, kn, vn)])

    full = Decoder(prompt + steps, pages_read)
    full.prompt(keys, values, orders["prompt order"])
    want = [full.step(*t, every_key=True) for t in tokens]
    result = {}
    for name, order in orders.items():
        dec = Decoder(prompt + steps, pages_read)
        dec.prompt(keys, values, order)
        mass, err = 0.0, 0.0
        for t, (o, l) in zip(tokens, want):
            out, lse = dec.step(*t)
            mass += float(torch.exp(lse - l).mean()) / steps
            err += float((out.float() - o.float()).norm() / o.float().norm()) / steps
        result[name] = (mass, err)
        say(f"{name}: {pages_read} of {(prompt + PAGE - 1) // PAGE} pages hold {100 * mass:.1f} % "
            f"of the softmax mass, relative error of the output {err:.3f}")
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompt", type=int, default=32768)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--pages-read", type=int, default=8)
    ns = ap.parse_args()
    run(ns.prompt, ns.steps, ns.pages_read)
