"""Drafted tokens over an evicted prompt, in a cache that is kept small.

    python examples/draft_trees.py [--tokens 8192] [--batch 16] [--steps 16] [--limit 256] [--budget 192]

The layer, prompt and paged cache of shared_prefix.py.  Every step drafts a tree of
tokens for each sequence (a chain with branches, as a small model would), all of whose
keys and values enter the cache (ecokv_append) and attend to what they follow
(ecokv_tree_mask, ecokv_attend_tree).  Of each tree a path is accepted; its rows
move to the front of the drafts (ecokv_commit), what the accepted tokens' attention gave
each key is added up (ecokv_weigh), and sequences past `limit` slots keep the `budget`
heaviest ones of each head (ecokv_prune).  Random weights: which path is accepted is
drawn.
"""
import argparse
import os
import random
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from shared_prefix import D, H_KV, H_Q, PAGE, Decoder, E, Layer, prefix_of  # noqa: E402

DRAFTS = 12  # of a sequence and step: a chain of six and branches of it
PARENTS = [-1, 0, 1, 2, 3, 4, -1, 0, 0, 1, 2, 3]


def path_to(draft):
    path = []
    while draft >= 0:
        path.append(draft)
        draft = PARENTS[draft]
    return path[::-1]


def run(tokens=8192, batch=16, steps=16, limit=256, budget=192, seed=0, log=print):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    layer = Layer(g)
    rnd = lambda n: torch.randn(n, 1024, generator=g, device="cuda").to(layer.dt)  # noqa: E731
    prefix, _ = prefix_of(layer, rnd(tokens), max(tokens // 10, 8))
    dec = Decoder(layer, prefix, tokens, batch, limit + DRAFTS)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    n = batch * DRAFTS
    starts = ints([DRAFTS * b for b in range(batch + 1)])
    parents = ints(PARENTS * batch)
    depth = ints([len(path_to(i)) - 1 for i in range(DRAFTS)] * batch)
    mask = E.tree_mask(parents, starts, words=1)  # (the same trees in every step)
    weights = torch.zeros(dec.cache.k_pages.shape[:3], device="cuda")
    prefix_weights = torch.zeros(prefix.k.shape[:-1], device="cuda")
    q, out = (torch.empty(n, H_Q, D, dtype=layer.dt, device="cuda") for _ in range(2))
    lse = torch.empty(n, H_Q, device="cuda")
    ws, ws_weigh = (f(n, batch, H_Q, H_KV, layer.dt) for f in (E.alloc_attend_workspace, E.alloc_weigh_workspace))
    written = torch.zeros(batch, dtype=torch.int32, device="cuda")  # tokens of each answer, evicted ones too
    accepted = []
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        pos = (tokens + written.repeat_interleave(DRAFTS) + depth).repeat(3, 1).int()
        dec.lengths += DRAFTS
        qkv = layer.project(rnd(n))
        E.append(dec.cache, qkv[1], qkv[2], starts, layer.rotary, pos, qkv[0], layer.q_norm, layer.k_norm, q_out=q, ws=ws)
        E.attend_tree(q, prefix, dec.cache, mask, starts, out=out, lse=lse, ws=ws)
        paths = [path_to(rng.randrange(DRAFTS)) for _ in range(batch)]  # (a verifier compares `out`'s tokens)
        most = max(len(p) for p in paths)
        counts = ints([len(p) for p in paths])
        E.commit(dec.cache, ints([p + [0] * (most - len(p)) for p in paths]), counts, starts, lengths_out=dec.lengths,
                 ws=ws)
        rows = torch.tensor([DRAFTS * b + i for b, p in enumerate(paths) for i in p], device="cuda")
        E.weigh(q[rows], lse[rows], prefix, dec.cache, prefix_weights, weights,
                torch.cat([counts.new_zeros(1), counts.cumsum(0).int()]), ws=ws_weigh)
        E.prune(dec.cache, weights, budget, limit, first=1, recent=budget // 4, to_weights=weights,
                lengths_out=dec.lengths, ws=ws)
        written += counts
        accepted.append(sum(len(p) for p in paths))
    torch.cuda.synchronize()
    log(f"{steps} steps of {batch} trees of {DRAFTS}: {(time.perf_counter() - t) / steps * 1e6:.1f} us a step, "
        f"{sum(accepted) / steps / batch:.2f} tokens a sequence; {PAGE}-slot pages, lengths {dec.lengths.tolist()}")
    for x in (ws, ws_weigh):
        status = E.ecokv_device_status(x)
        if status:
            raise E.EcokvError(status, "decode")
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(prefix_weights).all())
    return dec.lengths, accepted


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("tokens", 8192), ("batch", 16), ("steps", 16), ("limit", 256), ("budget", 192)):
        ap.add_argument(f"--{name}", type=int, default=default)
    run(**vars(ap.parse_args()))
