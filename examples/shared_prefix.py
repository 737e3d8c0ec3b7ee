"""Several questions about one video: evict its cache once, then decode a batch over it.

    python examples/shared_prefix.py [--tokens 8192] [--batch 16] [--steps 32]

One attention layer of the GQA shape (28 query heads, 4 KV heads), random weights.
The prompt's queries and keys are normed and rotated (ecokv_rotate), the eviction
pass keeps a tenth of them (ecokv_evict), and each sequence then asks a question of
its own length: its tokens enter a paged cache (ecokv_append) and attend to the shared
prefix and to their own past (ecokv_attend).  Decode steps follow, one token a
sequence, captured in a CUDA graph that is replayed as the lengths grow.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2609_06663_gb300 import ecokv as E  # noqa: E402

H_Q, H_KV, D, WINDOW, PAGE = 28, 4, 128, 8, 16


class Layer:
    """An attention layer: one projection to queries, keys and values, norms per head, rotary positions."""

    def __init__(self, g, dt=torch.bfloat16):
        self.dt = dt
        self.w = (torch.randn(1024, (H_Q + 2 * H_KV) * D, generator=g, device="cuda") / 32).to(dt)
        self.q_norm, self.k_norm = ((1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt) for _ in range(2))
        # time, height and width positions
        self.rotary = E.rotary(D, 1e6, sections=(16, 24, 24))

    def project(self, x):
        qkv = (x @ self.w).view(x.shape[0], H_Q + 2 * H_KV, D)
        return qkv[:, :H_Q], qkv[:, H_Q:H_Q + H_KV], qkv[:, H_Q + H_KV:]


def prefix_of(layer, x, budget):
    """The prompt's kept keys and values: an E.Prefix and the tensors it stands on."""
    n = x.shape[0]
    q, k, v = layer.project(x)
    pos = torch.arange(n, device="cuda", dtype=torch.int32).repeat(3, 1)
    # keys straight into the [heads, tokens, d] that the eviction pass reads
    keys = torch.empty(1, H_KV, n, D, dtype=layer.dt, device="cuda")
    q_win = torch.empty(1, H_Q, WINDOW, D, dtype=layer.dt, device="cuda")
    E.rotate(layer.rotary, pos, k, q_norm=layer.k_norm, q_out=keys[0].transpose(0, 1))
    E.rotate(layer.rotary, pos[:, -WINDOW:].contiguous(), q[-WINDOW:], q_norm=layer.q_norm,
             q_out=q_win[0].transpose(0, 1))
    p = E.make_params(n_layers=1, h_kv=H_KV, h_q=H_Q, n=n, window=WINDOW, budget=budget)
    idx, k_kept, v_kept, _, _ = E.evict(p, keys, v.transpose(0, 1).contiguous()[None], q_win)
    return E.Prefix(k_kept[0], v_kept[0]), idx


class Decoder:
    """A batch of sequences over one shared prefix."""

    def __init__(self, layer, prefix, prompt, batch, room):
        self.layer, self.prefix, self.prompt, self.batch = layer, prefix, prompt, batch
        cols = -(-room // PAGE)
        pages = torch.zeros(batch * cols, H_KV, PAGE, D, dtype=layer.dt, device="cuda")
        # (a serving system hands pages out as sequences grow; here each has its own from the start)
        table = torch.randperm(batch * cols, device="cuda").int().view(batch, cols)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.cache = E.PagedCache(pages, torch.zeros_like(pages), table, self.lengths)
        self.ws = {}

    def forward(self, x, starts, pos, q_buf, out):
        """New tokens x (those of sequence b: starts[b] .. starts[b + 1] - 1; starts None: one each); self.lengths
        counts them already.  Returns the attention's output [tokens, H_Q, D]."""
        q, k, v = self.layer.project(x)
        ws = self.ws.get(x.shape[0])
        if ws is None:
            ws = self.ws[x.shape[0]] = E.alloc_attend_workspace(x.shape[0], self.batch, H_Q, H_KV, self.layer.dt)
        E.append(self.cache, k, v, starts, self.layer.rotary, pos, q, self.layer.q_norm, self.layer.k_norm,
                 q_out=q_buf, ws=ws)
        return E.attend(q_buf, self.prefix, self.cache, starts, out=out, ws=ws)


def run(tokens=8192, batch=16, steps=32, seed=0, log=print):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    layer = Layer(g)
    rnd = lambda n: torch.randn(n, 1024, generator=g, device="cuda").to(layer.dt)  # noqa: E731
    prefix, idx = prefix_of(layer, rnd(tokens), max(tokens // 10, WINDOW))
    log(f"prefix: {idx.shape[-1]} of {tokens} rows a head")

    # the questions, 3 to 40 tokens each, all at once
    new = [3 + (7 * b) % 38 for b in range(batch)]
    dec = Decoder(layer, prefix, tokens, batch, max(new) + steps + 1)
    starts = torch.tensor([0] + new).cumsum(0).int().cuda()
    pos = torch.cat([torch.arange(n) + tokens for n in new]).int().cuda().repeat(3, 1)
    dec.lengths += torch.tensor(new, dtype=torch.int32, device="cuda")
    n = sum(new)
    out = dec.forward(rnd(n), starts, pos, torch.empty(n, H_Q, D, dtype=layer.dt, device="cuda"), None)
    last = out[starts[1:].long() - 1]

    # decode: the answer's tokens, one graph replayed
    x, q_buf, out = rnd(batch), torch.empty_like(last), torch.empty_like(last)
    pos = (tokens + dec.lengths).repeat(3, 1)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    dec.lengths += 1
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dec.forward(x, None, pos, q_buf, out)  # (kernels and workspaces are set up; the replay writes the same slots)
        with torch.cuda.graph(graph, stream=side):
            dec.forward(x, None, pos, q_buf, out)
    torch.cuda.current_stream().wait_stream(side)
    outs = []
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        graph.replay()
        outs.append(out.clone())
        x.copy_(out.reshape(batch, -1)[:, :1024] + x)  # the next token's input, made of this one's output
        dec.lengths += 1
        pos += 1
    torch.cuda.synchronize()
    log(f"{steps} steps of {batch} sequences: {(time.perf_counter() - t) / steps * 1e6:.1f} us a step")
    status = E.ecokv_device_status(dec.ws[batch])
    if status:
        raise E.EcokvError(status, "decode")
    return last, torch.stack(outs), dec


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    _, outs, _ = run(a.tokens, a.batch, a.steps)
    assert bool(torch.isfinite(outs).all()) and math.isfinite(float(outs.float().norm()))
