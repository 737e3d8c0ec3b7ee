"""The operators as they are used together: prompts evicted by the library, their
rows read as a shared prefix, and examples/shared_prefix.py."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from paper_2609_06663_gb300.workloads import make_inputs, small_workload
from tests.decode_ref import attend as ref_attend
from tests.test_gpu_decode import Batch, check_attend, gen

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def evicted(adaptive, dtype="bf16", n=900, h_kv=4, group=7, budget=150):
    w = small_workload(n=n, h_kv=h_kv, group=group, window=4, budget=budget, dtype=dtype, seed=5, clustered=True)
    K, V, Q = (x.cuda() for x in make_inputs(w))
    p = E.make_params(n_layers=1, h_kv=h_kv, h_q=w.h_q, n=n, window=4, budget=budget)
    if not adaptive:
        _, k, v, _, _ = E.evict(p, K, V, Q)
        return E.Prefix(k[0], v[0]), [(k[0, h].cpu(), v[0, h].cpu()) for h in range(h_kv)]
    _, off, k, v, _ = E.evict_adaptive(p, K, V, Q)
    o = off[0].tolist()
    return E.Prefix(k[0], v[0], off[0]), [(k[0, o[h]:o[h + 1]].cpu(), v[0, o[h]:o[h + 1]].cpu()) for h in range(h_kv)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("adaptive", [False, True])
def test_attend_over_an_evicted_prompt(adaptive, dt):
    pre, heads = evicted(adaptive, dt)
    b = Batch(3, 4, [1, 3, 1, 2], [40, 3, 300, 17], 16, dt)
    check_attend(b, heads, pre, 28, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_layered_budget_rows_as_prefixes(dt):
    """A layered call's layers: heads of a common stride, each layer its own number of rows."""
    w = small_workload(n=500, h_kv=2, group=4, window=4, budget=120, n_layers=3, dtype=dt, seed=8)
    K, V, Q = (x.cuda() for x in make_inputs(w))
    p = E.make_params(n_layers=3, h_kv=2, h_q=8, n=500, window=4, budget=120)
    budgets = [120, 70, 9]
    _, k, v, _, _ = E.evict_layered(p, K, V, Q, budgets)
    b = Batch(4, 2, [1, 1], [10, 150], 32, dt)
    for layer, n in enumerate(budgets):
        heads = [(k[layer, h, :n].cpu(), v[layer, h, :n].cpu()) for h in range(2)]
        check_attend(b, heads, E.Prefix(k[layer, :, :n], v[layer, :, :n]), 8, dt)


def test_example_decodes_what_the_definitions_say():
    spec = importlib.util.spec_from_file_location("shared_prefix", os.path.join(ROOT, "examples", "shared_prefix.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    steps, batch = 5, 6
    _, outs, dec = ex.run(tokens=700, batch=batch, steps=steps, log=lambda *_: None)
    # the cache at the end holds every key the steps appended: the last step again from the definition
    lens = (dec.lengths - 1).tolist()
    table, kp, vp = dec.cache.table.cpu(), dec.cache.k_pages.cpu(), dec.cache.v_pages.cpu()
    own = []
    for b, n in enumerate(lens):
        ids = table[b, :-(-n // ex.PAGE)].long()
        own.append(tuple(x[ids].transpose(0, 1).reshape(ex.H_KV, -1, ex.D)[:, :n] for x in (kp, vp)))
    heads = [(dec.prefix.k[h].cpu(), dec.prefix.v[h].cpu()) for h in range(ex.H_KV)]
    # the queries of the last step: run it again at the same lengths
    q = torch.empty(batch, ex.H_Q, ex.D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    x = torch.randn(batch, 1024, generator=gen(1)).bfloat16().cuda()
    dec.lengths -= 1
    pos = (700 + dec.lengths - 1).repeat(3, 1).int()
    got = dec.forward(x, None, pos, q, out)
    own = [(torch.cat([k[:, :-1], dec.cache.k_pages[int(table[b, (lens[b] - 1) // ex.PAGE]), :, (lens[b] - 1) % ex.PAGE]
                       .cpu()[:, None]], 1),
            torch.cat([v[:, :-1], dec.cache.v_pages[int(table[b, (lens[b] - 1) // ex.PAGE]), :, (lens[b] - 1) % ex.PAGE]
                       .cpu()[:, None]], 1)) for b, (k, v) in enumerate(own)]
    want, size, _, mag = ref_attend(q.cpu(), heads, own, [1] * batch, 1 / math.sqrt(ex.D))
    tol = (2 * (140 * mag + 40) * 2.0 ** -24 + 2.0 ** -8) * size + 2.0 ** -8 * want.abs() * (1 + 2 ** -7)
    assert bool(((got.cpu().double() - want).abs() <= tol).all())
    assert bool(torch.isfinite(outs).all())
