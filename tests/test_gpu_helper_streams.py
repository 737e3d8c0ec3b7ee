"""The eviction helpers on a stream that is not torch's current one, with no
workspace given and torch's current stream busy with readers of memory it has given
back; and with no stream given, inside a torch.cuda.stream block.  The same bits
as on the default stream."""
import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from paper_2609_06663_gb300.workloads import make_inputs, small_workload

pytestmark = pytest.mark.gpu


def calls(p, K, V, Q, **kw):
    yield E.score(p, K, Q, **kw)
    yield E.evict(p, K, V, Q, want_scores=True, **kw)
    yield E.evict_adaptive(p, K, V, Q, **kw)
    yield E.evict_layered(p, K, V, Q, [100, 37], **kw)
    yield E.evict_noalloc(p, K, V, Q, **kw)


def same(a, b):
    # (S is read where the helper returns it, the layered rows past a layer's budget are zeros)
    return all(torch.equal(x, y) if isinstance(x, torch.Tensor) else x == y for x, y in zip(a, b))


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_eviction_helpers_run_in_the_order_of_their_stream(how):
    w = small_workload(n=2000, h_kv=2, group=4, window=4, budget=100, n_layers=2, dtype="bf16", seed=8, clustered=True)
    K, V, Q = (x.cuda() for x in make_inputs(w))
    p = E.make_params(n_layers=2, h_kv=2, h_q=8, n=2000, window=4, budget=100)
    want = list(calls(p, K, V, Q))
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        for _ in range(20):
            big @ big
        old = [torch.ones_like(x) for x in want[1] if x is not None]
        kept = [x.clone() for x in old]
        del old
        if how == "current":
            with torch.cuda.stream(side):
                got = list(calls(p, K, V, Q))
        else:
            got = list(calls(p, K, V, Q, stream=side if how == "stream" else side.cuda_stream))
        side.synchronize()
        assert all(same(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        assert all(bool((x == 1).all()) for x in kept)


def test_compaction_and_selection_follow():
    w = small_workload(n=2000, h_kv=2, group=4, window=4, budget=100, n_layers=1, dtype="bf16", seed=9, clustered=True)
    K, V, Q = (x.cuda() for x in make_inputs(w))
    p = E.make_params(n_layers=1, h_kv=2, h_q=8, n=2000, window=4, budget=100)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    idx, k, v, s, _ = E.evict(p, K, V, Q, want_scores=True, stream=side)
    i2 = E.select(p, s, stream=side)
    k2, v2 = E.compact(p, K, V, i2, stream=side)
    side.synchronize()
    assert torch.equal(i2, idx) and torch.equal(k2, k) and torch.equal(v2, v)
