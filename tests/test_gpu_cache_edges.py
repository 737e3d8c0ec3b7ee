"""Weighing, tree attention and pruning where their kernels take another way: waits that run out,
sequences of fewer slots than new tokens, more caches than are resident at once."""
import pytest
import torch

from paper_2609_06663_gb300 import ecokv as E
from tests.test_gpu_decode import TYPES, Batch, gen, make_prefix

pytestmark = pytest.mark.gpu
D = 128


# ---------------------------------------------------------------- waits that run out
@pytest.mark.parametrize("h_q,h_kv,new,lens,page,rows", [(4, 1, [900, 10], [1000, 10], 64, 5), (28, 4, [61] * 8, [300] * 8, 16, 700)])
def test_weigh_that_gave_up_adds_nothing_left_by_others(h_q, h_kv, new, lens, page, rows):
    """Items that are cut between CTAs, none of which gets a tile: no weight changes, whatever the workspace held."""
    b = Batch(7, h_kv, new, lens, page, "bf16")
    heads, pre = make_prefix(gen(2), [rows] * h_kv, "bf16", False)
    q = torch.randn(b.tokens, h_q, D, generator=gen(1)).bfloat16().cuda()
    lse = torch.full((b.tokens, h_q), 5.0, device="cuda")
    pw, w = torch.rand(h_kv, rows, generator=gen(3)).cuda(), torch.rand(b.k.shape[:3], generator=gen(4)).cuda()
    ws = E.alloc_weigh_workspace(b.tokens, len(new), h_q, h_kv, q.dtype)
    ws[256:].fill_(255)  # (NaN where sums are left)
    got = E.weigh(q, lse, pre, b.cache, pw.clone(), w.clone(), b.starts.cuda(), decay=0.5, ws=ws, timeout_us=2000,
                  flags=E.ECOKV_FLAG_TEST_STALL)
    assert E.ecokv_device_status(ws) == E.ECOKV_ERR_TIMEOUT
    assert torch.equal(got[0], pw) and torch.equal(got[1], w)
    # the next call in this workspace as in a new one
    again = [E.weigh(q, lse, pre, b.cache, pw.clone(), w.clone(), b.starts.cuda(), decay=0.5, ws=x)
             for x in (ws, E.alloc_weigh_workspace(b.tokens, len(new), h_q, h_kv, q.dtype))]
    assert E.ecokv_device_status(ws) == 0
    assert torch.equal(again[0][0], again[1][0]) and torch.equal(again[0][1], again[1][1])
    assert not torch.equal(again[0][1], w)
