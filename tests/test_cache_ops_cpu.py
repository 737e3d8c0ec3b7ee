"""Drafted tokens and a cache that shrinks, on the host: argument errors returned before
anything is launched (fake pointers, never dereferenced)."""
import math
import os

import pytest

from paper_2609_06663_gb300 import ecokv as E
from tests.test_decode_cpu import FAKE, pages, params, prefix


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(E.LIB_PATH):
        from paper_2609_06663_gb300 import build
        build.build()
    return E.lib()


def weights(**kw):
    d = dict(w=FAKE, page_stride=64, head_stride=16, slot_stride=1)
    d.update(kw)
    return E.ecokv_weights(*(d[n] for n, _ in E.ecokv_weights._fields_))


BAD_PAGES = [(dict(k=None), 1), (dict(v=FAKE + 8), 1), (dict(table=None), 1), (dict(page_size=24), 1),
             (dict(n_pages=0), 1), (dict(table_stride=0), 1), (dict(page_stride=0), 1), (dict(head_stride=-128), 1),
             (dict(slot_stride=132), 1), (dict(page_size=4096, table_stride=4097), 2)]
BAD_WEIGHTS = [dict(w=None), dict(w=FAKE + 2), dict(page_stride=0), dict(head_stride=-1), dict(slot_stride=0)]


def test_tree_mask_refuses_arguments():
    call = E.ecokv_tree_mask
    assert call(None, FAKE, 4, 2, FAKE, 1) == 1
    assert call(FAKE, FAKE, 4, 2, None, 1) == 1
    assert call(FAKE + 2, FAKE, 4, 2, FAKE, 1) == 1
    assert call(FAKE, FAKE + 1, 4, 2, FAKE, 1) == 1
    assert call(FAKE, FAKE, 4, 2, FAKE + 4, 1) == 1
    assert call(FAKE, FAKE, -1, 2, FAKE, 1) == 1
    assert call(FAKE, FAKE, 4, 0, FAKE, 1) == 1
    assert call(FAKE, FAKE, 4, 2, FAKE, 0) == 1
    assert call(FAKE, None, 4, 2, FAKE, 1) == 1          # one draft a sequence
    assert call(FAKE, FAKE, 4, 2, FAKE, 65) == 2
    assert call(FAKE, FAKE, 4, 2, FAKE, 1, FAKE, 255) == 3
    assert call(FAKE, FAKE, 4, 2, FAKE, 1, FAKE + 4, 256) == 3
    assert call(None, None, 0, 2, None, 1) == 0          # nothing to do


def test_attend_tree_refuses_arguments():
    ws = E.ecokv_attend_workspace_size(2, 2, 8, 4, 1)

    def call(p=None, c=pages(), mask=FAKE, words=1, q=FAKE, out=FAKE, starts=None, n=ws, pre=None, dt=1):
        return E.ecokv_attend_tree(p or params(), dt, q, pre, c, starts, mask, words, out, None, FAKE, n)
    assert call(c=None) == 1 and call(mask=None) == 1 and call(mask=FAKE + 4) == 1
    assert call(words=0) == 1 and call(words=-1) == 1 and call(words=65) == 2
    assert call(q=None) == 1 and call(out=FAKE + 8) == 1 and call(dt=3) == 1 and call(starts=FAKE + 2) == 1
    assert call(n=ws - 1) == 3 and call(p=params(d=64)) == 2 and call(p=params(h_q=9)) == 1
    assert call(pre=prefix(rows=-1)) == 1
    assert call(p=params(tokens=3)) == 1
    assert call(p=params(tokens=0), mask=None) == 0
    for kw, code in BAD_PAGES:
        assert call(c=pages(**kw)) == code


def test_commit_refuses_arguments():
    def call(dt=1, c=pages(), h_kv=4, acc=FAKE, stride=4, counts=FAKE, starts=None, tokens=2, batch=2, w=None,
             out=1 << 24, ws=None, n=0):
        return E.ecokv_commit(dt, c, h_kv, acc, stride, counts, starts, tokens, batch, w, out, ws, n)
    assert call(dt=2) == 1 and call(h_kv=0) == 1 and call(acc=None) == 1 and call(stride=0) == 1
    assert call(counts=FAKE + 1) == 1 and call(starts=FAKE + 2) == 1 and call(tokens=3) == 1 and call(tokens=-1) == 1
    assert call(batch=0, tokens=0) == 1 and call(out=None) == 1 and call(out=FAKE + 4) == 1 and call(c=None) == 1
    assert call(ws=FAKE, n=255) == 3 and call(h_kv=(1 << 28) + 1) == 2
    # the lengths are written while others read the lists: they lie apart (but for the cache's own)
    far = 1 << 24
    assert call(counts=far) == 1 and call(counts=far + 4) == 1 and call(acc=far - 28) == 1 and call(starts=far - 8) == 1
    assert call(counts=far + 8, acc=far - 32, starts=far - 12, ws=FAKE, n=0) == 3
    for kw in BAD_WEIGHTS:
        assert call(w=weights(**kw)) == 1
    for kw, code in BAD_PAGES:
        assert call(c=pages(**kw)) == code


def weigh_params(**kw):
    d = dict(h_q=8, h_kv=4, d=128, tokens=2, batch=2, scale=0.0, decay=1.0, q_token=1024, q_head=128, flags=0,
             timeout_us=0)
    d.update(kw)
    return E.ecokv_weigh_params(*(d[n] for n, _ in E.ecokv_weigh_params._fields_))


@pytest.mark.parametrize("kw,code", [
    (dict(h_q=9), 1), (dict(h_kv=0), 1), (dict(tokens=-1), 1), (dict(batch=0), 1), (dict(d=64), 2), (dict(d=0), 1),
    (dict(h_q=260, h_kv=4), 2), (dict(scale=math.nan), 1), (dict(decay=math.inf), 1), (dict(decay=-0.5), 1),
    (dict(decay=math.nan), 1), (dict(q_token=0), 1), (dict(q_head=4), 1), (dict(flags=1), 1), (dict(tokens=3), 1)])
def test_weigh_refuses_parameters(kw, code):
    assert E.ecokv_weigh(weigh_params(**kw), 1, FAKE, FAKE, None, pages(), None, None, weights(), FAKE, 1 << 30) == code


def test_weigh_refuses_arguments():
    n = E.ecokv_weigh_workspace_size(2, 2, 8, 4, 1)
    assert n > 0 and E.ecokv_weigh_workspace_size(2, 2, 9, 4, 1) == 0 and E.ecokv_weigh_workspace_size(2, 0, 8, 4, 1) == 0

    def call(p=None, dt=1, q=FAKE, lse=FAKE, pre=prefix(), c=pages(), starts=None, pw=weights(), w=weights(), ws=FAKE,
             n=n):
        return E.ecokv_weigh(p or weigh_params(), dt, q, lse, pre, c, starts, pw, w, ws, n)
    assert call(dt=2) == 1 and call(q=None) == 1 and call(q=FAKE + 8) == 1 and call(lse=None) == 1 and call(lse=FAKE + 2) == 1
    assert call(pw=None) == 1 and call(w=None) == 1 and call(starts=FAKE + 2) == 1
    assert call(ws=None) == 3 and call(n=n - 1) == 3 and call(ws=FAKE + 8) == 3
    assert call(dt=0, p=weigh_params(flags=E.ECOKV_FLAG_TEST_STALL)) == 2
    assert call(p=weigh_params(tokens=0), q=None, lse=None) == 0
    for kw in BAD_WEIGHTS:
        assert call(w=weights(**kw)) == 1
    for kw in (dict(w=None), dict(w=FAKE + 2), dict(head_stride=-1), dict(slot_stride=0)):
        assert call(pw=weights(**kw)) == 1
    for kw, code in BAD_PAGES:
        if "v" not in kw:  # (not read)
            assert call(c=pages(**kw)) == code
    for kw, code in ((dict(k=None), 1), (dict(head_stride=100), 1), (dict(row_stride=0), 1), (dict(rows=-1), 1),
                     (dict(rows=(1 << 24) + 1), 2), (dict(head_off=FAKE + 2), 1)):
        assert call(pre=prefix(**kw)) == code


@pytest.mark.parametrize("dtype,flags", [(1, 0), (1, E.ECOKV_FLAG_FORCE_SIMT), (0, 0)])
@pytest.mark.parametrize("group", [1, 7, 8, 64])
@pytest.mark.parametrize("tokens,page,cols,rows", [(100000, 4096, 256, 0), (4096, 4096, 4096, 0), (10, 8, 1, 0),
                                                   (10000, 16, 8192, 131072), (1 << 20, 16, 4, 1 << 24)])
def test_weigh_size_limit(tokens, page, cols, rows, group, dtype, flags):
    """Taken up to the header's bound, refused far past it (no workspace is given: nothing is launched)."""
    h_kv, n, k = 2, tokens * group, lambda keys: -(-keys // 128)
    room = (2 ** 31 - 1) // h_kv - k(rows) * (32 + n)
    most = (room // k(page * cols) - n - 48) // 40
    c = pages(page_size=page, table_stride=cols, page_stride=h_kv * page * 128, head_stride=page * 128)

    def call(batch):
        p = weigh_params(h_q=h_kv * group, h_kv=h_kv, tokens=tokens, batch=batch, flags=flags)
        return E.ecokv_weigh(p, dtype, FAKE, FAKE, prefix(rows=rows, head_stride=max(rows, 1) * 128), c, FAKE, weights(),
                             weights(), FAKE, 0)
    if most >= 1:
        assert call(min(most, 2 ** 31 - 1)) == 3
    if cols > 1:
        assert call(2 ** 31 - 1) == 2


def prune_params(**kw):
    d = dict(h_kv=4, batch=2, budget=20, limit=30, first=4, recent=8)
    d.update(kw)
    return E.ecokv_prune_params(*(d[n] for n, _ in E.ecokv_prune_params._fields_))


@pytest.mark.parametrize("kw,code", [
    (dict(h_kv=0), 1), (dict(batch=0), 1), (dict(budget=0, first=0, recent=0), 1), (dict(limit=19), 1), (dict(first=-1), 1),
    (dict(recent=-1), 1), (dict(first=13), 1), (dict(recent=2 ** 31 - 1, first=1), 1), (dict(h_kv=1 << 29, batch=2), 2)])
def test_prune_refuses_parameters(kw, code):
    assert E.ecokv_prune(prune_params(**kw), 1, pages(), weights(), None, None, FAKE, 1 << 24) == code


def test_prune_refuses_arguments():
    def call(dt=1, c=pages(), w=weights(), to=None, tw=None, idx=1 << 26, out=1 << 24, ws=None, n=0):
        return E.ecokv_prune(prune_params(), dt, c, w, to, tw, idx, out, ws, n)
    assert call(dt=2) == 1 and call(w=None) == 1 and call(idx=None) == 1 and call(idx=(1 << 26) + 1) == 1
    assert call(out=None) == 1 and call(out=FAKE + 4) == 1 and call(out=FAKE + 2) == 1 and call(c=None) == 1
    assert call(ws=FAKE, n=255) == 3
    # in the same cache weights move within their tensor
    assert call(tw=weights(w=FAKE + 4)) == 1 and call(tw=weights(page_stride=128)) == 1
    assert call(tw=weights(), ws=FAKE, n=0) == 3 and call(to=pages(), tw=weights(w=FAKE + 4), ws=FAKE, n=0) == 3
    # the slots' list apart from both lengths
    assert call(idx=(1 << 24) + 4) == 1 and call(idx=FAKE - 4) == 1
    for kw in BAD_WEIGHTS:
        assert call(w=weights(**kw)) == 1 and call(tw=weights(**kw)) == 1
    for kw, code in BAD_PAGES:
        assert call(c=pages(**kw)) == code and call(to=pages(**kw)) == code


def test_helpers_want_cuda_tensors():
    import torch
    with pytest.raises(ValueError):
        E.tree_mask(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        E.attend_tree(torch.zeros(2, 4, 128), None, None, torch.zeros(2, 1, dtype=torch.int64))
    with pytest.raises(ValueError):
        E.weigh(torch.zeros(2, 4, 128), torch.zeros(2, 4), None, None)


@pytest.mark.parametrize("dtype,flags", [(1, 0), (1, E.ECOKV_FLAG_FORCE_SIMT), (0, 0)])
@pytest.mark.parametrize("group", [1, 2, 7, 32, 64])
@pytest.mark.parametrize("tokens,page,cols,rows", [(2560, 4096, 4096, 0), (40, 4096, 4096, 0), (1, 4096, 4096, 1000),
                                                   (300, 16, 8192, 100)])
def test_attend_tree_size_limit(tokens, page, cols, rows, group, dtype, flags):
    """The header's count of work, whichever tiles the call is cut in (no workspace is given: nothing is launched)."""
    tc = dtype == 1 and not flags
    n = -(-tokens // (2 * (128 // group) if tc else 64 // group))
    u = lambda keys: (2 * -(-keys // 128) + 4 if tc else -(-keys // 128)) if keys else 0  # noqa: E731
    most = (2 ** 31 - 1 - n * u(rows)) // u(page * cols) - n
    for batch, code in ((most, 3), (most + 1, 2)):
        p = params(h_q=group, h_kv=1, tokens=tokens, batch=batch, flags=flags)
        c = pages(page_size=page, table_stride=cols, page_stride=page * 128, head_stride=page * 128)
        pre = prefix(rows=rows, head_stride=max(rows, 1) * 128)
        assert E.ecokv_attend_tree(p, dtype, FAKE, pre, c, FAKE, FAKE, 1, FAKE, None, FAKE, 0) == code, batch
