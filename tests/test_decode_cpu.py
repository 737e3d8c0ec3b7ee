"""The decode step's entry points on the host: frequencies, and argument errors
returned before anything is launched (fake pointers, never dereferenced)."""
import ctypes
import math
import os

import pytest

from paper_2609_06663_gb300 import ecokv as E
from tests.decode_ref import frequencies

FAKE = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(E.LIB_PATH):
        from paper_2609_06663_gb300 import build
        build.build()
    return E.lib()


@pytest.mark.parametrize("rot,base,scaling,factor,original", [
    (128, 1e4, "none", 1.0, 0), (64, 1e6, "linear", 4.0, 0), (96, 5e5, "ntk", 8.0, 0), (128, 1e6, "yarn", 4.0, 32768),
    (16, 1e4, "yarn", 8.0, 8192), (32, 1e4, "yarn", 2.0, 100), (112, 1e4, "none", 1.0, 0)])
def test_frequencies_follow_their_formulas(rot, base, scaling, factor, original):
    r = E.rotary(rot, base, scaling=scaling, factor=factor, original=original)
    want, mag = frequencies(rot, base, scaling, factor, original)
    for f, w in enumerate(want):
        turns = w / (2 * math.pi) % 1.0
        # two libraries' pow, a quotient and the cut to 2^-64: a few units in the last of 53 bits
        assert abs(r.turns[f] / 2 ** 64 - turns) <= 8 * 2.0 ** -53 * turns + 2.0 ** -63
    assert abs(r.magnitude - mag) <= 2.0 ** -22 and r.axes == 1 and not any(r.axis[:rot // 2])


def test_own_frequencies_and_sections():
    r = E.rotary(32, inv_freq=[0.5 / (i + 1) for i in range(16)], magnitude=1.5, sections=(4, 6, 6))
    assert list(r.axis)[:16] == [0] * 4 + [1] * 6 + [2] * 6 and r.axes == 3 and r.magnitude == 1.5
    assert abs(r.turns[3] / 2 ** 64 - 0.125 / (2 * math.pi)) < 1e-16
    # whole turns a position do not count, and a frequency may be negative
    r = E.rotary(16, inv_freq=[2 * math.pi * 3 + 0.25, -0.25] + [0.0] * 6)
    assert abs(r.turns[0] / 2 ** 64 - 0.25 / (2 * math.pi)) < 1e-14
    assert abs(r.turns[1] / 2 ** 64 - (1 - 0.25 / (2 * math.pi))) < 1e-14 and r.turns[2] == 0


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(base=0.0), dict(base=1.0),
                                dict(base=math.inf), dict(scaling="linear", factor=0.0),
                                dict(scaling="yarn", factor=2.0, original=0), dict(sections=(60, 3)),
                                dict(sections=(10, 10, 10, 10, 24)), dict(sections=(-1, 65)), dict(magnitude=math.nan,
                                inv_freq=[0.1] * 64), dict(inv_freq=[math.inf] * 64)])
def test_rotary_refusals(kw):
    with pytest.raises(E.EcokvError) as e:
        E.rotary(**kw)
    assert e.value.code == 1


def test_rotary_needs_a_frequency_for_every_pair():
    with pytest.raises(ValueError):
        E.rotary(128, inv_freq=[0.1] * 63)
    with pytest.raises(KeyError):
        E.rotary(layout="quarter")


def rows(**kw):
    d = dict(x=FAKE, y=FAKE, x_token=512, x_head=128, y_token=512, y_head=128, norm=None, heads=4)
    d.update(kw)
    return E.ecokv_rows(*(d[n] for n, _ in E.ecokv_rows._fields_))


def pages(**kw):
    d = dict(k=FAKE, v=FAKE, page_stride=4 * 16 * 128, head_stride=16 * 128, slot_stride=128, n_pages=10, page_size=16,
             table=FAKE, table_stride=5, lengths=FAKE)
    d.update(kw)
    return E.ecokv_pages(*(d[n] for n, _ in E.ecokv_pages._fields_))


@pytest.mark.parametrize("kw", [dict(x=None), dict(x=FAKE + 8), dict(y=None), dict(y=FAKE + 2), dict(x_token=4),
                                dict(x_head=1), dict(y_token=130), dict(heads=0), dict(norm=FAKE + 4)])
def test_rotate_refuses_rows(kw):
    r = E.rotary()
    assert E.ecokv_rotate(r, 1, rows(**kw), None, FAKE, 3, 1e-6) == 1
    assert E.ecokv_rotate(r, 1, None, rows(**kw), FAKE, 3, 1e-6) == 1


def test_rotate_refuses_arguments():
    r = E.rotary()
    assert E.ecokv_rotate(r, 7, rows(), None, FAKE, 3, 1e-6) == 1          # dtype
    assert E.ecokv_rotate(r, 1, rows(), None, None, 3, 1e-6) == 1          # no positions
    assert E.ecokv_rotate(r, 1, rows(), None, FAKE + 2, 3, 1e-6) == 1      # misaligned positions
    assert E.ecokv_rotate(r, 1, rows(), None, FAKE, -1, 1e-6) == 1
    assert E.ecokv_rotate(r, 1, rows(), None, FAKE, 3, -1.0) == 1
    assert E.ecokv_rotate(r, 1, rows(), None, FAKE, 3, math.nan) == 1
    assert E.ecokv_rotate(r, 1, rows(heads=1 << 16), None, FAKE, 1 << 30, 0.0) == 2
    assert E.ecokv_rotate(r, 1, rows(), rows(), FAKE, 0, 1e-6) == 0        # nothing to do
    bad = E.rotary()
    bad.axis[5] = 1
    assert E.ecokv_rotate(bad, 1, rows(), None, FAKE, 3, 1e-6) == 1
    bad = E.rotary()
    bad.rot_dim = 20
    assert E.ecokv_rotate(bad, 1, rows(), None, FAKE, 3, 1e-6) == 1


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), 1), (dict(v=FAKE + 8), 1), (dict(table=None), 1), (dict(lengths=FAKE + 1), 1), (dict(page_size=24), 1),
    (dict(page_size=4), 1), (dict(page_size=8192), 1), (dict(n_pages=0), 1), (dict(table_stride=0), 1),
    (dict(page_stride=0), 1), (dict(head_stride=-128), 1), (dict(slot_stride=132), 1),
    (dict(page_size=4096, table_stride=4097), 2)])
def test_pages_are_checked(kw, code):
    c, p = pages(**kw), params()
    ws = E.ecokv_attend_workspace_size(2, 2, 8, 4, 1)
    assert E.ecokv_append(None, 1, None, rows(), rows(), c, None, None, 2, 2, 1e-6) == code
    assert E.ecokv_attend(p, 1, FAKE, None, c, None, FAKE, None, FAKE, ws) == code


def test_append_refuses_arguments():
    c, r = pages(), E.rotary()
    assert E.ecokv_append(r, 1, None, rows(), rows(heads=2), c, FAKE, None, 2, 2, 1e-6) == 1   # k and v differ
    assert E.ecokv_append(r, 1, None, rows(), rows(norm=FAKE), c, FAKE, None, 2, 2, 1e-6) == 1  # values are copied
    assert E.ecokv_append(r, 1, None, None, rows(), c, FAKE, None, 2, 2, 1e-6) == 1
    assert E.ecokv_append(r, 1, rows(y=None), rows(), rows(), c, FAKE, None, 2, 2, 1e-6) == 1
    assert E.ecokv_append(r, 1, None, rows(), rows(), c, FAKE, None, 3, 2, 1e-6) == 1           # one token a sequence
    assert E.ecokv_append(r, 1, None, rows(), rows(), c, FAKE, FAKE + 1, 3, 2, 1e-6) == 1
    assert E.ecokv_append(r, 1, None, rows(), rows(), c, FAKE, FAKE, 3, 0, 1e-6) == 1
    assert E.ecokv_append(r, 1, None, rows(), rows(), c, FAKE, None, 2, 2, 1e-6, FAKE, 255) == 3
    assert E.ecokv_append(r, 1, None, rows(), rows(), None, FAKE, None, 2, 2, 1e-6) == 1


def params(**kw):
    d = dict(h_q=8, h_kv=4, d=128, tokens=2, batch=2, scale=0.0, q_token=1024, q_head=128, out_token=1024, out_head=128,
             flags=0, timeout_us=0)
    d.update(kw)
    return E.ecokv_attend_params(*(d[n] for n, _ in E.ecokv_attend_params._fields_))


def prefix(**kw):
    d = dict(k=FAKE, v=FAKE, head_stride=1280, row_stride=128, rows=10, head_off=None)
    d.update(kw)
    return E.ecokv_prefix(*(d[n] for n, _ in E.ecokv_prefix._fields_))


@pytest.mark.parametrize("kw,code", [
    (dict(h_q=9), 1), (dict(h_kv=0), 1), (dict(tokens=-1), 1), (dict(batch=0), 1), (dict(d=64), 2), (dict(d=0), 1),
    (dict(h_q=260, h_kv=4), 2), (dict(scale=math.nan), 1), (dict(q_token=-1024), 1), (dict(q_head=4), 1),
    (dict(out_head=131), 1), (dict(flags=1), 1)])
def test_attend_refuses_parameters(kw, code):
    assert E.ecokv_attend(params(**kw), 1, FAKE, prefix(), None, None, FAKE, None, FAKE, 1 << 40) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), 1), (dict(v=FAKE + 8), 1), (dict(head_stride=100), 1), (dict(row_stride=0), 1), (dict(rows=-1), 1),
    (dict(rows=(1 << 24) + 1), 2), (dict(head_off=FAKE + 2), 1)])
def test_attend_refuses_prefixes(kw, code):
    assert E.ecokv_attend(params(), 1, FAKE, prefix(**kw), None, None, FAKE, None, FAKE, 1 << 40) == code


def test_attend_refuses_arguments():
    p, c, ws = params(), pages(), E.ecokv_attend_workspace_size(2, 2, 8, 4, 1)
    assert ws > 0 and E.ecokv_attend_workspace_size(2, 2, 9, 4, 1) == 0 and E.ecokv_attend_workspace_size(2, 0, 8, 4, 1) == 0
    assert E.ecokv_attend(p, 5, FAKE, None, c, None, FAKE, None, FAKE, ws) == 1
    assert E.ecokv_attend(p, 1, None, None, c, None, FAKE, None, FAKE, ws) == 1
    assert E.ecokv_attend(p, 1, FAKE + 4, None, c, None, FAKE, None, FAKE, ws) == 1
    assert E.ecokv_attend(p, 1, FAKE, None, c, None, FAKE, FAKE + 2, FAKE, ws) == 1
    assert E.ecokv_attend(p, 1, FAKE, None, c, None, FAKE, None, None, ws) == 3
    assert E.ecokv_attend(p, 1, FAKE, None, c, None, FAKE, None, FAKE, ws - 1) == 3
    assert E.ecokv_attend(params(tokens=3), 1, FAKE, None, c, None, FAKE, None, FAKE, 1 << 40) == 1  # one token a sequence
    assert E.ecokv_attend(p, 1, FAKE, None, c, FAKE + 2, FAKE, None, FAKE, ws) == 1
    assert E.ecokv_attend(params(tokens=0), 1, FAKE, None, c, FAKE, FAKE, None, FAKE, ws) == 0
    # more tiles than 31 bits count
    big = params(tokens=1 << 20, batch=1 << 16, h_q=64, h_kv=64)
    need = E.ecokv_attend_workspace_size(1 << 20, 1 << 16, 64, 64, 1)
    assert E.ecokv_attend(big, 1, FAKE, None, pages(page_size=4096, table_stride=4096), FAKE, FAKE, None, FAKE, need) == 2


def test_helpers_want_cuda_tensors():
    import torch
    x = torch.zeros(2, 4, 128)
    with pytest.raises(ValueError):
        E.rotate(E.rotary(), torch.zeros(1, 2, dtype=torch.int32), x)
    with pytest.raises(ValueError):
        E.Prefix(torch.zeros(4, 5, 128), torch.zeros(4, 5, 128))
    with pytest.raises(ValueError):
        E.PagedCache(torch.zeros(3, 4, 8, 128), torch.zeros(3, 4, 8, 128), torch.zeros(2, 2, dtype=torch.int32),
                     torch.zeros(2, dtype=torch.int32))
    assert ctypes.sizeof(E.ecokv_rotary) == 16 + 64 * 8 + 64


@pytest.mark.parametrize("kw", [dict(y_token=0), dict(y_head=0), dict(y_token=-512), dict(y_head=-128)])
def test_outputs_have_positive_strides(kw):
    """A stride of zero would have an output's rows race for one address."""
    r, c = E.rotary(), pages()
    assert E.ecokv_rotate(r, 1, rows(**kw), None, FAKE, 3, 1e-6) == 1
    assert E.ecokv_rotate(r, 1, None, rows(**kw), FAKE, 3, 1e-6) == 1
    assert E.ecokv_append(r, 1, rows(**kw), rows(), rows(), c, FAKE, None, 2, 2, 1e-6, FAKE, 256) == 1


@pytest.mark.parametrize("dtype,flags", [(1, 0), (1, E.ECOKV_FLAG_FORCE_SIMT), (0, 0)])
@pytest.mark.parametrize("group", [1, 7, 8, 64])
@pytest.mark.parametrize("tokens,page,cols,rows", [(100000, 4096, 256, 0), (4096, 4096, 4096, 0), (1, 8, 1, 0),
                                                   (10000, 16, 8192, 131072)])
def test_attend_size_limit(tokens, page, cols, rows, group, dtype, flags):
    """The header's count of work, met and passed by one sequence (no workspace is given: nothing is launched)."""
    tc = dtype == 1 and not flags
    n = -(-tokens // (2 * (128 // group) if tc else 64 // group))
    u = lambda keys: (2 * -(-keys // 128) + 4 if tc else -(-keys // 128)) if keys else 0  # noqa: E731
    h_kv = 2
    most = ((2 ** 31 - 1) // h_kv - n * u(rows)) // u(page * cols) - n
    assert most > 0
    for batch, code in ((most, 3), (most + 1, 2)):
        if batch >= 2 ** 31:
            continue
        p = params(h_q=h_kv * group, h_kv=h_kv, tokens=tokens, batch=batch, flags=flags)
        c = pages(page_size=page, table_stride=cols, page_stride=h_kv * page * 128, head_stride=page * 128)
        pre = prefix(rows=rows, head_stride=max(rows, 1) * 128)
        assert E.ecokv_attend(p, dtype, FAKE, pre, c, FAKE, FAKE, None, FAKE, 0) == code, batch
