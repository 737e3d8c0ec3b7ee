"""The walks over a call's items (csrc/attend.cuh, csrc/weigh.cuh), compiled for the CPU: every
tile of every item is one CTA's, and an item is whole in what next() returns, whatever the
object held before."""
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CUDA = "/usr/local/cuda/include"
TILE = 128


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists(CUDA):
        pytest.skip("no host compiler or CUDA headers")
    exe = str(tmp_path_factory.mktemp("walk") / "walk_host")
    subprocess.run(["g++", "-O1", "-fwrapv", "-std=c++17", "-Wno-attributes", "-I", CUDA, "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2609_06663_gb300", "csrc"), os.path.join(HERE, "walk_host.cpp"), "-o", exe],
                   check=True)

    def run(kind, numbers):
        """([a CTA's items in its order] by CTA, status)."""
        r = subprocess.run([exe, kind], input=" ".join(map(str, numbers)), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        lines = [x.split() for x in r.stdout.splitlines()]
        ctas = {}
        for x in lines[:-1]:
            c, *item = map(int, x)
            ctas.setdefault(c, []).append(tuple(item))
        return ctas, int(lines[-1][1])
    return run


def sequences(new, lens, single):
    """(first token, tokens, slots) of each."""
    out, t = [], 0
    for n, x in zip(new, lens):
        out.append((t, 1 if single else n, x))
        t += 1 if single else n
    return out


def tail(lens, new, single, offsets):
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return (lens or []) + ([] if single or not lens else starts) + (offsets or [])


def rows_of(rows, offsets, h_kv):
    return [(0, rows) if offsets is None else (offsets[h], offsets[h + 1] - offsets[h]) for h in range(h_kv)]


def together(ctas, key):
    """item -> [(CTA, tile0, ntiles)] in the CTAs' order; nothing but a CTA's first item goes on."""
    items = {}
    for c in sorted(ctas):
        for n, it in enumerate(ctas[c]):
            assert it[-2] == 0 or n == 0, "an item that goes on behind another one"
            assert it[-1] > 0
            items.setdefault(it[:-2], []).append((c, it[-2], it[-1]))
    return items


def tiles_in_order(parts, n):
    at, cta = 0, parts[0][0]
    for c, t0, k in parts:
        assert t0 == at and c == cta, (parts, n)
        at, cta = t0 + k, c + 1
    assert at == n, (parts, n)


# ---------------------------------------------------------------- ecokv_weigh
def div_up(a, b):
    return -(-a // b)


def check_weigh(walk, P, h_kv, g, new, lens, rows, offsets, tc, single=False):
    """The sizes as ecokv_weigh sets them."""
    tokens, batch = (sum(new) if new else 1), max(len(lens), 1)
    log2, most = (8, 128) if tc else (7, 64)
    span, t0 = 1 << log2, most // g
    if not tc and tokens > t0:
        t0 = div_up(tokens, div_up(tokens, t0))
    mean = 1 if single else div_up(tokens, batch)
    t1 = 1 if single else 2 * mean if mean < (t0 + 1) // 2 else t0
    unit = [div_up(min(tokens, t) * g, 32 if tc else 3) for t in (t0, t1)]
    lead, whole = 4 if tc else 2, 24
    need = [lead + u * div_up(n, t) for u, n, t in zip(unit, (tokens, 1 if single else tokens), (t0, t1))]
    cut = (rows > 0 and need[0] > whole) or (bool(lens) and need[1] > whole)
    numbers = [P, 0, P - 1, h_kv, tokens, batch, rows, 1 << 20, int(bool(lens)), int(bool(lens) and not single),
               int(offsets is not None), log2, t0, t1, *unit, lead, whole, max(unit) if cut else 1]
    ctas, status = walk("weigh", numbers + tail(lens, new, single, offsets))
    assert status == 0
    want = {}
    for h, (r0, n) in enumerate(rows_of(rows, offsets, h_kv)):
        for k in range(0, n, span):
            want[0, h, 0, k, min(n - k, span), 0, tokens, n, r0] = (tokens, t0)
    for b, (t, n, x) in enumerate(sequences(new, lens, single)):
        for h in range(h_kv):
            for k in range(0, x, span):
                want[1, h, b, k, min(x - k, span), t, n, x - n, 0] = (n, t1)
    got = together(ctas, want)
    assert got.keys() == want.keys(), (sorted(got.keys() - want.keys())[:3], sorted(want.keys() - got.keys())[:3])
    for item, (n, tpt) in want.items():
        tiles_in_order(got[item], max(div_up(n, tpt), 1))


WEIGH = [  # h_kv, group, new, lengths, prefix rows
    (1, 1, [1], [1], 0), (1, 1, [1], [5000], 0), (4, 7, [1] * 5, [1, 16, 17, 128, 529], 300), (8, 1, [3, 0, 5, 1], [3, 40, 200, 640], 128),
    (4, 7, [61, 30, 1, 17, 33], [61, 100, 1, 400, 33], 700), (1, 64, [1, 2, 35], [9, 20, 500], 64), (1, 4, [900, 10], [1000, 10], 5),
    (2, 2, [1] * 70, [7 * i for i in range(70)], 3000), (1, 7, [90], [1], 300), (3, 4, [50], [], 1000), (2, 1, [700], [700], 0),
]


@pytest.mark.parametrize("tc", [True, False])
@pytest.mark.parametrize("P", [1, 5, 152])
@pytest.mark.parametrize("h_kv,g,new,lens,rows", WEIGH)
def test_weigh_walk(walk, h_kv, g, new, lens, rows, P, tc):
    check_weigh(walk, P, h_kv, g, new, lens, rows, None, tc)


@pytest.mark.parametrize("tc", [True, False])
def test_weigh_walk_of_random_calls(walk, tc):
    rng = random.Random(5)
    for _ in range(40):
        h_kv, batch, single = rng.choice([1, 2, 4, 8, 40]), rng.randint(1, 70), rng.random() < 0.4
        new = [1] * batch if single else [rng.choice([0, 1, 3, 61]) for _ in range(batch)]
        new[0] = max(new[0], 1)
        offsets = None
        rows = rng.choice([0, 1, 255, 256, 257, 4000])
        if rows and rng.random() < 0.5:
            cuts = sorted(rng.randint(0, rows) for _ in range(h_kv - 1))
            offsets = [0] + cuts + [rows]
        check_weigh(walk, rng.choice([1, 3, 20, 152, 304]), h_kv, rng.choice([1, 4, 7]), new,
                    [rng.choice([0, 1, 100, 256, 700, 5000]) for _ in new], rows, offsets, tc, single)


# ---------------------------------------------------------------- ecokv_attend
def check_attend(walk, P, h_kv, g, new, lens, rows, offsets, tc, single=False, tree=False, ctas=None, most=None):
    tokens, batch = sum(new), max(len(lens), 1)
    tpt = (128 if tc else 64) // g
    span = 2 * tpt if tc else tpt
    numbers = [P, *(ctas or (0, P - 1)), h_kv, tokens, batch, rows, most or 1 << 20, int(bool(lens)),
               int(bool(lens) and not single), int(offsets is not None), tpt, span, int(tc), int(tree)]
    got, status = walk("attend", numbers + tail(lens, new, single, offsets))
    assert status == 0
    want = {}
    for h, (r0, n) in enumerate(rows_of(rows, offsets, h_kv)):
        if n:
            for t in range(0, tokens, span):
                want[0, h, 0, t, min(span, tokens - t), n, 0, n, r0] = n
    for b, (t, n, x) in enumerate(sequences(new, lens, single)):
        for i in range(0, n, span):
            vis = x if tree else max(x - n + min(n, i + span), 0)
            for h in range(h_kv):
                if vis:
                    want[1, h, b, t + i, min(span, n - i), x - n if tree else x - n + i + 1, 0 if tree else 1, vis, 0] = vis
    if ctas is not None:
        return got, want
    items = together(got, want)
    assert items.keys() == want.keys()
    for item, keys in want.items():
        tiles_in_order(items[item], div_up(keys, TILE))


@pytest.mark.parametrize("tc", [True, False])
def test_attend_walk_of_random_calls(walk, tc):
    rng = random.Random(6)
    for _ in range(40):
        h_kv, batch, single = rng.choice([1, 2, 4, 8, 40]), rng.randint(1, 70), rng.random() < 0.4
        new = [1] * batch if single else [rng.choice([0, 1, 3, 61, 300]) for _ in range(batch)]
        new[0] = max(new[0], 1)
        lens = [rng.choice([0, 1, 100, 256, 700, 5000]) for _ in new]  # (fewer slots than tokens among them)
        rows, offsets = rng.choice([0, 1, 128, 129, 4000]), None
        if rows and rng.random() < 0.5:
            offsets = [0] + sorted(rng.randint(0, rows) for _ in range(h_kv - 1)) + [rows]
        check_attend(walk, rng.choice([1, 3, 20, 152]), h_kv, rng.choice([1, 4, 7, 64]), new, lens, rows, offsets, tc, single,
                     tree=rng.random() < 0.5)


def test_attend_walk_of_as_much_work_as_is_taken(walk):
    """A prefix whose units are one less than 31 bits hold: every CTA has its equal run of them."""
    P, h_kv, groups, tiles = 152, 7, 3069, 99962
    total = h_kv * groups * tiles
    assert total == 2 ** 31 - 2
    run = div_up(total, P)
    for cta in (0, 1, 77, 150, 151):
        got, _ = check_attend(walk, P, h_kv, 1, [64 * groups], [], tiles * TILE, None, False, ctas=(cta, cta))
        assert sum(it[-1] for it in got[cta]) == min(run, total - cta * run), cta
        first, unit = got[cta][0], cta * run
        head, unit = divmod(unit, groups * tiles)
        assert first[1] == head and first[3] == unit // tiles * 64 and first[-2] == unit % tiles


def test_weigh_walk_of_as_much_work_as_is_taken(walk):
    P, h_kv, spans, tiles = 152, 8, 65536, 1022  # (a tile is 4 units, an item's keys 4)
    per, total = 4 + 4 * tiles, h_kv * spans * (4 + 4 * tiles)
    assert 2 ** 31 - per * h_kv * spans <= total < 2 ** 31
    run = div_up(total, P)
    for cta in (0, 75, 151):
        got, status = walk("weigh", [P, cta, cta, h_kv, 128 * tiles, 1, 256 * spans, 1 << 20, 0, 0, 0, 8, 128, 128, 4, 4, 4, 24, 4])
        x, end = cta * run, min((cta + 1) * run, total)
        want = []
        while x < end:
            item, y = divmod(x, per)
            z = min(per, y + end - x)
            t0, t1 = (div_up(max(v - 4, 0), 4) for v in (y, z))
            if t1 > t0:
                head, k = divmod(item, spans)
                want.append((0, head, 0, k * 256, 256, 0, 128 * tiles, 256 * spans, 0, t0, t1 - t0))
            x += z - y
        assert status == 0 and got[cta] == want
