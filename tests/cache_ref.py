"""Plain 64-bit forms of the operators for drafted tokens and for a cache that shrinks, from their definitions."""
import math

import torch

from tests.decode_ref import D


def reach(parents):
    """seen[i][j]: draft j is draft i or an ancestor of it."""
    n = len(parents)
    seen = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        at = i
        while at >= 0:
            seen[i, at] = True
            at = parents[at]
    return seen


def pack(seen, words):
    """[n][words] of 64 bits, as signed numbers, from a truth table [n][m]."""
    out = []
    for row in seen.tolist():
        bits = sum(1 << j for j, x in enumerate(row) if x)
        w = [(bits >> (64 * i)) & (2 ** 64 - 1) for i in range(words)]
        out.append([x - 2 ** 64 if x >= 2 ** 63 else x for x in w])
    return torch.tensor(out, dtype=torch.int64).view(len(out), words)


def causal(n):
    return torch.tril(torch.ones(n, n, dtype=torch.bool))


def rows_of(q, h, g, t, n):
    return q[t:t + n, h * g:(h + 1) * g].double()


def attend_masked(q, prefix, own, seen, scale):
    """decode_ref.attend where token i of a sequence sees the slots before its sequence's tokens and those of the
    tokens j with seen[b][i][j]."""
    tokens, h_q, _ = q.shape
    h_kv = len(prefix)
    g = h_q // h_kv
    out, size = torch.zeros(tokens, h_q, D, dtype=torch.float64), torch.zeros(tokens, h_q, D, dtype=torch.float64)
    lse = torch.full((tokens, h_q), -math.inf, dtype=torch.float64)
    mag, t = 0.0, 0
    for (ok, ov), m in zip(own, seen):
        n, L = m.shape[0], ok.shape[1]
        if n == 0:
            continue
        see = torch.cat([torch.ones(n, L - n, dtype=torch.bool), m], 1)
        for h in range(h_kv):
            k, v = torch.cat([prefix[h][0], ok[h]]).double(), torch.cat([prefix[h][1], ov[h]]).double()
            x = rows_of(q, h, g, t, n)
            s = x @ k.t() * scale
            full = torch.cat([torch.ones(n, k.shape[0] - L, dtype=torch.bool), see], 1)[:, None].expand(s.shape)
            mag = max(mag, float((x.abs() @ k.abs().t()).max()) * scale)
            s = s.masked_fill(~full, -math.inf)
            top = s.amax(-1, keepdim=True).clamp(min=-1e300)
            e = torch.exp(s - top).masked_fill(~full, 0.0)
            z = e.sum(-1, keepdim=True)
            at = (slice(t, t + n), slice(h * g, (h + 1) * g))
            lse[at] = (top + torch.log(z))[..., 0]
            p = e / z.clamp(min=1e-300)
            out[at], size[at] = p @ v, p @ v.abs()
        t += n
    return out, size, lse, mag


def weigh(q, lse, prefix_k, own_k, new, scale):
    """What each key is given: [h_kv] sums over the prefix's rows, per sequence [h_kv, len]; and the largest
    sum |q||k| scale + |lse| of a weight."""
    h_kv = len(prefix_k)
    g = q.shape[1] // h_kv
    pre = [torch.zeros(k.shape[0], dtype=torch.float64) for k in prefix_k]
    own, size, t = [], 0.0, 0
    for ok, n in zip(own_k, new):
        L = ok.shape[1]
        w = torch.zeros(h_kv, L, dtype=torch.float64)
        see = torch.cat([torch.ones(n, L - n, dtype=torch.bool), causal(n)], 1) if n else None
        for h in range(h_kv):
            if n == 0:
                continue
            x, z = rows_of(q, h, g, t, n), lse[t:t + n, h * g:(h + 1) * g, None].double()
            for k, mask, to in ((prefix_k[h], None, pre[h]), (ok[h], see, w[h])):
                if k.shape[0] == 0:
                    continue
                e = torch.exp(x @ k.double().t() * scale - z)
                e = torch.where((z == -math.inf) | (False if mask is None else ~mask[:, None]), 0.0, e)
                to += e.sum((0, 1))
                size = max(size, float((x.abs() @ k.double().abs().t()).max()) * scale +
                           float(z[z > -math.inf].abs().max() if bool((z > -math.inf).any()) else 0.0))
        own.append(w)
        t += n
    return pre, own, size


def prune(w, budget, limit, first, recent):
    """Kept slots of one head's weights [len]."""
    n = len(w)
    if n <= limit:
        return list(range(n))
    w = [-math.inf if x != x else x for x in w.tolist()]
    middle = range(first, n - recent)
    # (NaN below -inf)
    best = sorted(middle, key=lambda i: (-w[i], i))[:budget - first - recent]
    return list(range(first)) + sorted(best) + list(range(n - recent, n))
