"""Plain 64-bit forms of the decode step's operators (numpy-like torch on the CPU), written from their definitions."""
import math

import torch

D = 128


def frequencies(rot, base, scaling="none", factor=1.0, original=0):
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "yarn":
        def pair(turns):  # the pair that turns so often in `original` positions
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(32)), 0), min(math.ceil(pair(1)), rot - 1)
        out = []
        for i, x in enumerate(f):
            w = min(max((i - lo) / max(hi - lo, 1e-3), 0), 1)
            out.append(w * x / factor + (1 - w) * x)
        return out, 0.1 * math.log(factor) + 1
    return f, 1.0


def turn(x, pos, freq, axis, layout, magnitude=1.0, norm=None, eps=1e-6):
    """x [tokens, heads, D] -> (y, sum of the magnitudes each element is made of), in 64 bits."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + eps) * norm.double()
    y, size = x.clone(), x.abs().clone()
    if pos is None:
        return y, size
    half = len(freq)
    for f in range(half):
        a, b = (f, f + half) if layout == "half" else (2 * f, 2 * f + 1)
        ang = pos[axis[f]].double() * freq[f]
        c, s = magnitude * torch.cos(ang)[:, None], magnitude * torch.sin(ang)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = magnitude * (x[..., a].abs() + x[..., b].abs())
    return y, size


def attend(q, prefix, own, new, scale):
    """q [tokens, h_q, D]; prefix: (k, v) of every KV head; own: per sequence
    (k, v) [h_kv, len, D]; new: tokens of every sequence.  Returns out, sum p |v|
    / sum p, lse, all 64-bit, and the largest sum |q||k| scale of a score."""
    tokens, h_q, _ = q.shape
    h_kv = len(prefix)
    g = h_q // h_kv
    out, size = torch.zeros(tokens, h_q, D, dtype=torch.float64), torch.zeros(tokens, h_q, D, dtype=torch.float64)
    lse = torch.full((tokens, h_q), -math.inf, dtype=torch.float64)
    mag, t = 0.0, 0
    for (ok, ov), n in zip(own, new):
        L = ok.shape[1]
        for i in range(n):
            seen = max(L - n + i + 1, 0)
            for h in range(h_kv):
                k = torch.cat([prefix[h][0], ok[h, :seen]]).double()
                v = torch.cat([prefix[h][1], ov[h, :seen]]).double()
                if k.shape[0] == 0:
                    continue
                x = q[t, h * g:(h + 1) * g].double()
                s = x @ k.t() * scale
                mag = max(mag, float((x.abs() @ k.abs().t()).max()) * scale)
                lse[t, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
                p = torch.softmax(s, -1)
                out[t, h * g:(h + 1) * g] = p @ v
                size[t, h * g:(h + 1) * g] = p @ v.abs()
            t += 1
    return out, size, lse, mag
