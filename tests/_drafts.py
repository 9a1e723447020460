"""What the tests of drafted tokens share: references in 64 bits, written from the definitions."""
import math

import numpy as np


def random_tree(rng, n, reach=6):
    return [-1] + [int(rng.integers(max(-1, i - reach), i)) for i in range(1, n)]


def sees_of(parents):
    """Bit j of node i: j is i or an ancestor, by walking up."""
    out = []
    for i in range(len(parents)):
        m, j = 0, i
        while j >= 0:
            m |= 1 << j
            j = parents[j]
        out.append(m)
    return out


def attention(q, K, V, active, k, v, sees, count):
    """One sequence's outputs [N, Hq, D] in 64 bits, and the bound of every output's error.

    q [N, Hq, D], k, v [N, Hkv, D], K, V [n, Hkv, D] the cache's rows, active the positions attended.
    The bound is that of the prompts: rounding a weight to bf16 moves it by half a step of itself at
    most, the output's own rounding the output by half a step; a score is a sum of D products
    in fp32, off by at most D 2^-24 sum |q k|, which moves its weight by that over sqrt(D),
    relatively, and the sum of the weights as much; the exponential, the sums over the
    tokens (n 2^-24), the partials' factors and the division come on top.  Values that are not
    finite are left out of the bound."""
    import torch
    N, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    half_step = torch.finfo(q.dtype).eps / 2
    out = torch.zeros((N, Hq, D), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    at = torch.as_tensor(np.asarray(active), dtype=torch.int64, device=q.device)
    Kl, Vl = (x[at].double().transpose(0, 1).contiguous() for x in (K, V))              # [Hkv, n, D]
    for i in range(count):
        mine = [j for j in range(count) if sees[i] >> j & 1]
        n = len(at) + len(mine)
        if n == 0:
            continue
        Q = q[i].double().view(Hkv, G, D)
        Kh, Vh = (torch.cat([x, y[mine].double().transpose(0, 1)], 1) for x, y in ((Kl, k), (Vl, v)))
        Kt = Kh.transpose(1, 2).contiguous()
        p = torch.softmax(torch.matmul(Q, Kt) / math.sqrt(D), -1)
        size = torch.matmul(Q.abs(), Kt.abs()).amax((1, 2), keepdim=True)
        o, A = torch.matmul(p, Vh), torch.matmul(p, Vh.abs())
        rel = 2 * D * 2.0 ** -24 * size / math.sqrt(D) + 2 * n * 2.0 ** -24 + 2.0 ** -20
        out[i] = o.view(Hq, D)
        tol[i] = (half_step * (o.abs() + 1.01 * A) + rel * A).view(Hq, D)
    return out, tol


def check(got, ref, tol):
    err = (got.double() - ref).abs()
    worst = float((err / tol.clamp(min=1e-300)).max()) if err.numel() else 0.0
    assert worst <= 1.0, worst


def verify(tokens, parents, count, root, logits, probs, T, u):
    """One sequence's walk as it is defined: w as a vector.  (path, next token)"""
    V = len(root)

    def target(row):
        z = np.asarray(root if row < 0 else logits[row], np.float64)
        if np.isnan(z).any() or (z == np.inf).any() or not (z > -np.inf).any():
            return None
        if T == 0:
            return (np.arange(V) == int(np.argmax(z))).astype(np.float64)
        z = np.exp((z - z.max()) / T)
        return z / z.sum()

    path, last, w = [], -1, target(-1)
    for i in range(count):
        if parents[i] != last or not -1 <= parents[i] < i or w is None:
            continue
        x = int(tokens[i])
        inside = 0 <= x < V
        q = 1.0 if probs is None else (float(probs[last + 1][x]) if inside else 1.0)
        if T == 0:
            keep = inside and w[x] > 0
        else:
            keep = inside and float(u[i]) * q * w.sum() < w[x]
        if keep:
            path.append(i)
            last, w = i, target(i)
        elif T != 0:
            rest = w.copy()
            if probs is not None:
                rest = np.maximum(w / w.sum() - np.asarray(probs[last + 1], np.float64), 0.0)
            elif inside:
                rest[x] = 0.0
            w = rest if rest.sum() > 0 else w
    if w is None:
        return path, -1
    if T == 0:
        return path, int(np.argmax(w))
    run = np.cumsum(w)
    past = run > float(u[-1]) * run[-1]
    return path, int(np.argmax(past)) if past.any() else int(np.nonzero(w)[0][-1])


def turned(x, pos, freq, layout, magnitude=1.0, inverse=False):
    """[n, heads, D] turned by pos [n], in 64 bits, pair by pair, and the bound of every error: the
    output's rounding, sine and cosine rounded to fp32, two products and their sum (2^-24 of their
    terms each); angles in 64 bits are off by 2^-52 of themselves."""
    import torch
    dim, y = 2 * len(freq), x.double()
    sgn = -1.0 if inverse else 1.0
    mag = 1.0 / magnitude if inverse else magnitude
    ang = pos.double()[:, None] * torch.as_tensor(freq, dtype=torch.float64, device=x.device) * sgn
    co, si = torch.cos(ang)[:, None] * mag, torch.sin(ang)[:, None] * mag
    i = torch.arange(dim // 2, device=x.device)
    ia, ib = (i, i + dim // 2) if layout == "halves" else (2 * i, 2 * i + 1)
    a, b = y[..., ia], y[..., ib]
    out, size = y.clone(), torch.zeros_like(y)
    out[..., ia], out[..., ib] = a * co - b * si, b * co + a * si
    size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * mag
    far = 1 + ang.abs().max() * 2.0 ** -26 if ang.numel() else 1.0
    return out, torch.finfo(x.dtype).eps / 2 * out.abs() * 1.01 + 4 * 2.0 ** -24 * size * far
