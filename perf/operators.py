"""Cases of the prompt attention and of the cache held in 4 bits.

Three kinds of passes:

  prompt   asrkf_prefill_packed on one layer: causal attention over the prompts
           of a batch, packed one after another, and their rows into the cache;
  store    prompts written into a cache held in 4 bits and read back as the
           values that the codes stand for (asrkf_prefill_packed without
           queries, asrkf_get_rows);
  decode   one batch of requests on a context whose cache is held in 4 bits:
           reset, prompts, `steps` decode steps with the freeze schedule, and
           the counters, as a serving program runs it.

The 4-bit format: groups of 32 values of a row share a power-of-two scale X, the
smallest with max|x| < 7 X; a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6
times X with its sign (ties to the even one of the eight, 6 the largest).
"""
import math
import random

import numpy as np
import torch

own = False

BASE = {"kind": "prompt", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "kv_bits": 0,
        "ctx_lo": 8192, "ctx_hi": 8192, "len_seed": 1, "steps": 0, "window": 128, "k_soft": 2.0, "f_hh": 0.35}


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # the repository's smallest configuration, fp32 rows of 64: one short prompt (latency)
        _case("prompt-tiny-f32-512", q_heads=8, kv_heads=2, head_dim=64, dtype="f32", ctx_lo=512, ctx_hi=512),
        # a batch of one-line prompts, from one token up
        _case("prompt-8b-b64-short", batch=64, ctx_lo=1, ctx_hi=64),
        # the 8B shape: one prompt of the repository's single-layer configuration
        _case("prompt-8b-8k"),
        # the same at the headline configuration's context
        _case("prompt-8b-32k", ctx_lo=32768, ctx_hi=32768),
        # a ragged batch of chats, packed, into a cache held in 4 bits
        _case("prompt-8b-b32-ragged", batch=32, ctx_lo=100, ctx_hi=4000, kv_bits=4),
        # rows of 256
        _case("prompt-d256-b4", batch=4, q_heads=16, head_dim=256, ctx_lo=1000, ctx_hi=4097),
        # prompts kept in 4 bits and read back
        _case("store-d64-b3", kind="store", batch=3, q_heads=16, kv_heads=2, head_dim=64, ctx_lo=33, ctx_hi=700,
              kv_bits=4),
        _case("store-8b-b8-16k", kind="store", batch=8, ctx_lo=16384, ctx_hi=16384, kv_bits=4),
        # one short sequence: every step is a handful of launches (latency)
        _case("decode-tiny-512", kind="decode", q_heads=8, kv_heads=2, head_dim=64, ctx_lo=512, ctx_hi=512, steps=32,
              window=32, kv_bits=4),
        # one layer of the headline configuration: 8 sequences of 32k
        _case("decode-8b-b8-32k", kind="decode", batch=8, ctx_lo=32768, ctx_hi=32768, steps=32, kv_bits=4),
        # the repository's ragged batch at half its length
        _case("decode-8b-ragged-b64", kind="decode", batch=64, ctx_lo=1024, ctx_hi=16384, steps=24, kv_bits=4),
        # wide query groups
        _case("decode-64q8kv-b4-16k", kind="decode", batch=4, q_heads=64, ctx_lo=12000, ctx_hi=16384, steps=24,
              kv_bits=4),
    ]


# head layouts that the library serves: (q heads, KV heads, head dim)
LAYOUTS = [(8, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 8, 256), (32, 32, 128),
           (32, 16, 128), (16, 2, 64), (8, 8, 128), (4, 1, 128)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    hq, hkv, d = rng.choice(LAYOUTS)
    kind = rng.choice(["prompt", "prompt", "store", "decode", "decode"])
    c = dict(BASE, kind=kind, q_heads=hq, kv_heads=hkv, head_dim=d, len_seed=rng.randrange(1 << 20))
    if kind == "prompt":
        if d < 256 and rng.random() < 0.25 and hkv * d <= 2048:
            c["dtype"] = "f32"
        elif rng.random() < 0.3:
            c["kv_bits"] = 4
        c["batch"] = _log_int(rng, 1, 64)
        # at most a quarter of the longest listed prompt's products (fp32: of a tenth of those)
        most = math.sqrt(2.0 ** 42 / (4 * hq * d * c["batch"]) / (10 if c["dtype"] == "f32" else 1))
        c["ctx_hi"] = _log_int(rng, 1, min(16384, int(most)))
    elif kind == "store":
        c["kv_bits"], c["batch"] = 4, _log_int(rng, 1, 64)
        c["ctx_hi"] = _log_int(rng, 1, min(16384, (1 << 27) // (hkv * d * c["batch"])))
    else:
        c.update(kv_bits=4, batch=_log_int(rng, 1, 64), steps=rng.randint(8, 32), window=_log_int(rng, 16, 256),
                 k_soft=rng.choice([1.0, 2.0]), f_hh=round(rng.uniform(0.2, 0.5), 3))
        c["ctx_hi"] = _log_int(rng, 64, min(32768, (1 << 28) // (hkv * d * c["batch"])))
    c["ctx_lo"] = c["ctx_hi"] if rng.random() < 0.3 else max(1, int(c["ctx_hi"] * rng.uniform(0.05, 1)))
    return c


def _lengths(c):
    r = random.Random(c["len_seed"])
    return [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["batch"])]


def _inputs(c, seed):
    """Packed prompts [T][heads][dim] and, for decode, every step's rows, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, Hq, Hkv, D, N = (c[k] for k in ("batch", "q_heads", "kv_heads", "head_dim", "steps"))
    plen = _lengths(c)
    T = sum(plen)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    if c["kind"] != "decode":
        return plen, (normal(T, Hq, D) * 1.5).to(dt), normal(T, Hkv, D), normal(T, Hkv, D)
    # heavy-hitter keys: +-beta on an axis of each (sequence, KV head), next to nothing there otherwise, and
    # queries along that axis: every score stays clear of tau = 0.5, before and after rounding to 4 bits
    axis = torch.randint(0, D, (B, Hkv), generator=g, device="cuda")
    sign = (torch.randint(0, 2, (B, Hkv), generator=g, device="cuda") * 2 - 1).float()

    def keys(x, a, s):
        hot = torch.rand(x.shape[:-2] + (1,), generator=g, device="cuda") < c["f_hh"]
        beta = 8 + 56 * torch.rand(x.shape[:-1], generator=g, device="cuda")
        at = a.unsqueeze(-1)
        small = x.gather(-1, at).squeeze(-1).float() / 16
        return x.scatter_(-1, at, torch.where(hot, s * beta, small).to(dt).unsqueeze(-1))

    of = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(plen, device="cuda"))
    K, V = keys(normal(T, Hkv, D), axis[of], sign[of]), normal(T, Hkv, D)
    kn = keys(normal(N, B, Hkv, D), axis.expand(N, B, Hkv), sign.expand(N, B, Hkv))
    vn = normal(N, B, Hkv, D)
    q = normal(N, B, Hq, D).float() / 8192
    alpha = 0.2 + 0.1 * torch.rand((N, B, Hq), generator=g, device="cuda")
    ah = axis.repeat_interleave(Hq // Hkv, 1).expand(N, B, Hq)
    sh = sign.repeat_interleave(Hq // Hkv, 1)
    q.scatter_add_(-1, ah.unsqueeze(-1), (alpha * sh).unsqueeze(-1))
    return plen, K, V, kn, vn, q.to(dt)


class State:
    """The inputs, and the context and output buffers that a serving program keeps."""
    ctx = None

    def __del__(self):
        if self.ctx:
            self.lib.asrkf_destroy(self.ctx)
            self.ctx = None


def prepare(case, seed):
    c, s = case, State()
    s.case, s.inputs = c, _inputs(c, seed)
    s.plen = s.inputs[0]
    if own:
        import paper_2512_11221_amd as A
        s.lib = A
        s.seqs = list(range(c["batch"]))
        s.ctx = A.asrkf_init(A.make_config(
            1, c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], max(s.plen) + max(c["steps"], 2), c["window"],
            0.5, c["k_soft"], 1024, dtype=c["dtype"], kv_bits=c["kv_bits"]))
        if c["kind"] == "prompt":
            s.out = torch.empty_like(s.inputs[1])
        elif c["kind"] == "store":
            s.out = torch.empty_like(s.inputs[2]), torch.empty_like(s.inputs[3])
        else:
            s.out = torch.empty(s.inputs[5].shape, device="cuda")
    return s


def run(state):
    kind = state.case["kind"]
    if own:
        return {"prompt": _own_prompt, "store": _own_store, "decode": _own_decode}[kind](state)
    return {"prompt": _plain_prompt, "store": _plain_store, "decode": _plain_decode}[kind](state)


def _own_prompt(s):
    _, q, k, v = s.inputs
    s.lib.asrkf_prefill_packed(s.ctx, 0, s.seqs, s.plen, q, k, v, s.out)
    return s.out


def _own_store(s):
    _, _, k, v = s.inputs
    s.lib.asrkf_prefill_packed(s.ctx, 0, s.seqs, s.plen, None, k, v, None)
    at = 0
    for b, n in enumerate(s.plen):
        s.lib.asrkf_get_rows(s.ctx, 0, b, 0, n, s.out[0][at:at + n], s.out[1][at:at + n])
        at += n
    return s.out


def _own_decode(s):
    _, K, V, kn, vn, q = s.inputs
    A = s.lib
    A.asrkf_reset(s.ctx)
    A.asrkf_prefill_packed(s.ctx, 0, s.seqs, s.plen, None, K, V, None)
    for t in range(s.case["steps"]):
        A.asrkf_decode_step(s.ctx, 0, q[t], kn[t], vn[t], s.out[t])
        A.asrkf_restore(s.ctx, None, A.NONE)
    st = A.asrkf_stats(s.ctx)
    return {"out": s.out, "counters": np.array([st[k] for k in ("attended_total", "active_positions")], np.int64)}


def _padded(x, plen, length):
    """Packed rows [T, H, D] as [B, H, length, D] with zeros behind each sequence."""
    n = torch.tensor(plen, device=x.device)
    pos = torch.arange(length, device=x.device)
    at = (n.cumsum(0) - n).unsqueeze(1) + pos
    inside = pos < n.unsqueeze(1)
    rows = x[at.clamp(max=x.shape[0] - 1)] * inside[:, :, None, None].to(x.dtype)
    return rows.transpose(1, 2), inside


def _plain_prompt(s):
    plen, q, k, v = s.inputs
    B, top = len(plen), max(plen)
    Hq, Hkv, D = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hkv
    qp, inside = _padded(q.float(), plen, top)
    kp, vp = _padded(k.float(), plen, top)[0], _padded(v.float(), plen, top)[0]
    qp = qp.reshape(B, Hkv, G, top, D)
    kt = kp.transpose(2, 3).contiguous()
    out = torch.empty((B, Hkv, G, top, D), device=q.device)
    pos = torch.arange(top, device=q.device)
    step = max(1, (1 << 30) // (B * Hq * top))
    for i in range(0, top, step):       # as many queries at a time as the scores have room for
        e = min(top, i + step)
        x = torch.matmul(qp[:, :, :, i:e].reshape(B, Hkv, G * (e - i), D), kt[..., :e]).view(B, Hkv, G, e - i, e)
        x = (x * D ** -0.5).masked_fill(pos[:e] > pos[i:e, None], -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        x = x / x.sum(-1, keepdim=True)
        out[:, :, :, i:e] = torch.matmul(x.view(B, Hkv, G * (e - i), e), vp[:, :, :e]).view(B, Hkv, G, e - i, D)
    return out.reshape(B, Hq, top, D).transpose(1, 2)[inside].to(q.dtype)


def _rounded4(x):
    """The values that a row's 4-bit codes stand for, in 32 bits."""
    g = x.float().unflatten(-1, (-1, 32))
    amax = g.abs().amax(-1, keepdim=True)
    mant, exp = torch.frexp(amax)                       # amax = mant 2^exp, mant in [0.5, 1)
    e = (exp - 3 + (mant >= 0.875).int()).clamp(-100, 125)
    y = torch.ldexp(g, -e).clamp(-6, 6)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.ldexp(torch.round(y / step) * step, e).flatten(-2)


def _plain_store(s):
    _, _, k, v = s.inputs
    return _rounded4(k).to(k.dtype), _rounded4(v).to(v.dtype)


def _plain_decode(s):
    c = s.case
    plen, K, V, kn, vn, q = s.inputs
    N, B, Hq, D = q.shape
    Hkv, cap = c["kv_heads"], max(plen) + N
    kc, vc = _padded(_rounded4(K), plen, cap)[0].contiguous(), _padded(_rounded4(V), plen, cap)[0].contiguous()
    kn, vn = _rounded4(kn), _rounded4(vn)
    qt = q.float().view(N, B, Hkv, Hq // Hkv, D).transpose(3, 4).contiguous()
    n = torch.tensor(plen, device=q.device)
    pos, seq = torch.arange(cap, device=q.device), torch.arange(B, device=q.device)
    until = torch.zeros((B, cap), dtype=torch.int64, device=q.device)      # attends at step t where until <= t
    seen = torch.zeros_like(until)
    attended = torch.zeros((), dtype=torch.int64, device=q.device)
    out = torch.empty((N, B, Hq, D), device=q.device)
    for t in range(1, N + 1):
        kc[seq, :, n] = kn[t - 1]
        vc[seq, :, n] = vn[t - 1]
        n = n + 1
        on = (pos < n[:, None]) & (until <= t)
        x = torch.matmul(kc, qt[t - 1])                                    # [B, Hkv, cap, G]
        low = x.abs().sum((1, 3)) / Hq < 0.5
        p = (x * D ** -0.5).masked_fill(~on[:, None, :, None], -math.inf)
        p = torch.exp(p - p.amax(2, keepdim=True))
        p = (p / p.sum(2, keepdim=True)).transpose(2, 3).contiguous()
        out[t - 1] = torch.matmul(p, vc).view(B, Hq, D)
        low &= on & (pos < n[:, None] - c["window"])
        seen += low
        d = torch.floor(torch.sqrt(seen.double()) / c["k_soft"]).long()
        until = torch.where(low & (d >= 1), t + d, until)
        attended = attended + on.sum()
    active = ((pos < n[:, None]) & (until <= N + 1)).sum()
    return {"out": out, "counters": torch.stack([attended, active])}


def _steps(c):
    """Expected attended tokens summed over the steps: the heavy hitters and the window always, the others on the
    schedule of one that is found low whenever it attends."""
    total, until, seen = 0.0, 0, 0
    plen = _lengths(c)
    for t in range(1, c["steps"] + 1):
        total += sum(p + t for p in plen)
        if until > t:
            total -= (1 - c["f_hh"]) * sum(max(0, p + t - c["window"]) for p in plen)
            continue
        seen += 1
        d = int(math.sqrt(seen) / c["k_soft"])
        until = t + d if d else until
    return total


def work(case):
    c = case
    Hq, Hkv, D, esz = c["q_heads"], c["kv_heads"], c["head_dim"], 2 if c["dtype"] == "bf16" else 4
    plen = _lengths(c)
    T, row = sum(plen), 2 * Hkv * D * esz                                  # K and V of one token
    kept = 2 * Hkv * (D // 2 + D // 32) if c["kv_bits"] == 4 else row      # the same in the cache
    if c["kind"] == "prompt":
        return {"bytes": T * (2 * Hq * D * esz + row + kept), "flops": sum(2 * Hq * D * n * (n + 1) for n in plen)}
    if c["kind"] == "store":
        return {"bytes": T * 2 * (row + kept), "flops": 0}
    att = _steps(c)
    step = c["batch"] * (Hq * D * (esz + 4) + row + kept)
    return {"bytes": T * (row + kept) + att * kept + c["steps"] * step, "flops": att * 4 * Hq * D}


# ---- the results in 64 bits ----

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest4(x):
    """The 4-bit format by its definition: the nearest of the eight values, ties to the even code."""
    g = x.double().reshape(-1, 32)
    top = g.abs().max(dim=1, keepdim=True).values
    X = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -126) / 7)) + 1)
    X = torch.where(top < 7 * X / 2, X / 2, X)
    X = torch.where(top >= 7 * X, X * 2, X).clamp(2.0 ** -100, 2.0 ** 125)
    a = g.abs() / X
    code = torch.zeros_like(a)
    for i in range(1, 8):               # past the middle of two neighbours, or on it where the upper is even
        mid = (_VALUES[i - 1] + _VALUES[i]) / 2
        code += (a >= mid) if i % 2 == 0 else (a > mid)
    vals = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)[code.long()]
    return (torch.copysign(vals, g) * X).reshape(x.shape)


def exact(case, seed):
    c = case
    if c["kind"] == "store":
        _, _, k, v = _inputs(c, seed)
        return _nearest4(k), _nearest4(v)
    G, D = c["q_heads"] // c["kv_heads"], c["head_dim"]
    if c["kind"] == "prompt":
        plen, q, k, v = _inputs(c, seed)
        if sum(p * p for p in plen) * c["q_heads"] * D > 1e13:
            return None
        out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
        at = 0
        for n in plen:
            for h in range(c["kv_heads"]):
                K, V = k[at:at + n, h].double().t().contiguous(), v[at:at + n, h].double()
                for i in range(0, n, 2048):
                    m = min(n, i + 2048)
                    x = q[at + i:at + m, h * G:(h + 1) * G].double().reshape(-1, D) @ K[:, :m] / math.sqrt(D)
                    row = torch.arange(i, m, device="cuda").repeat_interleave(G)
                    x[torch.arange(m, device="cuda") > row[:, None]] = -math.inf
                    out[at + i:at + m, h * G:(h + 1) * G] = (torch.softmax(x, -1) @ V[:m]).view(m - i, G, D)
            at += n
        return out
    plen, K, V, kn, vn, q = _inputs(c, seed)
    N, B, Hq, _ = q.shape
    if sum(plen) * N * c["kv_heads"] * D * 16 > 3e12:
        return None
    out = torch.empty((N, B, Hq, D), dtype=torch.float64, device="cuda")
    at = 0
    for b, P in enumerate(plen):
        Kb = _nearest4(torch.cat([K[at:at + P], kn[:, b]])).permute(1, 2, 0).contiguous()
        Vb = _nearest4(torch.cat([V[at:at + P], vn[:, b]])).permute(1, 0, 2).contiguous()
        at += P
        back = torch.zeros(P + N, dtype=torch.int64, device="cuda")        # the step at which a token attends again
        hits = torch.zeros_like(back)
        for t in range(1, N + 1):
            n = P + t
            use = (back[:n] <= t).nonzero().squeeze(1)
            x = torch.matmul(q[t - 1, b].double().view(-1, G, D), Kb[:, :, use])
            out[t - 1, b] = torch.matmul(torch.softmax(x / math.sqrt(D), -1), Vb[:, use]).reshape(Hq, D)
            drop = use[(x.abs().sum((0, 1)) / Hq < 0.5) & (use < n - c["window"])]
            hits[drop] += 1
            d = (hits[drop].double().sqrt() / c["k_soft"]).floor().long()
            back[drop[d >= 1]] = t + d[d >= 1]
    return {"out": out, "counters": None}
