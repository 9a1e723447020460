"""Cases of speculative decoding on the cache: rotary positions, attention of drafted tokens over the active cache,
their verification, and the accepted ones' rows into the cache.

Four kinds of passes:

  rotate   asrkf_rotate: queries and keys turned by their positions, for one token of every sequence (positions from
           the context) or for the packed tokens of a prompt (positions given, slices of a fused projection);
  draft    asrkf_attend_drafts on one layer: every drafted token of every sequence attends to the sequence's active
           cache and to the drafted tokens that its mask names;
  verify   asrkf_verify_drafts: the drafted tokens against the target's logits, from given random numbers;
  round    a batch of requests decoded with drafts: reset, prompts, and per round and layer the rotations, the decode
           step of the last token and the drafts' attention, then the freeze schedule, the verification and
           asrkf_accept_drafts; the counters and the appended rows are read back at the end.

Trees: node i of a sequence has parent parents[i] < i, or -1 for a child of the sequence's last token.  A node is
looked at if its parent was the last one accepted, in the order of the nodes.  With w = the target's probabilities behind the
last accepted token, W = sum w and u a given random number in [0, 1), a drafted token x is accepted where
u q(x) W < w(x); q = 1 without draft probabilities, and after a rejection w(x) = 0; with them w = max(w / W - q, 0).
The next token is the first whose running sum of w passes u W.
"""
import math
import random

import numpy as np
import torch

own = False

BASE = {"kind": "draft", "batch": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16", "kv_bits": 0,
        "ctx_lo": 8192, "ctx_hi": 8192, "len_seed": 1, "nodes": 4, "tree": "chain", "ragged": False, "freeze": True,
        "f_hh": 0.35, "window": 128, "vocab": 1024, "temperature": 1.0, "probs": False, "layers": 1, "rounds": 0,
        "rot_dim": 128, "rot_base": 500000.0, "rot_layout": "halves", "rot_scaling": "none", "rot_factor": 1.0,
        "rot_original": 8192, "rot_magnitude": 1.0, "tokens": 0}


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # one token of every sequence of a batch, as every layer of a step does it (latency)
        _case("rotate-step-8b-b8", kind="rotate", batch=8, ctx_lo=100, ctx_hi=4000),
        # part of an fp32 head, values in pairs
        _case("rotate-f32-part", kind="rotate", q_heads=8, kv_heads=2, head_dim=64, dtype="f32", tokens=5001, rot_dim=32,
              rot_layout="pairs", rot_scaling="linear", rot_factor=4.0, rot_base=10000.0),
        # a long prompt past the trained context, slices of the fused projection
        _case("rotate-prompt-8b-32k", kind="rotate", tokens=32768, rot_scaling="ramp", rot_factor=4.0, rot_magnitude=1.1386),
        # the repository's smallest configuration: a chain over one short sequence (latency)
        _case("draft-tiny-f32", q_heads=8, kv_heads=2, head_dim=64, dtype="f32", ctx_lo=512, ctx_hi=512, nodes=5, window=32),
        # the headline configuration's sequences, most of the cache frozen
        _case("draft-8b-b8-32k-chain", batch=8, ctx_lo=32768, ctx_hi=32768, nodes=5),
        # wide trees over a dense cache
        _case("draft-8b-b4-16k-tree", batch=4, ctx_lo=12000, ctx_hi=16384, nodes=60, tree="wide", freeze=False),
        # a ragged batch of chats on a cache held in 4 bits
        _case("draft-8b-b32-four", batch=32, ctx_lo=1000, ctx_hi=8000, nodes=16, tree="random", ragged=True, kv_bits=4),
        # greedy decoding of one sequence (latency)
        _case("verify-tiny-greedy", kind="verify", nodes=4, temperature=0.0),
        # chains from a draft model that gives its probabilities
        _case("verify-8b-b8-probs", kind="verify", batch=8, nodes=5, vocab=128256, probs=True),
        # trees from a lookup, without probabilities, another vocabulary
        _case("verify-b32-tree", kind="verify", batch=32, nodes=16, tree="random", ragged=True, vocab=50257, temperature=0.8),
        # one short sequence with drafts: every round is a handful of launches (latency)
        _case("round-tiny-f32", kind="round", q_heads=8, kv_heads=2, head_dim=64, dtype="f32", ctx_lo=512, ctx_hi=512,
              nodes=4, rounds=16, window=32, rot_dim=64, f_hh=0.35),
        # a few layers of the 8B shape, a batch of different lengths
        _case("round-8b-4layer-b8", kind="round", batch=8, layers=4, ctx_lo=4000, ctx_hi=8192, nodes=8, tree="random", ragged=True,
              rounds=12, vocab=32000, probs=True),
    ]


# head layouts that the library serves: (q heads, KV heads, head dim)
LAYOUTS = [(8, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 8, 256), (32, 32, 128),
           (32, 16, 128), (16, 2, 64), (8, 8, 128), (4, 1, 128)]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    hq, hkv, d = rng.choice(LAYOUTS)
    kind = rng.choice(["rotate", "draft", "draft", "draft", "verify", "verify", "round"])
    c = dict(BASE, kind=kind, q_heads=hq, kv_heads=hkv, head_dim=d, len_seed=rng.randrange(1 << 20),
             nodes=_log_int(rng, 1, 64), tree=rng.choice(["chain", "random", "random", "wide"]), ragged=rng.random() < 0.5,
             f_hh=round(rng.uniform(0.2, 0.5), 3), window=_log_int(rng, 16, 256), rot_dim=d)
    if d < 256 and rng.random() < 0.2 and hkv * d <= 2048 and kind != "verify":
        c["dtype"] = "f32"
    elif rng.random() < 0.3 and kind in ("draft", "round"):
        c["kv_bits"] = 4
    if kind in ("rotate", "round"):
        c.update(rot_layout=rng.choice(["halves", "pairs"]), rot_scaling=rng.choice(["none", "linear", "bands", "ramp"]))
        if c["rot_scaling"] != "none":
            c.update(rot_factor=rng.choice([2.0, 4.0, 8.0, 32.0]))
    if kind == "rotate":
        c.update(rot_dim=rng.choice([d, d, d // 2, d // 4, 48]), rot_magnitude=rng.choice([1.0, 1.2]), batch=_log_int(rng, 1, 64),
                 rot_base=rng.choice([10000.0, 500000.0]))
        c["tokens"] = rng.choice([0, 1, 1, 1]) and _log_int(rng, 1, (1 << 27) // ((hq + hkv) * d))
        c["ctx_hi"] = _log_int(rng, 1, 4000)
    elif kind == "draft":
        c.update(batch=_log_int(rng, 1, 64), freeze=rng.random() < 0.6)
        # at most the rows of the longest listed batch and half of the products of the widest tree
        most = (1 << 28) // (hkv * d * c["batch"]) // (2 if c["dtype"] == "f32" else 1)
        most = min(most, (1 << 33) // (hq * d * c["nodes"] * c["batch"]) // (10 if c["dtype"] == "f32" else 1))
        c["ctx_hi"] = _log_int(rng, 1, min(32768, max(most, 64)))
    elif kind == "verify":
        c.update(batch=_log_int(rng, 1, 64), vocab=rng.choice([1000, 1024, 32000, 50257, 128256]), probs=rng.random() < 0.5,
                 temperature=rng.choice([0.0, 0.7, 1.0, 1.0]))
        if c["temperature"] == 0:
            c["probs"] = False
        c["nodes"] = min(c["nodes"], max(1, 25000000 // (c["batch"] * c["vocab"]) - 1))
    else:
        c.update(batch=_log_int(rng, 1, 16), layers=rng.randint(1, 3), rounds=rng.randint(4, 10), vocab=rng.choice([1000, 32000]),
                 probs=rng.random() < 0.5, nodes=min(c["nodes"], 16))
        c["ctx_hi"] = _log_int(rng, 64, min(8192, (1 << 25) // (hkv * d * c["batch"] * c["layers"])))
    c["ctx_lo"] = c["ctx_hi"] if rng.random() < 0.3 else max(1, int(c["ctx_hi"] * rng.uniform(0.05, 1)))
    return c


def _lengths(c):
    r = random.Random(c["len_seed"])
    return [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["batch"])]


def _trees(c, key=0):
    """parents [batch][nodes] and how many nodes each sequence has."""
    r = random.Random(c["len_seed"] * 31 + 7 + key)
    N = c["nodes"]
    parents, count = [], []
    for _ in range(c["batch"]):
        if c["tree"] == "chain":
            p = list(range(-1, N - 1))
        elif c["tree"] == "wide":          # four children to a node
            p = [(i - 4) // 4 if i >= 4 else -1 for i in range(N)]
        else:
            p = [r.randrange(max(-1, i - 6), i) if i else -1 for i in range(N)]
        parents.append(p)
        count.append(r.randint((N + 1) // 2, N) if c["ragged"] else N)
    return parents, count


def _sees(parents):
    """Bit j of node i: node j is node i or one of its ancestors.  Also the nodes' depths."""
    masks, depths = [], []
    for p in parents:
        m, d = [], []
        for i, a in enumerate(p):
            m.append((m[a] if a >= 0 else 0) | 1 << i)
            d.append(d[a] + 1 if a >= 0 else 0)
        masks.append(m)
        depths.append(d)
    return masks, depths


def _signed64(masks):
    return [[x - (1 << 64) if x >> 63 else x for x in m] for m in masks]


def _gen(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 61)
    return g, (torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)


class _Keys:
    """Heavy-hitter keys: +-beta on an axis of each (sequence, KV head), next to nothing there otherwise, and queries
    along that axis: every score stays clear of tau = 0.5, before and after rounding to 4 bits.  The axis is one that the
    rotations hardly turn."""

    def __init__(self, c, g, dt):
        self.c, self.g, self.dt = c, g, dt
        B, Hkv, D = c["batch"], c["kv_heads"], c["head_dim"]
        x = torch.randint(0, 4, (B, Hkv), generator=g, device="cuda")
        if c["rot_layout"] == "halves":
            self.axis = torch.where(x < 2, D // 2 - 1 - x, D - 1 - x % 2)
        else:
            self.axis = D - 1 - x
        self.sign = (torch.randint(0, 2, (B, Hkv), generator=g, device="cuda") * 2 - 1).float()

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=self.dt)

    def keys(self, x, of=None):
        """x [..., Hkv, D], its sequences given by `of` or by the dimension before the heads."""
        a, s = (self.axis[of], self.sign[of]) if of is not None else (self.axis, self.sign)
        hot = torch.rand(x.shape[:-2] + (1,), generator=self.g, device="cuda") < self.c["f_hh"]
        beta = 8 + 56 * torch.rand(x.shape[:-1], generator=self.g, device="cuda")
        at = a.expand(x.shape[:-1]).unsqueeze(-1)
        small = x.gather(-1, at).squeeze(-1).float() / 16
        return x.scatter_(-1, at, torch.where(hot, s * beta, small).to(self.dt).unsqueeze(-1))

    def queries(self, *lead):
        """[*lead, B, Hq, D] along the axis."""
        B, Hkv = self.axis.shape
        Hq, D = self.c["q_heads"], self.c["head_dim"]
        q = self.normal(*lead, B, Hq, D).float() / 8192
        alpha = 0.2 + 0.1 * torch.rand((*lead, B, Hq), generator=self.g, device="cuda")
        a = self.axis.repeat_interleave(Hq // Hkv, 1).expand(*lead, B, Hq).unsqueeze(-1)
        return q.scatter_(-1, a, (alpha * self.sign.repeat_interleave(Hq // Hkv, 1)).unsqueeze(-1)).to(self.dt)


def _of(plen):
    return torch.repeat_interleave(torch.arange(len(plen), device="cuda"), torch.tensor(plen, device="cuda"))


def _choices(c, g, parents, count):
    """What a verification is given: tokens, the target's logits behind the root and behind every node, the draft
    model's probabilities (row 0 for the root's children, row 1 + i for node i's), random numbers."""
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    logits = torch.randn((B, N + 1, V), generator=g, device="cuda") * 3
    u = torch.rand((B, N + 1), generator=g, device="cuda")
    par = torch.tensor(parents, device="cuda")
    tokens = torch.randint(0, V, (B, N), generator=g, device="cuda")
    probs = None
    if c["probs"]:
        probs = torch.softmax(logits[:, :N] + torch.randn((B, N, V), generator=g, device="cuda") * 0.7, -1)
        for i in range(N):                 # drawn from the row of the parent
            row = probs[torch.arange(B, device="cuda"), par[:, i] + 1]
            race = -torch.log(torch.rand((B, V), generator=g, device="cuda").clamp(min=1e-30)) / row.clamp(min=1e-30)
            tokens[:, i] = race.argmin(-1)
    else:
        # a drafted token has a probability of 0.05 to 0.95 behind its parent, two siblings hardly ever the same token
        p = 0.05 + 0.9 * torch.rand((B, N), generator=g, device="cuda")
        value = math.log(V) + 4.5 + torch.log(p / (1 - p))
        for i in range(N):
            logits[torch.arange(B, device="cuda"), par[:, i] + 1, tokens[:, i]] = value[:, i]
    return {"tokens": tokens.int(), "root": logits[:, 0].contiguous(), "logits": logits[:, 1:].contiguous(), "probs": probs, "u": u,
            "parents": par.int(), "count": torch.tensor(count, device="cuda").int()}


def _inputs(c, seed):
    """Everything that the seed decides, on the GPU."""
    g, dt = _gen(c, seed)
    B, Hq, Hkv, D, N = (c[k] for k in ("batch", "q_heads", "kv_heads", "head_dim", "nodes"))
    kind, x = c["kind"], {}
    if kind == "rotate":
        if c["tokens"]:
            fused = torch.randn((c["tokens"], Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=dt)
            x["q"], x["k"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv]
            x["pos"] = torch.arange(c["tokens"], device="cuda", dtype=torch.int32) + int(seed) % 100
        else:
            x["q"], x["k"] = (torch.randn((B, h, D), generator=g, device="cuda", dtype=dt) for h in (Hq, Hkv))
        x["plen"] = _lengths(c)
        return x
    parents, count = _trees(c)
    if kind == "verify":
        return _choices(c, g, parents, count)
    keys = _Keys(c, g, dt)
    plen = x["plen"] = _lengths(c)
    T = sum(plen)
    x["K"], x["V"] = keys.keys(keys.normal(T, Hkv, D), _of(plen)), keys.normal(T, Hkv, D)
    if kind == "draft":
        masks, _ = _sees(parents)
        x.update(q0=keys.queries(), k0=keys.keys(keys.normal(B, Hkv, D)), v0=keys.normal(B, Hkv, D),
                 q=(keys.normal(B, N, Hq, D) * 1.5).to(dt), k=keys.normal(B, N, Hkv, D), v=keys.normal(B, N, Hkv, D),
                 sees=torch.tensor(_signed64(masks), device="cuda"), count=torch.tensor(count, device="cuda").int())
        return x
    R, L = c["rounds"], c["layers"]
    x["K"], x["V"] = [x["K"]], [x["V"]]
    for _ in range(1, L):
        x["K"].append(keys.keys(keys.normal(T, Hkv, D), _of(plen)))
        x["V"].append(keys.normal(T, Hkv, D))
    x.update(q0=keys.queries(R, L), k0=keys.keys(keys.normal(R, L, B, Hkv, D)), v0=keys.normal(R, L, B, Hkv, D),
             q=(keys.normal(R, L, B, N, Hq, D) * 1.5).to(dt),
             k=keys.keys(keys.normal(R, L, N, B, Hkv, D)).transpose(2, 3).contiguous(), v=keys.normal(R, L, B, N, Hkv, D))
    x["rounds"] = []
    for r in range(R):
        parents, count = _trees(c, r)
        masks, depths = _sees(parents)
        ch = _choices(c, g, parents, count)
        ch["sees"] = torch.tensor(_signed64(masks), device="cuda")
        ch["pos"] = 1 + torch.tensor(depths, device="cuda").int()
        x["rounds"].append(ch)
    return x


class State:
    """The inputs, and the context and output buffers that a serving program keeps."""
    ctx = None

    def __del__(self):
        if self.ctx:
            self.lib.asrkf_destroy(self.ctx)
            self.ctx = None


def prepare(case, seed):
    c, s = case, State()
    s.case, s.x = c, _inputs(c, seed)
    x, kind = s.x, c["kind"]
    B, Hq, Hkv, D, N, V = (c[k] for k in ("batch", "q_heads", "kv_heads", "head_dim", "nodes", "vocab"))
    if kind == "draft":                    # which tokens the step before has left active, in the plain form's layout
        s.on = _active_after_one_step(c, x)
    if not own:
        return s
    import paper_2512_11221_amd as A
    s.lib = A
    longest = max(x["plen"]) if kind != "verify" else 2
    k_soft = 0.25 if kind == "draft" else 1.0
    s.ctx = A.asrkf_init(A.make_config(
        c["layers"], B, Hq, Hkv, D, longest + 2 + c["rounds"] * (N + 1) + N, c["window"],
        0.5 if c["freeze"] else 0.0, k_soft, V, dtype=c["dtype"], kv_bits=c["kv_bits"]))
    if kind in ("rotate", "round"):
        A.asrkf_set_rotary(s.ctx, c["rot_dim"], c["rot_base"], layout=c["rot_layout"], scaling=c["rot_scaling"],
                           factor=c["rot_factor"], original_ctx=c["rot_original"], low=1.0, high=32.0 if c["rot_scaling"] == "ramp" else 4.0,
                           magnitude=c["rot_magnitude"])
    if kind != "rotate":
        A.asrkf_reserve_drafts(s.ctx, N)
    seqs = s.seqs = list(range(B))
    if kind == "rotate":
        s.out = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in (x["q"], x["k"])]
        if not c["tokens"]:                # sequences of these lengths, whatever their rows
            rows = torch.zeros((sum(x["plen"]), Hkv, D), dtype=x["k"].dtype, device="cuda")
            A.asrkf_prefill_packed(s.ctx, 0, seqs, x["plen"], None, rows, rows, None)
    elif kind == "draft":
        A.asrkf_prefill_packed(s.ctx, 0, seqs, x["plen"], None, x["K"], x["V"], None)
        A.asrkf_decode_step(s.ctx, 0, x["q0"], x["k0"], x["v0"], torch.empty((B, Hq, D), device="cuda"))
        A.asrkf_restore(s.ctx, None, A.NONE)
        s.out = torch.zeros_like(x["q"])
    else:
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")   # noqa: E731
        s.choice = [(new(B, N), new(B), new(B)) for _ in range(max(1, c["rounds"]))]
        if kind == "round":
            s.rot = [torch.empty_like(x[k][0, 0]) for k in ("q0", "k0", "q")]
            s.kd = torch.empty_like(x["k"][0])                     # the drafts' turned keys, every layer's
            s.out = torch.empty(x["q0"].shape, device="cuda"), torch.zeros_like(x["q"])
            s.rows = [torch.zeros((B, c["rounds"] * (N + 1), Hkv, D), dtype=x["k"].dtype, device="cuda") for _ in range(2)]
    return s


def run(state):
    kind = state.case["kind"]
    if own:
        return {"rotate": _own_rotate, "draft": _own_draft, "verify": _own_verify, "round": _own_round}[kind](state)
    return {"rotate": _plain_rotate, "draft": _plain_draft, "verify": _plain_verify, "round": _plain_round}[kind](state)


# ---- the framework's calls ----

def _own_rotate(s):
    if s.case["tokens"]:
        s.lib.asrkf_rotate(s.ctx, s.x["pos"], s.x["q"], s.out[0], s.x["k"], s.out[1])
    else:
        s.lib.asrkf_rotate(s.ctx, None, s.x["q"], s.out[0], s.x["k"], s.out[1], rows_per_seq=1)
    return s.out


def _own_draft(s):
    x = s.x
    s.lib.asrkf_attend_drafts(s.ctx, 0, x["sees"], x["q"], x["k"], x["v"], s.out, count=x["count"] if s.case["ragged"] else None)
    return s.out


def _own_choose(s, ch, into):
    c = s.case
    s.lib.asrkf_verify_drafts(s.ctx, ch["tokens"], ch["parents"], ch["root"], ch["logits"], ch["u"], *into, probs=ch["probs"],
                              temperature=c["temperature"], count=ch["count"] if c["ragged"] else None)
    return into


def _own_verify(s):
    return _own_choose(s, s.x, s.choice[0])


def _own_round(s):
    A, c, x = s.lib, s.case, s.x
    L, N = c["layers"], c["nodes"]
    A.asrkf_reset(s.ctx)
    for layer in range(L):
        A.asrkf_prefill_packed(s.ctx, layer, s.seqs, x["plen"], None, x["K"][layer], x["V"][layer], None)
    q0, k0, q = s.rot
    for r in range(c["rounds"]):
        ch = x["rounds"][r]
        count = ch["count"] if c["ragged"] else None
        for layer in range(L):
            A.asrkf_rotate(s.ctx, None, x["q0"][r, layer], q0, x["k0"][r, layer], k0, rows_per_seq=1)
            A.asrkf_rotate(s.ctx, ch["pos"], x["q"][r, layer], q, x["k"][r, layer], s.kd[layer], rows_per_seq=N)
            A.asrkf_decode_step(s.ctx, layer, q0, k0, x["v0"][r, layer], s.out[0][r, layer])
            A.asrkf_attend_drafts(s.ctx, layer, ch["sees"], q, s.kd[layer], x["v"][r, layer], s.out[1][r, layer], count=count)
        A.asrkf_restore(s.ctx, None, A.NONE)
        path, n_path, _ = _own_choose(s, ch, s.choice[r])
        A.asrkf_accept_drafts(s.ctx, path, n_path, s.kd, x["v"][r])
    st = A.asrkf_stats(s.ctx)
    made = torch.stack([n for _, n, _ in s.choice]).sum(0).tolist()         # the tokens go to the clients here
    for b, n in enumerate(made):
        n += c["rounds"]
        A.asrkf_get_rows(s.ctx, L - 1, b, x["plen"][b], n, s.rows[0][b, :n], s.rows[1][b, :n])
    return {"out": s.out[0], "drafts": s.out[1], "choice": s.choice, "k": s.rows[0], "v": s.rows[1],
            "counters": np.array([st[k] for k in ("attended_total", "active_positions")], np.int64)}


# ---- the plain form ----

def _frequencies(c):
    """Turns of every pair per position, as Python floats."""
    dim, base, factor = c["rot_dim"], c["rot_base"], c["rot_factor"]
    f = [base ** (-2.0 * i / dim) for i in range(dim // 2)]
    if c["rot_scaling"] == "linear":
        return [x / factor for x in f]
    if c["rot_scaling"] == "bands":        # by turns over the original context: 1 and less stretched, 4 and more kept
        keep = [min(1.0, max(0.0, (c["rot_original"] * x / (2 * math.pi) - 1.0) / (4.0 - 1.0))) for x in f]
    elif c["rot_scaling"] == "ramp":       # by pair, between those of 32 turns and of one
        def pair(turns):
            return dim * math.log(c["rot_original"] / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), dim - 1)
        keep = [1.0 - min(1.0, max(0.0, (i - lo) / ((hi - lo) or 0.001))) for i in range(dim // 2)]
    else:
        return f
    return [x * (k + (1.0 - k) / factor) for x, k in zip(f, keep)]


def _turned(c, x, pos):
    """x [..., heads, D] turned by pos [...]: angles in 64 bits, the rest in 32."""
    dim = c["rot_dim"]
    ang = pos.double()[..., None, None] * torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
    co, si = (torch.cos(ang) * c["rot_magnitude"]).float(), (torch.sin(ang) * c["rot_magnitude"]).float()
    y = x.float()
    if c["rot_layout"] == "halves":
        a, b = y[..., :dim // 2], y[..., dim // 2:dim]
        parts = [a * co - b * si, b * co + a * si]
    else:
        a, b = y[..., 0:dim:2], y[..., 1:dim:2]
        parts = [torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)]
    return torch.cat(parts + [y[..., dim:]], -1).to(x.dtype)


def _plain_rotate(s):
    c, x = s.case, s.x
    pos = x["pos"] if c["tokens"] else torch.tensor(x["plen"], device="cuda")
    return [_turned(c, x["q"], pos), _turned(c, x["k"], pos)]


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


def _held(c, x):
    return _rounded4(x) if c["kv_bits"] == 4 else x.float()


def _padded(x, plen, length):
    """Packed rows [T, H, D] as [B, H, length, D] with zeros behind each sequence."""
    n = torch.tensor(plen, device=x.device)
    pos = torch.arange(length, device=x.device)
    at = (n.cumsum(0) - n).unsqueeze(1) + pos
    inside = pos < n.unsqueeze(1)
    rows = x[at.clamp(max=max(x.shape[0] - 1, 0))] * inside[:, :, None, None].to(x.dtype)
    return rows.transpose(1, 2).contiguous()


def _active_after_one_step(c, x):
    """[B, longest + 1]: whether a position attends at step 2, after a first step that froze what scored below 0.5."""
    plen, K = x["plen"], x["K"]
    n = torch.tensor(plen, device="cuda") + 1
    pos = torch.arange(max(plen) + 1, device="cuda")
    on = pos < n[:, None]
    if not c["freeze"]:
        return on
    G = c["q_heads"] // c["kv_heads"]
    q = x["q0"].float().view(c["batch"], c["kv_heads"], G, -1)
    score = torch.empty(K.shape[0], device="cuda")
    at = 0
    for b, p in enumerate(plen):
        kb = _held(c, K[at:at + p]).transpose(0, 1).contiguous()                    # [Hkv, p, D]
        score[at:at + p] = torch.matmul(kb, q[b].transpose(1, 2).contiguous()).abs().sum((0, 2)) / c["q_heads"]
        at += p
    low = torch.zeros(on.shape, dtype=torch.bool, device="cuda")
    low[pos < n[:, None] - 1] = score < 0.5
    return on & ~(low & (pos < n[:, None] - c["window"]))


def _softmax_rows(x):
    """Weights over the last dimension; a row of -inf only has none."""
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    return x / torch.where(total == 0, 1.0, total)


def _attend_plain(q, kc, vc, on, k, v, sees, count, out):
    """q [B, N, Hq, D] over kc, vc [B, Hkv, cap, D] where on [B, cap], and over the drafts k, v [B, N, Hkv, D] that
    sees names: rows below count into out."""
    B, N, Hq, D = q.shape
    Hkv = kc.shape[1]
    G = Hq // Hkv
    qp = q.float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    kd, vd = (t.float().transpose(1, 2).contiguous() for t in (k, v))               # [B, Hkv, N, D]
    bits = (sees[:, :, None] >> torch.arange(N, device="cuda")) & 1
    seen = (bits == 1) & (torch.arange(N, device="cuda") < count[:, None, None])
    x0 = torch.matmul(qp, kc.transpose(2, 3).contiguous()).masked_fill(~on[:, None, None, :], -math.inf)
    x1 = torch.matmul(qp, kd.transpose(2, 3).contiguous())
    x1 = x1.masked_fill(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    p = _softmax_rows(torch.cat([x0, x1], -1) * D ** -0.5)
    del x0, x1
    cap = kc.shape[2]
    o = torch.matmul(p[..., :cap].contiguous(), vc) + torch.matmul(p[..., cap:].contiguous(), vd)
    o = o.view(B, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).to(out.dtype)
    live = torch.arange(N, device="cuda") < count[:, None]
    out.copy_(torch.where(live[:, :, None, None], o, out))


def _plain_draft(s):
    c, x = s.case, s.x
    plen, B = x["plen"], c["batch"]
    length = max(plen) + 1
    seq, n = torch.arange(B, device="cuda"), torch.tensor(plen, device="cuda")
    kc, vc = _padded(_held(c, x["K"]), plen, length), _padded(_held(c, x["V"]), plen, length)
    kc[seq, :, n], vc[seq, :, n] = _held(c, x["k0"]), _held(c, x["v0"])
    out = torch.zeros_like(x["q"])
    _attend_plain(x["q"], kc, vc, s.on, x["k"], x["v"], x["sees"], x["count"], out)
    return out


def _probabilities(c, logits):
    z = logits.double() / c["temperature"]
    z = torch.exp(z - z.amax(-1, keepdim=True))
    return z / z.sum(-1, keepdim=True)


def _plain_choose(c, ch):
    """path [B, N] (-1 behind its end), its length, the next token."""
    tokens, par, count = ch["tokens"].long(), ch["parents"].long(), ch["count"]
    B, N = tokens.shape
    seq = torch.arange(B, device="cuda")
    at = torch.full((B,), -1, device="cuda")
    path = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
    n_path = torch.zeros(B, dtype=torch.int64, device="cuda")
    greedy = c["temperature"] == 0
    if greedy:
        best = torch.cat([ch["root"][:, None], ch["logits"]], 1).argmax(-1)        # [B, N + 1]
    else:
        w = _probabilities(c, ch["root"])
        u = ch["u"].double()
    for i in range(N):
        here = (par[:, i] == at) & (i < count)
        if greedy:
            yes = here & (tokens[:, i] == best[seq, at + 1])
        else:
            W = w.sum(-1)
            mass = w[seq, tokens[:, i]]
            if ch["probs"] is not None:
                q = ch["probs"][seq, par[:, i] + 1].double()
                yes = here & (u[:, i] * q[seq, tokens[:, i]] * W < mass)
                left = (w / W[:, None] - q).clamp(min=0)
            else:
                yes = here & (u[:, i] * W < mass)
                left = w.clone()
                left[seq, tokens[:, i]] = 0
            no = (here & ~yes)[:, None] & (left.sum(-1, keepdim=True) > 0)
            w = torch.where(yes[:, None], _probabilities(c, ch["logits"][:, i]), torch.where(no, left, w))
        path[seq, n_path.clamp(max=N - 1)] = torch.where(yes, i, path[seq, n_path.clamp(max=N - 1)].long()).int()
        n_path = n_path + yes
        at = torch.where(yes, i, at)
    if greedy:
        nxt = best[seq, at + 1]
    else:
        run = w.cumsum(-1)
        nxt = (run > (u[:, N] * run[:, -1])[:, None]).int().argmax(-1)
    return path, n_path.int(), nxt.int()


def _plain_verify(s):
    return _plain_choose(s.case, s.x)


def _plain_round(s):
    c, x = s.case, s.x
    R, L, B, N, Hq, D = x["q"].shape
    plen, Hkv = x["plen"], c["kv_heads"]
    cap = max(plen) + R * (N + 1) + N
    kc = [_padded(_held(c, t), plen, cap) for t in x["K"]]
    vc = [_padded(_held(c, t), plen, cap) for t in x["V"]]
    n = torch.tensor(plen, device="cuda")
    pos, seq = torch.arange(cap, device="cuda"), torch.arange(B, device="cuda")
    until = torch.zeros((L, B, cap), dtype=torch.int64, device="cuda")       # attends at step t where until <= t
    seen = torch.zeros_like(until)
    attended = torch.zeros((), dtype=torch.int64, device="cuda")
    out, drafts = torch.empty(x["q0"].shape, device="cuda"), torch.zeros_like(x["q"])
    choice = []
    for r in range(R):
        t, ch = r + 1, x["rounds"][r]
        turned = []
        for layer in range(L):
            q0, k0 = _turned(c, x["q0"][r, layer], n), _turned(c, x["k0"][r, layer], n)
            at = n[:, None] + ch["pos"]
            q, k = _turned(c, x["q"][r, layer], at), _turned(c, x["k"][r, layer], at)
            turned.append(k)
            kc[layer][seq, :, n], vc[layer][seq, :, n] = _held(c, k0), _held(c, x["v0"][r, layer])
            on = (pos <= n[:, None]) & (until[layer] <= t)
            y = torch.matmul(kc[layer], q0.float().view(B, Hkv, Hq // Hkv, D).transpose(2, 3).contiguous())
            low = y.abs().sum((1, 3)) / Hq < 0.5
            p = _softmax_rows((y * D ** -0.5).masked_fill(~on[:, None, :, None], -math.inf).transpose(2, 3).contiguous())
            out[r, layer] = torch.matmul(p, vc[layer]).view(B, Hq, D)
            _attend_plain(q, kc[layer], vc[layer], on, k, x["v"][r, layer], ch["sees"], ch["count"], drafts[r, layer])
            low &= on & (pos < n[:, None] + 1 - c["window"])
            seen[layer] += low
            d = torch.floor(torch.sqrt(seen[layer].double())).long()
            until[layer] = torch.where(low & (d >= 1), t + d, until[layer])
            attended = attended + on.sum()
        n = n + 1
        path, n_path, nxt = _plain_choose(c, ch)
        choice.append((path, n_path, nxt))
        for i in range(N):                  # node path[:, i] goes to position n + i
            take = i < n_path
            node = path[:, i].long().clamp(min=0)
            to = (n + i)[take]
            for layer in range(L):
                kc[layer][seq[take], :, to] = _held(c, turned[layer][seq, node])[take]
                vc[layer][seq[take], :, to] = _held(c, x["v"][r, layer][seq, node])[take]
        n = n + n_path
    active = ((pos < n[:, None]) & (until <= R + 1)).sum()
    # the rows behind the prompts, zeros behind the last
    at = torch.tensor(plen, device="cuda")[:, None] + torch.arange(R * (N + 1), device="cuda")
    rows = [t[L - 1].transpose(1, 2)[seq[:, None], at] * (at < n[:, None])[..., None, None] for t in (kc, vc)]
    return {"out": out, "drafts": drafts, "choice": choice, "k": rows[0].to(x["k"].dtype), "v": rows[1].to(x["v"].dtype),
            "counters": torch.stack([attended, active])}


# ---- what a pass cannot do without ----

def _attended(c, plen, steps):
    """Expected attended tokens of a layer summed over the steps: the heavy hitters and the window always, the others
    on the schedule of one that is found low whenever it attends."""
    total, until, seen = 0.0, 0, 0
    for t in range(1, steps + 1):
        total += sum(p + t for p in plen)
        if until > t:
            total -= (1 - c["f_hh"]) * sum(max(0, p + t - c["window"]) for p in plen)
            continue
        seen += 1
        d = int(math.sqrt(seen))
        until = t + d if d else until
    return total


def work(case):
    c = case
    B, Hq, Hkv, D, N, V = (c[k] for k in ("batch", "q_heads", "kv_heads", "head_dim", "nodes", "vocab"))
    esz = 2 if c["dtype"] == "bf16" else 4
    row = 2 * Hkv * D * esz                                                # K and V of one token
    kept = 2 * Hkv * (D // 2 + D // 32) if c["kv_bits"] == 4 else row      # the same in the cache
    if c["kind"] == "rotate":
        T = c["tokens"] or B
        return {"bytes": T * (2 * (Hq + Hkv) * D * esz + 4), "flops": T * (Hq + Hkv) * c["rot_dim"] * 3}
    if c["kind"] == "verify":
        _, count = _trees(c)
        rows = sum(count) + B                                              # one row of the draft's, where a walk ends
        return {"bytes": (rows + (B if c["probs"] else 0)) * V * 4 + B * N * 16, "flops": rows * V * 4}
    plen = _lengths(c)
    if c["kind"] == "draft":
        _, count = _trees(c)
        att = [p + 1 if not c["freeze"] else min(p + 1, c["window"] + c["f_hh"] * max(0, p + 1 - c["window"])) for p in plen]
        return {"bytes": sum(att) * kept + sum(count) * (2 * Hq * D * esz + row),
                "flops": sum(4 * Hq * D * m * (a + m / 2) for a, m in zip(att, count))}
    R, L = c["rounds"], c["layers"]
    att = L * _attended(c, plen, R)
    nodes = sum(sum(_trees(c, r)[1]) for r in range(R))
    return {"bytes": L * sum(plen) * (row + kept) + att * kept + L * nodes * (2 * Hq * D * esz + row) + L * R * B * (Hq * D * (esz + 4) + row + kept)
            + (nodes + R * B * (2 if c["probs"] else 1)) * V * 4,
            "flops": att * 4 * Hq * D * (1 + nodes / (R * B))}


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


def _exact_turn(c, x, pos):
    """Each pair as a complex number times magnitude e^(i pos f)."""
    dim = c["rot_dim"]
    i = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(-(2 * i / dim) * math.log(c["rot_base"]))
    if c["rot_scaling"] == "linear":
        f = f / c["rot_factor"]
    elif c["rot_scaling"] == "bands":
        part = ((c["rot_original"] * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        f = (1 - part) * f / c["rot_factor"] + part * f
    elif c["rot_scaling"] == "ramp":
        where = [dim / 2 * math.log(c["rot_original"] / (2 * math.pi * t)) / math.log(c["rot_base"]) for t in (32.0, 1.0)]
        lo, hi = max(math.floor(where[0]), 0), min(math.ceil(where[1]), dim - 1)
        part = ((i - lo) / (hi - lo if hi != lo else 0.001)).clamp(0, 1)
        f = part * f / c["rot_factor"] + (1 - part) * f
    turn = torch.polar(torch.full((), c["rot_magnitude"], dtype=torch.float64, device="cuda").expand(pos.shape + f.shape).contiguous(),
                       pos.double()[..., None] * f)[..., None, :]
    y = x.double()
    out = y.clone()
    if c["rot_layout"] == "halves":
        z = torch.complex(y[..., :dim // 2].contiguous(), y[..., dim // 2:dim].contiguous()) * turn
        out[..., :dim // 2], out[..., dim // 2:dim] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :dim].unflatten(-1, (-1, 2)).contiguous()) * turn
        out[..., :dim] = torch.view_as_real(z).flatten(-2)
    return out


def _exact_choice(c, ch):
    """Sequence by sequence, on the host."""
    B, N = ch["tokens"].shape
    tokens, par, u, count = (ch[k].cpu().numpy() for k in ("tokens", "parents", "u", "count"))
    root, logits = ch["root"], ch["logits"]

    def target(b, i):
        z = (root[b] if i < 0 else logits[b, i]).cpu().numpy().astype(np.float64)
        if c["temperature"] == 0:
            return np.where(np.arange(len(z)) == np.argmax(z), 1.0, 0.0)
        z = np.exp((z - z.max()) / c["temperature"])
        return z / z.sum()

    path, n_path, nxt = np.full((B, N), -1, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        last, w = -1, target(b, -1)
        for i in range(int(count[b])):
            if par[b, i] != last:
                continue
            x, q = int(tokens[b, i]), None
            if ch["probs"] is not None:
                q = ch["probs"][b, par[b, i] + 1].cpu().numpy().astype(np.float64)
            if np.float64(u[b, i]) * (1.0 if q is None else q[x]) * w.sum() < w[x]:
                path[b, n_path[b]] = last = i
                n_path[b] += 1
                w = target(b, i)
                continue
            rest = np.where(np.arange(len(w)) == x, 0.0, w) if q is None else np.maximum(w / w.sum() - q, 0.0)
            w = rest if rest.sum() > 0 else w
        run = np.cumsum(w)
        nxt[b] = np.argmax(run > np.float64(u[b, N]) * run[-1])
    return path, n_path, nxt


def _exact_attention(q, K, V, on, k, v, sees, count):
    """One sequence: q [N, Hq, D] over K, V [n, Hkv, D] where on, and over the drafts; rows below count."""
    N, Hq, D = q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    out = torch.zeros((N, Hq, D), dtype=torch.float64, device="cuda")
    use = on.nonzero().squeeze(1)
    named = torch.tensor([[bool(m >> j & 1) and j < count for j in range(N)] for m in sees], device="cuda")
    for h in range(Hkv):
        Q = q[:, h * G:(h + 1) * G].reshape(N * G, D) / math.sqrt(D)
        z = torch.cat([Q @ K[use, h].t().contiguous(), Q @ k[:, h].t().contiguous()], 1)
        z[:, len(use):][~named.repeat_interleave(G, 0)] = -math.inf
        out[:, h * G:(h + 1) * G] = (torch.softmax(z, -1) @ torch.cat([V[use, h], v[:, h]])).view(N, G, D)
    out[count:] = 0
    return out.nan_to_num(0.0)          # a row that sees nothing


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    if c["kind"] == "rotate":
        pos = x["pos"] if c["tokens"] else torch.tensor(x["plen"], device="cuda")
        return [_exact_turn(c, x["q"], pos), _exact_turn(c, x["k"], pos)]
    if c["kind"] == "verify":
        return _exact_choice(c, x)
    held = (lambda t: _nearest4(t)) if c["kv_bits"] == 4 else (lambda t: t.double())
    if c["kind"] == "draft":
        B, N = x["q"].shape[:2]
        if sum(x["plen"]) * N * c["kv_heads"] * c["head_dim"] * 3 > 4e11:
            return None
        on = _active_after_one_step(c, x)
        out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for b, p in enumerate(x["plen"]):
            K, V = (torch.cat([held(x[a][at:at + p]), held(x[z][b:b + 1])]) for a, z in (("K", "k0"), ("V", "v0")))
            out[b] = _exact_attention(x["q"][b].double(), K, V, on[b, :p + 1], x["k"][b].double(), x["v"][b].double(),
                                      x["sees"][b].tolist(), int(x["count"][b]))
            at += p
        return out
    R, L, B, N, Hq, D = x["q"].shape
    plen, Hkv = x["plen"], c["kv_heads"]
    if sum(plen) * R * L * (N + 1) * Hkv * D * 3 > 4e11:
        return None
    out, drafts = torch.empty(x["q0"].shape, dtype=torch.float64, device="cuda"), torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    choice = [_exact_choice(c, ch) for ch in x["rounds"]]
    start = [sum(plen[:b]) for b in range(B)]
    rows = torch.zeros((2, B, R * (N + 1), Hkv, D), dtype=torch.float64, device="cuda")
    dt = x["k"].dtype
    for layer in range(L):
        for b in range(B):
            K, V = (held(t[layer][start[b]:start[b] + plen[b]]) for t in (x["K"], x["V"]))
            back = torch.zeros(plen[b], dtype=torch.int64, device="cuda")
            hits = torch.zeros_like(back)
            for r in range(R):
                t, ch, n = r + 1, x["rounds"][r], K.shape[0]
                here = torch.tensor([n], device="cuda")
                # rows are rounded to their type where a call hands them on
                q0, k0 = (_exact_turn(c, x[a][r, layer, b:b + 1], here).to(dt).double() for a in ("q0", "k0"))
                q, k = (_exact_turn(c, x[a][r, layer, b], n + ch["pos"][b]).to(dt).double() for a in ("q", "k"))
                K, V = torch.cat([K, held(k0)]), torch.cat([V, held(x["v0"][r, layer, b:b + 1])])
                back, hits = (torch.cat([a, torch.zeros(1, dtype=torch.int64, device="cuda")]) for a in (back, hits))
                on = back <= t
                use = on.nonzero().squeeze(1)
                y = torch.matmul(q0[0].view(Hkv, Hq // Hkv, D), K[use].permute(1, 2, 0).contiguous())
                out[r, layer, b] = torch.matmul(torch.softmax(y / math.sqrt(D), -1), V[use].transpose(0, 1).contiguous()).reshape(Hq, D)
                drafts[r, layer, b] = _exact_attention(q, K, V, on, k, x["v"][r, layer, b].double(), ch["sees"][b].tolist(), int(ch["count"][b]))
                drop = use[(y.abs().sum((0, 1)) / Hq < 0.5) & (use < n + 1 - c["window"])]
                hits[drop] += 1
                back[drop] = t + hits[drop].double().sqrt().floor().long()
                path, n_path, _ = choice[r]
                took = path[b, :n_path[b]].tolist()
                K, V = torch.cat([K, held(k[took])]), torch.cat([V, held(x["v"][r, layer, b][took])])
                back, hits = (torch.cat([a, torch.zeros(len(took), dtype=torch.int64, device="cuda")]) for a in (back, hits))
            if layer == L - 1:
                rows[0, b, :K.shape[0] - plen[b]], rows[1, b, :V.shape[0] - plen[b]] = K[plen[b]:], V[plen[b]:]
    return {"out": out, "drafts": drafts, "choice": choice, "k": rows[0], "v": rows[1], "counters": None}
