"""Every form of the attention over packed prompts, by name: the four walks over all types, head
dims and query groups, and each of them with a cache held in 4 bits, whose rows the same launch
writes.  Lengths off the tiles' 32, 64 and 128 keys and the workgroups' rows."""
import math

import numpy as np
import pytest

from synth import gen
from tests import _harness as H
from tests._four import rounded
from tests._walks import HALVES, SPLIT, TEAM4, TEAM8, walk
from tests.test_gpu_four_bits import Rounded, _same
from tests.test_gpu_prompt import _check, _init, _inputs, _reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_11221_amd as A
    A.load()
    return torch


# at least 4096 units of 32 rows, over groups of 1, 2, 4 and 8 query heads (rows of 256: 16 KV heads for one)
MANY = {1: [1063, 501] * 11, 2: [307, 99] * 21, 4: [137] * 40 + [0, 1], 8: [97, 0, 33] * 16}
EIGHT = [(g * 8, 8, D, t, MANY[g]) for g in (1, 2, 4, 8) for D, t in ((64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32"))]
EIGHT += [(16, 16, 256, "bf16", [801, 263] * 8)] + [(g * 8, 8, 256, "bf16", MANY[g]) for g in (2, 4, 8)]
# fewer, and prompts below 512 tokens
FOUR = [(8, 8, 128, "bf16", [300, 0, 77] * 5), (16, 8, 128, "bf16", [301, 45] * 4), (32, 8, 128, "bf16", [137, 31] * 3),
        (64, 8, 128, "bf16", [99, 33, 1] * 3), (8, 8, 64, "bf16", [301, 77] * 12), (16, 8, 64, "bf16", [301, 45] * 8),
        (32, 8, 64, "bf16", [137, 31] * 8), (64, 8, 64, "bf16", [97, 33] * 4)]
FOUR += [(g * 2, 2, 256, "bf16", [130, 0, 1, 65, 700]) for g in (1, 2, 4, 8)]
# two waves to a row
TWO = [(16, 8, 128, "bf16", [1025, 0, 3]), (8, 8, 64, "bf16", [4200]), (16, 8, 64, "bf16", [2100, 65]),
       (64, 8, 64, "bf16", [521, 17]), (8, 8, 64, "f32", [141] * 30), (16, 8, 128, "f32", [139, 5] * 16),
       (64, 8, 64, "f32", [33, 0] * 16), (8, 8, 128, "f32", [4300, 33])]
# few rows, keys split over the waves
FEW = [(8, 8, 128, "bf16", [700, 33]), (16, 4, 128, "bf16", [0, 301, 5]), (16, 2, 64, "bf16", [1500]), (64, 8, 64, "f32", [120, 1])]
CASES = [(TEAM8, *c) for c in EIGHT] + [(TEAM4, *c) for c in FOUR] + [(HALVES, *c) for c in TWO] + [(SPLIT, *c) for c in FEW]


def _id(c):
    name, Hq, Hkv, D, dtype, lens = c
    return f"{name.replace(' ', '-')}-{Hq}q{Hkv}kv-{D}-{dtype}"


@pytest.mark.parametrize("what", ["plain", "grow", "fall", "inf", "nan"])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_every_walk(case, what):
    """Outputs, scores that rise or fall along each prompt by far more than one exponent's range, and
    values that are not finite in the first and the last prompt, which reach the tokens from their own
    on in their dim; run again, bitwise the same; the rows in the cache."""
    import torch
    name, Hq, Hkv, D, dtype, lens = case
    assert walk(Hq, Hkv, D, dtype, lens) == name
    G, T = Hq // Hkv, sum(lens)
    A, ctx = _init(len(lens), Hq, Hkv, D, dtype, max(lens) + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype, seed=17)
        if what in ("grow", "fall"):
            ramp = torch.cat([torch.arange(n, device="cuda", dtype=torch.float32) / max(1, n) for n in lens]) * 40
            k[:, :, 3] += (ramp if what == "grow" else 40 - ramp)[:, None].to(k.dtype)
            q[:, :, 3] = 20
        ref, tol = _reference(lens, q, k, v)
        hit = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
        bad = {"inf": math.inf, "nan": math.nan}.get(what)
        vb = v.clone()
        if bad is not None:
            for first, n in ((0, lens[0]), (T - lens[-1], lens[-1])):
                for i, p in enumerate(sorted({0, 31, n // 2, n - 2, n - 1} & set(range(n)))):
                    h = i % Hkv
                    vb[first + p, h, 9 * i + 1] = bad
                    hit[first + p:first + n, h * G:(h + 1) * G, 9 * i + 1] = True
        out = torch.full_like(q, 7.0)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, vb, out)
        got = out[hit].float()
        assert torch.isnan(got).all() if what == "nan" else (got == math.inf).all()
        keep = ~hit
        assert ((out.double() - ref).abs()[keep] <= tol[keep]).all()
        again = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, vb, again)
        bits = torch.int16 if dtype == "bf16" else torch.int32
        assert torch.equal(out.view(bits), again.view(bits))
        at = 0
        for b, n in enumerate(lens):
            if n and (b < 3 or b + 3 > len(lens)):
                kb, vc = torch.empty_like(k[:n]), torch.empty_like(v[:n])
                A.asrkf_get_rows(ctx, 0, b, 0, n, kb, vc)
                assert torch.equal(kb, k[at:at + n]) and torch.equal(vc.view(bits), vb[at:at + n].contiguous().view(bits))
            at += n
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("case", [c for c in CASES if c[4] == "bf16"], ids=_id)
def test_every_walk_into_a_cache_of_4_bits(case):
    """Attention over k and v as given, and their rows rounded into the cache by the same launch; rows
    of the other layer stay as they are."""
    import torch
    name, Hq, Hkv, D, dtype, lens = case
    assert walk(Hq, Hkv, D, dtype, lens) == name
    A, ctx = _init(len(lens), Hq, Hkv, D, dtype, max(lens) + 2, L=2, kv_bits=4)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype, seed=18)
        other = (k * 3).contiguous()
        A.asrkf_prefill_packed(ctx, 1, range(len(lens)), lens, None, other, v, None)
        out = torch.full_like(q, 7.0)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, v, out)
        _check(out, *_reference(lens, q, k, v), sum(lens))
        wk, wv, wo = (rounded(x.float().cpu().numpy()) for x in (k, v, other))
        at = 0
        for b, n in enumerate(lens):
            if n:
                kb, vb = torch.full_like(k[:n], 9.0), torch.full_like(v[:n], 9.0)
                A.asrkf_get_rows(ctx, 0, b, 0, n, kb, vb)
                _same(kb, wk[at:at + n])
                _same(vb, wv[at:at + n])
                A.asrkf_get_rows(ctx, 1, b, 0, n, kb, vb)
                _same(kb, wo[at:at + n])
                _same(vb, wv[at:at + n])
            at += n
    finally:
        A.asrkf_destroy(ctx)


def test_prompts_with_attention_then_4_bit_steps_match_the_oracle():
    """Both operators as a serving program runs them: the prompts of every layer with their attention
    into a cache held in 4 bits (one sequence without a prompt), then freezing decode steps, whose
    states are those of the oracle fed the values that the codes stand for."""
    import torch
    import paper_2512_11221_amd as A
    lens = [90, 0, 41]
    w = gen.Workload(name="packed four", seed=gen.SEED + 317, n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64,
                     dtype="bf16", prefill=lens, steps=30, window_K=8, tau=0.5, k_soft=1.0, vocab=64,
                     logit_sigma=2.0, recipe="hh", f_hh=[0.35, 0.3, 0.25])
    inst = [(l, b) for l in range(2) for b in range(3)]
    inp = H.Inputs(w)
    ctx = A.asrkf_init(A.make_config(2, 3, 8, 2, 64, w.max_ctx, w.window_K, w.tau, w.k_soft, w.vocab,
                                     entropy_spike=w.entropy_spike, dtype="bf16", kv_bits=4))
    try:
        for l in range(2):
            K, V = zip(*(inp.prompt(l, b) for b in range(3)))
            K, V = (H._dev(np.concatenate(x), "bf16") for x in (K, V))
            q = torch.randn((sum(lens), 8, 64), device="cuda", dtype=torch.bfloat16)
            out = torch.empty_like(q)
            A.asrkf_prefill_packed(ctx, l, [0, 1, 2], lens, q, K, V, out)
            _check(out, *_reference(lens, q, K, V), sum(lens))

        class NoPrompts(H.Inputs):          # the harness stores none: they are there
            def prompt(self, layer, seq):
                K, V = super().prompt(layer, seq)
                return K[:0], V[:0]

        g, _, _ = H.run_gpu(w, NoPrompts(w), inst, with_logits=False, ctx=ctx)
    finally:
        A.asrkf_destroy(ctx)
    o = H.run_oracle(w, Rounded(w), inst, with_logits=False)
    assert sum(int(r["frozen"].sum()) for key in inst for r in o[key]) > 0
    for key in inst:
        assert H.compare_instance(g[key], o[key]) < 1e-5
