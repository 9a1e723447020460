"""Packed prompts and 4-bit rows where offsets pass 32 bits, in spill mode, and in several calls."""
import math

import numpy as np
import pytest

from synth import gen
from tests import _harness as H
from tests._four import rounded
from tests.test_gpu_four_bits import _same
from tests.test_gpu_prompt import _check, _init, _inputs, _reference, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def test_prompts_past_4_gib():
    """Queries and outputs of 5 GB: the first, some middle and the last prompts against 64 bits, and the
    rows of the last."""
    import torch
    B, n, Hq, Hkv, D = 130, 4801, 32, 8, 128              # two launches
    lens = [n] * B
    A, ctx = _init(B, Hq, Hkv, D, "bf16", n + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, "bf16")
        assert q.numel() * 2 > 1 << 32
        out = torch.full_like(q, 7.0)
        A.asrkf_prefill_packed(ctx, 0, range(B), lens, q, k, v, out)
        for b in (0, 63, B - 3, B - 1):
            at = slice(b * n, b * n + n)
            _check(out[at], *_reference([n], q[at], k[at], v[at]), n)
        kb, vb = torch.empty_like(k[:n]), torch.empty_like(v[:n])
        A.asrkf_get_rows(ctx, 0, B - 1, 0, n, kb, vb)
        assert torch.equal(kb, k[-n:]) and torch.equal(vb, v[-n:])
    finally:
        A.asrkf_destroy(ctx)


def test_a_cache_of_4_bits_past_4_gib():
    """Codes of 6 GB a pool: the last sequence's rows of every layer, and decode steps that append to
    and attend over them."""
    import torch
    B, L, Hkv, D, n = 64, 3, 8, 128, 300
    A, ctx = _init(B, Hkv, Hkv, D, "bf16", 65600, L=L, kv_bits=4)
    try:
        assert L * B * 65600 * Hkv * D // 2 > 1 << 32
        g = torch.Generator(device="cuda")
        g.manual_seed(8)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)   # noqa: E731
        k, v = rnd(L, n, Hkv, D), rnd(L, n, Hkv, D)
        for l in range(L):
            A.asrkf_prefill_packed(ctx, l, [B - 1], [n], None, k[l], v[l], None)
        q, kn, vn = rnd(2, L, B, Hkv, D), rnd(2, L, B, Hkv, D), rnd(2, L, B, Hkv, D)
        out = torch.empty((2, L, B, Hkv, D), device="cuda")
        for t in range(2):
            for l in range(L):
                A.asrkf_decode_step(ctx, l, q[t, l], kn[t, l], vn[t, l], out[t, l])
            A.asrkf_restore(ctx, None, A.NONE)
        for l in range(L):
            kb, vb = torch.empty((2, n + 2, Hkv, D), device="cuda", dtype=torch.bfloat16)
            A.asrkf_get_rows(ctx, l, B - 1, 0, n + 2, kb, vb)
            _same(kb, rounded(torch.cat([k[l], kn[:, l, B - 1]]).float().cpu().numpy()))
            _same(vb, rounded(torch.cat([v[l], vn[:, l, B - 1]]).float().cpu().numpy()))
            for t in range(2):
                K, V = kb[:n + t + 1].double(), vb[:n + t + 1].double()
                x = torch.matmul(K.permute(1, 0, 2).contiguous(), q[t, l, B - 1].double().unsqueeze(2)).squeeze(2) / math.sqrt(D)
                p = torch.softmax(x, -1).unsqueeze(1)
                ref = torch.matmul(p, V.transpose(0, 1).contiguous()).squeeze(1)
                size = torch.matmul(p, V.abs().transpose(0, 1).contiguous()).squeeze(1)
                # scores in fp32 (D 2^-24 of sum |q k| <= 8 D, over sqrt(D)), twice; sums of n weights
                rel = 2 * D * 2.0 ** -24 * 8 * math.sqrt(D) + 2 * (n + 2) * 2.0 ** -24 + 2.0 ** -21
                assert ((out[t, l, B - 1].double() - ref).abs() <= rel * size).all()
            # the others have their new rows only
            A.asrkf_get_rows(ctx, l, 5, 0, 2, kb[:2], vb[:2])
            _same(kb[:2], rounded(kn[:, l, 5].float().cpu().numpy()))
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("device_rows", [0, 215])
def test_packed_prompts_then_spill_steps_match_the_oracle(device_rows):
    """Prompts of two sequences in two calls with their attention, and one without a prompt; then steps
    whose frozen rows leave the device."""
    import torch
    import paper_2512_11221_amd as A
    lens = [200, 0, 130]
    w = gen.Workload(name="packed spill", seed=gen.SEED + 331, n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64,
                     dtype="bf16", prefill=lens, steps=24, window_K=32, tau=math.inf, k_soft=1.0, vocab=64,
                     logit_sigma=1.0, recipe="gauss", spill_min_D=2, device_rows=device_rows)
    inst = [(l, b) for l in range(2) for b in range(3)]
    inp = H.Inputs(w)
    ctx = A.asrkf_init(A.make_config(2, 3, 8, 2, 64, w.max_ctx, w.window_K, w.tau, w.k_soft, w.vocab, dtype="bf16",
                                     entropy_spike=w.entropy_spike, spill_min_D=2, device_rows=device_rows))
    try:
        for l in range(2):
            for b in (2, 0):
                K, V = (H._dev(x, "bf16") for x in inp.prompt(l, b))
                q = torch.randn((lens[b], 8, 64), device="cuda", dtype=torch.bfloat16)
                out = torch.empty_like(q)
                A.asrkf_prefill_packed(ctx, l, [b], [lens[b]], q, K, V, out)
                _check(out, *_reference([lens[b]], q, K, V), lens[b])
            A.asrkf_prefill_packed(ctx, l, [1], [0], None, None, None, None)

        class NoPrompts(H.Inputs):          # the harness stores none: they are there
            def prompt(self, layer, seq):
                K, V = super().prompt(layer, seq)
                return K[:0], V[:0]

        g, _, stats = H.run_gpu(w, NoPrompts(w), inst, with_logits=False, ctx=ctx)
    finally:
        A.asrkf_destroy(ctx)
    o = H.run_oracle(w, inp, inst, with_logits=False)
    assert stats[-1]["rows_to_host"] > 0
    for key in inst:
        assert H.compare_instance(g[key], o[key]) < 1e-5
        H.compare_residency(w, g[key], o[key])
    assert np.isfinite([r["out"] for r in g[0, 1]]).all()
