"""A cache held in 4 bits: the format over every bf16 value, rows written by every
path, and decode steps against the oracle fed the values that the codes stand for."""
import math

import numpy as np
import pytest

from synth import gen
from tests import _harness as H
from tests._four import rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_11221_amd as A
    A.load()
    return torch


def _init(B, Hq, Hkv, D, max_ctx, **kw):
    import paper_2512_11221_amd as A
    return A, A.asrkf_init(A.make_config(kw.pop("L", 1), B, Hq, Hkv, D, max_ctx, 4, 0.5, 2.0, 32, kv_bits=4, **kw))


def _same(x, want):
    """x (bf16 tensor) holds the values of `want`, NaN where it is NaN."""
    np.testing.assert_array_equal(x.float().cpu().numpy(), want.astype(np.float32))


def _store(A, ctx, k, v, seq=0):
    import torch
    n = k.shape[0]
    A.asrkf_prefill_packed(ctx, 0, [seq], [n], None, k, v, None)
    kb, vb = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    A.asrkf_get_rows(ctx, 0, seq, 0, n, kb, vb)
    return kb, vb


def test_every_bf16_value():
    """All 65536 bit patterns, each as the largest of a group (K) and below a few larger ones (V)."""
    import torch
    n = 65536
    bits = torch.arange(n, dtype=torch.int32, device="cuda").to(torch.int16)
    x = bits.view(torch.bfloat16)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    scale = torch.where(x.float().isfinite(), x.float().abs(), torch.ones_like(x.float()))
    k = (torch.rand((n, 1, 64), generator=g, device="cuda") * 2 - 1) * scale[:, None, None]
    v = (torch.rand((n, 1, 64), generator=g, device="cuda") * 2 - 1) * scale[:, None, None] * 16
    k, v = k.clamp(-3e38, 3e38).to(torch.bfloat16), v.clamp(-3e38, 3e38).to(torch.bfloat16)
    k[:, 0, 17] = x
    k[:, 0, 40] = x
    v[:, 0, 63] = x
    A, ctx = _init(1, 1, 1, 64, n + 2)
    try:
        kb, vb = _store(A, ctx, k, v)
        _same(kb, rounded(k.float().cpu().numpy()))
        _same(vb, rounded(v.float().cpu().numpy()))
    finally:
        A.asrkf_destroy(ctx)


def test_ties_and_borders_of_the_scale():
    """The middles between neighbouring values, and largest magnitudes at 7 X and either side of it."""
    import torch
    rows = []
    for e in (-101, -100, -99, -1, 0, 3, 120, 125):
        for top in (3.984375, 4, 5, 6, 6.96875, 7, 7.03125, 7.96875):
            x = np.zeros(64)
            x[0] = top * 2.0 ** e
            x[1:16] = np.arange(1, 16) * 0.25 * 2.0 ** e          # 0.25, 0.75, 1.25, ... are ties
            x[16:31] = -x[1:16]
            x[32:48] = (np.arange(16) * 0.25 + 0.03125) * 2.0 ** e
            rows.append(x)
    x = torch.tensor(np.clip(np.array(rows), -3.3e38, 3.3e38)[:, None, :], device="cuda").to(torch.bfloat16)
    A, ctx = _init(1, 2, 1, 64, len(rows) + 2)
    try:
        kb, vb = _store(A, ctx, x, -x)
        want = rounded(x.float().cpu().numpy())
        _same(kb, want)
        _same(vb, -want)
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 64), (2, 128), (8, 128), (32, 128), (4, 256)])
@pytest.mark.parametrize("lens", [[1], [15, 16, 17], [130, 0, 3]], ids=str)
def test_rows_of_every_layout(Hkv, D, lens):
    """Packed prompts, asrkf_prefill and the appended row hold the same codes; rows of other
    sequences and layers are left as they were."""
    import torch
    B = len(lens)
    A, ctx = _init(B, Hkv, Hkv, D, max(lens) + 4, L=2)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(D + Hkv)
        T = sum(lens)
        k, v = (torch.randn((T, Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16) * 3 for _ in range(2))
        A.asrkf_prefill_packed(ctx, 0, range(B), lens, None, k, v, None)
        at = 0
        for b, n in enumerate(lens):
            if n:
                A.asrkf_prefill(ctx, 1, b, v[at:at + n], k[at:at + n], n)
            at += n
        kn, vn = (torch.randn((B, Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        out = torch.empty((B, Hkv, D), device="cuda")
        A.asrkf_decode_step(ctx, 0, kn, kn, vn, out)
        A.asrkf_decode_step(ctx, 1, kn, vn, kn, out)
        A.asrkf_restore(ctx, None, A.NONE)
        at = 0
        for b, n in enumerate(lens):
            want_k = rounded(torch.cat([k[at:at + n], kn[b:b + 1]]).float().cpu().numpy())
            want_v = rounded(torch.cat([v[at:at + n], vn[b:b + 1]]).float().cpu().numpy())
            at += n
            kb, vb = (torch.full((n + 2, Hkv, D), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            for l, (wk, wv) in enumerate([(want_k, want_v), (want_v, want_k)]):
                A.asrkf_get_rows(ctx, l, b, 0, n + 1, kb[:n + 1], vb[:n + 1])
                _same(kb[:n + 1], wk)
                _same(vb[:n + 1], wv)
                assert (kb[n + 1] == 7).all() and (vb[n + 1] == 7).all()
            A.asrkf_get_rows(ctx, 0, b, n, 1, kb[:1], vb[:1])         # one row in the middle
            _same(kb[:1], want_k[n:])
    finally:
        A.asrkf_destroy(ctx)


def test_rows_read_back_enter_unchanged():
    import torch
    A, ctx = _init(2, 8, 8, 128, 70)
    try:
        k, v = (torch.randn((60, 8, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
        kb, vb = _store(A, ctx, k, v)
        kc, vc = _store(A, ctx, kb, vb, seq=1)
        assert torch.equal(kb, kc) and torch.equal(vb, vc)
    finally:
        A.asrkf_destroy(ctx)


class Rounded(H.Inputs):
    """The inputs as a cache in 4 bits holds them (K and V of every position)."""

    def kv(self, layer, seq):
        key = (layer, seq)
        if key not in self._kv:
            K, V = super().kv(layer, seq)
            self._kv[key] = rounded(K), rounded(V)
        return self._kv[key]


def _run(w, out_tol=1e-5, modes=None, with_logits=True, **kw):
    import paper_2512_11221_amd as A
    inst = [(l, b) for l in range(w.n_layers) for b in range(w.batch)]
    cfg = A.make_config(w.n_layers, w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, w.max_ctx, w.window_K, w.tau,
                        w.k_soft, w.vocab, entropy_spike=w.entropy_spike, conf_drop=w.conf_drop, wr_last_N=w.wr_last_N,
                        dtype=w.dtype, history_W=w.history_W, relevance=w.relevance, scope=w.scope,
                        candidates=w.candidates, kv_bits=4)
    ctx = A.asrkf_init(cfg)
    try:
        g, _, _ = H.run_gpu(w, H.Inputs(w), inst, modes, with_logits, ctx=ctx, **kw)
    finally:
        A.asrkf_destroy(ctx)
    o = H.run_oracle(w, Rounded(w), inst, modes, with_logits)
    frozen = sum(int(r["frozen"].sum()) for k in inst for r in o[k])
    # fp32 sums over at most a few hundred tokens of values of size 1: as with bf16 rows
    worst = max(H.compare_instance(g[k], o[k]) for k in inst)
    assert worst < out_tol, worst
    return frozen


def _workload(**kw):
    base = dict(name="four", seed=gen.SEED + 311, n_layers=1, batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64,
                dtype="bf16", prefill=[150, 71], steps=24, window_K=8, tau=0.5, k_soft=1.0, vocab=256, logit_sigma=2.0,
                recipe="hh", f_hh=[0.35, 0.25])
    base.update(kw)
    return gen.Workload(**base)


@pytest.mark.parametrize("Hq,Hkv,D", [(g * h, h, d) for d, h in ((64, 2), (128, 2), (256, 2), (128, 8)) for g in (1, 2, 4, 8)] +
                         [(32, 32, 128), (1, 1, 64)])
def test_decode_against_the_oracle(Hq, Hkv, D):
    assert _run(_workload(n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D), with_logits=False) > 0


def test_decode_with_recovery_and_layers():
    assert _run(_workload(n_layers=3, steps=28), modes={9: 1, 15: 2, 21: 3}, with_logits=False) > 0


def test_decode_softmax_relevance():
    w = _workload(relevance="softmax", tau=0.004, prefill=[150, 71])
    _check_margin(w, 1e-6)
    _run(w, with_logits=False)


def _check_margin(w, margin):
    """No score that the oracle compares lies within the margin of tau."""
    near = []

    def on(l, b, t, n, Aset, s):
        near.append(float(np.min(np.abs(s - w.tau))))
    H.run_oracle(w, Rounded(w), [(l, b) for l in range(w.n_layers) for b in range(w.batch)], with_logits=False, on_scores=on)
    assert min(near) > margin, min(near)


def test_decode_token_scope_and_history():
    assert _run(_workload(n_layers=2, scope="token", history_W=16, f_hh=[0.1, 0.1]), with_logits=False) > 0


@pytest.mark.parametrize("lens", [[0, 1, 2], [31, 32, 33], [63, 64, 65], [127, 128, 129]], ids=str)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_lengths_around_the_tiles(D, lens):
    _run(_workload(batch=3, prefill=lens, head_dim=D, steps=6, f_hh=[0.3, 0.3, 0.3]), with_logits=False)


def test_decode_large_batches_and_splits():
    """More than 64 sequences (the plan in LDS), and one long sequence that many workgroups share."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 120, 70)]
    _run(_workload(batch=70, prefill=lens, steps=5, f_hh=[0.3] * 70), with_logits=False)
    _run(_workload(batch=1, prefill=[6000], steps=3, f_hh=[0.3], head_dim=128, n_q_heads=8, n_kv_heads=2), with_logits=False)


def _long_step(lens, Hq, Hkv, D, tau, relevance):
    """One step over long lists against 64 bits on the GPU, from the rows as they are held: the
    outputs, and which tokens are found low (those whose score lies clear of tau)."""
    import torch
    B, G, top = len(lens), Hq // Hkv, max(lens)
    import paper_2512_11221_amd as A
    ctx = A.asrkf_init(A.make_config(1, B, Hq, Hkv, D, top + 2, 16, tau, 1.0, 32, relevance=relevance, kv_bits=4))
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(11)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)   # noqa: E731
        T = sum(lens)
        A.asrkf_prefill_packed(ctx, 0, range(B), lens, None, rnd(T, Hkv, D), rnd(T, Hkv, D), None)
        q, out = rnd(B, Hq, D), torch.empty((B, Hq, D), device="cuda")
        A.asrkf_decode_step(ctx, 0, q, rnd(B, Hkv, D), rnd(B, Hkv, D), out)
        A.asrkf_restore(ctx, None, A.NONE)
        for b, n in enumerate(lens):
            k, v = (torch.empty((n + 1, Hkv, D), device="cuda", dtype=torch.bfloat16) for _ in range(2))
            A.asrkf_get_rows(ctx, 0, b, 0, n + 1, k, v)
            K, V = k.double().permute(1, 2, 0).contiguous(), v.double().transpose(0, 1).contiguous()
            x = torch.matmul(q[b].double().view(Hkv, G, D), K)
            p = torch.softmax(x / math.sqrt(D), -1)
            ref, size = torch.matmul(p, V).view(Hq, D), torch.matmul(p, V.abs()).view(Hq, D)
            # scores in fp32 (D 2^-24 of sum |q k| <= 8 D here, over sqrt(D)), twice; sums of n weights
            rel = 2 * D * 2.0 ** -24 * 8 * math.sqrt(D) + 2 * n * 2.0 ** -24 + 2.0 ** -21
            assert ((out[b].double() - ref).abs() <= rel * size).all()
            s = (x.abs() if relevance == "abs" else p).sum((0, 1)) / Hq
            low = (s < tau)[: n + 1 - 16].cpu().numpy()
            clear = ((s - tau).abs() > tau * rel)[: n + 1 - 16].cpu().numpy()
            st = A.asrkf_get_state(ctx, 0, b, top + 2)
            # the check says something: the band left out, 2 rel tau wide (rel <= 3e-3 and tau <= 13:
            # 0.08), holds a small share of scores that spread over several units (softmax: 2 rel
            # of the weights)
            assert n < 1000 or clear.mean() > 0.9 and 0 < low.mean() < 1
            np.testing.assert_array_equal((st["count"][: n + 1 - 16] == 1)[clear], low[clear])
            assert (st["count"][n + 1 - 16:] == 0).all()
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("lens,Hq,Hkv,D,tau,relevance", [
    ([20000, 9000], 8, 2, 128, 8.0, "abs"),             # many workgroups share a pair
    ([33000] * 8 + [1, 700], 16, 8, 64, 6.3, "abs"),    # every wave a head of its own: the relevance room is emptied on the way
    ([33000] * 4, 32, 8, 64, 4e-5, "softmax"),          # a plane per query head: the room holds a quarter of the tiles
    ([17000] * 5, 16, 8, 256, 12.7, "abs"),
], ids=["shared", "heads", "softmax", "rows256"])
def test_long_lists(lens, Hq, Hkv, D, tau, relevance):
    _long_step(lens, Hq, Hkv, D, tau, relevance)


def test_static_entry_graph_and_repeat_are_bitwise_the_same():
    import torch
    A, ctx = _init(2, 8, 2, 128, 600)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(4)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)   # noqa: E731
        k, v = rnd(700, 2, 128), rnd(700, 2, 128)
        q, kn, vn = rnd(8, 2, 8, 128), rnd(8, 2, 2, 128), rnd(8, 2, 2, 128)

        def steps(fn, out, first=0):
            for t in range(first, 8):
                fn(ctx, 0, q[t], kn[t], vn[t], out[t])
                A.asrkf_restore(ctx, None, A.NONE)

        outs = []
        for fn in (A.asrkf_decode_step, A.asrkf_decode_step_static, A.asrkf_decode_step):
            A.asrkf_reset(ctx)
            A.asrkf_prefill_packed(ctx, 0, [0, 1], [400, 300], None, k, v, None)
            outs.append(torch.empty((8, 2, 8, 128), device="cuda"))
            steps(fn, outs[-1])
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        # a captured step, replayed with the inputs of each step
        A.asrkf_reset(ctx)
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [400, 300], None, k, v, None)
        o1 = torch.empty((2, 8, 128), device="cuda")
        A.asrkf_decode_step(ctx, 0, q[0], kn[0], vn[0], o1)
        A.asrkf_restore(ctx, None, A.NONE)
        assert torch.equal(o1, outs[0][0])
        torch.cuda.synchronize()
        qs, ks, vs = q[1].clone(), kn[1].clone(), vn[1].clone()
        s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            A.asrkf_decode_step(ctx, 0, qs, ks, vs, o1, stream=s)
            A.asrkf_restore(ctx, None, A.NONE, stream=s)
        for t in range(1, 8):
            qs.copy_(q[t]), ks.copy_(kn[t]), vs.copy_(vn[t])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o1, outs[0][t]), t
        assert A.asrkf_stats(ctx)["step"] == 8
    finally:
        torch.cuda.synchronize()
        A.asrkf_destroy(ctx)


def test_groups_that_are_not_finite_read_as_nan():
    """A group of V with an infinity is NaN in its 32 dims of the attended output; a group of K
    makes its head's outputs NaN; other heads and sequences stay finite."""
    import torch
    A, ctx = _init(2, 4, 2, 64, 64)
    try:
        k, v = (torch.randn((40, 2, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
        v[7, 0, 40] = math.inf                    # sequence 0, KV head 0, dims 32 .. 63
        k[25, 1, 3] = math.nan                    # sequence 1 (tokens 20 ..), KV head 1
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [20, 20], None, k, v, None)
        q = torch.randn((2, 4, 64), device="cuda", dtype=torch.bfloat16)
        out = torch.empty((2, 4, 64), device="cuda")
        A.asrkf_decode_step(ctx, 0, q, k[:2].contiguous(), k[2:4].contiguous(), out)
        nan = torch.isnan(out)
        want = torch.zeros_like(nan)
        want[0, :2, 32:] = True
        want[1, 2:] = True
        assert torch.equal(nan, want)
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 64), (8, 2, 64), (16, 2, 64), (8, 2, 128), (16, 2, 128), (8, 2, 256)])
def test_keys_that_are_not_finite_leave_other_tokens_scores(Hq, Hkv, D):
    """Eq. 2 scores are each token's own.  Under a threshold above all of them every token outside
    the window is detected but those whose key holds a NaN, as with bf16 rows of the same values."""
    import torch
    import paper_2512_11221_amd as A
    n, K = 200, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(D)
    k, v = (torch.randn((n, Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    bad = (0, 37, 90, 133)
    for i, p in enumerate(bad):
        k[p, i % Hkv, i * 11 % D] = (math.nan, math.inf, -math.inf, math.nan)[i]
    q = torch.randn((1, Hq, D), generator=g, device="cuda", dtype=torch.bfloat16)
    out = torch.empty((1, Hq, D), device="cuda")
    counts = []
    rows = k, v
    for bits in (4, 0):
        ctx = A.asrkf_init(A.make_config(1, 1, Hq, Hkv, D, n + 8, K, 1e9, 2.0, 32, kv_bits=bits))
        try:
            A.asrkf_prefill_packed(ctx, 0, [0], [n], None, *rows, None)
            if bits:
                rows = torch.empty_like(k), torch.empty_like(v)
                A.asrkf_get_rows(ctx, 0, 0, 0, n, *rows)
            A.asrkf_decode_step(ctx, 0, q, k[50:51].contiguous(), v[50:51].contiguous(), out)
            A.asrkf_restore(ctx, None, A.NONE)
            counts.append(A.asrkf_get_state(ctx, 0, 0, n + 8)["count"])
        finally:
            torch.cuda.synchronize()
            A.asrkf_destroy(ctx)
    np.testing.assert_array_equal(counts[0], counts[1])
    want = np.ones(n - 2 * K, np.int32)               # well before the window
    want[list(bad)] = 0
    np.testing.assert_array_equal(counts[0][:n - 2 * K], want)


def test_refusals():
    import torch
    A, ctx = _init(1, 8, 2, 64, 64)
    try:
        k = torch.zeros((10, 2, 64), device="cuda", dtype=torch.bfloat16)
        for bad in (k.cpu(), torch.zeros(10 * 128 + 4, device="cuda", dtype=torch.bfloat16)[4:]):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_prefill(ctx, 0, 0, bad, k, 10)
            assert e.value.code == A._lib.EINVAL
        assert A.asrkf_get_state(ctx, 0, 0, 64)["n"] == 0
        A.asrkf_prefill(ctx, 0, 0, k, k, 10)
        with pytest.raises(ValueError):
            A.asrkf_get_rows(ctx, 0, 0, 0, 10, k.transpose(0, 1), k)
        with pytest.raises(A.AsrkfError) as e:
            A.asrkf_get_rows(ctx, 0, 0, 0, 10, k.cpu(), k)
        assert e.value.code == A._lib.EINVAL
    finally:
        A.asrkf_destroy(ctx)
