"""Attention over packed prompts (asrkf_prefill_packed): every type and head layout
at lengths around the tiles' edges against 64 bits, values that are not finite,
strides, refusals, streams and graphs, and a run with the decode steps behind it."""
import math

import numpy as np
import pytest

from synth import gen
from tests import _harness as H
from tests import _walks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_11221_amd as A
    A.load()
    return torch


def _init(B, Hq, Hkv, D, dtype, max_ctx, **kw):
    import paper_2512_11221_amd as A
    return A, A.asrkf_init(A.make_config(kw.pop("L", 1), B, Hq, Hkv, D, max_ctx, 4, 0.5, 2.0, 32, dtype=dtype, **kw))


def _inputs(lens, Hq, Hkv, D, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    T = max(1, sum(lens))
    return [torch.randn((T, h, D), generator=g, device="cuda", dtype=dt) * s for h, s in ((Hq, 1.5), (Hkv, 1), (Hkv, 1))]


def _reference(lens, q, k, v):
    """Outputs in 64 bits; the bound of every output's error, by its type.

    A = sum_j p_j |v_j| of an output.  Rounding a weight to bf16 moves it by 2^-8 of
    itself at most, the output's own rounding the output by 2^-8 (fp32: 2^-24 each).  A score
    is a sum of D products in fp32, off by at most D 2^-24 sum |q k|, which moves its
    weight by that over sqrt(D), relatively, and the sum of the weights as much; the
    exponential, the sums over the tokens (n 2^-24) and the division come on top."""
    import torch
    Hq, Hkv, D = q.shape[1], k.shape[1], q.shape[2]
    G = Hq // Hkv
    half_step = torch.finfo(q.dtype).eps / 2
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    tol = torch.empty_like(out)
    at = 0
    for n in lens:
        for h in range(Hkv if n else 0):
            Q = q[at:at + n, h * G:(h + 1) * G].double().reshape(n * G, D)
            K, V = k[at:at + n, h].double(), v[at:at + n, h].double()
            behind = torch.arange(n, device=q.device) > torch.arange(n, device=q.device).repeat_interleave(G)[:, None]
            p = torch.softmax((Q @ K.t().contiguous() / math.sqrt(D)).masked_fill(behind, -math.inf), -1)
            size = float((Q.abs() @ K.abs().t().contiguous()).max())
            o, A = p @ V, p @ V.abs()
            rel = 2 * D * 2.0 ** -24 * size / math.sqrt(D) + 2 * n * 2.0 ** -24 + 2.0 ** -21
            out[at:at + n, h * G:(h + 1) * G] = o.view(n, G, D)
            tol[at:at + n, h * G:(h + 1) * G] = (half_step * (o.abs() + 1.01 * A) + rel * A).view(n, G, D)
        at += n
    return out, tol


def _check(out, ref, tol, T):
    err = (out[:T].double() - ref[:T]).abs()
    worst = float((err / tol[:T].clamp(min=1e-300)).max()) if T else 0.0
    assert worst <= 1.0, worst


LAYOUTS = [(8, 8, 64), (4, 2, 64), (8, 2, 64), (16, 2, 64), (4, 4, 128), (8, 4, 128), (8, 2, 128), (8, 1, 128)]
LENGTHS = [[1], [2, 1, 3], [31, 32, 33, 1], [63, 65, 64], [0, 127, 0, 129, 128], [300, 5, 17]]


@pytest.mark.parametrize("lens", LENGTHS, ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("Hq,Hkv,D,dtype", [(*x, t) for x in LAYOUTS for t in ("bf16", "f32")] +
                         [(g * 2, 2, 256, "bf16") for g in (1, 2, 4, 8)])
def test_outputs(Hq, Hkv, D, dtype, lens):
    import torch
    A, ctx = _init(len(lens), Hq, Hkv, D, dtype, max(lens) + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype)
        out = torch.full_like(q, 7.0)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, v, out)
        ref, tol = _reference(lens, q, k, v)
        _check(out, ref, tol, sum(lens))
        at = 0
        for b, n in enumerate(lens):              # the rows in the cache
            if n == 0:
                continue
            kb, vb = torch.empty_like(k[:n]), torch.empty_like(v[:n])
            A.asrkf_get_rows(ctx, 0, b, 0, n, kb, vb)
            assert torch.equal(kb, k[at:at + n]) and torch.equal(vb, v[at:at + n])
            at += n
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("Hq,Hkv,D,dtype,n", [(32, 8, 128, "bf16", 1500), (32, 8, 128, "bf16", 2048),
                                              (8, 8, 128, "bf16", 3000), (16, 8, 256, "bf16", 1025),
                                              (16, 2, 64, "bf16", 2500), (8, 2, 64, "f32", 2000),
                                              (32, 8, 128, "f32", 700), (64, 8, 128, "bf16", 600)])
def test_long_prompts(Hq, Hkv, D, dtype, n):
    import torch
    lens = [n, n // 7]
    A, ctx = _init(2, Hq, Hkv, D, dtype, n + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype, seed=3)
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [1, 0], lens, q, k, v, out)
        ref, tol = _reference(lens, q, k, v)
        _check(out, ref, tol, sum(lens))
    finally:
        A.asrkf_destroy(ctx)


def test_many_sequences():
    """More sequences than one launch's table holds, in another order than the context's."""
    import torch
    B = 500
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 70, B)]
    seqs = [int(x) for x in rng.permutation(B)]
    A, ctx = _init(B, 8, 2, 64, "bf16", 80)
    try:
        q, k, v = _inputs(lens, 8, 2, 64, "bf16")
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, seqs, lens, q, k, v, out)
        ref, tol = _reference(lens, q, k, v)
        _check(out, ref, tol, sum(lens))
        at = 0
        for b, n in zip(seqs, lens):
            assert A.asrkf_get_state(ctx, 0, b, 80)["n"] == n
            if n:
                kb, vb = torch.empty_like(k[:n]), torch.empty_like(v[:n])
                A.asrkf_get_rows(ctx, 0, b, 0, n, kb, vb)
                assert torch.equal(kb, k[at:at + n]) and torch.equal(vb, v[at:at + n])
            at += n
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 256), ("f32", 64)])
def test_scores_that_grow(dtype, D):
    """Scores that rise along the prompt by far more than one exponent's range, so that
    every tile brings a new maximum, and scores that fall."""
    import torch
    n = 260
    A, ctx = _init(2, 4, 2, D, dtype, n + 2)
    try:
        q, k, v = _inputs([n, n], 4, 2, D, dtype)
        ramp = torch.arange(n, device="cuda", dtype=torch.float32) / n * 40
        axis = torch.zeros(D, device="cuda")
        axis[3] = 1
        k[:n] = k[:n] + (ramp[:, None, None] * axis).to(k.dtype)
        k[n:] = k[n:] + (ramp.flip(0)[:, None, None] * axis).to(k.dtype)
        q[:, :, 3] = 20
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [n, n], q, k, v, out)
        ref, tol = _reference([n, n], q, k, v)
        _check(out, ref, tol, 2 * n)
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_stay_behind_their_token(dtype, D, bad):
    """A value of v that is not finite reaches the tokens from its own on, in its dim; the
    others, and the other sequence, are as without it."""
    import torch
    n, at = 200, (70, 130, 199)
    A, ctx = _init(2, 4, 2, D, dtype, n + 2)
    try:
        q, k, v = _inputs([n, n], 4, 2, D, dtype)
        ref, tol = _reference([n, n], q, k, v)
        vb = v.clone()
        for i, p in enumerate(at):
            vb[p, 1, 5 + 20 * i] = bad
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [n, n], q, k, vb, out)
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        for i, p in enumerate(at):
            hit[p:n, 2:4, 5 + 20 * i] = True
        got = out[hit].float()
        assert torch.isnan(got).all() if math.isnan(bad) else (got == bad).all()
        keep = ~hit
        assert ((out.double() - ref).abs()[keep] <= tol[keep]).all()
    finally:
        A.asrkf_destroy(ctx)


# two waves to a row, with half of a tile's keys each: medium prompts
HALVES = [(32, 8, 128, "bf16", [513, 65, 1]), (32, 8, 128, "bf16", [0, 640]), (8, 8, 128, "bf16", [2049, 300]),
          (64, 8, 128, "bf16", [512]), (32, 8, 64, "bf16", [1100]), (32, 8, 64, "f32", [1030, 1, 0, 40]),
          (32, 8, 128, "f32", [1025, 31]), (32, 8, 128, "f32", [140] * 8)]


@pytest.mark.parametrize("Hq,Hkv,D,dtype,lens", HALVES, ids=str)
@pytest.mark.parametrize("what", ["plain", "grow", "fall", "inf", "nan"])
def test_medium_prompts(Hq, Hkv, D, dtype, lens, what):
    """Outputs, scores that rise or fall along the prompt, and values that are not finite in
    either half of a tile, which reach the tokens from their own on in their dim."""
    import torch
    T, n = sum(lens), max(lens)
    first = sum(lens[:lens.index(n)])
    A, ctx = _init(len(lens), Hq, Hkv, D, dtype, n + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype, seed=9)
        if what in ("grow", "fall"):
            ramp = torch.arange(T, device="cuda", dtype=torch.float32) / T * 40
            k[:, :, 3] += (ramp if what == "grow" else ramp.flip(0))[:, None].to(k.dtype)
            q[:, :, 3] = 20
        ref, tol = _reference(lens, q, k, v)
        hit = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
        bad = {"inf": math.inf, "nan": math.nan}.get(what)
        vb = v.clone()
        if bad is not None:
            G = Hq // Hkv
            for i, p in enumerate((0, 33, 70, 101, 128 if n > 128 else 127, n - 1)):
                h = i % min(Hkv, 2)
                vb[first + p, h, 7 * i] = bad
                hit[first + p:first + n, h * G:(h + 1) * G, 7 * i] = True
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, vb, out)
        got = out[hit].float()
        assert torch.isnan(got).all() if what == "nan" else (got == math.inf).all()
        keep = ~hit
        assert ((out.double() - ref).abs()[keep] <= tol[keep]).all()
        again = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, vb, again)
        assert torch.equal(out.view(torch.int16 if dtype == "bf16" else torch.int32),
                           again.view(torch.int16 if dtype == "bf16" else torch.int32))
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_that_are_not_finite(dtype):
    """A NaN key makes the outputs of its token and the later ones NaN (of its KV head); a
    key whose score is -inf weighs nothing."""
    import torch
    n, p = 150, 77
    A, ctx = _init(1, 4, 2, 64, dtype, n + 2)
    try:
        q, k, v = _inputs([n], 4, 2, 64, dtype)
        ref, tol = _reference([n], q, k, v)
        kb = k.clone()
        kb[p, 0, 9] = math.nan
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, kb, v, out)
        assert torch.isnan(out[p:, :2]).all()
        assert ((out.double() - ref).abs() <= tol)[:p].all() and ((out.double() - ref).abs() <= tol)[:, 2:].all()
        q2, kb = q.clone(), k.clone()
        q2[:, :2, 9] = q2[:, :2, 9].abs() + 0.5
        kb[p, 0, 9] = -math.inf
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q2, kb, v, out)
        rows = [i for i in range(n) if i != p]
        Q, K, V = q2[:, :2].double(), kb[rows, 0].double(), v[rows, 0].double()
        for i in (0, p - 1, p, p + 1, n - 1):
            m = sum(r <= i for r in rows)
            w = torch.softmax(Q[i] @ K[:m].t() / 8, -1)
            # weights and output rounded by half a step each, and the scores' rounding as above
            assert ((out[i, :2].double() - w @ V[:m]).abs() <= 1.1 * torch.finfo(q.dtype).eps * (w @ V[:m].abs()) + 1e-5).all()
    finally:
        A.asrkf_destroy(ctx)


def test_large_values_do_not_overflow():
    """Values at the type's largest: the outputs are averages and stay finite."""
    import torch
    n = 300
    A, ctx = _init(1, 4, 2, 64, "bf16", n + 2)
    try:
        q, k, v = _inputs([n], 4, 2, 64, "bf16")
        big = torch.finfo(torch.bfloat16).max / 512          # n of them stay within fp32
        v = torch.full_like(v, big)
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, k, v, out)
        # weights and output rounded by half a step each
        assert ((out.double() / big - 1).abs() <= 2.0 ** -7).all()
    finally:
        A.asrkf_destroy(ctx)


# (q heads, KV heads, head dim, lengths) in each walk: one key set for few rows, two waves to a
# row, four waves, eight waves
LARGE = [(4, 2, 64, "bf16", [300, 1]), (8, 2, 64, "bf16", [3000]), (32, 8, 128, "bf16", [700]), (32, 8, 128, "bf16", [400] * 3),
         (32, 8, 128, "bf16", [2100] * 2), (8, 4, 256, "bf16", [513]), (8, 2, 64, "f32", [2000]),
         (32, 8, 64, "f32", [1100]), (32, 8, 128, "f32", [700] * 6)]


@pytest.mark.parametrize("Hq,Hkv,D,dtype,lens", LARGE, ids=str)
@pytest.mark.parametrize("what", ["same", "even", "signs"])
def test_values_at_the_largest(Hq, Hkv, D, dtype, lens, what):
    """Outputs are averages: with values at their type's largest (fp32: below it by more than the sums'
    rounding, 2 n 2^-24 < 2^-10) they are finite and as near as others.  All values alike under
    scores that differ and that do not, and values of both signs."""
    import torch
    A, ctx = _init(len(lens), Hq, Hkv, D, dtype, max(lens) + 2)
    try:
        q, k, v = _inputs(lens, Hq, Hkv, D, dtype, seed=21)
        big = torch.finfo(v.dtype).max * (1 - (2.0 ** -9 if dtype == "f32" else 0))
        if what == "signs":
            v = torch.where(v > 0.3, big, -big).to(v.dtype)
        else:
            v = torch.full_like(v, big)
        if what == "even":
            q.zero_()
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, q, k, v, out)
        assert torch.isfinite(out).all()
        _check(out, *_reference(lens, q, k, v), sum(lens))
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_strides(dtype):
    """q, k and v as slices of one fused projection, and rows far apart."""
    import torch
    n = 140
    A, ctx = _init(1, 8, 2, 64, dtype, n + 2)
    try:
        q, k, v = _inputs([n], 8, 2, 64, dtype)
        ref, tol = _reference([n], q, k, v)
        fused = torch.cat([q, k, v], 1)
        out = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], fused[:, :8], fused[:, 8:10], fused[:, 10:], out)
        _check(out, ref, tol, n)
        kb, vb = torch.empty_like(k), torch.empty_like(v)
        A.asrkf_get_rows(ctx, 0, 0, 0, n, kb, vb)
        assert torch.equal(kb, k) and torch.equal(vb, v)
        wide = torch.zeros((n, 300, 64), dtype=k.dtype, device="cuda")
        wide[:, 100:102] = k
        out2 = torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, wide[:, 100:102], v, out2)
        assert torch.equal(out, out2)
    finally:
        A.asrkf_destroy(ctx)


def test_longest_token_stride():
    """A stride of 16 MiB from one token to the next: tiles reach past 2 GiB in all."""
    import torch
    n, stride = 200, (16 << 20) // 2
    A, ctx = _init(1, 2, 1, 64, "bf16", n + 2)
    try:
        q, k, v = _inputs([n], 2, 1, 64, "bf16")
        far = torch.empty((n - 1) * stride + 64, dtype=torch.bfloat16, device="cuda").as_strided((n, 1, 64), (stride, 64, 1))
        far.copy_(k)
        out, out2 = torch.empty_like(q), torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, k, v, out)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, far, v, out2)
        assert torch.equal(out, out2)
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("Hq,Hkv,D,n,walk", [(16, 2, 128, 520, _walks.HALVES), (64, 8, 64, 520, _walks.HALVES),
                                             (32, 8, 128, 300, _walks.TEAM4)])
def test_longest_token_stride_in_larger_tiles(Hq, Hkv, D, n, walk):
    """... in tiles of 64 and 128 keys, k and v slices of one array whose tiles span up to 2 GiB."""
    import torch
    assert _walks.walk(Hq, Hkv, D, "bf16", [n]) == walk
    stride = (16 << 20) // 2
    A, ctx = _init(1, Hq, Hkv, D, "bf16", n + 2)
    try:
        q, k, v = _inputs([n], Hq, Hkv, D, "bf16")
        far = torch.empty((n - 1) * stride + 2 * Hkv * D, dtype=torch.bfloat16, device="cuda")
        far = far.as_strided((n, 2 * Hkv, D), (stride, D, 1))
        far[:, :Hkv] = k
        far[:, Hkv:] = v
        out, out2 = torch.empty_like(q), torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, k, v, out)
        _check(out, *_reference([n], q, k, v), n)
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, far[:, :Hkv], far[:, Hkv:], out2)
        assert torch.equal(out, out2)
        kb, vb = torch.empty_like(k), torch.empty_like(v)
        A.asrkf_get_rows(ctx, 0, 0, 0, n, kb, vb)
        assert torch.equal(kb, k) and torch.equal(vb, v)
    finally:
        A.asrkf_destroy(ctx)


def test_outputs_do_not_depend_on_the_batch_and_repeat():
    """A sequence's outputs are bitwise the same alone and packed with others, run again, on
    another stream, and on calls that overlap in time."""
    import torch
    lens = [200, 333, 64]
    A, ctx = _init(3, 8, 2, 128, "bf16", 340)
    try:
        q, k, v = _inputs(lens, 8, 2, 128, "bf16")
        out, again = torch.empty_like(q), torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0, 1, 2], lens, q, k, v, out)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        A.asrkf_prefill_packed(ctx, 0, [0, 1, 2], lens, q, k, v, again, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, again)
        one = torch.empty_like(q[200:533])
        A.asrkf_prefill_packed(ctx, 0, [1], [333], q[200:533], k[200:533], v[200:533], one)
        assert torch.equal(one, out[200:533])
    finally:
        A.asrkf_destroy(ctx)


def test_two_contexts_at_once():
    import torch
    n = 700
    runs = []
    try:
        for i in range(2):
            A, ctx = _init(1, 8, 2, 64, "bf16", n + 2)
            x = _inputs([n], 8, 2, 64, "bf16", seed=i)
            runs.append((A, ctx, x, torch.empty_like(x[0]), torch.cuda.Stream()))
        torch.cuda.synchronize()
        for _ in range(3):
            for A, ctx, x, out, s in runs:
                A.asrkf_prefill_packed(ctx, 0, [0], [n], *x, out, stream=s)
        torch.cuda.synchronize()
        for A, ctx, x, out, s in runs:
            _check(out, *_reference([n], *x), n)
    finally:
        for A, ctx, *_ in runs:
            A.asrkf_destroy(ctx)


def test_captured_and_replayed():
    import torch
    lens = [150, 70]
    A, ctx = _init(2, 8, 2, 64, "bf16", 160)
    try:
        q, k, v = _inputs(lens, 8, 2, 64, "bf16")
        eager, out = torch.empty_like(q), torch.empty_like(q)
        A.asrkf_prefill_packed(ctx, 0, [0, 1], lens, q, k, v, eager)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            A.asrkf_prefill_packed(ctx, 0, [0, 1], lens, q, k, v, out, stream=s)
        for i in range(3):
            out.zero_()
            q.mul_(1.25)
            g.replay()
            A.asrkf_prefill_packed(ctx, 0, [0, 1], lens, q, k, v, eager)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
    finally:
        torch.cuda.synchronize()
        A.asrkf_destroy(ctx)


def test_refusals():
    import torch
    A, ctx = _init(2, 8, 2, 64, "bf16", 64, L=2)
    E = A._lib

    def code(*a, **kw):
        with pytest.raises(A.AsrkfError) as e:
            A.asrkf_prefill_packed(ctx, *a, **kw)
        return e.value.code

    try:
        q, k, v = _inputs([20, 20], 8, 2, 64, "bf16")
        out = torch.zeros_like(q)
        ok = (q, k, v, out)
        assert code(2, [0], [20], *ok) == E.EINVAL
        assert code(-1, [0], [20], *ok) == E.EINVAL
        assert code(0, [], [], *ok) == E.EINVAL
        assert code(0, [0, 1, 0], [5, 5, 5], *ok) == E.EINVAL
        assert code(0, [0, 0], [5, 5], *ok) == E.EINVAL
        assert code(0, [2], [5], *ok) == E.EINVAL
        assert code(0, [-1], [5], *ok) == E.EINVAL
        assert code(0, [0], [-1], *ok) == E.EINVAL
        assert code(0, [0], [64], *ok) == E.EINVAL
        assert code(0, [0], [20], None, k, v, out) == E.EINVAL
        assert code(0, [0], [20], q, k, v, None) == E.EINVAL
        assert code(0, [0], [20], q, None, v, out) == E.EINVAL
        assert code(0, [0], [20], q.cpu(), k, v, out) == E.EINVAL
        flat = torch.zeros(40 * 8 * 64 + 4, dtype=torch.bfloat16, device="cuda")
        assert code(0, [0], [20], q, k, v, flat[4:]) == E.EINVAL             # 8-byte offset
        thin = torch.zeros((40, 2, 68), dtype=torch.bfloat16, device="cuda")[:, :, :64]
        with pytest.raises(ValueError):
            A.asrkf_prefill_packed(ctx, 0, [0], [20], q, thin, v, out)
        with pytest.raises(ValueError):
            A.asrkf_prefill_packed(ctx, 0, [0, 1], [20], *ok)
        with pytest.raises(ValueError):
            A.asrkf_prefill_packed(ctx, 0, [0], [20], q, k, v, out[:, :, :32])
        lib = A.load()
        import ctypes
        i32 = ctypes.c_int32

        def raw(qs, ks, vs):
            return lib.asrkf_prefill_packed(ctx, 0, 1, (i32 * 1)(0), (i32 * 1)(20), q.data_ptr(), qs, k.data_ptr(), ks,
                                            v.data_ptr(), vs, out.data_ptr(), None)
        for bad in ((-8, 0, 0), (64, 0, 0), (0, 127, 0), (0, 132, 0), (0, 0, (16 << 20) // 2 + 8), (1 << 40, 0, 0)):
            assert raw(*bad) == E.EINVAL, bad
        assert lib.asrkf_prefill_packed(ctx, 0, 1, None, None, None, 0, k.data_ptr(), 0, v.data_ptr(), 0, None, None) == E.EINVAL
        assert float(out.abs().max()) == 0 and A.asrkf_get_state(ctx, 0, 0, 64)["n"] == 0     # nothing was done
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [20, 0], q, k, v, out)
        assert code(1, [0], [19], *ok) == E.EINVAL          # another length in another layer
        assert code(1, [1], [3], *ok) == E.EINVAL
        with pytest.raises(A.AsrkfError):
            A.asrkf_prefill(ctx, 1, 1, k, v, 3)
        A.asrkf_prefill_packed(ctx, 1, [1, 0], [0, 20], None, k, v, None)
        rows = torch.empty_like(k[:20])
        for a in ((0, 0, 0, 21), (0, 0, -1, 2), (0, 0, 0, 0), (0, 1, 0, 1), (2, 0, 0, 1), (0, 2, 0, 1)):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_get_rows(ctx, *a, rows, rows)
            assert e.value.code == E.EINVAL
        qn, kn, on = q[:2].clone(), k[:2].clone(), torch.empty((2, 8, 64), device="cuda")
        for l in range(2):
            A.asrkf_decode_step(ctx, l, qn, kn, kn, on)
        A.asrkf_restore(ctx, None, A.NONE)
        assert code(0, [0], [20], *ok) == E.ESTATE
    finally:
        A.asrkf_destroy(ctx)


def test_prompts_that_are_all_empty():
    """Empty tensors have null pointers; the sequences then have no prompt, as if never named."""
    import torch
    A, ctx = _init(2, 8, 2, 64, "bf16", 64)
    try:
        q, k = (torch.empty((0, h, 64), device="cuda", dtype=torch.bfloat16) for h in (8, 2))
        A.asrkf_prefill_packed(ctx, 0, [1, 0], [0, 0], q, k, k, torch.empty_like(q))
        A.asrkf_prefill_packed(ctx, 0, [0, 1], [0, 0], None, None, None, None)
        qn, kn = (torch.randn((2, h, 64), device="cuda").to(torch.bfloat16) for h in (8, 2))
        out = torch.empty((2, 8, 64), device="cuda")
        A.asrkf_decode_step(ctx, 0, qn, kn, kn, out)
        assert torch.equal(out, kn.float().repeat_interleave(4, 1))
    finally:
        A.asrkf_destroy(ctx)


def test_outputs_over_inputs_are_refused():
    import torch
    n = 20
    A, ctx = _init(1, 2, 2, 64, "bf16", 64)
    try:
        x = torch.zeros((5 * n, 2, 64), dtype=torch.bfloat16, device="cuda")
        q, k, v, out = (x[i * n:(i + 1) * n] for i in range(4))
        for args in ((q, k, v, q), (q, k, v, k), (q, k, v, v), (q, k, v, x[n - 1:2 * n - 1]), (q, k, v, x[3 * n - 1:])):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_prefill_packed(ctx, 0, [0], [n], *args)
            assert e.value.code == A._lib.EINVAL and "overlaps" in A.asrkf_last_error()
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, k, v, out)              # side by side
        A.asrkf_prefill_packed(ctx, 0, [0], [n], q, q, q, out)              # inputs may be the same
        for a, b in ((k, k), (k, x[2 * n - 1:3 * n - 1])):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_get_rows(ctx, 0, 0, 0, n, a, b)
            assert e.value.code == A._lib.EINVAL
        A.asrkf_get_rows(ctx, 0, 0, 0, n, k, v)
    finally:
        A.asrkf_destroy(ctx)


def test_rows_are_refused_in_spill_mode_and_prompts_are_not():
    import torch
    A, ctx = _init(1, 8, 2, 64, "bf16", 64, spill_min_D=2, device_rows=30)
    try:
        q, k, v = _inputs([29], 8, 2, 64, "bf16")
        out = torch.empty_like(q)
        with pytest.raises(A.AsrkfError) as e:                # no device row left for the first step
            A.asrkf_prefill_packed(ctx, 0, [0], [30], *_inputs([30], 8, 2, 64, "bf16"), torch.empty((30, 8, 64), device="cuda", dtype=torch.bfloat16))
        assert e.value.code == A._lib.EINVAL
        A.asrkf_prefill_packed(ctx, 0, [0], [29], q, k, v, out)
        _check(out, *_reference([29], q, k, v), 29)
        with pytest.raises(A.AsrkfError) as e:
            A.asrkf_get_rows(ctx, 0, 0, 0, 5, torch.empty_like(k), torch.empty_like(v))
        assert e.value.code == A._lib.ESTATE
    finally:
        A.asrkf_destroy(ctx)


def test_decode_steps_behind_packed_prompts_match_the_oracle():
    """Prompts through the packed call in both layers (one sequence without any), then
    freezing decode steps: states bit-exact against the oracle, as behind asrkf_prefill."""
    import torch
    import paper_2512_11221_amd as A
    w = gen.Workload(name="packed", seed=gen.SEED + 301, n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64,
                     dtype="bf16", prefill=[90, 0, 41], steps=30, window_K=8, tau=0.5, k_soft=1.0, vocab=64,
                     logit_sigma=2.0, recipe="hh", f_hh=[0.35, 0.3, 0.25])
    inst = [(l, b) for l in range(2) for b in range(3)]
    inp = H.Inputs(w)
    ctx = A.asrkf_init(A.make_config(2, 3, 8, 2, 64, w.max_ctx, w.window_K, w.tau, w.k_soft, w.vocab,
                                     entropy_spike=w.entropy_spike, dtype="bf16"))
    try:
        for l in range(2):
            K, V = zip(*(inp.prompt(l, b) for b in range(3)))
            K, V = (H._dev(np.concatenate(x), "bf16") for x in (K, V))
            q = torch.randn((131, 8, 64), device="cuda", dtype=torch.bfloat16)
            out = torch.empty_like(q)
            A.asrkf_prefill_packed(ctx, l, [0, 1, 2], [90, 0, 41], q, K, V, out)
            _check(out, *_reference([90, 0, 41], q, K, V), 131)

        class NoPrompts(H.Inputs):          # the harness stores none: they are there
            def prompt(self, layer, seq):
                K, V = super().prompt(layer, seq)
                return K[:0], V[:0]

        g, _, _ = H.run_gpu(w, NoPrompts(w), inst, with_logits=False, ctx=ctx)
    finally:
        A.asrkf_destroy(ctx)
    o = H.run_oracle(w, inp, inst, with_logits=False)
    assert sum(int(r["frozen"].sum()) for key in inst for r in o[key]) > 0
    for key in inst:
        assert H.compare_instance(g[key], o[key]) < 1e-5
