"""Rotary positions (asrkf_rotate): layouts, scalings, far positions, strides, in place and back, positions
that follow the context's steps, graphs, and refusals."""
import numpy as np
import pytest

from tests import _drafts as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_11221_amd as A
    A.load()
    return torch


def _init(B=2, Hq=8, Hkv=2, D=64, dtype="bf16", max_ctx=64, L=1, **kw):
    import paper_2512_11221_amd as A
    return A, A.asrkf_init(A.make_config(L, B, Hq, Hkv, D, max_ctx, 4, 0.5, 2.0, 32, dtype=dtype, **kw))


def _rows(n, h, D, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((n, h, D), generator=g, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)


SCALINGS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="bands", factor=8.0, original_ctx=8192, low=1.0, high=4.0),
            dict(scaling="ramp", factor=32.0, original_ctx=4096, low=1.0, high=32.0, magnitude=1.3466)]


@pytest.mark.parametrize("setting", SCALINGS, ids=lambda s: s.get("scaling", "none"))
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("Hq,Hkv,D,dim,dtype", [(8, 2, 64, 64, "bf16"), (8, 2, 64, 48, "f32"), (32, 8, 128, 128, "bf16"), (4, 4, 128, 16, "f32"),
                                                (1, 1, 128, 128, "f32"), (16, 8, 256, 256, "bf16"), (2, 2, 256, 80, "bf16")])
def test_outputs(Hq, Hkv, D, dim, dtype, layout, setting):
    """Both launch forms (a row to a workgroup below 4096 rows, four from there on), positions of either sign and far ones."""
    import torch
    A, ctx = _init(2, Hq, Hkv, D, dtype)
    try:
        A.asrkf_set_rotary(ctx, dim, 500000.0, layout=layout, **setting)
        freq = A.asrkf_rotary_table(D, dim, base=500000.0, layout=layout, **setting)
        mag = setting.get("magnitude", 1.0)
        for n in (1, 7, 4097):
            q, k = _rows(n, Hq, D, dtype, n), _rows(n, Hkv, D, dtype, n + 1)
            pos = torch.arange(n, device="cuda", dtype=torch.int32) * 37 - 5
            pos[n // 2] = 1 << 28
            qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
            A.asrkf_rotate(ctx, pos, q, qo, k, ko)
            for x, y in ((q, qo), (k, ko)):
                R.check(y, *R.turned(x, pos, freq, layout, mag))
                assert torch.equal(y[..., dim:], x[..., dim:])
            back = torch.empty_like(k)
            A.asrkf_rotate(ctx, pos, None, None, k, back, inverse=True)
            R.check(back, *R.turned(k, pos, freq, layout, mag, inverse=True))
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("Hkv", [1, 2])
def test_one_kind_of_rows_alone(Hkv):
    import torch
    A, ctx = _init(2, Hkv, Hkv, 64)
    try:
        A.asrkf_set_rotary(ctx, 64)
        freq = A.asrkf_rotary_table(64, 64)
        x, pos = _rows(300, Hkv, 64, "bf16"), torch.arange(300, device="cuda", dtype=torch.int32)
        for which in (0, 1):
            y = torch.empty_like(x)
            args = [None] * 4
            args[2 * which], args[2 * which + 1] = x, y
            A.asrkf_rotate(ctx, pos, *args)
            R.check(y, *R.turned(x, pos, freq, "halves"))
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_on_slices_of_a_fused_projection(dtype, layout):
    """Values beside the rows stay; the same bits as into dense rows."""
    import torch
    A, ctx = _init(3, 8, 2, 128, dtype)
    try:
        A.asrkf_set_rotary(ctx, 96, 10000.0, layout=layout)
        n = 5000
        fused = _rows(n, 12, 128, dtype, 3)
        before = fused.clone()
        pos = torch.randint(0, 100000, (n,), device="cuda", dtype=torch.int32)
        q, k = torch.empty_like(fused[:, :8]).contiguous(), torch.empty_like(fused[:, 8:10]).contiguous()
        A.asrkf_rotate(ctx, pos, fused[:, :8], q, fused[:, 8:10], k)
        assert torch.equal(fused, before)
        A.asrkf_rotate(ctx, pos, fused[:, :8], fused[:, :8], fused[:, 8:10], fused[:, 8:10])
        assert torch.equal(fused[:, :8], q) and torch.equal(fused[:, 8:10], k) and torch.equal(fused[:, 10:], before[:, 10:])
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("heads,dim,n", [(1, 64, 1 << 25), (32, 128, (1 << 23) + 4096)])
def test_the_most_rows(heads, dim, n):
    """2^25 rows of 128 bytes, and more rows of 8 KiB than a grid has workgroups for (64 GiB): turned in place."""
    import torch
    A, ctx = _init(2, heads, heads, dim)
    try:
        A.asrkf_set_rotary(ctx, dim)
        freq = A.asrkf_rotary_table(dim, dim)
        x = _rows(4096, heads, dim, "bf16").repeat(n // 4096, 1, 1)
        some = torch.cat([torch.arange(i, i + 100) for i in (0, (1 << 22) - 50, n - 100)]).cuda()
        before = x[some]
        pos = torch.arange(n, device="cuda", dtype=torch.int32)
        A.asrkf_rotate(ctx, pos, None, None, x, x)
        R.check(x[some], *R.turned(before, some, freq, "halves"))
    finally:
        A.asrkf_destroy(ctx)
        del x
        torch.cuda.empty_cache()


def test_values_that_are_not_finite_stay_in_their_pair():
    import torch
    A, ctx = _init(2, 8, 2, 64, "f32")
    try:
        A.asrkf_set_rotary(ctx, 32)
        x = _rows(4, 2, 64, "f32")
        clean = x.clone()
        x[1, 0, 3], x[2, 1, 40], x[3, 1, 20] = float("nan"), float("inf"), float("inf")
        pos = torch.tensor([1, 2, 3, 4], device="cuda", dtype=torch.int32)
        y, z = torch.empty_like(x), torch.empty_like(x)
        A.asrkf_rotate(ctx, pos, None, None, x, y)
        A.asrkf_rotate(ctx, pos, None, None, clean, z)
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[1, 0, 3] = hit[1, 0, 19] = hit[2, 1, 40] = hit[3, 1, 20] = hit[3, 1, 4] = True
        assert torch.equal(y[~hit], z[~hit]) and not torch.isfinite(y[hit]).any()
    finally:
        A.asrkf_destroy(ctx)


def _steps(A, ctx, L, q, k):
    import torch
    out = torch.empty(q.shape, device="cuda")
    for layer in range(L):
        A.asrkf_decode_step(ctx, layer, q, k, k, out)


@pytest.mark.parametrize("lens", [[3, 0, 17]])
def test_positions_of_the_step(lens):
    """rows_per_seq: the position that the step's token takes, the same before and behind the step's first
    attention launch, one more after the step; offsets on top."""
    import torch
    L, B = 2, len(lens)
    A, ctx = _init(B, 8, 2, 64, "bf16", 64, L)
    try:
        A.asrkf_set_rotary(ctx, 64)
        freq = A.asrkf_rotary_table(64, 64)
        rows = _rows(sum(lens), 2, 64, "bf16")
        for layer in range(L):
            A.asrkf_prefill_packed(ctx, layer, range(B), lens, None, rows, rows, None)
        q, k = _rows(B, 8, 64, "bf16", 1), _rows(B, 2, 64, "bf16", 2)
        d = _rows(B * 3, 2, 64, "bf16", 5).view(B, 3, 2, 64)
        off = torch.tensor([[1, 2, -1]] * B, device="cuda", dtype=torch.int32)
        n = torch.tensor(lens, device="cuda")
        for t in range(3):
            for layer in range(L):
                qo, ko, do = torch.empty_like(q), torch.empty_like(k), torch.empty_like(d)
                A.asrkf_rotate(ctx, None, q, qo, k, ko, rows_per_seq=1)
                A.asrkf_rotate(ctx, off, None, None, d, do, rows_per_seq=3)
                R.check(qo, *R.turned(q, n + t, freq, "halves"))
                R.check(ko, *R.turned(k, n + t, freq, "halves"))
                ref, tol = R.turned(d.view(B * 3, 2, 64), (n[:, None] + t + off).flatten(), freq, "halves")
                R.check(do.view(B * 3, 2, 64), ref, tol)
                A.asrkf_decode_step(ctx, layer, qo, ko, k, torch.empty((B, 8, 64), device="cuda"))
            A.asrkf_rotate(ctx, None, q, qo, None, None, rows_per_seq=1)      # before restore: the same step
            R.check(qo, *R.turned(q, n + t, freq, "halves"))
            A.asrkf_restore(ctx, None, A.NONE)
    finally:
        A.asrkf_destroy(ctx)


def test_replayed_steps_move_the_positions():
    import torch
    lens, B = [5, 9], 2
    A, ctx = _init(B, 8, 2, 64, "f32", 64)
    try:
        A.asrkf_set_rotary(ctx, 64)
        freq = A.asrkf_rotary_table(64, 64)
        rows = _rows(sum(lens), 2, 64, "f32")
        A.asrkf_prefill_packed(ctx, 0, range(B), lens, None, rows, rows, None)
        q, k = _rows(B, 8, 64, "f32", 1), _rows(B, 2, 64, "f32", 2)
        _steps(A, ctx, 1, q, k)
        A.asrkf_restore(ctx, None, A.NONE)
        qo, ko, out = torch.empty_like(q), torch.empty_like(k), torch.empty(q.shape, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        with torch.cuda.graph(g, stream=s):
            A.asrkf_rotate(ctx, None, q, qo, k, ko, rows_per_seq=1)
            A.asrkf_decode_step(ctx, 0, qo, ko, k, out)
            A.asrkf_restore(ctx, None, A.NONE)
        A.asrkf_set_rotary(ctx, 32, 77.0)           # captured calls keep theirs
        n = torch.tensor(lens, device="cuda") + 1
        for t in range(4):
            g.replay()
            torch.cuda.synchronize()
            R.check(qo, *R.turned(q, n + t, freq, "halves"))
            R.check(ko, *R.turned(k, n + t, freq, "halves"))
            torch.zeros(1000, device="cuda").sum().item()
        assert A.asrkf_stats(ctx)["step"] == 5
    finally:
        A.asrkf_destroy(ctx)


def test_another_stream():
    import torch
    A, ctx = _init(2, 8, 2, 128)
    try:
        A.asrkf_set_rotary(ctx, 128)
        freq = A.asrkf_rotary_table(128, 128)
        s = torch.cuda.Stream()
        x, pos = _rows(9000, 8, 128, "bf16"), torch.arange(9000, device="cuda", dtype=torch.int32)
        y = torch.empty_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            A.asrkf_rotate(ctx, pos, x, y, None, None)
        A.asrkf_rotate(ctx, pos, y, y, None, None, inverse=True)        # waits for the other stream's
        torch.cuda.synchronize()
        once, _ = R.turned(x, pos, freq, "halves")
        ref, tol = R.turned(once.bfloat16(), pos, freq, "halves", inverse=True)
        # a rounding of the first turn may fall the other way: a step of both values of a pair
        a = once.abs()
        R.check(y, ref, tol + 2.0 ** -7 * (a + a.roll(64, -1)))
    finally:
        A.asrkf_destroy(ctx)


def test_refusals():
    import torch
    A, ctx = _init(2, 8, 2, 64)
    try:
        lib, EINVAL, ESTATE = A.load(), A._lib.EINVAL, A._lib.ESTATE
        buf = torch.zeros((40, 12, 64), device="cuda", dtype=torch.bfloat16)
        pos = torch.zeros(10, device="cuda", dtype=torch.int32)
        q, k = buf[:10, :8].contiguous(), buf[:10, 8:10].contiguous()
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        P = lambda t: t.data_ptr()                                             # noqa: E731
        call = lambda *a: lib.asrkf_rotate(ctx, *a, 0, None)                   # noqa: E731
        good = [10, 0, P(pos), P(q), 0, P(qo), 0, P(k), 0, P(ko), 0]
        assert call(*good) == ESTATE                                           # no setting yet
        for bad in (dict(dim=8), dict(dim=24), dict(dim=80), dict(dim=64, base=1.0), dict(dim=64, layout=2), dict(dim=64, scaling=4),
                    dict(dim=64, scaling="linear", factor=0.0), dict(dim=64, magnitude=0.0), dict(dim=64, scaling="ramp"),
                    dict(dim=64, scaling="bands", original_ctx=100, low=2.0, high=2.0), dict(dim=64, base=float("nan"))):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_set_rotary(ctx, **bad)
            assert e.value.code == EINVAL
        A.asrkf_set_rotary(ctx, 64)
        assert call(*good) == 0

        def but(**kw):
            names = ["n", "per", "pos", "q", "qs", "qo", "qos", "k", "ks", "ko", "kos"]
            return [kw.get(n, v) for n, v in zip(names, good)]
        big = 1 << 30
        for bad in (dict(n=-1), dict(n=(1 << 25) + 1), dict(per=-1), dict(per=3), dict(per=10), dict(pos=0), dict(q=0), dict(qo=0), dict(ko=0),
                    dict(q=0, qo=0, k=0, ko=0), dict(qs=-512), dict(qs=8), dict(qs=514), dict(qos=big), dict(q=P(q) + 2), dict(ko=P(ko) + 8),
                    dict(pos=P(pos) + 2), dict(qo=P(q) + 1024), dict(ko=P(q)), dict(qo=P(k)), dict(ko=P(qo)), dict(qos=1024, qo=P(q)),
                    dict(n=1 << 20), dict(pos=P(qo)), dict(k=torch.zeros(4096).data_ptr())):
            assert call(*but(**bad)) == EINVAL, bad
        assert call(*but(n=0, q=0, qo=0)) == 0                                 # no rows: nothing is looked at
        # slices of one buffer beside each other are apart; ones that cross are not
        f = P(buf)
        assert call(10, 0, P(pos), f, 768, f, 768, f + 1024, 768, f + 1024, 768) == 0
        assert call(10, 0, P(pos), 0, 0, 0, 0, f, 768, f + 256, 768) == 0      # into a neighbour's place
        assert call(10, 0, P(pos), 0, 0, 0, 0, f, 768, f + 128, 768) == EINVAL
        assert call(10, 0, P(pos), 0, 0, 0, 0, f + 10 * 128, 768, f + 11 * 128, 768) == EINVAL
        torch.cuda.synchronize()
    finally:
        A.asrkf_destroy(ctx)
