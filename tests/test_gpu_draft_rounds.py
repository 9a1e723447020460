"""Rounds with drafted tokens where the host knows less than the device: the layout of a step, room within a capture
and in replays, replayed rounds bit by bit."""
import numpy as np
import pytest

from tests.test_gpu_accept import Run, _i32, gpu                             # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw,lens", [(dict(Hq=32, Hkv=32), [300, 310, 0, 37, 900, 64, 65, 300]),
                                     (dict(Hq=32, Hkv=32, kv_bits=4, relevance="softmax", tau=0.002), [300, 310, 0, 37, 900, 64, 65, 300])],
                         ids=["bf16", "four"])
def test_the_layout_of_a_step_does_not_hang_on_what_the_host_knows(kw, lens):
    """Rejected drafts by the thousand, which the host counts as accepted until a call waits: the steps behind them have
    the bits of a context that looked in between, and the same verdicts."""
    import torch
    N, max_ctx = 64, 18000
    a, b = (Run(lens, L=1, N=N, max_ctx=max_ctx, seed=2, **kw) for _ in range(2))
    try:
        A = a.A
        k, v = a.nodes()
        path, none = _i32(np.tile(np.arange(N), (len(lens), 1))), _i32([0] * len(lens))
        rows = [[tuple(a.randn(a.B, h, a.D) for h in (32, 32, 32))] for _ in range(4)]
        for r in (a, b):
            r.step(rows[0])
            for _ in range(max_ctx // N - 17):       # lists that might hold 16384 tokens and more
                A.asrkf_accept_drafts(r.ctx, path, none, k, v)
        for x in rows[1:]:
            A.asrkf_stats(b.ctx)
            assert torch.equal(a.step(x), b.step(x))
            for r in (a, b):
                A.asrkf_accept_drafts(r.ctx, path, none, k, v)
        for i in range(len(lens)):
            x, y = a.state(0, i), b.state(0, i)
            assert all(np.array_equal(x[key], y[key]) for key in x)
    finally:
        a.close()
        b.close()


def test_a_round_is_captured_behind_drafts_that_were_counted_as_accepted():
    """Ten rounds of rejected drafts: by the host's count the sequences are full, and a capture cannot look.  The
    captured round runs until the room is really used up."""
    import torch
    r = Run([10, 3], N=4, max_ctx=40, L=2)
    try:
        A = r.A
        k, v = r.nodes()
        path, n_path = _i32([[0, 1, 2, 3]] * 2), _i32([0, 0])
        q0 = [r.randn(2, h, 64) for h in (8, 2, 2)]
        out = torch.empty((2, 2, 8, 64), device="cuda")

        def calls():
            for layer in range(2):
                A.asrkf_decode_step(r.ctx, layer, *q0, out[layer])
            A.asrkf_restore(r.ctx, None, A.NONE)
            A.asrkf_accept_drafts(r.ctx, path, n_path, k, v)
        calls()
        assert r.state(0, 0)["n"] == 11
        for _ in range(7):                           # 11 + 28 of 40
            A.asrkf_accept_drafts(r.ctx, path, n_path, k, v)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            calls()
        n_path.copy_(_i32([4, 1]))
        torch.cuda.synchronize()
        for t in range(1, 6):
            g.replay()
            torch.cuda.synchronize()
            assert [r.state(1, b)["n"] for b in range(2)] == [11 + 5 * t, 4 + 2 * t]
            torch.zeros(5000, device="cuda").sum().item()
        # 36 of 40 are known now: a capture refuses what can never be replayed
        torch.cuda.synchronize()
        A.asrkf_accept_drafts(r.ctx, path, _i32([4, 0]), k, v)
        assert r.state(0, 0)["n"] == 40
        refused = []
        g2 = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g2, stream=torch.cuda.Stream()):
            torch.zeros(1, device="cuda")
            for call in (lambda: A.asrkf_decode_step(r.ctx, 0, *q0, out[0]), lambda: A.asrkf_accept_drafts(r.ctx, path, n_path, k, v)):
                with pytest.raises(A.AsrkfError) as e:
                    call()
                refused.append(e.value.code)
        assert refused == [A._lib.ECAPACITY] * 2
    finally:
        r.close()


def test_replayed_acceptance_without_room_leaves_the_rest_as_it_is():
    """Replays whose drafts have no room in one of two sequences: the next waiting call says so, once, and the context
    goes on with the bits of one in which that sequence accepted nothing."""
    import torch
    a, b = (Run([22, 4], N=4, max_ctx=30, L=2, seed=4, tau=6.0) for _ in range(2))
    try:
        A = a.A
        k, v = a.nodes()
        rows = [[tuple(a.randn(2, h, 64) for h in (8, 2, 2)) for _ in range(2)] for _ in range(3)]
        path, takes, graphs = _i32([[0, 1, 2, 3], [3, 1, 0, 2]]), [_i32([0, 0]) for _ in range(2)], []
        for r, n_path in zip((a, b), takes):
            r.step(rows[0])
            torch.cuda.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=torch.cuda.Stream()):
                A.asrkf_accept_drafts(r.ctx, path, n_path, k, v)

        def replay(*most):
            for g, n_path, n in zip(graphs, takes, most):
                n_path.copy_(_i32(n))
                torch.cuda.synchronize()
                g.replay()
            torch.cuda.synchronize()
        for t in range(1, 4):
            replay([2, 3], [2, 3])
            assert [a.state(1, i)["n"] for i in range(2)] == [23 + 2 * t, 5 + 3 * t]
        for _ in range(2):                           # no room for two behind 29 of 30, room in the other sequence
            replay([2, 3], [0, 3])
            with pytest.raises(A.AsrkfError, match="room") as e:
                A.asrkf_stats(a.ctx)
            assert e.value.code == A._lib.ECAPACITY
            x, y = A.asrkf_stats(a.ctx), A.asrkf_stats(b.ctx)
            assert x["total_positions"] == y["total_positions"] == 2 * sum(b.state(0, i)["n"] for i in range(2))
        replay([1, 0], [1, 0])                       # one fits
        assert [a.state(0, i)["n"] for i in range(2)] == [30, 20]
        for layer in range(2):
            for i in range(2):
                x, y = a.state(layer, i), b.state(layer, i)
                assert all(np.array_equal(x[key], y[key]) for key in x)
                assert all(torch.equal(p, q) for p, q in zip(a.rows(layer, i, 0, x["n"]), b.rows(layer, i, 0, x["n"])))
        for r in (a, b):                             # a full sequence takes no further step
            with pytest.raises(A.AsrkfError) as e:
                r.step(rows[1])
            assert e.value.code == A._lib.ECAPACITY
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("kw,tau", [(dict(), 8.0), (dict(dtype="f32"), 8.0), (dict(kv_bits=4, D=128), 11.0), (dict(scope="token"), 8.0),
                                    (dict(history_W=3), 8.0), (dict(relevance="softmax"), 0.02)], ids=str)
def test_counts_behind_an_acceptance(kw, tau):
    """Steps behind an acceptance against those of a context whose prompt held the tokens, with a tau that the tokens
    outside the window fall below in every variant: outputs, counts, lists."""
    import torch
    N = 5
    a = Run([60, 58], N=N, seed=3, tau=tau, window_K=61, **kw)
    try:
        k, v = a.nodes()
        rows = [[tuple(a.randn(2, h, a.D) for h in (8, a.Hkv, a.Hkv)) for _ in range(a.L)] for _ in range(6)]
        a.step(rows[0])
        a.A.asrkf_accept_drafts(a.ctx, _i32([[0, 1, 2, 3, 4]] * 2), _i32([N, 3]), k, v)
        got = [a.step(x) for x in rows[1:]]
        b = Run([60 + 1 + N, 58 + 1 + 3], N=N, seed=3, tau=tau, window_K=61, **kw)
        try:
            for layer in range(a.L):
                K, V = [], []
                for i, (p, take) in enumerate(zip((0, 60), (N, 3))):
                    for out, x, j, d in ((K, a.prompts[layer][0], 1, k), (V, a.prompts[layer][1], 2, v)):
                        out += [x[p:p + a.lens[i]], rows[0][layer][j][i:i + 1], d[layer, i, :take]]
                b.A.asrkf_prefill_packed(b.ctx, layer, range(2), b.lens, None, torch.cat(K), torch.cat(V), None)
            for x, y in zip(got, [b.step(x) for x in rows[1:]]):
                # fp32 sums of up to 71 terms of |v| < 5 either way
                assert (x - y).abs().max() <= 200 * 2.0 ** -24 * 5
            for layer in range(a.L):
                for i in range(2):
                    x, y = a.state(layer, i), b.state(layer, i)
                    assert x["n"] == y["n"] and list(x["count"]) == list(y["count"]) and list(x["active"]) == list(y["active"])
                    assert x["count"].any() and x["frozen"].any()
        finally:
            b.close()
    finally:
        a.close()


@pytest.mark.parametrize("kw", [dict(dtype="f32"), dict(), dict(kv_bits=4, D=128), dict(scope="token"), dict(D=256, Hkv=4)], ids=str)
def test_replayed_rounds_have_the_bits_of_eager_ones(kw):
    """A captured round, step, drafts and acceptance, against a context that runs the same calls: every replay's outputs
    bit by bit, with lists that freeze and grow."""
    import torch
    a, b = (Run([40, 300], N=6, max_ctx=400, L=2, seed=9, tau=6.0, **kw) for _ in range(2))
    try:
        A, N, D, Hkv = a.A, 6, a.D, a.Hkv
        q, q0 = a.randn(2, N, 8, D), [[a.randn(2, h, D) for h in (8, Hkv, Hkv)] for _ in range(2)]
        k, v = a.nodes()
        sees = torch.tensor([[1, 3, 5, 9, 17, 33], [1, 3, 7, 15, 31, 63]], device="cuda")
        path, n_path = _i32([[0, 1, -1, 0, 0, 0], [2, 3, 5, 0, 0, 0]]), _i32([2, 1])
        outs = {}

        def calls(r):
            o0, o = outs.setdefault(r, (torch.empty((2, 2, 8, D), device="cuda"), torch.empty((2,) + q.shape, dtype=q.dtype, device="cuda")))
            for layer in range(2):
                A.asrkf_decode_step(r.ctx, layer, *q0[layer], o0[layer])
                A.asrkf_attend_drafts(r.ctx, layer, sees, q, k[layer], v[layer], o[layer])
            A.asrkf_restore(r.ctx, None, A.NONE)
            A.asrkf_accept_drafts(r.ctx, path, n_path, k, v)
        for r in (a, b):
            calls(r)
            torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            calls(a)
        for t in range(6):
            n_path.copy_(_i32([t % 3, 3 - t % 4]))
            q.copy_(b.randn(*q.shape))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            calls(b)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(outs[a], outs[b]))
            for layer in range(2):
                for i in range(2):
                    x, y = a.state(layer, i), b.state(layer, i)
                    assert all(np.array_equal(x[key], y[key]) for key in x)
            torch.zeros(5000, device="cuda").sum().item()
        assert any(a.state(layer, 1)["frozen"].any() for layer in range(2))
    finally:
        a.close()
        b.close()
