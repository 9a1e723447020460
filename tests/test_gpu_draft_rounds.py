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
