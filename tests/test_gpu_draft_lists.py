"""Attention of drafted tokens (asrkf_attend_drafts) over lists that all layers share, and beside decoding the same
tokens over lists that freeze."""
import numpy as np
import pytest

from tests import _drafts as R
from tests._four import rounded
from tests.test_gpu_drafts import Setting, _counts, _kind, _masks, _sees, gpu    # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,t,N", [(8, 2, 64, "bf16", 5), (8, 4, 128, "f32", 9), (8, 2, 128, "four", 17), (16, 4, 256, "bf16", 33), (8, 1, 64, "f32", 64)])
def test_lists_shared_by_all_layers(Hq, Hkv, D, t, N):
    """Token scope: one list for three layers, each with rows of its own; between steps, and within one before and
    behind a layer's own token."""
    import torch
    s = Setting([0, 31, 130, 700, 1], Hq, Hkv, D, L=3, steps=2, scope="token", **_kind(t))
    try:
        rng = np.random.default_rng(N)
        sees, count = _masks(rng, s.B, N, "tree"), _counts(s.B, N)
        nodes = [s.nodes(N) for _ in range(3)]
        counts = torch.tensor(count, device="cuda", dtype=torch.int32)

        def attend(layer):
            q, k, v = nodes[layer]
            out = torch.full_like(q, 7.0)
            s.A.asrkf_attend_drafts(s.ctx, layer, _sees(sees), q, k, v, out, count=counts)
            return out

        def check(out, layer, active):
            q, k, v = nodes[layer]
            for b in range(s.B):
                K, V = s.rows(layer, b, s.lens[b] + len_now)
                ref, tol = R.attention(q[b], K, V, active[b], k[b], v[b], sees[b], count[b])
                R.check(out[b, :count[b]], ref[:count[b]], tol[:count[b]])
                assert (out[b, count[b]:] == 7.0).all()
        len_now = 2
        lists = [s.A.asrkf_get_state(s.ctx, 0, b, s.max_ctx)["active"] for b in range(s.B)]
        assert any(len(x) < n + 3 for x, n in zip(lists, s.lens))            # some are frozen
        for layer in range(3):
            assert all(np.array_equal(s.A.asrkf_get_state(s.ctx, layer, b, s.max_ctx)["active"], lists[b]) for b in range(s.B))
            check(attend(layer), layer, [x[:-1] for x in lists])
        s.decode(0)
        s.decode(1)
        outs = [attend(layer) for layer in range(3)]
        s.decode(2)
        s.A.asrkf_restore(s.ctx, None, s.A.NONE)
        len_now = 3
        for layer in range(3):
            check(outs[layer], layer, lists if layer < 2 else [x[:-1] for x in lists])
    finally:
        s.close()


@pytest.mark.parametrize("Hq,Hkv,D,t", [(8, 2, 64, "bf16"), (8, 4, 128, "f32"), (8, 2, 128, "four"), (16, 4, 256, "bf16"), (8, 2, 64, "four"), (8, 8, 128, "bf16")])
def test_a_drafted_token_beside_decoding_it(Hq, Hkv, D, t):
    """Siblings behind the last token, each seeing itself, then a decode step of one of them: it attends to the same rows.
    The drafts' output has its weights and itself rounded to the context's type, the step's is fp32; both are within
    the bound of the drafts' error of the exact value.  (Rows of values that 4 bits hold, where the cache does.)"""
    import torch
    s = Setting([0, 31, 130, 700, 1], Hq, Hkv, D, steps=2, **_kind(t))
    try:
        N = 7
        sees = [[1 << i for i in range(N)]] * s.B
        for turn in range(3):
            q, k, v = s.nodes(N)
            if t == "four":
                k, v = (torch.tensor(rounded(x.double().cpu().numpy()), device="cuda").to(q.dtype) for x in (k, v))
            out, step = torch.empty_like(q), torch.empty((s.B, Hq, D), device="cuda")
            tol = [s.reference(0, b, q, k, v, sees, [N] * s.B)[1] for b in range(s.B)]
            s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
            which = [(b + turn) % N for b in range(s.B)]
            at = torch.arange(s.B, device="cuda"), torch.tensor(which, device="cuda")
            s.A.asrkf_decode_step(s.ctx, 0, q[at].contiguous(), k[at].contiguous(), v[at].contiguous(), step)
            s.A.asrkf_restore(s.ctx, None, s.A.NONE)
            for b in range(s.B):
                R.check(out[b, which[b]], step[b].double(), 2 * tol[b][which[b]])
        assert s.A.asrkf_get_state(s.ctx, 0, 3, s.max_ctx)["frozen"].any()
    finally:
        s.close()
