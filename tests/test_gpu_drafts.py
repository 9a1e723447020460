"""Attention of drafted tokens over the active cache (asrkf_attend_drafts): every type, head layout and kind of
workgroup against 64 bits, with lists that have gaps, ragged counts and masks that leave a row empty;
values that are not finite, strides, long lists, large batches, graphs, streams and refusals."""
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


def _randn(g, *shape, dtype):
    import torch
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)


class Setting:
    """A context after its prompts and `steps` decode steps that froze about half of what lies outside the window."""

    def __init__(self, lens, Hq, Hkv, D, dtype="bf16", nodes=64, L=1, steps=1, seed=0, max_ctx=None, **kw):
        import torch
        import paper_2512_11221_amd as A
        self.A, self.lens, self.L, self.B = A, lens, L, len(lens)
        self.Hq, self.Hkv, self.D, self.dtype = Hq, Hkv, D, dtype
        self.max_ctx = max_ctx or max(lens) + 80
        g = self.g = torch.Generator(device="cuda")
        g.manual_seed(99 + seed)
        # |q.k| averaged over heads has a mean of 0.8 sqrt(D): tau in its middle, frozen at once and for long
        kw = {"tau": 0.8 * D ** 0.5, "k_soft": 0.05, "window_K": 3, **kw}
        self.ctx = A.asrkf_init(A.make_config(L, self.B, Hq, Hkv, D, self.max_ctx, kw.pop("window_K"), kw.pop("tau"), kw.pop("k_soft"), 32,
                                              dtype=dtype, **kw))
        A.asrkf_reserve_drafts(self.ctx, nodes)
        T = sum(lens)
        for layer in range(L):
            K, V = self.randn(T, Hkv, D), self.randn(T, Hkv, D)
            if T:
                A.asrkf_prefill_packed(self.ctx, layer, range(self.B), lens, None, K, V, None)
        for _ in range(steps):
            self.step()

    def randn(self, *shape):
        return _randn(self.g, *shape, dtype=self.dtype)

    def decode(self, layer):
        import torch
        B = self.B
        self.A.asrkf_decode_step(self.ctx, layer, self.randn(B, self.Hq, self.D), self.randn(B, self.Hkv, self.D), self.randn(B, self.Hkv, self.D),
                                 torch.empty((B, self.Hq, self.D), device="cuda"))

    def step(self):
        for layer in range(self.L):
            self.decode(layer)
        self.A.asrkf_restore(self.ctx, None, self.A.NONE)

    def nodes(self, N):
        """q, k, v of N drafted nodes a sequence."""
        B = self.B
        return (self.randn(B, N, self.Hq, self.D) * 1.5).to(self.randn(1).dtype), self.randn(B, N, self.Hkv, self.D), self.randn(B, N, self.Hkv, self.D)

    def rows(self, layer, b, n):
        import torch
        K = torch.empty((max(n, 1), self.Hkv, self.D), dtype=self.randn(1).dtype, device="cuda")
        V = torch.empty_like(K)
        if n:
            self.A.asrkf_get_rows(self.ctx, layer, b, 0, n, K, V)
        return K, V

    def reference(self, layer, b, q, k, v, sees, count):
        """Between two steps: the list's last entry is the token to come."""
        st = self.A.asrkf_get_state(self.ctx, layer, b, self.max_ctx)
        K, V = self.rows(layer, b, st["n"])
        return R.attention(q[b], K, V, st["active"][:-1], k[b], v[b], sees[b], count[b])

    def close(self):
        self.A.asrkf_destroy(self.ctx)


def _sees(masks):
    import torch
    return torch.tensor(np.array(masks, np.uint64).view(np.int64), device="cuda")


def _masks(rng, B, N, kind):
    if kind == "tree":
        return [R.sees_of(R.random_tree(rng, N)) for _ in range(B)]
    if kind == "chain":
        return [R.sees_of(range(-1, N - 1)) for _ in range(B)]
    m = rng.integers(0, 1 << 62, (B, N), dtype=np.int64) * 4 + rng.integers(0, 4, (B, N))       # any bits, some rows none
    m[:, ::3] = 0
    return m.view(np.uint64).tolist()


def _counts(B, N):
    return [(N, 0, 1, max(1, N // 2), N - 1)[b % 5] for b in range(B)]


LAYOUTS = [(8, 8, 64), (4, 2, 64), (8, 2, 64), (16, 2, 64), (4, 4, 128), (8, 4, 128), (8, 2, 128), (8, 1, 128)]
KINDS = [(*x, t) for x in LAYOUTS for t in ("bf16", "f32", "four")] + [(g * 2, 2, 256, t) for g in (1, 2, 4, 8) for t in ("bf16", "four")]


def _kind(t):
    return dict(dtype="bf16", kv_bits=4) if t == "four" else dict(dtype=t)


@pytest.mark.parametrize("N,mask", [(1, "chain"), (3, "any"), (8, "tree"), (17, "tree"), (33, "any"), (64, "tree"), (64, "any")])
@pytest.mark.parametrize("Hq,Hkv,D,t", KINDS)
def test_outputs(Hq, Hkv, D, t, N, mask):
    """Between two steps, over lists with gaps, one of them empty; rows behind the counts stay."""
    import torch
    s = Setting([0, 31, 64, 130, 700, 1], Hq, Hkv, D, **_kind(t))
    try:
        rng = np.random.default_rng(N)
        sees, count = _masks(rng, s.B, N, mask), _counts(s.B, N)
        q, k, v = s.nodes(N)
        out = torch.full_like(q, 7.0)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out, count=torch.tensor(count, device="cuda", dtype=torch.int32))
        for b in range(s.B):
            ref, tol = s.reference(0, b, q, k, v, sees, count)
            R.check(out[b, :count[b]], ref[:count[b]], tol[:count[b]])
            assert (out[b, count[b]:] == 7.0).all()
    finally:
        s.close()


@pytest.mark.parametrize("Hq,Hkv,D,t", [(8, 2, 64, "bf16"), (8, 4, 128, "four"), (4, 4, 64, "f32"), (16, 8, 256, "bf16")])
def test_before_and_behind_the_steps_own_token(Hq, Hkv, D, t):
    """Within a step a layer's drafts attend to its token once its decode_step was called; without that, and between two
    steps, the list ends before the token to come.  Every sequence empty but for its tokens, too."""
    import torch
    s = Setting([0, 5, 90], Hq, Hkv, D, L=2, steps=2, **_kind(t))
    try:
        N = 6
        sees = _masks(np.random.default_rng(1), s.B, N, "tree")
        q, k, v = s.nodes(N)
        count = [N] * s.B
        before = [[s.A.asrkf_get_state(s.ctx, layer, b, s.max_ctx)["active"] for b in range(s.B)] for layer in range(2)]

        def attend(layer):
            out = torch.empty_like(q)
            s.A.asrkf_attend_drafts(s.ctx, layer, _sees(sees), q, k, v, out)
            return out
        s.decode(0)
        outs = {0: attend(0), 1: attend(1)}         # layer 1's token is not there yet
        s.decode(1)
        outs[2] = attend(1)
        s.A.asrkf_restore(s.ctx, None, s.A.NONE)
        for key, layer, own in ((0, 0, True), (1, 1, False), (2, 1, True)):
            for b in range(s.B):
                active = before[layer][b] if own else before[layer][b][:-1]
                K, V = s.rows(layer, b, s.lens[b] + 3)
                R.check(outs[key][b], *R.attention(q[b], K, V, active, k[b], v[b], sees[b], N))
    finally:
        s.close()


@pytest.mark.parametrize("t", ["bf16", "f32", "four"])
def test_a_node_that_sees_nothing_gets_zeros(t):
    """No list, no mask: also with values there that are not finite, and where only scores of -inf are seen."""
    import torch
    s = Setting([0, 0], 8, 2, 64, L=2, steps=0, max_ctx=40, **_kind(t))
    try:
        s.decode(0)                                  # layer 1's lists hold no row yet
        q, k, v = s.nodes(4)
        v[:, 2:] = float("nan")
        k[:, 3] = float("inf")
        out = torch.full_like(q, 7.0)
        s.A.asrkf_attend_drafts(s.ctx, 1, _sees([[0, 1, 0, 3]] * 2), q, k, v, out)
        assert (out[:, 0] == 0).all() and (out[:, 2] == 0).all()
        ref, tol = R.attention(q[0], k[0][:0], v[0][:0], [], k[0], v[0], [0, 1, 0, 3], 4)
        R.check(out[0], ref, tol)
        q[:], k[:] = 1.0, 0.0
        k[:, 0, :, 5] = float("-inf")
        out.fill_(7.0)
        s.A.asrkf_attend_drafts(s.ctx, 1, _sees([[1, 0, 0, 1]] * 2), q, k, v, out)
        assert (out == 0).all()
    finally:
        s.close()


@pytest.mark.parametrize("Hq,Hkv,D,t,N", [(8, 2, 64, "bf16", 8), (8, 8, 128, "f32", 5), (8, 1, 128, "four", 40), (4, 2, 256, "bf16", 20),
                                          (8, 1, 128, "bf16", 16), (16, 2, 64, "f32", 64)])
def test_values_that_are_not_finite_reach_those_that_see_them(Hq, Hkv, D, t, N):
    import torch
    s = Setting([40, 300], Hq, Hkv, D, **_kind(t))
    try:
        sees = _masks(np.random.default_rng(3), s.B, N, "chain")
        q, k, v = s.nodes(N)
        bad = N // 2
        clean = torch.empty_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, clean)
        for what, where in ((float("nan"), "k"), (float("inf"), "v"), (float("nan"), "v"), (float("-inf"), "v")):
            k2, v2 = k.clone(), v.clone()
            (k2 if where == "k" else v2)[:, bad, 0, 7] = what
            out = torch.empty_like(q)
            s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k2, v2, out)
            G = Hq // Hkv
            hit = torch.zeros_like(out, dtype=torch.bool)
            if where == "k":
                hit[:, bad:, :G] = True
                assert torch.isnan(out[hit]).all()
                # which rows are rescaled together depends on all of a tile's scores: the others by their bounds
                for b in range(s.B):
                    ref, tol = s.reference(0, b, q, k, v, sees, [N] * s.B)
                    mine = ~hit[b]
                    R.check(out[b][mine], ref[mine], tol[mine])
                continue
            else:
                hit[:, bad:, :G, 7] = True
                assert (torch.isnan(out[hit]) if what != what else out[hit] == what).all()
            assert torch.equal(out[~hit], clean[~hit])
        # behind the counts: not read
        k[:, bad:], v[:, bad:] = float("nan"), float("nan")
        q[:, bad:] = float("nan")
        every = _sees([[~0 & (2 ** 64 - 1)] * N] * s.B)
        count = torch.tensor([bad] * s.B, device="cuda", dtype=torch.int32)
        out = torch.zeros_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, every, q, k, v, out, count=count)
        assert torch.isfinite(out).all()
    finally:
        s.close()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_large_values_and_scores(t):
    """Values at their type's largest give finite outputs; scores of 10^4 apart weigh one key."""
    import torch
    s = Setting([200], 4, 2, 64, tau=0.0, **_kind(t))
    try:
        N = 5
        sees = _masks(np.random.default_rng(2), 1, N, "tree")
        q, k, v = s.nodes(N)
        v = torch.full_like(v, torch.finfo(v.dtype).max) * (1 if t == "bf16" else 1 - 2.0 ** -14)     # (200 roundings of 2^-23)
        out = torch.empty_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q * 1000, k * 1000, v, out)
        assert torch.isfinite(out).all()
        q, k, v = s.nodes(N)
        q, k = q * 300, k * 300
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
        ref, tol = s.reference(0, 0, q, k, v, sees, [N])
        R.check(out[0], ref, tol)
    finally:
        s.close()


@pytest.mark.parametrize("Hq,Hkv,D,t,N,lens", [
    (32, 8, 128, "bf16", 5, [9000]), (32, 8, 128, "bf16", 60, [5000, 33]), (8, 1, 128, "four", 16, [20000, 700]), (16, 2, 64, "bf16", 64, [12000]),
    (16, 8, 256, "bf16", 12, [3000, 17]), (8, 2, 64, "f32", 30, [6000]), (32, 32, 128, "four", 3, [2000] * 3), (8, 2, 64, "bf16", 2, [30, 5000] * 5),
    (4, 4, 128, "f32", 9, [100, 900, 2500]), (32, 8, 128, "four", 16, [20000, 700]), (16, 2, 64, "four", 7, [12000, 60]),
    (8, 2, 128, "four", 13, [40] * 300)])
def test_long_lists_are_shared(Hq, Hkv, D, t, N, lens):
    """Pairs cut over many workgroups, in equal parts and across the pairs; the same bits again."""
    import torch
    s = Setting(lens, Hq, Hkv, D, **_kind(t))
    try:
        sees, count = _masks(np.random.default_rng(5), s.B, N, "tree"), [N] * s.B
        q, k, v = s.nodes(N)
        out, again = torch.empty_like(q), torch.empty_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, again)
        assert torch.equal(out, again)
        for b in range(s.B):
            ref, tol = s.reference(0, b, q, k, v, sees, count)
            R.check(out[b], ref, tol)
    finally:
        s.close()


@pytest.mark.parametrize("B,N,t", [(64, 3, "bf16"), (65, 3, "bf16"), (70, 20, "four"), (300, 1, "f32"), (1024, 2, "bf16")])
def test_large_batches(B, N, t):
    """More sequences than a wave has lanes, lengths of all kinds, many without drafts."""
    import torch
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 200, B)]
    s = Setting(lens, 4, 2, 64, **_kind(t))
    try:
        sees, count = _masks(rng, B, N, "tree"), [int(x) for x in rng.integers(0, N + 1, B)]
        q, k, v = s.nodes(N)
        out = torch.full_like(q, 7.0)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out, count=torch.tensor(count, device="cuda", dtype=torch.int32))
        for b in list(range(0, B, max(1, B // 40))) + [B - 1]:
            ref, tol = s.reference(0, b, q, k, v, sees, count)
            R.check(out[b, :count[b]], ref[:count[b]], tol[:count[b]])
        for b in range(B):
            assert (out[b, count[b]:] == 7.0).all()
    finally:
        s.close()


@pytest.mark.parametrize("B,D,t,N", [(1024, 256, "bf16", 3), (1024, 128, "f32", 2), (1024, 128, "bf16", 5), (100, 256, "four", 24)])
def test_large_batches_of_wide_rows(B, D, t, N):
    """The plan of more than 64 sequences beside the largest tiles that a workgroup has."""
    import torch
    rng = np.random.default_rng(D + B)
    s = Setting([int(x) for x in rng.integers(0, 40, B)], 4, 1, D, **_kind(t))
    try:
        sees, count = _masks(rng, B, N, "tree"), [int(x) for x in rng.integers(0, N + 1, B)]
        q, k, v = s.nodes(N)
        out = torch.full_like(q, 7.0)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out, count=torch.tensor(count, device="cuda", dtype=torch.int32))
        for b in list(range(0, B, max(1, B // 40))) + [B - 1]:
            ref, tol = s.reference(0, b, q, k, v, sees, count)
            R.check(out[b, :count[b]], ref[:count[b]], tol[:count[b]])
        for b in range(B):
            assert (out[b, count[b]:] == 7.0).all()
    finally:
        s.close()


@pytest.mark.parametrize("Hq,Hkv,D,t", [(32, 8, 128, "bf16"), (16, 4, 128, "four"), (8, 2, 64, "f32"), (16, 4, 256, "bf16")])
def test_room_that_grows(Hq, Hkv, D, t):
    """Room for more nodes on the same context, then few and many nodes over lists that many workgroups share."""
    s = Setting([6000, 300, 45], Hq, Hkv, D, nodes=1, **_kind(t))
    try:
        import torch
        for room, ns in ((1, [1]), (9, [9, 2]), (64, [64, 1, 16, 31, 9])):
            s.A.asrkf_reserve_drafts(s.ctx, room)
            for N in ns:
                sees, count = _masks(np.random.default_rng(N), s.B, N, "tree"), [N] * s.B
                q, k, v = s.nodes(N)
                out = torch.empty_like(q)
                s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
                for b in range(s.B):
                    ref, tol = s.reference(0, b, q, k, v, sees, count)
                    R.check(out[b], ref, tol)
    finally:
        s.close()


def test_rows_past_two_gigabytes_of_a_pool():
    """The longest context: 2 GiB of K a sequence, the second sequence's rows beyond 32-bit offsets."""
    import torch
    n = 1_000_000
    s = Setting([3, n], 8, 8, 128, max_ctx=n + 100, tau=0.0, nodes=4)
    try:
        sees, count = _masks(np.random.default_rng(0), 2, 4, "chain"), [4, 4]
        q, k, v = s.nodes(4)
        q = q * 2
        out = torch.empty_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
        for h in range(8):
            K = torch.empty((n + 1, 8, 128), dtype=torch.bfloat16, device="cuda") if h == 0 else K
            V = torch.empty_like(K) if h == 0 else V
            if h == 0:
                s.A.asrkf_get_rows(s.ctx, 0, 1, 0, n + 1, K, V)
            ref, tol = R.attention(q[1][:, h:h + 1], K[:, h:h + 1].contiguous(), V[:, h:h + 1].contiguous(), np.arange(n + 1), k[1][:, h:h + 1],
                                   v[1][:, h:h + 1], sees[1], 4)
            R.check(out[1][:, h:h + 1], ref, tol)
    finally:
        s.close()


def test_strides_and_views():
    """Slices of a fused projection, and a batch whose sequences are views of a wider tensor's nodes."""
    import torch
    s = Setting([50, 90], 8, 2, 64)
    try:
        N = 9
        sees = _masks(np.random.default_rng(4), 2, N, "tree")
        fused = s.randn(2, N, 12, 64)
        q, k, v = fused[:, :, :8], fused[:, :, 8:10], fused[:, :, 10:]
        out, ref = torch.empty((2, N, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((2, N, 8, 64), dtype=torch.bfloat16, device="cuda")
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q, k, v, out)
        s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), q.contiguous(), k.contiguous(), v.contiguous(), ref)
        assert torch.equal(out, ref)
        for bad in (s.randn(2, N + 1, 8, 64)[:, :N], s.randn(2, N, 8, 128)[..., ::2], s.randn(2, N, 8, 128)[..., :64], s.randn(2, N, 64, 8).transpose(2, 3),
                    s.randn(N, 2, 8, 64).transpose(0, 1), s.randn(2, 1, 8, 64).expand(2, N, 8, 64)):
            with pytest.raises(ValueError):
                s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), bad, k, v, out)
        for bad in (s.randn(2, N, 4, 64), s.randn(1, N, 8, 64), s.randn(2, N, 8, 64).float(), s.randn(2, 8, 64)):
            with pytest.raises(s.A.AsrkfError):
                s.A.asrkf_attend_drafts(s.ctx, 0, _sees(sees), bad, k, v, out)
    finally:
        s.close()


def test_replays_and_two_graphs_share_the_workspace():
    """A captured step with its drafts, and a graph of the drafts alone, replayed in turn with eager calls between."""
    import torch
    s = Setting([800, 3000], 8, 2, 128, tau=0.0)
    try:
        N = 8
        sees = _sees(_masks(np.random.default_rng(6), 2, N, "tree"))
        masks = sees.cpu().numpy().view(np.uint64).tolist()
        q, k, v = s.nodes(N)
        q0, k0, v0 = s.randn(2, 8, 128), s.randn(2, 2, 128), s.randn(2, 2, 128)
        o0, o1, o2 = torch.empty((2, 8, 128), device="cuda"), torch.empty_like(q), torch.empty_like(q)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(one, stream=st):
            s.A.asrkf_decode_step(s.ctx, 0, q0, k0, v0, o0)
            s.A.asrkf_attend_drafts(s.ctx, 0, sees, q, k, v, o1)
            s.A.asrkf_restore(s.ctx, None, s.A.NONE)
        s.A.asrkf_stats(s.ctx)
        with torch.cuda.graph(two, stream=st):
            s.A.asrkf_attend_drafts(s.ctx, 0, sees, q, k, v, o2)
        for t in range(3):
            one.replay()
            two.replay()
            torch.cuda.synchronize()
            s.A.asrkf_stats(s.ctx)
            eager = torch.empty_like(q)
            s.A.asrkf_attend_drafts(s.ctx, 0, sees, q, k, v, eager)
            torch.cuda.synchronize()
            # between the steps both have the same list: the step's token is in it by then
            for o in (o1, o2):
                assert torch.equal(o, eager)
            for b in range(2):
                ref, tol = s.reference(0, b, q, k, v, masks, [N] * 2)
                R.check(eager[b], ref, tol)
    finally:
        s.close()


def test_alternating_streams():
    import torch
    s = Setting([4000, 100], 8, 2, 64)
    try:
        N = 16
        sees = _sees(_masks(np.random.default_rng(7), 2, N, "tree"))
        q, k, v = s.nodes(N)
        ref = torch.empty_like(q)
        s.A.asrkf_attend_drafts(s.ctx, 0, sees, q, k, v, ref)
        streams = [torch.cuda.Stream() for _ in range(3)]
        outs = [torch.empty_like(q) for _ in range(9)]
        torch.cuda.synchronize()
        for i, o in enumerate(outs):                  # one workspace: the calls order themselves
            s.A.asrkf_attend_drafts(s.ctx, 0, sees, q, k, v, o, stream=streams[i % 3])
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs)
    finally:
        s.close()


def test_refusals():
    import torch
    s = Setting([10, 20], 8, 2, 64, nodes=8, steps=0)
    try:
        A, ctx, lib = s.A, s.ctx, s.A.load()
        EINVAL, ESTATE = A._lib.EINVAL, A._lib.ESTATE
        N = 8
        sees, count = _sees([[1] * N] * 2), torch.tensor([N, N], device="cuda", dtype=torch.int32)
        q, k, v = s.nodes(N)
        out = torch.empty_like(q)
        P = lambda t: t.data_ptr()                                             # noqa: E731
        good = dict(layer=0, n=N, count=P(count), sees=P(sees), q=P(q), qs=0, k=P(k), ks=0, v=P(v), vs=0, out=P(out))

        def call(**kw):
            return lib.asrkf_attend_drafts(ctx, *{**good, **kw}.values(), None)
        assert call() == ESTATE                                                # before the first decode step
        s.step()
        assert call() == 0 and call(count=0) == 0 and call(n=7) == 0
        for bad in (dict(layer=-1), dict(layer=1), dict(n=0), dict(n=9), dict(sees=0), dict(q=0), dict(k=0), dict(v=0), dict(out=0),
                    dict(qs=-8), dict(qs=504), dict(qs=516), dict(ks=64), dict(vs=1 << 40), dict(q=P(q) + 8), dict(sees=P(sees) + 4),
                    dict(count=P(count) + 2), dict(out=P(q)), dict(out=P(k)), dict(out=P(v) + 16), dict(qs=1 << 20),
                    dict(q=torch.zeros(1 << 14).data_ptr())):
            assert call(**bad) == EINVAL, bad
        assert lib.asrkf_reserve_drafts(ctx, 0) == EINVAL and lib.asrkf_reserve_drafts(ctx, 65) == EINVAL
        assert lib.asrkf_reserve_drafts(ctx, 3) == 0                           # less than there is: as it was
        assert call() == 0
        assert lib.asrkf_reserve_drafts(ctx, 64) == 0
        torch.cuda.synchronize()
    finally:
        s.close()
    from tests.test_abi_cpu import BASE
    ctx = A.asrkf_init(A.make_config(**{**BASE, "spill_min_D": 2}))
    try:
        with pytest.raises(A.AsrkfError) as e:
            A.asrkf_reserve_drafts(ctx, 4)
        assert e.value.code == EINVAL
        assert lib.asrkf_attend_drafts(ctx, *good.values(), None) == ESTATE
    finally:
        A.asrkf_destroy(ctx)
