"""Verification of drafted tokens (asrkf_verify_drafts) against the walk as it is defined, on vectors in 64 bits;
rows that are no distribution, odd vocabularies, the distribution of the next token, graphs and refusals."""
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


def _init(B, V, nodes):
    import paper_2512_11221_amd as A
    ctx = A.asrkf_init(A.make_config(1, B, 4, 2, 64, 16, 4, 0.5, 2.0, V))
    A.asrkf_reserve_drafts(ctx, nodes)
    return A, ctx


class Case:
    """Trees whose tokens have a fair chance: drawn from the draft's rows, or given one behind their parent."""

    def __init__(self, B, N, V, probs, seed, sigma=2.0, ragged=True, reach=4):
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.N, self.V = B, N, V
        self.parents = np.array([R.random_tree(rng, N, reach) for _ in range(B)], np.int32)
        self.count = np.array([(N, max(1, N - 2), 0, N, 1)[b % 5] if ragged else N for b in range(B)], np.int32)
        z = rng.standard_normal((B, N + 1, V)).astype(np.float32) * np.float32(sigma)
        self.u = rng.random((B, N + 1)).astype(np.float32)
        self.tokens = rng.integers(0, V, (B, N)).astype(np.int32)
        self.probs = None
        if probs:
            y = (z[:, :N] + rng.standard_normal((B, N, V)) * 0.6).astype(np.float64)
            y = np.exp(y - y.max(-1, keepdims=True))
            self.probs = (y / y.sum(-1, keepdims=True)).astype(np.float32)
            for b in range(B):
                for i in range(N):
                    p = self.probs[b, self.parents[b, i] + 1].astype(np.float64)
                    self.tokens[b, i] = rng.choice(V, p=p / p.sum())
        else:
            for b in range(B):
                for i in range(N):
                    z[b, self.parents[b, i] + 1, self.tokens[b, i]] = np.log(V) + sigma ** 2 / 2 + rng.normal() * 1.5
        self.root, self.logits = z[:, 0].copy(), z[:, 1:].copy()

    def run(self, A, ctx, T, count=True, stream=None):
        import torch
        d = lambda x: None if x is None else torch.tensor(x, device="cuda")          # noqa: E731
        path = torch.full((self.B, self.N), 99, dtype=torch.int32, device="cuda")
        n, nxt = (torch.full((self.B,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        self.args = (d(self.tokens), d(self.parents), d(self.root), d(self.logits), d(self.u), path, n, nxt)
        self.kw = dict(probs=d(self.probs), temperature=T, count=d(self.count) if count else None)
        torch.cuda.synchronize()
        A.asrkf_verify_drafts(ctx, *self.args, **self.kw, stream=stream)
        torch.cuda.synchronize()
        return path.cpu().numpy(), n.cpu().numpy(), nxt.cpu().numpy()

    def check(self, got, T):
        path, n, nxt = got
        for b in range(self.B):
            want, tok = R.verify(self.tokens[b], self.parents[b], int(self.count[b]), self.root[b], self.logits[b],
                                 None if self.probs is None else self.probs[b], T, self.u[b])
            assert n[b] == len(want) and list(path[b]) == want + [-1] * (self.N - len(want)), b
            assert nxt[b] == tok, (b, nxt[b], tok)


@pytest.mark.parametrize("T", [0.0, 0.3, 1.0, 2.5])
@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("B,N,V", [(5, 1, 1), (5, 3, 2), (10, 8, 5), (20, 17, 63), (5, 64, 100), (6, 9, 1023), (5, 6, 1025), (5, 5, 4099), (6, 4, 32000),
                                   (3, 3, 50257), (2, 5, 128256)])
def test_walks(B, N, V, probs, T):
    if probs and T == 0:
        pytest.skip("no draft probabilities in greedy decoding")
    A, ctx = _init(B, V, N)
    try:
        took = 0
        for seed in range(3):
            c = Case(B, N, V, probs, 100 * seed + N, sigma=1.0 if V < 10 else 2.0)
            got = c.run(A, ctx, T)
            c.check(got, T)
            took += got[1].sum()
        if T == 1.0 and B * N >= 50:                # (a handful of nodes may all be rejected)
            assert took > 0
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("probs", [False, True])
def test_siblings_with_one_token(probs):
    """Wide trees over few tokens: the same token again below one parent, many rejections in a row."""
    A, ctx = _init(40, 4, 24)
    try:
        for seed in range(4):
            c = Case(40, 24, 4, probs, seed, sigma=1.0, reach=24)
            c.parents = np.array([[-1] * 12 + [int(x) for x in c.rng.integers(0, 12, 12)] for _ in range(40)], np.int32)
            c.check(c.run(A, ctx, 1.0), 1.0)
    finally:
        A.asrkf_destroy(ctx)


def test_greedy_takes_the_lowest_of_equals():
    A, ctx = _init(4, 1000, 2)
    try:
        c = Case(4, 2, 1000, False, 0, ragged=False)
        c.parents[:] = [-1, 0]
        c.root[:] = -1.0
        c.root[:, [700, 123, 999]] = 5.0
        c.logits[:] = 3.0
        c.tokens[:] = [[123, 0], [700, 0], [123, 1], [999, 5]]
        path, n, nxt = got = c.run(A, ctx, 0.0, count=False)
        c.check(got, 0.0)
        assert list(n) == [2, 0, 1, 0] and list(nxt) == [0, 123, 0, 123]
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("probs", [False, True])
@pytest.mark.parametrize("T", [0.0, 1.0])
def test_rows_that_are_no_distribution(T, probs):
    """A NaN, +inf, or nothing above -inf: no child of that row is kept, and no token follows; -inf alone weighs nothing."""
    if probs and T == 0:
        return
    A, ctx = _init(5, 777, 3)
    try:
        for row in (0, 1, 2, 3):
            c = Case(5, 3, 777, probs, 7 + row, ragged=False)
            c.parents[:] = [-1, 0, 1]
            c.u[:] = 0.0                            # keeps what has any weight
            rows = np.concatenate([c.root[:, None], c.logits], 1)
            for i in range(3):                      # the chain follows the largest logits
                c.tokens[:, i] = rows[:, i].argmax(-1)
            rows[0, row, 600] = np.nan
            rows[1, row, 0] = np.inf
            rows[2, row, :] = -np.inf
            rows[3, row, 1:] = -np.inf              # one token left
            rows[4, row, 100:700] = -np.inf
            c.root, c.logits = rows[:, 0].copy(), rows[:, 1:].copy()
            got = c.run(A, ctx, T)
            c.check(got, T)
            assert list(got[1][:3]) == [row] * 3 and list(got[2][:3]) == [-1] * 3 and (got[2][3:] >= 0).all()
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("probs", [False, True])
def test_tokens_and_parents_out_of_range(probs):
    A, ctx = _init(6, 50, 5)
    try:
        c = Case(6, 5, 50, probs, 3, ragged=False)
        c.parents[:] = [-1, 0, 1, -1, 3]
        c.tokens[0, 0], c.tokens[1, 0], c.tokens[2, 1] = 50, -1, 1 << 30
        c.parents[3, 0], c.parents[4, 1], c.parents[5, 2] = -2, 1, 1 << 30
        c.u[:, :5] = 0.0
        c.check(c.run(A, ctx, 1.0), 1.0)
    finally:
        A.asrkf_destroy(ctx)


def test_the_draft_is_nearly_the_target():
    """q = p but for the logits' rounding to fp32 (10^-8): everything is kept, and behind a drafted token of probability 0
    the draw is from those 10^-8."""
    A, ctx = _init(2, 6, 2)
    try:
        c = Case(2, 2, 6, True, 1, ragged=False)
        c.parents[:] = [-1, 0]
        z = np.log(np.array([0.5, 0.25, 0.125, 0.125, 1e-300, 1e-300])).astype(np.float32)
        z[4:] = -np.inf
        c.root[:], c.logits[:] = z, z
        c.probs[:] = [0.5, 0.25, 0.125, 0.125, 0.0, 0.0]
        c.tokens[:] = [[0, 1], [5, 1]]
        c.u[:] = [[0.99, 0.99, 0.6], [0.0, 0.0, 0.6]]
        path, n, nxt = got = c.run(A, ctx, 1.0)
        c.check(got, 1.0)
        assert list(n) == [2, 0] and nxt[0] == 1
    finally:
        A.asrkf_destroy(ctx)


def test_the_draft_is_the_target():
    """q = p to the last bit: where a token of probability 0 was drafted nothing remains, and p stays, also behind a
    second one and behind one that is kept."""
    A, ctx = _init(4, 5000, 3)
    try:
        c = Case(4, 3, 5000, True, 1, ragged=False)
        hot = [3, 1500, 2500, 4999]
        z = np.full(5000, -np.inf, np.float32)
        z[hot] = 1.0
        q = np.zeros(5000, np.float32)
        q[hot] = 0.25
        c.root[:], c.logits[:], c.probs[:] = z, z, q
        c.parents[:] = [[-1, 0, 1], [-1, -1, -1], [-1, 0, 0], [-1, -1, 1]]
        c.tokens[:] = [[1500, 3, 4999], [7, 8, 2500], [3, 9, 10], [11, 1500, 12]]
        c.u[:] = [[0.99, 0.99, 0.99, 0.6], [0.0, 0.0, 0.9, 0.1], [0.0, 0.0, 0.0, 0.6], [0.0, 0.5, 0.0, 0.3]]
        path, n, nxt = got = c.run(A, ctx, 1.0)
        c.check(got, 1.0)
        assert list(n) == [3, 1, 1, 1] and list(nxt) == [2500, 3, 2500, 1500]
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("u", [0.0, 1 - 2.0 ** -24])
def test_the_ends_of_the_random_numbers(u):
    """0 takes the first token of any weight, the largest below 1 one of the last: also where whole parts weigh nothing."""
    A, ctx = _init(3, 20000, 1)
    try:
        c = Case(3, 1, 20000, False, 5, ragged=False)
        c.root[:] = -np.inf
        c.root[0, 12345], c.root[0, 777] = 1.0, 1.0
        c.root[1, 19999] = -3.0
        c.root[2, :10] = 0.0
        c.tokens[:] = 5
        c.u[:, 0] = 0.999
        c.u[:, 1] = u
        got = c.run(A, ctx, 1.0)
        c.check(got, 1.0)
        assert list(got[2]) == ([777, 19999, 0] if u == 0 else [12345, 19999, 9])
    finally:
        A.asrkf_destroy(ctx)


def test_the_last_token_of_any_weight():
    """Three tokens have all of the weight and the first two drafts of them are rejected: the third is kept, or, where
    the rounded rest of 10^-7 says no, the next one."""
    A, ctx = _init(1024, 20000, 3)
    try:
        for T in (0.7, 1.0, 1.9):
            c = Case(1024, 3, 20000, False, int(T * 10), ragged=False)
            c.parents[:] = -1
            c.tokens[:] = [5000, 10, 15000]
            c.root[:] = -np.inf
            c.root[:, 5000] = c.rng.uniform(-9, 9, 1024)
            c.root[:, 10] = c.root[:, 5000] + c.rng.uniform(-1, 1, 1024).astype(np.float32)
            c.root[:, 15000] = c.root[:, 5000] + T * np.log(10.0 ** c.rng.uniform(-6.5, -5.5, 1024)).astype(np.float32)
            c.u[:] = 1 - 2.0 ** -24
            path, n, nxt = c.run(A, ctx, T)
            kept = n == 1
            assert kept.sum() + (n == 0).sum() == 1024
            assert (path[kept, 0] == 2).all() and (nxt[kept] >= 0).all() and (nxt[~kept] == 15000).all()
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("probs", [False, True])
def test_next_tokens_have_the_targets_distribution(probs):
    """The token behind the root, drafted or drawn, over 40 x 1024 sequences whose two siblings are drawn from q:
    within six standard deviations of p for each of the 7 tokens."""
    B, V, runs = 1024, 7, 40
    A, ctx = _init(B, V, 2)
    try:
        rng = np.random.default_rng(11)
        z = rng.standard_normal(V).astype(np.float32)
        p = np.exp(z.astype(np.float64))
        p /= p.sum()
        y = rng.standard_normal(V)
        q = (np.exp(y) / np.exp(y).sum()).astype(np.float32)
        seen = np.zeros(V)
        c = Case(B, 2, V, probs, 0, ragged=False)
        c.parents[:] = [-1, -1]
        c.root[:], c.logits[:] = z, 0.0
        if probs:
            c.probs[:] = q
        for _ in range(runs):
            c.u = rng.random((B, 3)).astype(np.float32)
            c.tokens = rng.choice(V, size=(B, 2), p=q.astype(np.float64) / q.astype(np.float64).sum()).astype(np.int32)
            path, n, nxt = c.run(A, ctx, 1.0)
            first = np.where(n > 0, c.tokens[np.arange(B), np.maximum(path[:, 0], 0)], nxt)
            seen += np.bincount(first, minlength=V)
        total = B * runs
        assert (np.abs(seen - total * p) <= 6 * np.sqrt(total * p * (1 - p))).all()
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("probs,T", [(False, 0.0), (False, 1.0), (True, 1.0)])
def test_replays(probs, T):
    """New inputs in the same buffers, each replay against the definition; the workspace is clean between."""
    import torch
    A, ctx = _init(6, 5000, 7)
    try:
        c = Case(6, 7, 5000, probs, 1)
        c.check(c.run(A, ctx, T), T)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            A.asrkf_verify_drafts(ctx, *c.args, **c.kw)
        for seed in range(2, 5):
            d = Case(6, 7, 5000, probs, seed)
            d.count = c.count
            for dst, src in zip(c.args[:5] + ((c.kw["probs"],) if probs else ()), (d.tokens, d.parents, d.root, d.logits, d.u, d.probs)):
                dst.copy_(torch.tensor(src))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            d.check([x.cpu().numpy() for x in c.args[5:]], T)
            other = Case(6, 7, 5000, probs, seed + 50)
            other.check(other.run(A, ctx, T), T)
    finally:
        A.asrkf_destroy(ctx)


def test_alternating_streams():
    import torch
    A, ctx = _init(6, 3000, 7)
    try:
        streams = [torch.cuda.Stream() for _ in range(2)]
        cases = [Case(6, 7, 3000, i % 2 == 1, i) for i in range(6)]
        for c in cases:
            c.run(A, ctx, 1.0)
        for i, c in enumerate(cases):
            for x in c.args[5:]:
                x.fill_(99)
        torch.cuda.synchronize()
        for i, c in enumerate(cases):
            A.asrkf_verify_drafts(ctx, *c.args, **c.kw, stream=streams[i % 2])
        torch.cuda.synchronize()
        for c in cases:
            c.check([x.cpu().numpy() for x in c.args[5:]], 1.0)
    finally:
        A.asrkf_destroy(ctx)


def test_refusals():
    import torch
    A, ctx = _init(2, 64, 4)
    try:
        c = Case(2, 4, 64, True, 0)
        c.run(A, ctx, 1.0)
        lib, EINVAL = A.load(), A._lib.EINVAL
        names = ("tokens", "parents", "root", "logits", "u", "path", "n_path", "next")
        good = dict(zip(names, (x.data_ptr() for x in c.args)), probs=c.kw["probs"].data_ptr(), count=c.kw["count"].data_ptr(), n=4, T=1.0)

        def call(**kw):
            a = {**good, **kw}
            return lib.asrkf_verify_drafts(ctx, a["n"], a["count"], a["tokens"], a["parents"], a["root"], a["logits"], a["probs"], a["T"], a["u"],
                                           a["path"], a["n_path"], a["next"], None)
        assert call() == 0 and call(count=None) == 0 and call(probs=None) == 0 and call(probs=None, T=0.0, u=None) == 0
        inf, nan = float("inf"), float("nan")
        for bad in ([dict(n=0), dict(n=5), dict(T=-1.0), dict(T=inf), dict(T=nan), dict(T=1e-7), dict(T=0.0)] +
                    [{x: None} for x in names] + [{x: good[x] + 2} for x in names] +
                    [dict(path=good["tokens"]), dict(next=good["n_path"]), dict(next=good["logits"] + 64), dict(n_path=good["path"] + 4),
                     dict(logits=torch.zeros(512).data_ptr())]):
            assert call(**bad) == EINVAL, bad
        for i, wrong in ((0, c.args[0].long()), (0, c.args[0][:1]), (2, c.args[2][:, :63]), (3, c.args[3].double()), (4, c.args[4][:, :4]),
                         (5, c.args[5][:, :3]), (6, c.args[6].float())):
            with pytest.raises(A.AsrkfError):
                A.asrkf_verify_drafts(ctx, *[wrong if j == i else x for j, x in enumerate(c.args)], **c.kw)
        with pytest.raises(ValueError):
            A.asrkf_verify_drafts(ctx, *[torch.zeros((64, 2), device="cuda").t() if j == 2 else x for j, x in enumerate(c.args)], **c.kw)
        torch.cuda.synchronize()
    finally:
        A.asrkf_destroy(ctx)
