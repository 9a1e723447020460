"""What rejections leave of a row, where that is next to nothing of a part or of the whole (asrkf_verify_drafts)."""
import numpy as np
import pytest

from tests.test_gpu_verify import Case, _init, gpu                           # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,T", [(70000, 1.0), (131072, 0.7), (262144, 1.0), (300000, 1.3)])
def test_parts_of_which_next_to_nothing_is_left(V, T):
    """A heavy token in every part of the row, all of them rejected one after the other: the draw is from the 10^-4 that
    stand beside them, which every part is summed again for, by several waves in turn."""
    B, heavy = 8, 60
    A, ctx = _init(B, V, heavy)
    try:
        for seed in range(3):
            c = Case(B, heavy, V, False, seed, ragged=False)
            c.parents[:] = -1
            c.tokens[:] = (np.arange(heavy) * (V / heavy) + c.rng.integers(0, V // heavy, (B, heavy))).astype(np.int32)
            c.root[:] = c.rng.standard_normal((B, V)).astype(np.float32) * 0.5
            light = T * np.log(1e-4 * heavy / V / np.exp(0.125 / T ** 2))       # all light ones of a part weigh 10^-4 of its heavy one
            for b in range(B):
                c.root[b] += np.float32(light)
                c.root[b, c.tokens[b]] = c.rng.uniform(-0.1, 0.1, heavy)
            c.u[:, :heavy] = 1 - 2.0 ** -24
            path, n, nxt = got = c.run(A, ctx, T, count=False)
            c.check(got, T)
            assert (n == 0).all() and not (nxt[:, None] == c.tokens).any()
    finally:
        A.asrkf_destroy(ctx)


def _beside(about, octave, which):
    """A temperature near `about` at which two logits, neighbours among the fp32 numbers from `octave` to twice that, have
    a probability (of the larger or the smaller one) just beside an fp32 number: 10^-12 to 5 * 10^-10 of it."""
    rng = np.random.default_rng(1)
    T = (about * rng.uniform(0.9, 1.1, 100000)).astype(np.float32).astype(np.float64)
    z = np.exp(-octave * 2.0 ** -23 / T)
    p = (1 / (1 + z), z / (1 + z))[which]
    u = p.astype(np.float32)
    off = np.abs(u - p) / p
    at = int(np.nonzero((off > 1e-12) & (off < 5e-10))[0][0])
    return float(T[at]), u[at]


@pytest.mark.parametrize("about,octave", [(1.2e-6, 16.0), (2.4e-6, 32.0), (2e-5, 256.0), (2e-3, 32768.0)])
@pytest.mark.parametrize("V", [5000, 262144 + 9000])
@pytest.mark.parametrize("first", [0, 1])
def test_cold_rows_over_several_parts(about, octave, V, first):
    """Temperatures at which a step of fp32 logits weighs e and more: two tokens in different parts of the row have all
    of the weight, and the random numbers lie 10^-12 to 5 * 10^-10 beside the drafted token's probability, or beside
    where the draw passes from the first of them in the vocabulary to the other."""
    B = 512 if V < 10000 else 24
    A, ctx = _init(B, V, 1)
    try:
        at = (V - 700, 12) if first else (12, V - 700)       # of the larger one and the smaller one
        for draw in (False, True):
            which = first if draw else 1
            T, u = _beside(about, octave, which)
            c = Case(B, 1, V, False, 0, ragged=False)
            x = (octave * c.rng.uniform(1.001, 1.999, B)).astype(np.float32)
            c.parents[:] = -1
            c.root[:] = -np.inf
            c.root[:, at[0]], c.root[:, at[1]] = x, np.nextafter(x, np.float32(0))
            c.tokens[:] = -1 if draw else at[1]              # (one outside the vocabulary leaves the row as it is)
            c.u[:, 0], c.u[:, 1] = (0.5, u) if draw else (u, 0.5)
            c.check(c.run(A, ctx, T, count=False), T)
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("scale,T", [(1e12, 1e-6), (3e38, 1.0), (3e38, 1e-6), (1e30, 0.7)])
@pytest.mark.parametrize("probs", [False, True])
def test_the_largest_logits(scale, T, probs):
    """Logits whose quotient by the temperature is known to more than a factor no longer: equal ones share the weight."""
    T = float(np.float32(T))
    B, V = 40, 9000
    A, ctx = _init(B, V, 3)
    try:
        c = Case(B, 3, V, probs, 5, ragged=False)
        rows = np.concatenate([c.root[:, None], c.logits], 1)
        rows *= np.float32(scale / 100)
        for b in range(B):
            for i in range(4):
                rows[b, i, c.rng.integers(0, V, 3)] = np.float32(scale) * np.float32(c.rng.uniform(0.5, 1))
                if i < 3:
                    c.tokens[b, i] = rows[b, i].argmax()
        c.parents[:] = [-1, 0, 1]
        c.root, c.logits = rows[:, 0].copy(), rows[:, 1:].copy()
        got = c.run(A, ctx, T, count=False)
        c.check(got, T)
        assert got[1].any() and (got[2] >= 0).all()
    finally:
        A.asrkf_destroy(ctx)


@pytest.mark.parametrize("T", [0.7, 1.0, 1.9])
@pytest.mark.parametrize("V", [20000, 300000])
def test_the_last_token_of_any_weight_is_kept(V, T):
    """Three tokens have all of the weight and the first two drafts of them are rejected: W is the third's weight, which
    u < 1 keeps, however little it is."""
    B = 1024 if V < 100000 else 64
    T = float(np.float32(T))
    A, ctx = _init(B, V, 4)
    try:
        c = Case(B, 4, V, False, int(T * 10), ragged=False)
        c.parents[:] = [-1, -1, -1, 2]
        c.tokens[:] = [5000, 10, 15000, 77]
        c.root[:] = -np.inf
        c.root[:, 5000] = c.rng.uniform(-9, 9, B)
        c.root[:, 10] = c.root[:, 5000] + c.rng.uniform(-1, 1, B).astype(np.float32)
        c.root[:, 15000] = c.root[:, 5000] + T * np.log(10.0 ** c.rng.uniform(-6.5, -5.5, B)).astype(np.float32)
        c.u[:, :3] = 1 - 2.0 ** -24
        got = c.run(A, ctx, T, count=False)
        c.check(got, T)
        assert (got[1] >= 1).all() and (got[0][:, 0] == 2).all()
    finally:
        A.asrkf_destroy(ctx)


def test_siblings_that_weigh_less_and_less():
    """Up to five siblings, each with all but 10^-1 to 10^-6.5 of what the ones before it have left, over a floor of
    further tokens or none, and random numbers near 1: many rejections in a row, W down to 10^-30."""
    B, N, V = 1024, 5, 9000
    A, ctx = _init(B, V, N)
    try:
        deep = 0
        for seed in range(4):
            c = Case(B, N, V, False, seed, ragged=False)
            c.parents[:] = -1
            c.root[:] = -np.inf
            c.root[B // 2:, 6000:] = -80.0
            left = np.zeros(B)
            for i in range(N):
                c.tokens[:, i] = c.rng.permutation(V)[:B] % 6000
                share = 10.0 ** c.rng.uniform(-6.5, -1, B)
                c.root[np.arange(B), c.tokens[:, i]] = (left + np.log1p(-share)).astype(np.float32)
                left += np.log(share)
            c.u[:, :N] = 1 - c.rng.choice([2.0 ** -24, 2.0 ** -22, 2.0 ** -18], (B, N))
            path, n, nxt = got = c.run(A, ctx, 1.0, count=False)
            c.check(got, 1.0)
            deep += ((n == 0) | (path[:, 0] >= 2)).sum()
        assert deep > 1000
    finally:
        A.asrkf_destroy(ctx)
