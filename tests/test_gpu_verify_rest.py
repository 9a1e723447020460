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
