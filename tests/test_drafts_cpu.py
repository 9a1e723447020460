"""Checks of rotary positions and drafted tokens that need no GPU: the frequencies, the masks of trees, refused
arguments, the binding's own checks, and the references that the GPU tests use."""
import ctypes
import math
import os

import numpy as np
import pytest

import paper_2512_11221_amd as A
from tests import _drafts as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_frequencies_without_scaling():
    for dim in (16, 64, 128, 256):
        f = A.asrkf_rotary_table(256, dim, base=10000.0)
        np.testing.assert_allclose(f, 10000.0 ** (-np.arange(0, dim, 2) / dim), rtol=1e-14)
    assert (A.asrkf_rotary_table(64, 64, layout="pairs") == A.asrkf_rotary_table(64, 64, layout="halves")).all()


def test_scaled_frequencies():
    dim, base, ctx, factor = 128, 500000.0, 8192, 8.0
    plain = A.asrkf_rotary_table(dim, dim, base=base)
    np.testing.assert_allclose(A.asrkf_rotary_table(dim, dim, base=base, scaling="linear", factor=factor), plain / factor, rtol=1e-15)
    # bands: kept above `high` turns over the original context, stretched below `low`, straight between in turns
    bands = A.asrkf_rotary_table(dim, dim, base=base, scaling="bands", factor=factor, original_ctx=ctx, low=1.0, high=4.0)
    turns = ctx * plain / (2 * math.pi)
    assert (turns > 4).any() and (turns < 1).any() and ((turns > 1) & (turns < 4)).any()
    np.testing.assert_allclose(bands[turns >= 4], plain[turns >= 4], rtol=1e-15)
    np.testing.assert_allclose(bands[turns <= 1], plain[turns <= 1] / factor, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    s = (turns[mid] - 1) / 3
    np.testing.assert_allclose(bands[mid], plain[mid] * s + plain[mid] / factor * (1 - s), rtol=1e-14)
    # ramp: by pair, between the pairs of 32 turns (down) and of one (up)
    ramp = A.asrkf_rotary_table(dim, dim, base=base, scaling="ramp", factor=factor, original_ctx=ctx, low=1.0, high=32.0)
    p = math.floor(64 * math.log(ctx / (32 * 2 * math.pi)) / math.log(base))
    q = math.ceil(64 * math.log(ctx / (2 * math.pi)) / math.log(base))
    i = np.arange(64)
    s = 1 - np.clip((i - p) / (q - p), 0, 1)
    np.testing.assert_allclose(ramp, plain * s + plain / factor * (1 - s), rtol=1e-14)
    assert 0 < p < q < 64 and (ramp[: p + 1] == plain[: p + 1]).all()
    # a context so short that the ramp has no width, and one whose low end lies past the last pair
    step = A.asrkf_rotary_table(64, 64, base=1e4, scaling="ramp", factor=2.0, original_ctx=1, low=1.0, high=2.0)
    np.testing.assert_allclose(step[1:], A.asrkf_rotary_table(64, 64, base=1e4)[1:] / 2, rtol=1e-15)
    far = A.asrkf_rotary_table(64, 64, base=10.0, scaling="ramp", factor=2.0, original_ctx=1 << 20, low=1.0, high=32.0)
    assert np.isfinite(far).all() and (far > 0).all()


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=8), dict(dim=72), dict(dim=144), dict(dim=-16), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
                                 dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1), dict(magnitude=0.0), dict(magnitude=math.nan),
                                 dict(magnitude=math.inf), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=math.nan),
                                 dict(scaling="bands", factor=2.0), dict(scaling="ramp", factor=2.0, original_ctx=9, low=0.0),
                                 dict(scaling="ramp", factor=2.0, original_ctx=9, low=2.0, high=2.0),
                                 dict(scaling="bands", factor=2.0, original_ctx=9, low=2.0, high=math.inf)])
def test_rotary_settings_refused(bad):
    kw = {"dim": 64, **bad}
    with pytest.raises(A.AsrkfError) as e:
        A.asrkf_rotary_table(128, kw.pop("dim"), **kw)
    assert e.value.code == A._lib.EINVAL
    for kw in (dict(layout="thirds"), dict(scaling="some")):
        with pytest.raises(ValueError):
            A.make_rotary(64, **kw)


def test_masks_and_depths_of_trees():
    rng = np.random.default_rng(0)
    for n in (1, 2, 7, 63, 64):
        for parents in (R.random_tree(rng, n, 64), list(range(-1, n - 1)), [-1] * n):
            sees, depth = A.asrkf_tree_masks(parents)
            assert sees.tolist() == R.sees_of(parents)
            assert depth.tolist() == [bin(m).count("1") - 1 for m in R.sees_of(parents)]
    for bad in ([], [0], [-2], [-1, 1], [-1, 0, 5], [-1] * 65):
        with pytest.raises(A.AsrkfError) as e:
            A.asrkf_tree_masks(bad)
        assert e.value.code == A._lib.EINVAL
    lib = A.load()
    p = np.array([-1, 0], np.int32)
    assert lib.asrkf_tree_masks(2, p.ctypes.data, None, None) == 0 and lib.asrkf_tree_masks(2, None, None, None) == A._lib.EINVAL


def test_null_context():
    lib, EINVAL = A.load(), A._lib.EINVAL
    assert lib.asrkf_set_rotary(None, ctypes.byref(A.make_rotary(64))) == EINVAL
    assert lib.asrkf_rotate(None, 1, 0, None, None, 0, None, 0, None, 0, None, 0, 0, None) == EINVAL
    assert lib.asrkf_reserve_drafts(None, 4) == EINVAL
    assert lib.asrkf_attend_drafts(None, 0, 1, None, None, None, 0, None, 0, None, 0, None, None) == EINVAL
    assert lib.asrkf_verify_drafts(None, 1, None, None, None, None, None, None, 1.0, None, None, None, None, None) == EINVAL
    assert lib.asrkf_accept_drafts(None, 1, None, None, None, 0, 0, None, 0, 0, None) == EINVAL
    assert "null context" in A.asrkf_last_error()
    assert lib.asrkf_rotary_table(None, 64, None) == EINVAL


def test_binding_struct_matches_the_header(tmp_path):
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    fields = [f for f, _ in A._lib.asrkf_rotary._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "asrkf.h"\nint main(void) {\n    printf("%zu\\n", sizeof(asrkf_rotary));\n' +
                   "".join(f'    printf("%zu\\n", offsetof(asrkf_rotary, {f}));\n' for f in fields) + "    return 0;\n}\n")
    exe = str(tmp_path / "layout")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-pedantic", str(src), "-I", os.path.join(ROOT, "include"), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, timeout=60).stdout.split()]
    assert got == [ctypes.sizeof(A._lib.asrkf_rotary)] + [getattr(A._lib.asrkf_rotary, f).offset for f in fields]


def _context():
    import torch
    ctx = A._lib.Context(1 << 12)
    ctx.layout, ctx.sizes = (8, 2, 64, torch.bfloat16), (3, 2, 50)
    return ctx


class _Called(Exception):
    pass


class _NoLibrary:
    def __getattr__(self, name):
        def call(*a):
            raise _Called(name, a)
        return call


def test_rows_of_views():
    """Evenly spaced rows of any leading dimensions, with their stride; everything else is refused."""
    import torch
    ctx, f = _context(), A._lib._rows
    x = torch.zeros((2, 5, 12, 64), dtype=torch.bfloat16)
    q = x[:, :, :8]
    assert f(ctx, "q", q, 0) == (10, 768) and f(ctx, "k", x[:, :, 8:10], 1) == (10, 768) and f(ctx, "q", q[0], 0) == (5, 768)
    assert f(ctx, "q", q[:, :1], 0) == (2, 3840) and f(ctx, "q", q[:1, :1], 0) == (1, 0) and f(ctx, "q", q[:, 0], 0) == (2, 3840)
    assert f(ctx, "q", q[:0], 0) == (0, 0) and f(ctx, "q", q[:, ::2][:, :1], 0) == (2, 3840) and f(ctx, "q", x[0, ::2, :8], 0) == (3, 1536)
    for bad in (q[:, :4], q.transpose(0, 1), q[:1].expand(2, 5, 8, 64), torch.zeros((10, 8, 128), dtype=torch.bfloat16)[..., :64],
                torch.zeros((10, 16, 64), dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError):
            f(ctx, "q", bad, 0)
    for bad in (q.float(), x, q[..., :32], q[0, 0]):
        with pytest.raises(A.AsrkfError):
            f(ctx, "q", bad, 0)


def test_binding_refuses_tensors_of_other_shapes_and_types(monkeypatch):
    import torch
    monkeypatch.setattr(A._lib, "load", _NoLibrary)
    ctx = _context()
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)                        # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)                          # noqa: E731
    good = dict(layer=0, sees=torch.zeros((2, 5), dtype=torch.int64), q=bf(2, 5, 8, 64), k=bf(2, 5, 2, 64), v=bf(2, 5, 2, 64), out=bf(2, 5, 8, 64))

    def attend(**kw):
        A.asrkf_attend_drafts(ctx, *{**good, **{k: v for k, v in kw.items() if k != "count"}}.values(), count=kw.get("count"), stream=0)
    for kw in (dict(), dict(count=i32(2)), dict(sees=torch.zeros((2, 5), dtype=torch.uint64))):
        with pytest.raises(_Called):
            attend(**kw)
    for kw in (dict(sees=torch.zeros((2, 4), dtype=torch.int64)), dict(sees=i32(2, 5)), dict(count=i32(3)), dict(count=i32(2).long()), dict(q=bf(2, 4, 8, 64)),
               dict(k=bf(2, 6, 2, 64)), dict(v=bf(2, 5, 4, 64)), dict(out=bf(2, 5, 8, 64).float()), dict(out=bf(1, 5, 8, 64))):
        with pytest.raises(A.AsrkfError) as e:
            attend(**kw)
        assert e.value.code == A._lib.EINVAL
    with pytest.raises(ValueError):
        attend(out=bf(2, 5, 10, 64)[:, :, :8])

    with pytest.raises(_Called) as e:
        A.asrkf_accept_drafts(ctx, i32(2, 5), i32(2), bf(3, 2, 5, 2, 64), bf(3, 2, 5, 4, 64)[:, :, :, 2:], stream=0)
    assert e.value.args[1][5:7] == (128, 1280) and e.value.args[1][8:10] == (256, 2560)
    for k in (bf(2, 2, 5, 2, 64), bf(3, 2, 4, 2, 64), bf(3, 2, 5, 2, 32), bf(2, 5, 2, 64)):
        with pytest.raises(A.AsrkfError):
            A.asrkf_accept_drafts(ctx, i32(2, 5), i32(2), k, bf(3, 2, 5, 2, 64), stream=0)

    rot = lambda **kw: A.asrkf_rotate(ctx, *{**dict(pos=i32(10), q=bf(10, 8, 64), q_out=bf(2, 5, 8, 64), k=None, k_out=None), **kw}.values(), stream=0)  # noqa: E731
    with pytest.raises(_Called):
        rot()
    with pytest.raises(_Called):
        rot(k=bf(10, 2, 64), k_out=bf(10, 2, 64), pos=i32(2, 5))
    for kw in (dict(pos=i32(9)), dict(pos=i32(10).long()), dict(q_out=bf(9, 8, 64)), dict(k=bf(11, 2, 64), k_out=bf(11, 2, 64)), dict(q=bf(10, 2, 64))):
        with pytest.raises(A.AsrkfError):
            rot(**kw)
    for kw in (dict(q_out=None), dict(q=None, q_out=None), dict(k=bf(10, 2, 64))):
        with pytest.raises(ValueError):
            rot(**kw)


def test_the_walks_reference_keeps_the_distribution():
    """The reference walk itself, over a grid of random numbers: the token behind the root has the target's distribution,
    with a draft's probabilities and without."""
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.2, 0.6], np.float32)
    root, n = np.log(p).astype(np.float32), 60
    grid = (np.arange(n) + 0.5) / n
    for probs in (None, [q, q]):
        got = np.zeros(3)
        for x, y in ((x, y) for x in range(3) for y in range(3)):
            weight = float(q[x]) * float(q[y])
            for a in grid:
                for b in grid:
                    path, tok = R.verify([x, y], [-1, -1], 2, root, [root, root], probs, 1.0, [a, b, 0.0])
                    if path:
                        got[[x, y][path[0]]] += weight / n ** 2
                        continue
                    # the draw over a grid of its own random number
                    for c in (np.arange(12) + 0.5) / 12:
                        got[R.verify([x, y], [-1, -1], 2, root, [root, root], probs, 1.0, [a, b, c])[1]] += weight / n ** 2 / 12
        # each test and the draw are off by a step of their grid at most, the draw of what was rejected only
        assert np.abs(got - p).max() <= 2 / n + 1 / 12, got
