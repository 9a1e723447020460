"""Checks of the packed prompts and the 4-bit cache that need no GPU: refused
configurations, the binding's checks, and the 4-bit format's own reference."""
import os

import numpy as np
import pytest

import paper_2512_11221_amd as A
from tests._four import VALUES, rounded
from tests.test_abi_cpu import BASE


@pytest.mark.parametrize("bad", [dict(kv_bits=3), dict(kv_bits=8), dict(kv_bits=-4), dict(kv_bits=16),
                                 dict(kv_bits=4, dtype="f32"), dict(kv_bits=4, spill_min_D=2)])
def test_configurations_refused(bad):
    with pytest.raises(A.AsrkfError) as e:
        A.asrkf_init(A.make_config(**{**BASE, **bad}))
    assert e.value.code == A._lib.EINVAL


@pytest.mark.parametrize("bits", [0, 4])
def test_the_longest_context_is_counted_in_the_type_of_the_rows_given(bits):
    """... whatever the cache holds, and the refusal says so: 2^23 positions of 256 bytes."""
    with pytest.raises(A.AsrkfError) as e:
        A.asrkf_init(A.make_config(**{**BASE, "max_ctx": (1 << 23) - 1, "kv_bits": bits}))
    assert e.value.code == A._lib.EINVAL and "256 bytes in dtype" in str(e.value)
    assert ("4 bits" in str(e.value)) == (bits == 4)
    with open(os.path.join(os.path.dirname(A.__file__), "..", "include", "asrkf.h")) as f:
        text = f.read()
    doc = text[text.index("int32_t max_ctx;"):text.index("int32_t window_K;")]
    assert "2 GiB" in doc and "4 bits" in doc


def test_null_context():
    lib = A.load()
    assert lib.asrkf_prefill_packed(None, 0, 1, None, None, None, 0, None, 0, None, 0, None, None) == A._lib.EINVAL
    assert lib.asrkf_get_rows(None, 0, 0, 0, 1, None, None, None) == A._lib.EINVAL
    assert "null context" in A.asrkf_last_error()


def test_binding_takes_token_strides_and_refuses_other_layouts():
    import torch
    f = A._lib._token_stride
    x = torch.zeros((5, 12, 64))
    assert f("q", x) == 768 and f("q", x[:, 2:4]) == 768 and f("q", None) == 0 and f("q", x.view(-1)) == 0
    assert f("q", x[:1, 2:4]) == 0                 # one token has no next
    for bad in (x[:, ::2], x[:, :, :32], x.transpose(0, 1), x.view(-1)[::2]):
        with pytest.raises(ValueError):
            f("q", bad)


def test_binding_refuses_tokens_that_share_memory():
    """An expanded tensor's token stride of 0 is not the 0 that stands for dense rows."""
    import torch
    x = torch.zeros((1, 2, 64)).expand(7, 2, 64)
    y = torch.zeros(4096).as_strided((7, 2, 64), (64, 64, 1))
    for bad in (x, y):
        with pytest.raises(ValueError):
            A._lib._token_stride("k", bad)


def test_four_bit_reference():
    """The reference itself: its values are its own, X is the smallest that the rule allows, and
    no value is off by more than X."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4000, 32)) * np.exp2(rng.integers(-90, 90, (4000, 1)).astype(float))
    r = rounded(x)
    assert np.array_equal(rounded(r), r)
    top = np.abs(x).max(1)
    X = np.exp2(np.floor(np.log2(top / 7)) + 1)
    assert (top < 7 * X).all() and (top >= 3.5 * X).all()
    assert (np.abs(r - x) <= X[:, None]).all()
    assert np.isin(np.abs(r / X[:, None]), VALUES).all()
    assert np.isnan(rounded(np.r_[np.inf, np.zeros(31)])).all() and (rounded(np.zeros(32)) == 0).all()
    assert (rounded(np.full(32, 2.0 ** -130)) == 0).all()


class _Called(Exception):
    pass


class _NoLibrary:
    """In the place of the library: says that the call got that far."""
    def asrkf_prefill_packed(self, *a):
        raise _Called

    asrkf_get_rows = asrkf_prefill_packed


def _context():
    import torch
    ctx = A._lib.Context(1 << 12)
    ctx.layout = (8, 2, 64, torch.bfloat16)
    return ctx


def test_binding_refuses_tensors_that_hold_too_little(monkeypatch):
    """A tensor that ends before the rows of the lengths' sum, or of another type, lies in an allocation
    that may go on behind it: the library would take its neighbour's bytes for rows.  Every other
    view of the same rows is taken as before."""
    import torch
    monkeypatch.setattr(A._lib, "load", _NoLibrary)
    ctx = _context()
    rows = lambda n, h, d=64, t=torch.bfloat16: torch.zeros((n, h, d), dtype=t)   # noqa: E731
    q, k, out = rows(12, 8), rows(12, 2), rows(12, 8)
    good = dict(q=q, k=k, v=k, out=out)

    def call(lens=(5, 0, 7), ctx=ctx, **kw):
        A.asrkf_prefill_packed(ctx, 0, range(len(lens)), lens, *{**good, **kw}.values(), stream=0)

    fused = rows(12, 12)
    taken = [dict(), dict(q=None, out=None), dict(lens=(3, 4)), dict(k=k.view(-1), v=k.view(12, 128)),
             dict(q=q.view(1, 12, 512), k=k.view(1, 12, 2, 64)), dict(q=fused[:, :8], k=fused[:, 8:10], v=fused[:, 10:]),
             dict(q=fused), dict(lens=(0,), q=None, k=None, v=None, out=None), dict(lens=(0, 0), k=rows(0, 2)),
             dict(lens=(-3, 2)), dict(ctx=int(ctx), q=rows(11, 8))]    # (the library's to refuse; a bare handle)
    for kw in taken:
        with pytest.raises(_Called):
            call(**kw)
    wide = torch.float32
    for name, h in (("q", 8), ("k", 2), ("v", 2), ("out", 8)):
        for bad in (rows(11, h), rows(12, h, t=wide), rows(12, h).view(torch.int16), rows(12, h, 32), rows(12, h).half(),
                    rows(12, h).view(-1)[:-1], rows(11, h).view(11, -1), rows(1, h), rows(0, h)):
            with pytest.raises(A.AsrkfError) as e:
                call(**{name: bad})
            assert e.value.code == A._lib.EINVAL and str(e.value).split(": ")[1].startswith(name), e.value
    for bad in (fused[:11, :8], fused[:, 5:12]):                       # slices of a fused projection
        with pytest.raises(A.AsrkfError):
            call(q=bad)

    for k12 in (k, k.view(-1), rows(13, 2)):
        with pytest.raises(_Called):
            A.asrkf_get_rows(ctx, 0, 0, 3, 12, k12, k.clone(), stream=0)
    for bad in (rows(11, 2), rows(12, 2, t=wide), rows(12, 2).view(-1)[:-1], rows(0, 2)):
        for a, b in ((bad, k), (k, bad)):
            with pytest.raises(A.AsrkfError) as e:
                A.asrkf_get_rows(ctx, 0, 0, 0, 12, a, b, stream=0)
            assert e.value.code == A._lib.EINVAL
