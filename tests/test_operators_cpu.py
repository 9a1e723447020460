"""Checks of the packed prompts and the 4-bit cache that need no GPU: refused
configurations, the binding's checks, and the 4-bit format's own reference."""
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
