"""Numbers of rows of a rotation (asrkf_rotate): none, and those that leave a remainder in a workgroup for every number
of rows that one takes."""
import pytest

from tests import _drafts as R
from tests.test_gpu_rotate import _init, _rows, gpu                          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(dtype):
    """Empty tensors, whose address is none, are no rows: nothing is done.  Where there are rows, q or k is needed."""
    import torch
    A, ctx = _init(2, 8, 2, 64, dtype)
    try:
        A.asrkf_set_rotary(ctx, 64)
        q, k, pos = _rows(0, 8, 64, dtype), _rows(0, 2, 64, dtype), torch.empty(0, dtype=torch.int32, device="cuda")
        A.asrkf_rotate(ctx, pos, q, torch.empty_like(q), k, torch.empty_like(k))
        A.asrkf_rotate(ctx, pos, None, None, k, torch.empty_like(k))
        x = _rows(4, 8, 64, dtype)
        y = torch.full_like(x, 9.0)
        A.asrkf_rotate(ctx, torch.arange(4, device="cuda", dtype=torch.int32)[:0], x[:0], y[:0], None, None)
        torch.cuda.synchronize()
        assert (y == 9.0).all()
        lib, pos = A.load(), torch.arange(4, device="cuda", dtype=torch.int32)
        assert lib.asrkf_rotate(ctx, 4, 0, pos.data_ptr(), None, 0, None, 0, None, 0, None, 0, 0, None) == A._lib.EINVAL
        assert lib.asrkf_rotate(ctx, 0, 2, None, None, 0, None, 0, None, 0, None, 0, 0, None) == A._lib.EINVAL
    finally:
        A.asrkf_destroy(ctx)


# rows to a workgroup: 256 threads by the pairs of 16-byte pieces of a row's heads, at most 8
@pytest.mark.parametrize("Hq,Hkv,D,dtype,per", [(1, 1, 64, "bf16", 8), (2, 2, 128, "bf16", 8), (8, 2, 64, "bf16", 6), (8, 2, 64, "f32", 3), (8, 4, 128, "bf16", 2),
                                                (16, 2, 64, "bf16", 3), (8, 8, 64, "f32", 2), (32, 8, 128, "bf16", 1), (4, 4, 64, "f32", 4)])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_the_last_workgroups_rows(Hq, Hkv, D, dtype, per, layout):
    """Every remainder of rows in the last workgroup, and rows behind the last one that stay as they are."""
    import torch
    A, ctx = _init(2, Hq, Hkv, D, dtype)
    try:
        assert min(8, max(1, 256 // ((Hq + Hkv) * D // (16 if dtype == "bf16" else 8)))) == per
        A.asrkf_set_rotary(ctx, D, 500000.0, layout=layout)
        freq = A.asrkf_rotary_table(D, D, base=500000.0, layout=layout)
        for n in [1] + [3 * per + i for i in range(per)]:
            q, k = _rows(n, Hq, D, dtype, n), _rows(n, Hkv, D, dtype, n + 1)
            pos = torch.arange(n, device="cuda", dtype=torch.int32) * 1013 + 5
            qo, ko = (torch.full((n + 8,) + x.shape[1:], 9.0, dtype=x.dtype, device="cuda") for x in (q, k))
            A.asrkf_rotate(ctx, pos, q, qo[:n], k, ko[:n])
            for x, y in ((q, qo), (k, ko)):
                R.check(y[:n], *R.turned(x, pos, freq, layout))
                assert (y[n:] == 9.0).all()
    finally:
        A.asrkf_destroy(ctx)
