"""Attention of few rows over many keys, and of few keys read by many rows, on the GPU: the long axis dealt to more than
sixteen and more than sixty-four parts, against the 64-bit plain form with the tolerances of test_layers.py."""
import pytest

torch = pytest.importorskip("torch")

from test_layers import BF16, F32, Case, _say  # noqa: E402

pytestmark = pytest.mark.gpu


# (query lengths, key lengths, H, Hk, d, share of absent keys, p)
FEW = [
    ([1], [20011], 8, 8, 100, 0, 0), ([3], [17000], 2, 1, 24, 0.5, 0), ([1, 0, 2], [9001, 40, 16000], 4, 2, 64, 0.1, 0.2),
    ([1], [2500], 1, 1, 128, 0, 0), ([2], [16500], 2, 2, 200, 0.2, 0.1), ([1], [16385], 1, 1, 256, 0, 0),
    ([17000], [2], 2, 2, 40, 0, 0.1), ([9000, 5], [3, 70], 4, 1, 72, 0.2, 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ql,kl,H,Hk,d,masked,p", FEW)
def test_many_parts(ql, kl, H, Hk, d, masked, p, dtype):
    _say(f"attention q={ql} k={kl} H={H}/{Hk} d={d} masked={masked} p={p} {dtype}")
    c = Case(dtype, ql, kl, H, Hk, d, masked, p)
    o, lse = c.forward()
    torch.cuda.synchronize()
    c.check_forward(o, lse)
    g = c.backward(o, lse)
    torch.cuda.synchronize()
    c.check_backward(o, lse, g)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parts_without_a_key(dtype):
    """Whole parts of absent keys, holding NaN, count nothing; without any key a row is zero and its lse -infinity."""
    c = Case(dtype, [2], [18000], 2, 2, 64, masked=0.5)
    c.mask[:9000] = 0
    c.k[:9000] = float("nan")
    c.v[:9000] = float("inf")
    o, lse = c.forward()
    c.check_forward(o, lse)
    c.mask[:] = 0
    o, lse = c.forward()
    assert not bool(o.any()) and bool((lse == -float("inf")).all())
    g = c.backward(o, lse)
    assert not any(bool(g[n].any()) for n in g)
