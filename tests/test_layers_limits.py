"""The layers around the product on the CPU: sizes that one launch cannot hold are refused before it, layouts of outputs
that do not overlap are not, and the plain 64-bit forms of the GPU tests against autograd."""
import pytest

torch = pytest.importorskip("torch")

from test_layers_host import INVALID, OK, UNSUPPORTED, at, drop  # noqa: E402,F401


def test_dropout_refuses_more_than_a_launch_holds():
    far = dict(res=None, rng=at(1 << 20), y=at(2000), dtype=1)
    assert drop(groups=1 << 37, K=1, **far) == UNSUPPORTED
    assert drop(groups=(1 << 37) // 49 + 1, K=49, **far) == UNSUPPORTED
    assert drop(groups=1, K=1 << 31, **far) == UNSUPPORTED
