"""The example block (examples/molecule_block.py) on the GPU: it commutes with rotations, draws included; its gradients
agree with differences; training lowers the loss."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import gtp_oracle as O  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("molecule_block", os.path.join(ROOT, "examples", "molecule_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def small(m, L, p, C=16, heads=4):
    offsets, longest = m.molecules(5, 9)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((int(offsets[-1]), C, (L + 1) ** 2), generator=g, device="cuda")
    rng = torch.tensor([[11, 2], [11, 3]], dtype=torch.int64, device="cuda")
    return m.Block(C, L, heads, p), x, offsets, longest, rng


@pytest.mark.parametrize("L", [1, 2])
def test_block_commutes_with_rotations(example, L):
    block, x, offsets, longest, rng = small(example, L, 0.2)
    q, _ = np.linalg.qr(np.random.default_rng(0).standard_normal((3, 3)))
    R = q * np.sign(np.linalg.det(q))
    D = torch.from_numpy(O.wigner_d_real(L, R)).float().cuda()
    a, _ = block.forward(x, offsets, longest, rng)
    b, _ = block.forward((x @ D.T).contiguous(), offsets, longest, rng)
    # fp32: some 2^-20 of values of a few units
    assert float((a @ D.T - b).abs().max()) < 1e-4 * float(a.abs().max())


def test_gradients_against_differences(example):
    block, x, offsets, longest, rng = small(example, 2, 0.2)
    g = torch.Generator(device="cuda").manual_seed(5)
    out, s = block.forward(x, offsets, longest, rng)
    dout = torch.randn(out.shape, generator=g, device="cuda")
    dx, grads = block.backward(s, dout)
    f = lambda z: float((block.forward(z, offsets, longest, rng)[0].double() * dout.double()).sum())  # noqa: E731
    for name, grad in [("x", dx), *grads.items()]:
        t = x if name == "x" else block.params[name]
        u = torch.randn(t.shape, generator=g, device="cuda").abs() * grad.sign()  # no cancelling of the sum
        h = 5e-4
        up, dn = t + h * u, t - h * u
        if name == "x":
            got = f(up) - f(dn)
        else:
            block.params[name] = up
            got = f(x)
            block.params[name] = dn
            got -= f(x)
            block.params[name] = t
        want = float((grad.double() * (up.double() - dn.double())).sum())
        size = float((grad.double() * (up.double() - dn.double())).abs().sum())
        # the third order: logits move by some 0.05 along u, 0.05^2 / 6 of the size; fp32 outputs' 2^-20 |dout| each
        tol = 1e-3 * size + 2.0 ** -20 * float((dout * out).abs().double().sum())
        print(f"  {name}: difference {got:.6f} gradient {want:.6f} tolerance {tol:.6f}", flush=True)
        assert abs(got - want) <= tol, name


def test_training_lowers_the_loss(example):
    losses = example.train(count=8, atoms=12, C=16, steps=15, heads=4, say=lambda *_: None)
    assert losses[-1] < 0.8 * losses[0], losses
