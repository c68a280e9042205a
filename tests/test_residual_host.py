"""The residual step on the CPU: refusals of the C entries (made-up pointers: every argument is checked before the first
HIP call) and of the binding, work sizes, and the plain 64-bit forms of the GPU tests against autograd."""
import math
import struct

import pytest

torch = pytest.importorskip("torch")

import residual_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
OK, INVALID, UNSUPPORTED = gtp.GTP_OK, gtp.GTP_ERR_INVALID_ARG, gtp.GTP_ERR_UNSUPPORTED
GB = 1 << 30


def at(i):
    """A made-up device address: the i-th GiB."""
    return (100 + i) * GB


def desc(L=2, dtype=0, N=10, C=8, post=1, eps=1e-5, scale=at(0), w_post=at(1), b_post=at(2), w_pre=at(3), b_pre=at(4),
         gate=at(5)):
    return struct.pack("<2i2qif6Q", L, dtype, N, C, post, eps, *(p or 0 for p in (scale, w_post, b_post, w_pre, b_pre, gate)))


def stats_of(i=10, **more):
    d = dict(mean_post=at(i), rstd_post=at(i + 1), mean_pre=at(i + 2), rstd_pre=at(i + 3))
    d.update(more)
    return struct.pack("<4Q", *(p or 0 for p in d.values()))


def forward(x=at(20), a=at(21), r=at(22), h=at(23), stats="", **more):
    return gtp.lib().gtp_residual_norm(desc(**more), x, a, r, h, stats_of() if stats == "" else stats, None)


GRADS = dict(dx=at(30), da=at(31), dgate=at(32), dscale=at(33), dw_post=at(34), db_post=at(35), dw_pre=at(36), db_pre=at(37))


def backward(r=at(20), a=at(21), stats="", dh=at(24), dr=at(25), work=at(40), nbytes=1 << 26, grads=GRADS, **more):
    own = {n: more.pop(n) for n in list(more) if n in GRADS}
    g = None if grads is None else struct.pack("<8Q", *(p or 0 for p in {**grads, **own}.values()))
    return gtp.lib().gtp_residual_norm_backward(desc(**more), r, a, stats_of() if stats == "" else stats, dh, dr, g, work,
                                                nbytes, None)


DESC = [dict(L=-1), dict(L=65), dict(dtype=2), dict(N=-1), dict(C=-1), dict(post=2), dict(post=-1), dict(eps=0.0),
        dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(N=1 << 62), dict(post=0), dict(post=0, w_post=None),
        dict(post=0, b_post=None), dict(scale=at(0) + 2), dict(w_post=at(1) + 1), dict(b_post=at(2) + 2),
        dict(w_pre=at(3) + 1), dict(b_pre=at(4) + 2), dict(gate=at(5) + 2), dict(gate=at(5) + 1, dtype=1)]


@pytest.mark.parametrize("bad", DESC)
def test_bad_descriptions(bad):
    assert forward(**bad) == INVALID and backward(**bad) == INVALID
    assert gtp.lib().gtp_last_error()
    assert gtp.lib().gtp_residual_norm_backward_work(desc(**bad)) == -1


def test_forward_refusals():
    for bad in (dict(x=None), dict(a=None), dict(r=None), dict(h=None), dict(x=at(20) + 2), dict(a=at(21) + 1),
                dict(r=at(22) + 2), dict(h=at(23) + 3), dict(r=at(21)), dict(r=at(20) + 16), dict(h=at(20)), dict(h=at(21)),
                dict(h=at(22)), dict(h=at(5)), dict(r=at(0)), dict(r=at(1)), dict(r=at(2)), dict(h=at(3)), dict(h=at(4)),
                dict(stats=stats_of(mean_post=at(22))), dict(stats=stats_of(rstd_pre=at(23))),
                dict(stats=stats_of(rstd_post=at(10))), dict(stats=stats_of(mean_pre=at(12) + 2)),
                dict(stats=stats_of(), post=0, w_post=None, b_post=None)):
        assert forward(**bad) == INVALID, bad
    assert gtp.lib().gtp_residual_norm(None, at(0), at(1), at(2), at(3), None, None) == INVALID
    assert forward(N=1 << 31, C=1, L=0, x=at(100), r=at(200), a=at(300), h=at(400)) == UNSUPPORTED
    assert forward(N=1, C=1 << 31, L=0, x=at(100), r=at(200), a=at(300), h=at(400)) == UNSUPPORTED
    assert forward(N=0, x=None, a=None, r=None, h=None) == OK and forward(C=0, x=None, a=None, r=None, h=None) == OK


def test_backward_refusals():
    for bad in (dict(r=None), dict(a=None), dict(dh=None), dict(stats=None), dict(stats=stats_of(mean_pre=None)),
                dict(stats=stats_of(rstd_pre=None)), dict(stats=stats_of(mean_post=None)),
                dict(stats=stats_of(rstd_post=None)), dict(work=None), dict(nbytes=15), dict(work=at(40) + 4),
                dict(grads=None), dict(gate=None), dict(dx=at(20)), dict(dx=at(24)), dict(dx=at(25) + 16), dict(da=at(21)),
                dict(da=at(25)), dict(dgate=at(5)), dict(dscale=at(0)), dict(dw_post=at(1)), dict(db_post=at(2)),
                dict(dw_pre=at(3)), dict(db_pre=at(4)), dict(db_pre=at(36)), dict(dx=at(31)), dict(dx=at(30) + 2),
                dict(dgate=at(32) + 1), dict(dscale=at(33) + 2), dict(work=at(24)), dict(work=at(30)), dict(dw_pre=at(13)),
                dict(dr=at(25) + 1), dict(post=0, w_post=None, b_post=None)):
        assert backward(**bad) == INVALID, bad
    assert backward(grads=dict.fromkeys(GRADS)) == OK
    assert backward(C=0) == OK
    assert backward(N=1 << 31, C=1, L=0) == UNSUPPORTED
    w = gtp.lib().gtp_residual_norm_backward_work
    assert w(None) == -1 and w(desc(N=0)) == 0 and w(desc(C=0)) == 0
    assert w(desc()) >= 4 * 8 * 8


def test_binding_refusals():
    z = lambda *s, dtype=F32: torch.zeros(s, dtype=dtype)  # noqa: E731
    x, a = z(4, 8, 9), z(4, 8, 9)
    st = (z(4), z(4, 3), z(4), z(4, 3))
    f, b = gtp.gtp_residual_norm, gtp.gtp_residual_norm_backward
    for call, error in (
            (lambda: f(z(4, 8, 8), a, 2), ValueError), (lambda: f(x, z(4, 8, 8), 2), ValueError),
            (lambda: f(x.double(), a, 2), TypeError), (lambda: f(x, a.bfloat16(), 2), TypeError),
            (lambda: f(x, a, 2, gate=z(4, 9)), ValueError), (lambda: f(x, a, 2, gate=z(4, 8, dtype=BF16)), TypeError),
            (lambda: f(x, a, 2, scale=z(2, 8)), ValueError), (lambda: f(x, a, 2, w_post=z(3, 8, dtype=BF16)), TypeError),
            (lambda: f(x, a, 2, w_post=z(3, 8), post=False), ValueError),
            (lambda: f(x, a, 2, b_post=z(8), post=False), ValueError), (lambda: f(x, a, 2, b_pre=z(9)), ValueError),
            (lambda: f(z(8, 4, 9).transpose(0, 1), a, 2), ValueError), (lambda: f(x, a, 2, r=z(4, 8, 9, dtype=BF16)), TypeError),
            (lambda: f(x, a, 2, h=z(3, 8, 9)), ValueError), (lambda: f(x, a, 2), ValueError),  # not device tensors
            (lambda: b(x, a, 2, st, z(4, 8, 9, dtype=BF16)), TypeError), (lambda: b(x, a, 2, st[:3], x), ValueError),
            (lambda: b(x, a, 2, (z(4), z(4, 2), z(4), z(4, 3)), x), ValueError),
            (lambda: b(x, a, 2, (None, None, z(4), z(4, 3)), x), TypeError),
            (lambda: b(x, a, 2, st, x, need=("dgate",)), ValueError), (lambda: b(x, a, 2, st, x, need=("dy",)), ValueError),
            (lambda: b(x, a, 2, st, x, post=False, need=("dw_post",)), ValueError),
            (lambda: b(x, a, 2, st, x, dr=z(4, 8, 4)), ValueError), (lambda: b(x, a, 2, st, x), ValueError)):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("L", [0, 1, 3])
def test_plain_forms_against_autograd(L, gated, post):
    g = torch.Generator().manual_seed(L)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    N, C, K = 5, 6, (L + 1) ** 2
    leaves = {"dx": n(N, C, K), "da": n(N, C, K), "dgate": n(N, C), "dscale": n(L + 1, C), "dw_post": n(L + 1, C),
              "db_post": n(C), "dw_pre": n(L + 1, C), "db_pre": n(C)}
    if not gated:
        leaves["dgate"] = None
    if not post:
        leaves["dw_post"] = leaves["db_post"] = None
    for t in leaves.values():
        if t is not None:
            t.requires_grad_()
    args = [leaves[k] for k in ("dgate", "dscale", "dw_post", "db_post", "dw_pre", "db_pre")]
    r, h, stats = R.forward(leaves["dx"], leaves["da"], L, *args, post)
    dh, dr = n(N, C, K), n(N, C, K)
    ((h * dh).sum() + (r * dr).sum()).backward()
    with torch.no_grad():
        out, _, _ = R.backward(r, leaves["da"], L, stats, dh, dr, *args, post)
    for name, t in leaves.items():
        if t is not None:
            assert torch.allclose(out[name], t.grad, rtol=1e-9, atol=1e-11), name
