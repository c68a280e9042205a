"""The layers around the product on the GPU against plain 64-bit forms
(tests/layers_ref.py): normalisation of SH features, dropout, attention, and
their gradients; types, lengths from none to long, odd sizes, strides and
alignment, absent keys, streams, graphs, run-to-run equality, and the
poisoned-LDS build.

Tolerances.  u = 2^-24 is half a unit in the last place of fp32; bf16 has 8
significant bits, so rounding to it moves a value by at most 2^-8 of itself, and
an output in bf16 carries that.  fp32 sums of n terms here run over at
most a few hundred in sequence per lane: an error below 2^-16 (256 u) of the sum
of the terms' magnitudes.  With bf16 inputs the attention rounds P (or dS) to
bf16 before it sums: 2^-8 of the same sums besides.  Each comparison takes these
sums from the reference, element by element.
"""
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
C32 = 2.0 ** -16
POISON_LIB = os.path.join(os.path.dirname(gtp.__file__), "libgtp_poison.so")
RNG = (0x9E3779B97F4A7C15 >> 1, 5)


def _say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def off_by_one(t):
    """The same values one element past a 16-byte boundary."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    out = buf[1:].view(t.shape)
    out.copy_(t)
    return out


def close(got, want, tol, what):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    worst = float((err / tol.clamp_min(1e-300)).max()) if err.numel() else 0.0
    _say(f"  {what}: worst {worst:.3f} of the tolerance")
    assert not bool(bad.any()), (what, worst, int(bad.sum()))


def out_tol(want, dtype):
    return want.abs() * (2.0 ** -8 if dtype == BF16 else 2.0 ** -23)


# ------------------------------------------------------------------ normalisation

NORMS = [(1, 1, 0), (3, 1, 0), (5, 7, 0), (33, 256, 0), (3, 300, 0), (2, 5000, 0), (1, 70001, 0), (700, 17, 0),
         (1, 1, 1), (7, 5, 1), (65, 16, 1), (33, 16, 2), (257, 64, 2), (3, 1000, 3), (40, 33, 4), (9, 128, 6),
         (4, 64, 8), (3, 65, 12), (3, 64, 16), (2, 3, 20), (2, 2, 64), (1, 600, 8)]


def norm_case(N, C, L, dtype, seed=0, shift=0.3):
    g = gen(1000 + seed + N + 7 * C + 13 * L)
    x = randn(g, N, C, (L + 1) ** 2)
    x[..., 0] += shift
    return x.to(dtype), randn(g, N, C, (L + 1) ** 2, dtype=dtype), 1 + 0.2 * randn(g, L + 1, C), 0.2 * randn(g, C)


def norm_check(x, dy, w, b, L, y, mean, rstd, grads, what):
    dt = x.dtype
    d = lambda t: None if t is None else t.double()  # noqa: E731
    ry, rm, rr = R.norm(d(x), L, d(w), d(b), 1e-5)
    big = x.double().abs()
    size = (big + (big[..., :1].amax(1, keepdim=True))) * rr.amax(1)[:, None, None] + 1.0
    close(mean, rm, C32 * x[..., 0].double().abs().mean(1) + 1e-30, what + " mean")
    # the mean's own error, counted against the row's spread
    close(rstd, rr, C32 * rr * (1 + size.amax((1, 2)))[:, None], what + " rstd")
    wm = 1.0 if w is None else w.abs().max().double()
    close(y, ry, out_tol(ry, dt) + C32 * wm * size, what + " y")
    dx, dw, db, sw, sb = R.norm_backward(d(x), d(dy), L, d(w), d(mean), d(rstd))
    if "dx" in grads:
        rows = (d(dy).abs() * wm).amax((1, 2), keepdim=True) * d(rstd).amax(1)[:, None, None] * (1 + size) ** 2
        close(grads["dx"], dx, out_tol(dx, dt) + C32 * rows, what + " dx")
    if "dw" in grads:
        close(grads["dw"], dw, C32 * sw + 1e-30, what + " dw")
    if "db" in grads:
        close(grads["db"], db, C32 * sb + 1e-30, what + " db")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", NORMS)
def test_norm_and_gradient(N, C, L, dtype):
    x, dy, w, b = norm_case(N, C, L, dtype)
    _say(f"norm N={N} C={C} L={L} {dtype}")
    y, mean, rstd = gtp.gtp_layer_norm(x, L, w, b)
    grads = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, w)
    norm_check(x, dy, w, b, L, y, mean, rstd, grads, f"{N},{C},{L}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(9, 256, 0), (9, 66, 0), (17, 32, 2), (5, 128, 6), (3, 64, 16)])
def test_norm_off_alignment_without_parameters_and_parts(N, C, L, dtype):
    x, dy, w, b = norm_case(N, C, L, dtype, 1)
    x, dy = off_by_one(x), off_by_one(dy)
    _say(f"norm off alignment N={N} C={C} L={L} {dtype}")
    y = off_by_one(torch.zeros_like(x))
    y, mean, rstd = gtp.gtp_layer_norm(x, L, y=y)
    grads = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd)
    norm_check(x, dy, None, None, L, y, mean, rstd, grads, "no w, b")
    for need in (("dx",), ("dw",), ("db",), ("dw", "db")):
        part = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, need=need)
        assert set(part) == set(need)
        for n in need:
            assert torch.equal(part[n], grads[n]), n


def test_norm_in_place_and_large_mean():
    x, dy, w, b = norm_case(64, 200, 1, F32, 2, shift=1000.0)
    ry, rm, rr = R.norm(x.double(), 1, w.double(), b.double(), 1e-5)
    y0, mean, rstd = gtp.gtp_layer_norm(x, 1, w, b)
    # the mean of values near 1000 is good to a few of its own units: 2^-21 of 1000
    close(y0, ry, (2.0 ** -21 * 1000 * rr[:, :1, None] + 1e-5) * w.abs().max().double() * torch.ones_like(ry), "large mean")
    z = x.clone()
    y1, _, _ = gtp.gtp_layer_norm(z, 1, w, b, y=z)
    assert y1.data_ptr() == z.data_ptr() and torch.equal(y1, y0)


def test_norm_constant_rows_and_empty():
    for L in (0, 2):
        x = torch.full((5, 24, (L + 1) ** 2), 2.0, device="cuda")
        b = torch.arange(24, device="cuda", dtype=F32)
        y, mean, rstd = gtp.gtp_layer_norm(x, L, None, b)
        assert torch.equal(y[..., 0], b.expand(5, 24)) and bool((mean == 2).all())
        assert torch.allclose(rstd[:, 0], torch.full((5,), 1e5 ** 0.5, device="cuda"), rtol=1e-6)
    for N, C in ((0, 8), (4, 0)):
        x = torch.zeros((N, C, 4), device="cuda")
        y, mean, rstd = gtp.gtp_layer_norm(x, 1)
        g = gtp.gtp_layer_norm_backward(x, x, 1, torch.zeros(N, device="cuda"), torch.zeros((N, 2), device="cuda"))
        assert g["dw"].shape == (2, C) and not bool(g["dw"].any()) and not bool(g["db"].any())


def test_norm_nan_stays_in_its_row():
    for L in (0, 3):
        x, dy, w, b = norm_case(40, 64, L, F32, 3)
        y0, _, _ = gtp.gtp_layer_norm(x, L, w, b)
        x[7, 3, 0] = math.nan
        y, _, _ = gtp.gtp_layer_norm(x, L, w, b)
        rest = [i for i in range(40) if i != 7]
        assert torch.equal(y[rest], y0[rest]) and bool(torch.isnan(y[7, :, 0]).all())


def test_norm_commutes_with_rotation():
    """Degree 1 turned by a rotation matrix (Y_1 ~ (y, z, x): any orthogonal matrix keeps the sums)."""
    g = gen(5)
    x = randn(g, 50, 32, 4)
    D, _ = torch.linalg.qr(randn(g, 3, 3).cpu().double())
    D = D.float().cuda()
    turn = lambda t: torch.cat([t[..., :1], t[..., 1:] @ D.T], -1).contiguous()  # noqa: E731
    w, b = 1 + 0.1 * randn(g, 2, 32), randn(g, 32)
    a, _, _ = gtp.gtp_layer_norm(turn(x), 1, w, b)
    c, _, _ = gtp.gtp_layer_norm(x, 1, w, b)
    assert float((a - turn(c)).abs().max()) < 2e-5


def difference(f, x, direction, h):
    """Central difference of the fp64 scalar f along direction, with the step that fp32 inputs really take."""
    up, dn = x + h * direction, x - h * direction
    return (f(up) - f(dn)), (up.double() - dn.double())


@pytest.mark.parametrize("N,C,L", [(6, 24, 0), (6, 24, 2), (5, 300, 1)])
def test_norm_gradient_against_differences(N, C, L):
    x, dy, w, b = norm_case(N, C, L, F32, 4)
    _, mean, rstd = gtp.gtp_layer_norm(x, L, w, b)
    g = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, w)
    f = lambda x, w, b: float((gtp.gtp_layer_norm(x, L, w, b)[0].double() * dy.double()).sum())  # noqa: E731
    gg = gen(77)
    for name, t in (("dx", x), ("dw", w), ("db", b)):
        u = randn(gg, *t.shape)
        args = {"dx": lambda z: f(z, w, b), "dw": lambda z: f(x, z, b), "db": lambda z: f(x, w, z)}[name]
        got, step = difference(args, t, u, 1e-2)
        want = float((g[name].double() * step).sum())
        # a cubic term of relative size h^2, and fp32 outputs' errors of 2^-21 |dy| each over the difference
        noise = 2.0 ** -21 * float((dy.double().abs()).sum()) + 1e-3 * float((g[name].double() * step).abs().sum())
        _say(f"  {name}: difference {got:.6f} gradient {want:.6f}")
        assert abs(got - want) <= noise


# ------------------------------------------------------------------ dropout

def rng_tensor(seed=RNG[0], offset=RNG[1]):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


DROPS = [(1, 1), (7, 1), (8, 1), (4099, 1), (100003, 1), (5, 3), (1000, 4), (257, 9), (4001, 9), (129, 49), (77, 289),
         (3, 4225), (2049, 16), (513, 25), (2, 40001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("groups,K", DROPS)
def test_dropout(groups, K, dtype):
    g = gen(groups + K)
    x, res = randn(g, groups, K, dtype=dtype), randn(g, groups, K, dtype=dtype)
    rng = rng_tensor()
    for p in (0.0, 0.1, 0.5, 0.99999):
        _say(f"dropout groups={groups} K={K} p={p} {dtype}")
        keep = torch.from_numpy(R.keep_groups(groups, p, *RNG)).cuda()[:, None]
        scale = 65536.0 / (65536 - R.threshold(p))
        want = torch.where(keep, x.double() * scale, 0.0)
        y = gtp.gtp_dropout(x, p, rng)
        assert bool((y[~keep.expand_as(y)] == 0).all())
        close(y, want, out_tol(want, dtype) * 2, "y")
        want = want + res.double()
        close(gtp.gtp_dropout(x, p, rng, res=res), want, out_tol(want, dtype) + (x.double().abs() * scale + res.double().abs()) * 2.0 ** -22, "y + res")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("groups,K", [(1000, 1), (1003, 1), (333, 9), (100, 49)])
def test_dropout_in_place_and_off_alignment(groups, K, dtype):
    g = gen(3)
    x, res, rng = randn(g, groups, K, dtype=dtype), randn(g, groups, K, dtype=dtype), rng_tensor()
    want = gtp.gtp_dropout(x, 0.3, rng, res=res)
    for a, b in ((x.clone(), res), (off_by_one(x), off_by_one(res))):
        assert torch.equal(gtp.gtp_dropout(a, 0.3, rng, res=b, y=a), want)
        c = b.clone() if b is res else off_by_one(res)
        a = x if b is res else off_by_one(x)
        assert torch.equal(gtp.gtp_dropout(a, 0.3, rng, res=c, y=c), want)


def test_dropout_nan_dropped_and_rate():
    x = torch.full((1 << 20, 1), math.nan, device="cuda")
    y = gtp.gtp_dropout(x, 0.25, rng_tensor())
    rate = float((y == 0).double().mean())
    assert abs(rate - 0.25) < 5 * math.sqrt(0.25 * 0.75 / (1 << 20)), rate  # five standard deviations
    other = gtp.gtp_dropout(x, 0.25, rng_tensor(offset=6))
    both = float(((y == 0) & (other == 0)).double().mean())
    assert abs(both - 0.0625) < 5 * math.sqrt(0.0625 / (1 << 20))


def test_dropout_past_32_bits():
    n = (1 << 32) + 4097
    x = torch.ones((n, 1), dtype=BF16, device="cuda")
    y = gtp.gtp_dropout(x, 0.5, rng_tensor(), y=x)
    for first in ((1 << 32) - 1000, n - 999):
        keep = R.keep_groups(999, 0.5, *RNG, first=first)
        assert np.array_equal(y[first:first + 999, 0].float().cpu().numpy(), keep * 2.0)
    del x, y
    n = 87_700_000  # groups of 49: elements past 32 bits
    x = torch.ones((n, 49), dtype=BF16, device="cuda")
    y = gtp.gtp_dropout(x, 0.5, rng_tensor(), y=x)
    keep = R.keep_groups(2000, 0.5, *RNG, first=n - 2000)
    assert np.array_equal(y[n - 2000:].float().cpu().numpy(), np.repeat(keep[:, None] * 2.0, 49, 1))


# ------------------------------------------------------------------ attention

def offsets(lengths):
    return torch.tensor([0] + list(lengths), dtype=torch.int64).cumsum(0).cuda()


class Case:
    def __init__(self, dtype, ql, kl, H, Hk, d, masked=0.0, p=0.0, seed=0, scale=None, size=1.0):
        g = gen(17 * sum(ql) + sum(kl) + 100 * H + d + seed)
        self.dtype, self.ql, self.kl, self.p = dtype, ql, kl, p
        self.q, self.k, self.v = (randn(g, sum(n), h, d, dtype=dtype, scale=size) for n, h in ((ql, H), (kl, Hk), (kl, Hk)))
        self.do = randn(g, sum(ql), H, d, dtype=dtype)
        self.scale = 1 / math.sqrt(d) if scale is None else scale
        self.mask = (torch.rand(sum(kl), generator=g, device="cuda") >= masked).to(torch.uint8) if masked else None
        self.args = dict(q_off=offsets(ql), k_off=offsets(kl), max_q=max(ql), max_k=max(kl), key_mask=self.mask, p=p,
                         rng=rng_tensor() if p else None, scale=self.scale)

    def ref(self, grad=None):
        qs, ks = (R.segments(offsets(n).tolist(), len(n), 0, 0) for n in (self.ql, self.kl))
        t = [x.double() for x in (self.q, self.k, self.v)]
        if self.mask is not None:  # whatever absent rows hold
            t[1], t[2] = (torch.where(self.mask.bool()[:, None, None], x, 0.0) for x in t[1:])
        return R.attention(*t, self.scale, qs, ks, self.mask, self.p, RNG, max(self.ql), max(self.kl), grad)

    def forward(self, **more):
        return gtp.gtp_attention(self.q, self.k, self.v, **{**self.args, **more})

    def backward(self, o, lse, **more):
        return gtp.gtp_attention_backward(self.q, self.k, self.v, o, self.do, lse, **{**self.args, **more})

    def check_forward(self, o, lse):
        ro, rl, size = self.ref()
        half = 2.0 ** -8 if self.dtype == BF16 else 0.0
        # a score's fp32 error moves P by as much: u times the score's terms
        smax = 1 + (self.q.double().norm(dim=-1).amax() * self.k_norm() * abs(self.scale))
        close(o, ro, out_tol(ro, self.dtype) + (half + C32 * smax) * size + 1e-30, "o")
        none = torch.isinf(rl)
        assert torch.equal(torch.isinf(lse), none) and bool((lse[none] < 0).all())
        close(lse[~none], rl[~none], C32 * smax * torch.ones_like(rl[~none]), "lse")

    def k_norm(self):
        k = self.k if self.mask is None else self.k[self.mask.bool()]
        return k.double().norm(dim=-1).amax() if k.numel() else torch.zeros((), dtype=torch.float64, device="cuda")

    def check_backward(self, o, lse, grads, names=("dq", "dk", "dv")):
        ref = dict(zip(("dq", "dk", "dv"), self.ref((self.do.double(), o.double(), lse.double()))))
        half = 2.0 ** -8 if self.dtype == BF16 else 0.0
        smax = 1 + (self.q.double().norm(dim=-1).amax() * self.k_norm() * abs(self.scale))
        for n in names:
            want, size, e32 = ref[n]
            close(grads[n], want, out_tol(want, self.dtype) + half * size + C32 * smax * e32 + 1e-30, n)


# (query lengths, key lengths, H, Hk, d, share of absent keys, p)
ATTN = [
    ([1], [1], 1, 1, 1, 0, 0), ([1], [1], 2, 1, 9, 0, 0.3), ([1, 1, 1], [5, 1, 33], 3, 3, 16, 0, 0),
    ([27] * 4, [27] * 4, 8, 8, 32, 0, 0), ([5, 49, 32, 33, 1, 31], [5, 49, 32, 33, 1, 31], 2, 2, 72, 0, 0.1),
    ([0, 3, 0, 64], [4, 0, 0, 65], 2, 2, 64, 0, 0), ([40, 7], [40, 90], 6, 2, 75, 0.3, 0),
    ([129, 128, 127], [63, 64, 65], 2, 1, 100, 0, 0.2), ([300], [257], 1, 1, 128, 0, 0),
    ([1], [3001], 4, 1, 64, 0.1, 0), ([2, 2], [1000, 1999], 8, 2, 128, 0, 0.1), ([33], [1], 5, 1, 3, 0, 0),
    ([200], [131], 2, 2, 144, 0, 0), ([70], [70], 2, 1, 200, 0.2, 0.1), ([65, 20], [65, 20], 1, 1, 256, 0, 0),
    ([511], [513], 1, 1, 48, 0.5, 0), ([1025], [1023], 2, 2, 40, 0, 0), ([31], [700], 12, 4, 24, 0.9, 0.5),
    ([2000], [3], 3, 1, 64, 0, 0), ([1500], [40], 4, 2, 96, 0.2, 0.1), ([3], [4], 1, 1, 217, 0, 0),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ql,kl,H,Hk,d,masked,p", ATTN)
def test_attention_and_gradient(ql, kl, H, Hk, d, masked, p, dtype):
    _say(f"attention q={ql} k={kl} H={H}/{Hk} d={d} masked={masked} p={p} {dtype}")
    c = Case(dtype, ql, kl, H, Hk, d, masked, p)
    o, lse = c.forward()
    torch.cuda.synchronize()
    c.check_forward(o, lse)
    g = c.backward(o, lse)
    torch.cuda.synchronize()
    c.check_backward(o, lse, g)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_equal_segments_without_offsets(dtype):
    c = Case(dtype, [50] * 3, [70] * 3, 4, 2, 64)
    o, lse = c.forward()
    for more in (dict(q_off=None, k_off=None), dict(q_off=None), dict(k_off=None)):
        o2, lse2 = c.forward(**more)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    g, g2 = c.backward(o, lse), c.backward(o, lse, q_off=None, k_off=None)
    assert all(torch.equal(g[n], g2[n]) for n in g)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 72, 75])
def test_attention_on_slices_of_a_packed_tensor(d, dtype):
    """q, k, v as slices of one [T, 3, H, d] tensor, the gradients written into slices of another; and, one element
    off 16-byte alignment."""
    c = Case(dtype, [33, 64, 90], [33, 64, 90], 4, 4, d)
    o, lse = c.forward()
    g = c.backward(o, lse)
    for shift in (0, 1):
        T = sum(c.ql)
        buf = torch.zeros(T * 3 * 4 * d + shift, dtype=dtype, device="cuda")[shift:].view(T, 3, 4, d)
        buf[:, 0], buf[:, 1], buf[:, 2] = c.q, c.k, c.v
        out = torch.full_like(buf, 7.0)
        q, k, v = buf.unbind(1)
        o2, lse2 = gtp.gtp_attention(q, k, v, **c.args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        gtp.gtp_attention_backward(q, k, v, o, c.do, lse, **c.args, dq=out[:, 0], dk=out[:, 1], dv=out[:, 2])
        assert all(torch.equal(out[:, i], g[n]) for i, n in enumerate(("dq", "dk", "dv")))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_expanded_inputs(dtype):
    """One key and value row for all heads and one query row for all rows, by strides of zero."""
    c = Case(dtype, [40], [50], 4, 4, 64)
    c.k, c.v = c.k[:, :1].expand(-1, 4, -1), c.v[:, :1].expand(-1, 4, -1)
    c.q = c.q[:1].expand(40, -1, -1)
    o, lse = c.forward()
    c.check_forward(o, lse)
    c.check_backward(o, lse, c.backward(o, lse))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_attention_absent_keys_hold_anything(dtype, p):
    c = Case(dtype, [40, 50, 20], [130, 60, 70], 4, 2, 64, masked=0.4, p=p)
    c.mask[130:190] = 0  # no key of the second segment: its rows are empty
    o, lse = c.forward()
    assert bool((o[40:90] == 0).all()) and bool((lse[40:90] == -math.inf).all())
    g = c.backward(o, lse)
    c.check_forward(o, lse)
    c.check_backward(o, lse, g)
    assert bool((g["dq"][40:90] == 0).all()) and bool((g["dk"][~c.mask.bool()] == 0).all())
    for junk in (math.nan, math.inf, -math.inf, torch.finfo(dtype).min, torch.finfo(dtype).max):
        for t in (c.k, c.v):
            t[~c.mask.bool()] = junk
        o2, lse2 = c.forward()
        g2 = c.backward(o, lse)
        assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(g[n], g2[n]) for n in g), junk


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_large_scores(dtype):
    """Scores up to some hundreds: the running maximum has to move, and exponentials far below it vanish."""
    c = Case(dtype, [100], [300], 2, 2, 64, scale=8.0)
    o, lse = c.forward()
    assert bool(torch.isfinite(o).all())
    c.check_forward(o, lse)
    c.check_backward(o, lse, c.backward(o, lse))
    c = Case(dtype, [100], [300], 2, 2, 64, scale=-1.5)
    o, lse = c.forward()
    c.check_forward(o, lse)
    c.check_backward(o, lse, c.backward(o, lse))


def test_attention_nan_stays_in_its_row_and_segment():
    c = Case(F32, [40, 40], [40, 40], 2, 2, 64)
    o, lse = c.forward()
    c.q[3, 1, 5] = math.nan
    o2, _ = c.forward()
    assert bool(torch.isnan(o2[3, 1]).all())
    o2[3, 1] = o[3, 1]
    assert torch.equal(o, o2)
    c.k[50, 0, 0] = math.nan
    o2, _ = c.forward()
    assert torch.equal(o[:3], o2[:3]) and bool(torch.isnan(o2[40:, 0]).all()) and torch.equal(o2[40:, 1], o[40:, 1])


def test_attention_infinite_scores():
    """A score of -infinity counts nothing; rows of nothing else are empty, as without keys."""
    c = Case(F32, [8], [8], 1, 1, 4)
    c.q.fill_(1.0)
    c.k.fill_(0.0)
    c.k[2] = -1e38
    c.k[3, 0, 0] = -math.inf
    o, lse = c.forward()
    keep = [0, 1, 4, 5, 6, 7]
    assert torch.allclose(o, c.v[keep].mean(0).expand_as(o), atol=1e-6)
    assert torch.allclose(lse, torch.full_like(lse, math.log(6)), atol=1e-6)
    c.k[:, 0, 0] = -math.inf
    c.k[:, 0, 1:] = 0
    o, lse = c.forward()
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    g = c.backward(o, lse)
    assert bool((g["dv"] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_far_into_a_long_cache(dtype):
    """Keys whose offsets pass 2^32 bytes and 2^31 elements."""
    d, n = 128, 17_000_000
    k = torch.zeros((n, 1, d), dtype=dtype, device="cuda")
    v = torch.zeros((n, 1, d), dtype=dtype, device="cuda")
    c = Case(dtype, [70], [300], 2, 1, d)
    k[-300:], v[-300:] = c.k, c.v
    off = torch.tensor([n - 300, n], dtype=torch.int64, device="cuda")
    args = {**c.args, "k_off": off}
    o, lse = gtp.gtp_attention(c.q, k, v, **args)
    want, wl = c.forward()
    assert torch.equal(o, want) and torch.equal(lse, wl)
    dk, dv = k.clone(), v.clone()
    gtp.gtp_attention_backward(c.q, k, v, o, c.do, lse, **args, dk=dk, dv=dv)
    g = c.backward(o, lse)
    assert torch.equal(dk[-300:], g["dk"]) and torch.equal(dv[-300:], g["dv"])
    assert not bool(dk[:1000].any())  # rows of no segment are not written


def test_attention_offsets_outside_the_tensor_are_cut():
    c = Case(F32, [20, 30], [20, 30], 2, 2, 32)
    o, lse = c.forward()
    off = torch.tensor([-5, 20, 1 << 40], dtype=torch.int64, device="cuda")
    o2, lse2 = c.forward(q_off=off, k_off=off)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_parts_of_the_gradient(dtype):
    c = Case(dtype, [80, 33], [80, 33], 4, 2, 40, masked=0.1, p=0.1)
    o, lse = c.forward()
    g = c.backward(o, lse)
    assert torch.equal(c.backward(o, lse, need=("dq",))["dq"], g["dq"])
    part = c.backward(o, lse, need=("dk", "dv"))
    assert set(part) == {"dk", "dv"} and torch.equal(part["dk"], g["dk"]) and torch.equal(part["dv"], g["dv"])
    assert set(c.backward(o, lse, need=("dv",))) == {"dv"}


@pytest.mark.parametrize("masked,p", [(0.0, 0.0), (0.2, 0.25)])
def test_attention_gradient_against_differences(masked, p):
    c = Case(F32, [30, 9], [30, 21], 4, 2, 24, masked=masked, p=p)
    o, lse = c.forward()
    g = c.backward(o, lse)
    f = lambda q, k, v: float((gtp.gtp_attention(q, k, v, **c.args)[0].double() * c.do.double()).sum())  # noqa: E731
    gg = gen(7)
    for name, t in (("dq", c.q), ("dk", c.k), ("dv", c.v)):
        u = randn(gg, *t.shape)
        args = {"dq": lambda z: f(z, c.k, c.v), "dk": lambda z: f(c.q, z, c.v), "dv": lambda z: f(c.q, c.k, z)}[name]
        got, step = difference(args, t, u, 1e-2)
        want = float((g[name].double() * step).sum())
        # a cubic term of relative size h^2, and outputs' errors of 2^-20 |do| each
        noise = 2.0 ** -20 * float(c.do.double().abs().sum()) + 1e-3 * float((g[name].double() * step).abs().sum())
        _say(f"  {name}: difference {got:.6f} gradient {want:.6f}")
        assert abs(got - want) <= noise


# ------------------------------------------------------------------ streams, graphs, equality, poisoned LDS

def everything(dtype, seed=0):
    """One call of each, the shapes that take different kernels: a list of outputs."""
    out = []
    for N, C, L in ((300, 256, 0), (40, 64, 2), (20, 128, 6), (5, 64, 16), (6, 9000, 0), (2, 2, 20)):
        x, dy, w, b = norm_case(N, C, L, dtype, 40 + seed)
        y, mean, rstd = gtp.gtp_layer_norm(x, L, w, b)
        out += [y, mean, rstd, *gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, w).values()]
    for groups, K in ((5000, 1), (600, 9)):
        x = randn(gen(seed), groups, K, dtype=dtype)
        out.append(gtp.gtp_dropout(x, 0.2, rng_tensor(), res=x))
    for ql, kl, H, Hk, d, p in (([30, 49], [30, 49], 4, 4, 72, 0.1), ([300], [300], 4, 2, 64, 0.0),
                                ([2], [4000], 4, 2, 64, 0.0), ([3000], [9], 2, 1, 128, 0.1), ([90], [80], 2, 2, 160, 0.0)):
        c = Case(dtype, ql, kl, H, Hk, d, 0.1, p, seed=seed)
        o, lse = c.forward()
        out += [o, lse, *c.backward(o, lse).values()]
    return out


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_same_bits_again_and_poisoned_lds(dtype):
    a, b = everything(dtype), everything(dtype)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with gtp.use_library(POISON_LIB):
        c = everything(dtype)
        torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, c))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_on_another_stream(dtype):
    """Every call on a stream that is not the current one, given as an argument."""
    s = torch.cuda.Stream()
    x, dy, w, b = norm_case(200, 64, 2, dtype)
    c = Case(dtype, [2], [9000], 4, 2, 64, 0.1, 0.1)
    y, mean, rstd = gtp.gtp_layer_norm(x, 2, w, b)
    g = gtp.gtp_layer_norm_backward(x, dy, 2, mean, rstd, w)
    o, lse = c.forward()
    h = c.backward(o, lse)
    z = gtp.gtp_dropout(x, 0.1, rng_tensor())
    torch.cuda.synchronize()
    for _ in range(5):
        y2, m2, r2 = gtp.gtp_layer_norm(x, 2, w, b, stream=s)
        g2 = gtp.gtp_layer_norm_backward(x, dy, 2, m2, r2, w, stream=s)
        o2, l2 = c.forward(stream=s)
        h2 = c.backward(o2, l2, stream=s)
        z2 = gtp.gtp_dropout(x, 0.1, c.args["rng"], stream=s)
        junk = torch.full((1 << 20,), 3.0, device="cuda")  # the current stream's allocator goes on meanwhile
        del junk
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(o, o2) and torch.equal(lse, l2) and torch.equal(z, z2)
    assert all(torch.equal(g[n], g2[n]) for n in g) and all(torch.equal(h[n], h2[n]) for n in h)


def test_captured_in_a_graph():
    """norm -> attention -> dropout + residual, replayed with changed inputs and draws, each replay against the same
    calls outside the graph."""
    c = Case(F32, [40, 25], [40, 25], 4, 4, 36, p=0.1)
    T = 65
    x, w, b, rng = randn(gen(1), T, 16, 9), torch.ones(3, 16, device="cuda"), torch.zeros(16, device="cuda"), rng_tensor()
    args = {**c.args, "rng": rng}

    def block():
        y, mean, rstd = gtp.gtp_layer_norm(x, 2, w, b)
        h = y.view(T, 4, 36)
        o, lse = gtp.gtp_attention(h, h, h, **args)
        z = gtp.gtp_dropout(o.view(T, 16, 9), 0.2, rng, res=x)
        gr = gtp.gtp_attention_backward(h, h, h, o, c.do, lse, **args)
        gn = gtp.gtp_layer_norm_backward(x, gr["dq"].view(T, 16, 9), 2, mean, rstd, w)
        return [z, gr["dq"], gr["dk"], gr["dv"], *gn.values()]

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block()
    for i in range(4):
        x.copy_(randn(gen(50 + i), T, 16, 9))
        rng[1] = i
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = block()
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(got, want)), i
