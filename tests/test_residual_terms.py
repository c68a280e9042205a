"""The residual step and its gradient, each element against a bound of the terms that enter it (tests/residual_bounds.py), on
every way that rows take: teams of lanes, a workgroup, rows too long for the registers, the general one.

On the CPU: the bounds' values are those of the plain forms, arithmetic in 32 bits is within the bounds, and a gradient with
any one of its terms left out is not, at every shape.  On the GPU (-m gpu): the kernels against the bounds; in place in
bf16; gradients of long rows and of the general way against differences.

An output has its own rounding besides: bf16 2^-8 of the value, fp32 2^-23 for its last operations.
"""
import pytest

torch = pytest.importorskip("torch")

import residual_bounds as B  # noqa: E402
import residual_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
NAMES = ("gate", "scale", "w_post", "b_post", "w_pre", "b_pre")
STATS = ("mean_post", "rstd_post", "mean_pre", "rstd_pre")
# (rows, channels, degree, what b_post is multiplied by: one term of a channel's K in dgate, it would not show among
# thousands)
TEAMS = [(5, 7, 0, 1), (33, 256, 0, 1), (700, 17, 0, 1), (65, 500, 0, 1), (7, 5, 1, 1), (1000, 16, 1, 1), (33, 16, 2, 1), (27, 128, 2, 1)]
GROUPS = [(3, 1100, 0, 1), (300, 256, 2, 1), (40, 33, 4, 1), (9, 128, 6, 1), (130, 30, 6, 1), (4, 64, 8, 1), (3, 120, 8, 1), (3, 65, 12, 1)]
LONG = [(7, 300, 8, 1), (1, 600, 8, 1), (3, 1000, 3, 1), (3, 64, 16, 1), (2, 24, 31, 10)]
GENERAL = [(2, 5000, 0, 1), (3, 9001, 0, 1), (130, 5003, 0, 1), (2, 6, 32, 10), (2, 2, 64, 40)]
SHAPES = TEAMS + GROUPS + LONG + GENERAL
# the gradient that shows a term where nothing hides it
SHOWN = {"along2": "dx", "mean2": "dx", "r2": "dx", "w2": "dx", "dr": "dx", "along1": "da", "mean1": "da", "r1": "da", "w1": "da",
         "sig": "da", "shift": "dgate", "scale": "dgate", "slope": "dgate"}
gpu = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


class Case:
    """Degrees of unequal size, an offset at degree 0; made on the CPU."""

    def __init__(self, N, C, L, more, dtype, post=True, gated=True, device="cpu", seed=0):
        g = torch.Generator().manual_seed(9000 + seed + N + 7 * C + 13 * L)
        n = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        K = (L + 1) ** 2
        deg = torch.tensor([l for l in range(L + 1) for _ in range(2 * l + 1)])
        x, a = n(N, C, K) * (1.7 - 0.2 * (deg % 5)), n(N, C, K) * (0.6 + 0.3 * (deg % 4))
        x[..., 0] += 0.3
        a[..., 0] -= 0.2
        self.L, self.post, self.dtype = L, post, dtype
        self.x, self.a, self.dh, self.dr = (t.to(dtype).to(device) for t in (x, a, n(N, C, K), n(N, C, K)))
        w = {"gate": n(N, C).to(dtype) if gated else None, "scale": 0.5 + 0.1 * n(L + 1, C),
             "w_post": 1 + 0.2 * n(L + 1, C) if post else None, "b_post": 0.2 * more * n(C) if post else None,
             "w_pre": 1 + 0.2 * n(L + 1, C), "b_pre": 0.2 * n(C)}
        self.w = {k: None if t is None else t.to(device) for k, t in w.items()}

    def args(self, dtype=torch.float64):
        return [None if self.w[n] is None else self.w[n].to(dtype) for n in NAMES]

    def step(self, dtype=torch.float64):
        return B.forward(self.x.to(dtype), self.a.to(dtype), self.L, *self.args(dtype), self.post)

    def gradient(self, r, stats, dtype=torch.float64, without=(), dr=True):
        stats = [None if t is None else t.to(dtype) for t in stats]
        g, e = B.backward(r.to(dtype), self.a.to(dtype), self.L, stats, self.dh.to(dtype), self.dr.to(dtype) if dr else None,
                          *self.args(dtype), self.post, without)
        gone = (() if self.w["gate"] is not None else ("dgate",)) + (() if self.post else ("dw_post", "db_post"))
        return {n: t for n, t in g.items() if n not in gone}, e

    def own(self, n, want):
        """An output's own rounding."""
        half = 2.0 ** -8 if self.dtype == BF16 and n in ("r", "h", "dx", "da", "dgate") else 2.0 ** -23
        return want.abs() * half

    def forward(self, **more):
        return gtp.gtp_residual_norm(self.x, self.a, self.L, **{**self.w, **more}, post=self.post)

    def backward(self, r, stats, **more):
        return gtp.gtp_residual_norm_backward(r, self.a, self.L, stats, self.dh, **{"dr": self.dr, **self.w, **more},
                                              post=self.post)

    def check_step(self, r, h, stats):
        want, err = self.step()
        got = {"r": r, "h": h, **{n: t for n, t in zip(STATS, stats) if t is not None}}
        assert set(got) == set(want)
        self.check(got, want, err)

    def check_gradient(self, r, stats, grads, dr=True):
        want, err = self.gradient(r, stats, dr=dr)
        assert set(grads) == set(want)
        self.check(grads, want, err)

    def check(self, got, want, err):
        for n in want:
            off = (got[n].double() - want[n]).abs()
            tol = err[n] + self.own(n, want[n]) + 1e-30
            _say(f"  {n}: worst {float((off / tol).max()):.3f} of the bound")
            assert got[n].shape == want[n].shape and bool((off <= tol).all()), n


def given(c):
    """r and the statistics that a gradient reads, rounded to what they are stored in."""
    v, _ = c.step()
    return v["r"].to(c.dtype), [v[n].float() if n in v else None for n in STATS]


# ------------------------------------------------------------------------------ the bounds

@pytest.mark.parametrize("post,gated", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("N,C,L,more", [(5, 7, 0, 1), (33, 16, 2, 1), (2, 3, 5, 1)])
def test_values_are_the_plain_forms(N, C, L, more, post, gated):
    c = Case(N, C, L, more, F32, post, gated)
    v, _ = c.step()
    r, h, stats = R.forward(c.x.double(), c.a.double(), L, *c.args(), post)
    for n, t in zip(("r", "h") + STATS, (r, h, *stats)):
        assert (t is None) == (n not in v) and (t is None or torch.allclose(t, v[n], rtol=1e-12, atol=1e-13)), n
    for dr in (True, False):
        g, _ = c.gradient(r, stats, dr=dr)
        want, _, _ = R.backward(r, c.a.double(), L, stats, c.dh.double(), c.dr.double() if dr else None, *c.args(), post)
        for n, t in g.items():
            assert torch.allclose(t, want[n], rtol=1e-10, atol=1e-11), n


@pytest.mark.parametrize("N,C,L,more", SHAPES)
def test_arithmetic_in_32_bits_is_within(N, C, L, more):
    for post, gated in ((True, True), (False, False)):
        c = Case(N, C, L, more, F32, post, gated)
        v, _ = c.step(F32)
        want, err = c.step()
        c.check(v, want, err)
        r, stats = given(c)
        g, _ = c.gradient(r, stats, F32)
        c.check_gradient(r, stats, g)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L,more", SHAPES)
def test_each_term_is_seen(N, C, L, more, dtype):
    """A gradient without a term leaves the bound, and few values are smaller than their bound: zeros would not pass."""
    c = Case(N, C, L, more, dtype)
    r, stats = given(c)
    want, err = c.gradient(r, stats)
    tol = {n: err[n] + c.own(n, want[n]) for n in want}
    for term, n in SHOWN.items():
        got, _ = c.gradient(r, stats, without=(term,))
        assert bool(((got[n] - want[n]).abs() > tol[n]).any()), term
    v, e = c.step()
    for n, t, b in [(n, want[n], tol[n]) for n in want] + [("h", v["h"], e["h"] + c.own("h", v["h"]))]:
        assert float((t.abs() < b).double().mean()) < 0.06, n


# ------------------------------------------------------------------------------ the kernels

@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L,more", SHAPES)
def test_step_and_gradient(N, C, L, more, dtype):
    for post, gated in ((True, True), (False, True), (True, False), (False, False)):
        _say(f"residual by terms N={N} C={C} L={L} {dtype} post={post} gated={gated}")
        c = Case(N, C, L, more, dtype, post, gated, "cuda")
        r, h, stats = c.forward()
        c.check_step(r, h, stats)
        c.check_gradient(r, stats, c.backward(r, stats))
        c.check_gradient(r, stats, c.backward(r, stats, dr=None), dr=False)


@gpu
@pytest.mark.parametrize("N,C,L", [(50, 128, 0), (9, 9001, 0), (50, 16, 1), (50, 48, 2), (6, 128, 6), (3, 300, 8), (2, 6, 32)])
def test_in_place_in_bf16(N, C, L):
    c = Case(N, C, L, 1, BF16, device="cuda", seed=2)
    r, h, stats = c.forward()
    z = c.x.clone()
    r2, h2, stats2 = gtp.gtp_residual_norm(z, c.a, L, **c.w, r=z)
    assert r2.data_ptr() == z.data_ptr() and torch.equal(r2, r) and torch.equal(h2, h)
    assert all(torch.equal(s, t) for s, t in zip(stats, stats2))
    grads = c.backward(r, stats)
    d = c.dr.clone()
    again = c.backward(r, stats, dr=d, dx=d)
    assert again["dx"].data_ptr() == d.data_ptr()
    for n in grads:
        assert torch.equal(again[n], grads[n]), n


@gpu
@pytest.mark.parametrize("N,C,L,post", [(3, 300, 8, True), (3, 300, 8, False), (2, 24, 31, True), (2, 6, 32, True), (2, 4099, 0, True)])
def test_gradient_against_differences(N, C, L, post):
    """Along one direction a tensor, up the gradient (along any other its terms cancel); f = <dh, h> + <dr, r> of the kernels'
    results in 32 bits."""
    c = Case(N, C, L, 1, F32, post=post, device="cuda", seed=7)
    r, _, stats = c.forward()
    grads = c.backward(r, stats)
    base = {"dx": c.x, "da": c.a, **{"d" + n: t for n, t in c.w.items() if t is not None}}

    def f(name, t):
        args = {**c.w}
        x, a = (t if name == "dx" else c.x), (t if name == "da" else c.a)
        if name not in ("dx", "da"):
            args[name[1:]] = t
        rr, hh, _ = gtp.gtp_residual_norm(x, a, L, **args, post=post)
        return float((hh.double() * c.dh.double()).sum() + (rr.double() * c.dr.double()).sum())

    g = torch.Generator().manual_seed(78)
    for name, t in base.items():
        u = torch.randn(t.shape, generator=g).abs().cuda() * torch.sign(grads[name].float())
        up, dn = t + 1e-2 * u, t - 1e-2 * u
        got, step = f(name, up) - f(name, dn), up.double() - dn.double()
        want = float((grads[name].double() * step).sum())
        # a cubic term of relative size h^2 over the smallest degree's size, 0.6, squared; fp32 outputs' errors of 2^-21 of the
        # cotangents' sizes over the difference
        noise = 2.0 ** -21 * float((c.dh.double().abs() + c.dr.double().abs()).sum()) * 3 + \
            1e-3 * float((grads[name].double() * step).abs().sum())
        _say(f"  {name}: difference {got:.6f} gradient {want:.6f} noise {noise:.6f}")
        assert abs(got - want) <= noise, name
