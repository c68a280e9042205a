"""The residual step and its gradient on the GPU against plain 64-bit forms (tests/residual_ref.py): types, rows from
one to many, degrees 0 to 64, odd channel counts, alignment, parts left out, in place, streams, graphs, NaN and
infinities, run-to-run equality, the poisoned-LDS build.

Tolerances.  u = 2^-24 is half a unit in the last place of fp32; rounding to bf16 moves a value by at most 2^-8 of
itself, and a bf16 output carries that (fp32: 2^-23 for its last operations).  A lane adds up at most some 300 terms in
sequence (rows of 70001 scalars on 256 threads), then a tree: a sum's error is below 2^-16 = 256 u of the sum of its
terms' magnitudes, and so is that of a result made of a few such sums, counted against the magnitudes that
enter it.  These are bounded by row: |xh| <= X = (max |v| + |mean|) max rstd, |D| <= MD = max |dr| + rstd max |g| (2 + X^2).
The weights' gradients sum over the rows what carries an error of D's (16 u of MD: its means have errors of 256 u of
mean |g xh| <= rms g, since xh has mean square 1 at most, and a row's largest value is several times its rms).
"""
import math
import os

import pytest

torch = pytest.importorskip("torch")

import residual_ref as R  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402
from test_layers import close, gen, off_by_one, out_tol, randn  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
C32, ROW = 2.0 ** -16, 2.0 ** -20
POISON_LIB = os.path.join(os.path.dirname(gtp.__file__), "libgtp_poison.so")
NAMES = ("gate", "scale", "w_post", "b_post", "w_pre", "b_pre")


def _say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


class Case:
    def __init__(self, N, C, L, dtype, post=True, gated=True, weights=True, seed=0, shift=0.3, away=False):
        g = gen(4000 + seed + N + 7 * C + 13 * L)
        place = off_by_one if away else lambda t: t
        K = (L + 1) ** 2
        self.L, self.dtype, self.post = L, dtype, post
        self.x, self.a, self.dh, self.dr = (randn(g, N, C, K) for _ in range(4))
        self.x[..., 0] += shift
        self.a[..., 0] -= shift
        self.x, self.a, self.dh, self.dr = (place(t.to(dtype)) for t in (self.x, self.a, self.dh, self.dr))
        w = {"gate": randn(g, N, C, dtype=dtype) if gated else None}
        w.update({n: 1 + 0.2 * randn(g, L + 1, C) if weights else None for n in ("scale", "w_post", "w_pre")})
        w.update({n: 0.2 * randn(g, C) if weights else None for n in ("b_post", "b_pre")})
        if w["scale"] is not None:
            w["scale"] *= 0.5
        if not post:
            w["w_post"] = w["b_post"] = None
        if away and w["gate"] is not None:
            w["gate"] = off_by_one(w["gate"])
        self.w = w

    def wide(self):
        return [None if self.w[n] is None else self.w[n].double() for n in NAMES]

    def forward(self, **more):
        return gtp.gtp_residual_norm(self.x, self.a, self.L, **{**self.w, **more}, post=self.post)

    def backward(self, r, stats, **more):
        return gtp.gtp_residual_norm_backward(r, self.a, self.L, stats, self.dh, **{"dr": self.dr, **self.w, **more},
                                              post=self.post)

    def check_forward(self, r, h, stats):
        x, a = self.x.double(), self.a.double()
        rr, rh, rs = R.forward(x, a, self.L, *self.wide(), self.post)
        ab = lambda t, i: t.abs().amax(i)  # noqa: E731
        _, s, w1, b1, w2, b2 = (1.0 if t is None else t.abs().max() for t in self.wide())
        M1 = ab(a, (1, 2)) + ab(a[..., 0], 1)
        if self.post:
            close(stats[0], rs[0], C32 * a[..., 0].abs().mean(1) + 1e-30, "mean_post")
            M1 = M1 * rs[1].amax(1) + 1
            close(stats[1], rs[1], C32 * rs[1] * M1[:, None], "rstd_post")
            M1 = w1 * M1 + (b1 if self.w["b_post"] is not None else 0.0)
        Mr = ab(x, (1, 2)) + s * M1
        close(r, rr, out_tol(rr, self.dtype) + C32 * Mr[:, None, None], "r")
        M2 = 2 * Mr * rs[3].amax(1) + 1
        close(stats[2], rs[2], C32 * Mr + 1e-30, "mean_pre")
        close(stats[3], rs[3], C32 * rs[3] * M2[:, None], "rstd_pre")
        # |xh2| <= M2; r's error and the size's each move it by C32 M2 of its magnitude
        close(h, rh, out_tol(rh, self.dtype) + C32 * (w2 * M2 * M2 + (b2 if self.w["b_pre"] is not None else 0.0))[:, None, None],
              "h")

    def check_backward(self, r, stats, grads, dr=True):
        wide = [None if t is None else t.double() for t in stats]
        want, rows, size = R.backward(r.double(), self.a.double(), self.L, wide, self.dh.double(),
                                      self.dr.double() if dr else None, *self.wide(), self.post)
        for n, got in grads.items():
            assert got.shape == want[n].shape, n
            if n in ("dx", "da"):
                tol = out_tol(want[n], self.dtype) + C32 * rows[n][:, None, None]
            elif n == "dgate":
                tol = out_tol(want[n], self.dtype) + C32 * rows[n][:, None]
            else:
                per = {"dscale": rows["sum"], "dw_post": rows["sum"], "db_post": rows["u"]}.get(n, 0.0)
                tol = C32 * size[n] + ROW * (2 * self.L + 1) * per + 1e-30
            close(got, want[n], tol, n)


SHAPES = [(1, 1, 0), (3, 1, 0), (5, 7, 0), (33, 256, 0), (3, 300, 0), (2, 5000, 0), (1, 70001, 0), (700, 17, 0), (4097, 20, 0),
          (65, 500, 0), (1, 1, 1), (7, 5, 1), (1000, 16, 1), (33, 16, 2), (27, 128, 2), (257, 64, 2), (300, 256, 2), (3, 1000, 3),
          (40, 33, 4), (9, 128, 6), (130, 30, 6), (4, 64, 8), (7, 300, 8), (3, 65, 12), (3, 64, 16), (2, 3, 20), (2, 2, 64),
          (1, 600, 8), (130, 5003, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", SHAPES)
def test_step_and_gradient(N, C, L, dtype):
    for post, gated in ((True, True), (False, True), (True, False), (False, False)):
        _say(f"residual N={N} C={C} L={L} {dtype} post={post} gated={gated}")
        c = Case(N, C, L, dtype, post, gated)
        r, h, stats = c.forward()
        c.check_forward(r, h, stats)
        c.check_backward(r, stats, c.backward(r, stats))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(9, 256, 0), (9, 66, 0), (17, 32, 2), (5, 128, 6), (3, 64, 16)])
def test_off_alignment_without_weights_and_parts(N, C, L, dtype):
    c = Case(N, C, L, dtype, weights=False, seed=1, away=True)
    r, h = off_by_one(torch.zeros_like(c.x)), off_by_one(torch.zeros_like(c.x))
    r, h, stats = c.forward(r=r, h=h)
    c.check_forward(r, h, stats)
    dx = off_by_one(torch.zeros_like(r))
    grads = c.backward(r, stats, dx=dx)
    assert grads["dx"].data_ptr() == dx.data_ptr()
    c.check_backward(r, stats, grads)
    for need in (("dx",), ("da",), ("dgate",), ("dscale",), ("dw_post", "db_pre"), ("dx", "dw_pre"), ("da", "db_post"), ()):
        part = c.backward(r, stats, need=need)
        assert set(part) == set(need)
        for n in need:
            assert torch.equal(part[n], grads[n]), (need, n)


@pytest.mark.parametrize("N,C,L", [(50, 128, 0), (50, 48, 2), (6, 128, 6), (3, 300, 8)])
def test_in_place_and_no_dr(N, C, L):
    c = Case(N, C, L, F32, seed=2)
    r, h, stats = c.forward()
    z = c.x.clone()
    r2, h2, _ = gtp.gtp_residual_norm(z, c.a, L, **c.w, r=z)
    assert r2.data_ptr() == z.data_ptr() and torch.equal(r2, r) and torch.equal(h2, h)
    grads = c.backward(r, stats)
    d = c.dr.clone()
    again = c.backward(r, stats, dr=d, dx=d)
    assert again["dx"].data_ptr() == d.data_ptr()
    for n in grads:
        assert torch.equal(again[n], grads[n]), n
    none = c.backward(r, stats, dr=None)
    c.check_backward(r, stats, none, dr=False)
    zero = c.backward(r, stats, dr=torch.zeros_like(r))
    for n in none:
        assert torch.equal(none[n], zero[n]), n


def test_empty():
    for N, C in ((0, 8), (4, 0)):
        x = torch.zeros((N, C, 4), device="cuda")
        r, h, stats = gtp.gtp_residual_norm(x, x.clone(), 1)
        z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        g = gtp.gtp_residual_norm_backward(x, x.clone(), 1, (z(N), z(N, 2), z(N), z(N, 2)), x.clone())
        assert set(g) == {"dx", "da", "dscale", "dw_post", "db_post", "dw_pre", "db_pre"}
        for n in set(g) - {"dx", "da"}:
            assert not bool(g[n].any()), n


@pytest.mark.parametrize("C,L", [(64, 0), (33, 2), (128, 6), (300, 8)])
def test_constant_rows_zero_rows_and_large_mean(C, L):
    K = (L + 1) ** 2
    x = torch.full((5, C, K), 2.0, device="cuda")
    a = torch.zeros_like(x)
    b = torch.arange(C, device="cuda", dtype=F32)
    r, h, stats = gtp.gtp_residual_norm(x, a, L, b_pre=b)
    assert torch.equal(r, x) and torch.equal(h[..., 0], b.expand(5, C)) and bool((stats[2] == 2).all())
    assert torch.allclose(stats[1], torch.full((5, L + 1), 1e5 ** 0.5, device="cuda"), rtol=1e-6)
    c = Case(9, C, L, F32, seed=3)
    c.x[..., 0] += 1000.0
    r, h, stats = c.forward()
    _, rh, rs = R.forward(c.x.double(), c.a.double(), L, *c.wide(), True)
    # r is rounded at 1000 (2^-14 a half unit of 1024: 2^-15), the mean carries a few such units
    tol = (2.0 ** -12 * rs[3].amax(1) + 1e-5) * (1 + rh.abs().amax())
    close(h, rh, tol[:, None, None] * torch.ones_like(rh), "large mean")


def test_nan_and_infinities_stay_in_their_rows():
    for C, L, dtype in ((64, 0, F32), (32, 3, F32), (128, 6, BF16), (300, 8, F32)):
        c = Case(40, C, L, dtype, seed=4)
        r0, h0, s0 = c.forward()
        g0 = c.backward(r0, s0)
        c.x[7, 3, 0] = math.nan
        c.a[9, 1, 0] = math.inf
        r, h, stats = c.forward()
        rest = [i for i in range(40) if i not in (7, 9)]
        assert torch.equal(r[rest], r0[rest]) and torch.equal(h[rest], h0[rest])
        assert bool(torch.isnan(r[7, 3, 0])) and bool(torch.isnan(h[7, :, 0]).all()) and bool(torch.isnan(h[9, :, 0]).all())
        g = c.backward(r, stats)
        for n in ("dx", "da", "dgate"):
            assert torch.equal(g[n][rest], g0[n][rest]), n


def test_gates_at_the_ends():
    c = Case(6, 40, 2, F32, seed=5)
    c.w["gate"][:, 0], c.w["gate"][:, 1], c.w["gate"][:, 2], c.w["gate"][:, 3] = math.inf, -math.inf, 100.0, -100.0
    r, h, stats = c.forward()
    assert torch.equal(r[:, 1], c.x[:, 1])
    c.check_forward(r, h, stats)
    g = c.backward(r, stats)
    assert not bool(g["dgate"][:, :2].any()) and not bool(g["da"][:, 1:2].isnan().any())
    c.check_backward(r, stats, g)


def test_commutes_with_rotation():
    """Degree 1 turned by an orthogonal matrix, x and a alike."""
    g = gen(6)
    c = Case(50, 32, 1, F32, seed=6)
    D, _ = torch.linalg.qr(randn(g, 3, 3).cpu().double())
    D = D.float().cuda()
    turn = lambda t: torch.cat([t[..., :1], t[..., 1:] @ D.T], -1).contiguous()  # noqa: E731
    r, h, _ = c.forward()
    r2, h2, _ = gtp.gtp_residual_norm(turn(c.x), turn(c.a), 1, **c.w)
    assert float((r2 - turn(r)).abs().max()) < 2e-5 and float((h2 - turn(h)).abs().max()) < 4e-5


@pytest.mark.parametrize("N,C,L,post", [(6, 24, 0, True), (6, 24, 2, True), (5, 300, 1, False), (3, 128, 6, True)])
def test_gradient_against_differences(N, C, L, post):
    c = Case(N, C, L, F32, post=post, seed=7)
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

    gg = gen(78)
    for name, t in base.items():
        u = randn(gg, *t.shape)
        up, dn = t + 1e-2 * u, t - 1e-2 * u
        got, step = f(name, up) - f(name, dn), up.double() - dn.double()
        want = float((grads[name].double() * step).sum())
        # a cubic term of relative size h^2, and fp32 outputs' errors of 2^-21 of the cotangents' sizes over the difference
        noise = 2.0 ** -21 * float((c.dh.double().abs() + c.dr.double().abs()).sum()) * 3 + \
            1e-3 * float((grads[name].double() * step).abs().sum())
        _say(f"  {name}: difference {got:.6f} gradient {want:.6f}")
        assert abs(got - want) <= noise, name


@pytest.mark.parametrize("N,C,L", [(300, 256, 2), (3000, 20, 0), (64, 128, 6), (9, 300, 8)])
def test_bits_repeat_on_streams_and_in_graphs(N, C, L):
    c = Case(N, C, L, F32, seed=8)
    r, h, stats = c.forward()
    grads = c.backward(r, stats)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r2, h2, stats2 = c.forward(stream=side)
    grads2 = c.backward(r2, stats2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(r, r2) and torch.equal(h, h2)
    for n in grads:
        assert torch.equal(grads[n], grads2[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r3, h3, stats3 = c.forward()
        grads3 = c.backward(r3, stats3)
    for turn in range(3):
        for t in (r3, h3, *grads3.values()):
            t.fill_(float(turn))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r, r3) and torch.equal(h, h3)
        for n in grads:
            assert torch.equal(grads[n], grads3[n]), (turn, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_poisoned_lds(dtype):
    for N, C, L in ((40, 24, 0), (300, 64, 2), (20, 300, 0), (9, 128, 6), (5, 200, 4), (3, 300, 8), (2, 70, 12)):
        for post, gated in ((True, True), (False, False)):
            _say(f"poisoned N={N} C={C} L={L} {dtype}")
            c = Case(N, C, L, dtype, post, gated, seed=9)
            r, h, stats = c.forward()
            grads = c.backward(r, stats)
            with gtp.use_library(POISON_LIB):
                r2, h2, stats2 = c.forward()
                grads2 = c.backward(r, stats)
            assert torch.equal(r, r2) and torch.equal(h, h2)
            for n in grads:
                assert torch.equal(grads[n], grads2[n]), n


def test_many_rows():
    """More rows than a launch takes at a time; every row of the weights' sums counts once."""
    N, C = 70001, 8
    x, a = torch.zeros((N, C, 1), device="cuda"), torch.zeros((N, C, 1), device="cuda")
    x[:, 0] = 1.0
    r, h, stats = gtp.gtp_residual_norm(x, a, 0, post=False)
    g = gtp.gtp_residual_norm_backward(r, a, 0, stats, torch.ones_like(x), dr=torch.ones_like(x), post=False)
    assert bool((g["db_pre"] == N).all()) and not bool(g["dscale"].any())
    assert bool((h == h[0]).all()) and bool((g["dx"] == g["dx"][0]).all())
