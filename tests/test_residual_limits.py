"""Limits of the residual step: outputs that are not asked for (on the CPU); infinities in the gradients of the last rows
(-m gpu)."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2401_10216_amd import gtp  # noqa: E402
from test_residual_terms import BF16, F32, Case  # noqa: E402


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(9, 17, 0), (37, 128, 0), (21, 4, 1), (5, 16, 2), (6, 128, 2), (3, 300, 8), (5, 4500, 0)])
def test_infinities_of_the_last_row_stay_in_their_sums(N, C, L, dtype):
    """An infinite dh or dr makes the weights' gradients that it enters infinite, not NaN: in a row that lanes without a row of
    their own load again, as in any other."""
    for n in (0, N - 1):
        print(f"residual infinities N={N} C={C} L={L} {dtype} row {n}", flush=True)
        c = Case(N, C, L, 1, dtype, device="cuda")
        r, _, stats = c.forward()
        clean = c.backward(r, stats)
        c.dh[n, 1, 0] = math.inf
        g = c.backward(r, stats)
        x = (r[:, 1, 0].double() - stats[2].double()) * stats[3][:, 0].double()
        assert float(g["db_pre"][1]) == math.inf and float(g["dw_pre"][0, 1]) == math.copysign(math.inf, float(x[n]))
        for name in ("db_pre", "dw_pre"):
            rest = torch.ones_like(g[name], dtype=torch.bool)
            rest[..., 1].view(-1)[0] = False
            assert torch.equal(g[name][rest], clean[name][rest]), name
        c = Case(N, C, L, 1, dtype, device="cuda")
        c.dr[n, 1, 0] = -math.inf
        g = c.backward(r, stats)
        xh = (c.a[:, 1, 0].double() - stats[0].double()) * stats[1][:, 0].double()
        s = math.copysign(math.inf, -float(c.w["scale"][0, 1]))
        assert float(g["db_post"][1]) == s and float(g["dw_post"][0, 1]) == math.copysign(s, -float(xh[n]) * float(c.w["scale"][0, 1]))
        for name in ("db_post", "dw_post", "dscale"):
            rest = torch.ones_like(g[name], dtype=torch.bool)
            rest[..., 1].view(-1)[0] = False
            assert torch.equal(g[name][rest], clean[name][rest]), name
        # dscale: the sum of infinite terms of two signs may be NaN; of one it is infinite
        t = xh[n] * c.w["w_post"][0, 1].double(), c.w["b_post"][1].double()
        if float(t[0]) * float(t[1]) > 0:
            assert float(g["dscale"][0, 1]) == math.copysign(math.inf, -float(t[0]))


def test_dx_that_is_not_asked_for():
    """Refused before anything else happens: it would stay as it was."""
    z = torch.zeros
    x, st = z(4, 8, 9), (z(4), z(4, 3), z(4), z(4, 3))
    for need in (("da",), ("dscale", "dw_pre"), ()):
        with pytest.raises(ValueError, match="dx is given"):
            gtp.gtp_residual_norm_backward(x, x, 2, st, x, need=need, dx=z(4, 8, 9))
    for need in (None, ("dx", "da")):  # asked for: the next refusal, of tensors in host memory
        with pytest.raises(ValueError, match="device tensor"):
            gtp.gtp_residual_norm_backward(x, x, 2, st, x, need=need, dx=z(4, 8, 9))


@pytest.mark.gpu
def test_need_may_be_any_iterable():
    c = Case(5, 16, 2, 1, F32, device="cuda")
    r, _, stats = c.forward()
    all_ = c.backward(r, stats)
    for names in (("dx", "dscale"), ("da",), ("dgate", "db_pre"), ("dw_post", "dw_post"), ()):
        for need in (names, iter(names), set(names), (n for n in names)):
            got = c.backward(r, stats, need=need)
            assert set(got) == set(names) and all(torch.equal(got[n], all_[n]) for n in names)
