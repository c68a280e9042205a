"""The layers around the product on long axes, on the GPU, with inputs of which one lost or doubled element is a large
error in some output: attention with equal scores, where single keys at the edges of tiles and parts hold the values; long
rows of the normalisation whose gradient's subtracted terms are of order one; weight gradients over more rows than one
workgroup's turn.

Tolerances: with all scores zero a probability is 1 / n and every sum over keys is of ones and zeros, exact in fp32 while
below 2^24; what is left of the forward is a division, a product and an output's rounding (2^-8 in bf16; fp32: a few units,
2^-20).  The gradients make P = exp(s - lse) again from lse in fp32: its error near 10, four units or 3.8e-6, is P's relative
error, with half a unit of 14 (lse in units of log 2) and the exponential's own: 4.5e-6, below 2^-17."""
import math

import pytest

torch = pytest.importorskip("torch")

import layers_ref as R  # noqa: E402
from test_layers import BF16, C32, F32, _say, close, norm_case, norm_check, out_tol  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


def edges(n, count):
    """`count` places of 0 .. n - 1: the first and last, and around multiples of 32, spread over the whole length."""
    at = sorted({0, n - 1, *(m + s for m in range(0, n + 32, 32) for s in (-1, 0) if 0 <= m + s < n)})
    step = max(1, -(-len(at) // count))
    picked = (at[::step] + at[-1:] + at[1::step])[:count]
    return torch.tensor((picked * count)[:count], device="cuda")


def near(got, want, rel, what):
    err = (got.double() - want).abs()
    _say(f"  {what}: worst {float((err / want.abs().clamp_min(1e-300)).max()) / rel:.3f} of the tolerance")
    assert bool((err <= rel * want.abs()).all()), (what, int((err > rel * want.abs()).sum()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq,nk,H,d", [(1, 20011, 8, 128), (1, 16384, 8, 100), (3, 17000, 12, 64), (40, 5001, 5, 72),
                                       (300, 2305, 2, 40), (1, 9001, 3, 200), (2, 16449, 4, 256)])
def test_every_key_counts_once(nq, nk, H, d, dtype):
    """Key J[h, i] alone holds element i of head h: o there is 1 / nk, and so on for the gradients."""
    _say(f"equal scores nq={nq} nk={nk} H={H} d={d} {dtype}")
    J = edges(nk, H * d).view(H, d)
    heads, cols = torch.arange(H, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    q = torch.zeros((nq, H, d), dtype=dtype, device="cuda")
    v = torch.zeros((nk, H, d), dtype=dtype, device="cuda")
    v[J, heads, cols] = 1.0
    k = v.clone()  # q = 0: the scores are equal all the same
    do = torch.ones_like(q)
    rel = 2.0 ** -7 if dtype == BF16 else 2.0 ** -20
    o, lse = gtp.gtp_attention(q, k, v, scale=0.5)
    near(o, torch.full(o.shape, 1.0 / nk, device="cuda").double(), rel, "o")
    # one key more or less moves lse by 1 / nk, at least 4.9e-5: four units of fp32 near 10 are 3.8e-6
    assert float((lse.double() - math.log(nk)).abs().max()) < 4e-6
    rel = 2.0 ** -7 if dtype == BF16 else 2.0 ** -17
    g = gtp.gtp_attention_backward(q, k, v, o, do, lse, scale=0.5)
    near(g["dv"], torch.full(v.shape, nq / nk, device="cuda").double(), rel, "dv")
    # dS = (dP - delta) / nk, dP the number of elements that the key holds, delta their sum's mean
    holds = v.double().sum(-1)
    ds = (holds - holds.mean(0)) / nk * 0.5
    want = (v.double() * ds[..., None]).sum(0)
    near(g["dq"], want.expand(nq, H, d), 2 * rel, "dq")
    assert not bool(g["dk"].any())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq,nk,H,Hk,d", [(17000, 2, 2, 2, 128), (9001, 3, 4, 1, 100), (2049, 65, 2, 1, 64), (16385, 40, 2, 2, 200)])
def test_every_row_counts_once(nq, nk, H, Hk, d, dtype):
    """Rows at tiles' edges alone hold the elements of q and dout: dv there is 1 / nk and dk dS of that row."""
    _say(f"equal scores nq={nq} nk={nk} H={H}/{Hk} d={d} {dtype}")
    G = H // Hk
    J = edges(nq * G, Hk * d).view(Hk, d)  # rows of a key head's query heads together
    hk, cols = torch.arange(Hk, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    q = torch.zeros((nq, H, d), dtype=dtype, device="cuda")
    q[J // G, hk * G + J % G, cols] = 1.0
    do = q.clone()
    k = torch.zeros((nk, Hk, d), dtype=dtype, device="cuda")
    v = (torch.arange(nk, device="cuda")[:, None, None] % 2 * 2.0 - 1.0 + torch.zeros_like(k)).to(dtype)  # -1, 1, ...
    o, lse = gtp.gtp_attention(q, k, v, scale=0.5)
    g = gtp.gtp_attention_backward(q, k, v, o, do, lse, scale=0.5)
    rel = 2.0 ** -7 if dtype == BF16 else 2.0 ** -17
    near(g["dv"], torch.full(v.shape, 1.0 / nk, device="cuda").double(), rel, "dv")
    # a row of c ones in dout: dS[row, j] = c (v[j] - mean v) / nk, o's rounding in the mean
    ones = do.double().sum(-1)[J // G, hk * G + J % G]
    mean = v.double()[:, 0, 0].mean()
    want = 0.5 / nk * ones[None] * (v.double() - mean)
    err = (g["dk"].double() - want).abs()
    assert bool((err <= rel * 0.5 / nk * ones[None] * 2).all()), int((err > rel / nk * ones[None]).sum())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(2, 70001, 0), (3, 9000, 0), (3, 4000, 0), (4, 512, 6), (2, 600, 8), (3, 64, 16), (40, 256, 0), (9, 64, 2)])
def test_norm_gradient_subtracts_its_means(N, C, L, dtype):
    """dy with a mean of one and half of x in it: both subtracted terms are of order one, and so is what a missing one
    leaves.  An element's error is counted against the terms that it is made of."""
    x, dy, _, _ = norm_case(N, C, L, dtype, 9)
    dy = (1.0 + 0.5 * x.float() + 0.1 * dy.float()).to(dtype)
    _, mean, rstd = gtp.gtp_layer_norm(x, L)
    got = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, need=("dx",))["dx"]
    d = [t.double() for t in (x, dy, mean, rstd)]
    want = R.norm_backward(d[0], d[1], L, None, d[2], d[3])[0]
    terms = torch.empty_like(want)
    for l, sl in enumerate(R.degree_slices(L)):
        r = d[3][:, l][:, None, None]
        xh = (d[0][..., sl] - (d[2][:, None, None] if l == 0 else 0.0)) * r
        g = d[1][..., sl].abs()
        terms[..., sl] = r * (g + xh.abs() * (g * xh.abs()).mean((1, 2), keepdim=True) + g.mean((1, 2), keepdim=True))
    close(got, want, out_tol(want, dtype) + C32 * terms, "dx")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(1500, 9000, 0), (700, 512, 6), (300, 400, 8), (5000, 3, 0), (3000, 1, 1), (200, 70001, 0)])
def test_norm_weight_gradients_over_many_rows(N, C, L, dtype):
    """Rows too long for the registers, more of them than parts of the sum; the general path in several chunks of rows."""
    x, dy, w, b = norm_case(N, C, L, dtype, 10)
    y, mean, rstd = gtp.gtp_layer_norm(x, L, w, b)
    grads = gtp.gtp_layer_norm_backward(x, dy, L, mean, rstd, w)
    norm_check(x, dy, w, b, L, y, mean, rstd, grads, f"{N},{C},{L}")
    # sums of ones: every row once
    one = gtp.gtp_layer_norm_backward(x, torch.ones_like(dy), L, mean, rstd, need=("db",))["db"]
    assert torch.equal(one, torch.full_like(one, float(N)))
