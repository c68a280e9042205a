"""The layers around the product on the GPU at the edges of what their entries
accept: gradients in place, infinities and values near fp32's largest, sizes
past one launch, many rows a workgroup."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from test_layers import BF16, C32, F32, Case, _say, close, norm_case, norm_check  # noqa: E402
from paper_2401_10216_amd import gtp  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gtp.lib()


def stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def code(t):
    return {F32: 0, BF16: 1}[t.dtype]


# ------------------------------------------------------------------ normalisation

def norm_backward_into(x, dy, L, mean, rstd, w, dx):
    """The C entry with dx given (it may be dy): dx, dw, db."""
    N, C, _ = x.shape
    lib = gtp.lib()
    n = lib.gtp_layer_norm_backward_work(L, code(x), N, C)
    work = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty((L + 1, C), device="cuda"), torch.empty(C, device="cuda")
    assert lib.gtp_layer_norm_backward(L, x.data_ptr(), code(x), w.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                       dy.data_ptr(), N, C, dx.data_ptr(), dw.data_ptr(), db.data_ptr(), work.data_ptr(),
                                       n, stream()) == gtp.GTP_OK
    return dx, dw, db


# rows in a wave, in registers (scalars; degrees), too long for them (degrees; scalars), and the general path (short; long)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(40, 256, 0), (9, 4000, 0), (40, 64, 2), (9, 512, 6), (5, 600, 8), (7, 9000, 0),
                                   (70, 1, 1), (3, 7, 0), (2, 70001, 0)])
def test_norm_gradient_in_place(N, C, L, dtype):
    _say(f"norm gradient in place N={N} C={C} L={L} {dtype}")
    x, dy, w, b = norm_case(N, C, L, dtype, 6)
    y, mean, rstd = gtp.gtp_layer_norm(x, L, w, b)
    want = norm_backward_into(x, dy, L, mean, rstd, w, torch.empty_like(dy))
    norm_check(x, dy, w, b, L, y, mean, rstd, dict(zip(("dx", "dw", "db"), want)), "apart")
    z = dy.clone()
    got = norm_backward_into(x, z, L, mean, rstd, w, z)
    assert all(torch.equal(g, e) for g, e in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,C,L", [(40, 256, 0), (9, 4000, 0), (9, 512, 6), (5, 600, 8), (3, 65, 12), (7, 9000, 0),
                                   (70, 1, 1), (3, 7, 0), (2, 70001, 0)])
def test_norm_in_place(N, C, L, dtype):
    x, _, w, b = norm_case(N, C, L, dtype, 7)
    want = gtp.gtp_layer_norm(x, L, w, b)
    z = x.clone()
    got = gtp.gtp_layer_norm(z, L, w, b, y=z)
    assert got[0].data_ptr() == z.data_ptr() and all(torch.equal(g, e) for g, e in zip(got, want))


def test_norm_of_many_short_rows():
    """More than 2^24 rows on the general path: more workgroups of 256 than one launch holds.  (Weight sums of up to 3072
    terms a lane with signs at random: some 46 units of the terms' magnitudes, below the 256 of C32.)"""
    x, dy, w, b = norm_case((1 << 24) + 5, 1, 1, F32, 8)
    y, mean, rstd = gtp.gtp_layer_norm(x, 1, w, b)
    grads = gtp.gtp_layer_norm_backward(x, dy, 1, mean, rstd, w)
    norm_check(x, dy, w, b, 1, y, mean, rstd, grads, "many rows")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_many_channels(dtype):
    """More than 2^25 channels: more workgroups of a channel, or of 16 columns of weight sums, than one launch holds.
    Values whose statistics and gradients are exact: x = 1, -1, ..., so mean 0, rstd 1 / sqrt(1 + 3)."""
    C = (1 << 25) + 4
    c = torch.arange(C, device="cuda")
    s = 1.0 - 2.0 * (c % 2)
    x = torch.stack([s, -s]).unsqueeze(-1).to(dtype)
    dy = torch.stack([(c % 4).float(), torch.ones_like(s)]).unsqueeze(-1).to(dtype)
    y, mean, rstd = gtp.gtp_layer_norm(x, 0, eps=3.0)
    assert torch.allclose(mean, torch.zeros_like(mean), atol=1e-6) and torch.allclose(rstd, torch.full_like(rstd, 0.5))
    assert torch.equal(y, x * 0.5)
    g = gtp.gtp_layer_norm_backward(x, dy, 0, mean, rstd)
    # row 0: mean of dy 3 / 2, of dy xh -1 / 4; row 1: 1 and 0
    want = torch.stack([0.5 * ((c % 4) - 1.5 + 0.25 * 0.5 * s), torch.zeros_like(s)]).unsqueeze(-1)
    assert float((g["dx"].float() - want).abs().max()) <= (2.0 ** -8 if dtype == BF16 else 1e-6)
    assert torch.allclose(g["dw"][0], 0.5 * s * ((c % 4) - 1), atol=1e-6) and torch.equal(g["db"], (c % 4) + 1.0)


# ------------------------------------------------------------------ attention: infinities, large values

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [4, 72, 200])
def test_attention_infinity_times_infinity(d, dtype):
    """Infinity times minus infinity is a score of minus infinity, as a finite number times it is."""
    c = Case(dtype, [8], [8], 1, 1, d)
    c.q.fill_(0.25)
    c.q[3, 0, 1] = math.inf
    c.k.fill_(0.0)
    c.k[:, 0, 1] = -math.inf  # every score of every row
    o, lse = c.forward()
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("d", [4, 72, 200])
def test_attention_values_near_the_largest(d):
    """fp32 values above the largest bf16 value (3.39e38) are what they are: a score of such a key with a small enough
    query is finite, and so are its gradients."""
    c = Case(F32, [40], [50], 1, 1, d, scale=1.0)
    c.q.fill_(0.0)
    c.q[:, 0, 0] = 1.0
    c.q[:, 0, 1] = 2.0 ** -126
    c.k[:, 0, 1:] = 0.0
    c.k[2, 0, 1] = torch.finfo(F32).max
    c.k[3, 0, 1] = -torch.finfo(F32).max
    ro, rl, size = c.ref()
    o, lse = c.forward()
    # a score's terms are below 4 + 4: P moves by C32 of that, with room for the sums
    tol = 16 * C32
    close(o, ro, tol * size + 1e-30, "o")
    close(lse, rl, tol * torch.ones_like(rl), "lse")
    g = c.backward(o, lse)
    for n, (want, terms, e32) in zip(("dq", "dk", "dv"), c.ref((c.do.double(), o.double(), lse.double()))):
        held = terms < torch.finfo(F32).max  # dq's terms dS k may pass fp32's range, as a product of finite numbers can
        assert float(held.double().mean()) > 0.5 and (n == "dq" or bool(held.all()))
        close(g[n][held], want[held], (tol * e32 + 2.0 ** -23 * want.abs() + 1e-30)[held], n)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ql,kl", [([8], [8]), ([1], [9000])])
def test_attention_gradient_of_rows_of_minus_infinity(ql, kl, dtype):
    """A row whose every score is minus infinity has an output of zeros, so no gradient comes from it or to it."""
    c = Case(dtype, ql, kl, 2, 2, 72)
    c.q.fill_(1.0)
    c.k.fill_(0.0)
    c.k[:, 0, 1] = -math.inf  # the first head's rows; the second's are ordinary
    o, lse = c.forward()
    assert bool((o[:, 0] == 0).all()) and bool((lse[:, 0] == -math.inf).all()) and bool(torch.isfinite(lse[:, 1]).all())
    g = c.backward(o, lse)
    for n in ("dq", "dk", "dv"):
        assert not bool(g[n][:, 0].any()), n
        assert bool(torch.isfinite(g[n]).all()) and (n != "dv" or bool(g[n][:, 1].any())), n


def test_attention_gradient_of_many_rows_and_heads():
    """More than 2^28 rows of heads: more threads than one launch holds, 16 a row."""
    B, nq, nk, H = 16385, 64, 4, 256
    assert B * nq * H > 1 << 28
    c = Case(BF16, [nq], [nk], H, 1, 1)
    g = torch.Generator(device="cuda").manual_seed(8)
    q, do = (torch.randn((B * nq, H, 1), generator=g, device="cuda", dtype=BF16) for _ in range(2))
    k, v = (torch.randn((B * nk, 1, 1), generator=g, device="cuda", dtype=BF16) for _ in range(2))
    o, lse = gtp.gtp_attention(q, k, v, scale=c.scale, max_q=nq, max_k=nk)
    grads = gtp.gtp_attention_backward(q, k, v, o, do, lse, scale=c.scale, max_q=nq, max_k=nk)
    for b in (0, 7000, B - 1):
        rows, keys = slice(b * nq, (b + 1) * nq), slice(b * nk, (b + 1) * nk)
        c.q, c.k, c.v, c.do = q[rows], k[keys], v[keys], do[rows]
        c.check_forward(o[rows], lse[rows])
        c.check_backward(o[rows], lse[rows], {"dq": grads["dq"][rows], "dk": grads["dk"][keys], "dv": grads["dv"][keys]})


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 75])
def test_attention_gradients_into_slices_by_head(d, dtype):
    """q, k, v and their gradients interleaved by head: slices of [T, H, 3, d], and of [H, T, 3, d]."""
    c = Case(dtype, [33, 64, 90], [33, 64, 90], 4, 4, d)
    o, lse = c.forward()
    g = c.backward(o, lse)
    T = sum(c.ql)
    for shape, turn in (((T, 4, 3, d), lambda t: t), ((4, T, 3, d), lambda t: t.transpose(0, 1))):
        buf = torch.zeros(shape, dtype=dtype, device="cuda")
        q, k, v = (turn(t) for t in buf.unbind(2))
        q.copy_(c.q), k.copy_(c.k), v.copy_(c.v)
        out = torch.full_like(buf, 7.0)
        dq, dk, dv = (turn(t) for t in out.unbind(2))
        o2, lse2 = gtp.gtp_attention(q, k, v, **c.args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        gtp.gtp_attention_backward(q, k, v, o, c.do, lse, **c.args, dq=dq, dk=dk, dv=dv)
        assert torch.equal(dq, g["dq"]) and torch.equal(dk, g["dk"]) and torch.equal(dv, g["dv"])


def test_attention_of_no_rows_against_equal_segments():
    """No query row, three segments of keys: gradients of zero; no key, three segments of rows: outputs of zero."""
    c = Case(F32, [5], [12], 2, 2, 8)
    q, do = c.q[:0], c.do[:0]
    o, lse = gtp.gtp_attention(q, c.k, c.v, max_q=0, max_k=4)
    g = gtp.gtp_attention_backward(q, c.k, c.v, o, do, lse, max_q=0, max_k=4)
    assert o.shape == q.shape and not bool(g["dk"].any()) and not bool(g["dv"].any())
    q, do, k = c.k, c.v, c.q[:0]
    o, lse = gtp.gtp_attention(q, k, k, max_q=4, max_k=0)
    g = gtp.gtp_attention_backward(q, k, k, o, do, lse, max_q=4, max_k=0)
    assert not bool(o.any()) and bool((lse == -math.inf).all()) and not bool(g["dq"].any()) and g["dk"].shape == k.shape
